// Softmax cross entropy and its gradients where one side is short: at most 64
// rows a worker (a small batch, the last tokens of a few sequences), or at most
// 64 classes.  The formulas are the large path's; what differs is what bounds
// them: the long side (the weight, or the rows) is read once a pass, and its
// products with the short side are few.  So nothing is laid out anew.
//
// "Stream" is the long side (n x cols), "side" the short one (up to 64 x cols).
//   few_side    the short side as operands of the logits, in their order (not
//               for the smallest calls)
//   few_logit   a workgroup takes 16 to 64 rows of the stream: the logits, with
//               the sum over columns cut among its waves and joined in LDS; then
//               forward what a row needs of them, backward g, stored both ways
//   few_rest    does the latter where several workgroups share the columns
//   few_sum     the side's gradient, g^T stream: a sum over the stream, which is
//               read again, cut among waves and workgroups
//   few_finish  adds the workgroups' sums up in a fixed order, if there are more
//               than one
//   few_outer   the stream's gradient, g side: a sum over the short side, bound
//               by what it writes
//
// Operands go from memory to registers and to the matrix cores as bfloat16
// pieces: a bfloat16 element is one, a binary32 element three that hold its 24
// bits (cut off, not rounded, so that the largest value does not overflow; for
// the logits each of the others is scaled to the first one's size and has sums of
// its own, or the smallest values' pieces would be under bfloat16's).  Of
// the pieces' products those under 2^-24 of a term are left out; of g, where the
// result is rounded to bfloat16, two pieces are taken (16 bits next to 1).
//
// The gradients' pieces share one sum, for which the registers are enough: there
// an operand whose values are all far under one is taken times a power of two
// (the stream's as long as a wave has seen no larger one, so others' calls do not
// pay for it), and so are factors.
//
// A matrix instruction sums over 32 elements, of which a lane has eight.  For
// the logits they are neighbours in a row.  For the other two products the sum
// runs over rows: a lane takes 16 bytes of the same columns of eight rows, and
// each column of them is an operand of a product of its own, so nothing is
// transposed in memory or in LDS.
#include <algorithm>
#include <type_traits>

#include "tc_lane.h"

namespace tc {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kWorkers = 16;  // of one launch
constexpr int kShort = 64;    // rows of the short side
// Steps from one workgroup's beginning to the next one's: odd, so that neighbours
// are at different halves of 64 columns too, and far enough for the memory's
// channels (8 rows of 4,096 over 131,072 classes in bfloat16 with 0, 1, 2, 5, 8,
// 32 steps: 261, 221, 312, 218, 257, 262 us; 16 of 8,192 over 32,000 155, 120, 118,
// 116, 191, 155; 5 of 4,096 over 32,000 in binary32 119, 111, 154, 102, 105, 119).
constexpr int kTurn = 5;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// --------------------------------------------------------------------- operands

// Eight elements as bfloat16 pieces, the largest first.
template <int P>
struct Pieces {
    u32x4 p[P];
};

__device__ __forceinline__ uint32_t high_halves(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x07060302u); }

// P pieces of eight binary32 values, cut off; UP: piece n times 2^8n, so that it
// is no smaller than bfloat16's values where the first one is not.
template <int P, bool UP = false>
__device__ __forceinline__ Pieces<P> cut(const float* f) {
    Pieces<P> r;
    float rest[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) rest[e] = f[e];
#pragma unroll
    for (int n = 0; n < P; ++n) {
#pragma unroll
        for (int i = 0; i < 4; ++i) r.p[n][i] = high_halves(__float_as_uint(rest[2 * i]), __float_as_uint(rest[2 * i + 1]));
        if (n + 1 < P)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                rest[e] -= __uint_as_float(__float_as_uint(rest[e]) & 0xffff0000u);
                if (UP) rest[e] *= 256.0f;
            }
    }
    return r;
}

// Sums of the products of pieces i and j that are times 2^8(i + j).
template <int PA, int PB>
struct Sums {
    static constexpr int kSums = PA > PB ? PA : PB;
    f32x4 v[kSums];
    __device__ __forceinline__ void add(const Pieces<PA>& a, const Pieces<PB>& b) {
#pragma unroll
        for (int i = 0; i < PA; ++i)
#pragma unroll
            for (int j = 0; j < PB; ++j)
                if (i + j < kSums)
                    v[i + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.p[i]), __builtin_bit_cast(bf16x8, b.p[j]), v[i + j], 0, 0, 0);
    }
    __device__ __forceinline__ f32x4 sum() const {
        f32x4 s = v[0];
        if constexpr (kSums == 3) s += (v[2] * 0x1p-8f + v[1]) * 0x1p-8f;
        return s;
    }
};

template <int PA, int PB>
__device__ __forceinline__ f32x4 multiply(const Pieces<PA>& a, const Pieces<PB>& b, f32x4 c) {
    constexpr int kMost = (PA > PB ? PA : PB) - 1;  // products of pieces i and j, i + j <= kMost, small ones first
#pragma unroll
    for (int s = kMost; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < PA; ++i) {
            const int j = s - i;
            if (j < 0 || j >= PB) continue;
            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.p[i]), __builtin_bit_cast(bf16x8, b.p[j]), c, 0, 0, 0);
        }
    return c;
}

// What the rows of an operand are: binary32, bfloat16 at addresses of whole
// words, or bfloat16 at any.
enum Kind { kF32, kBf16, kOdd };

// Eight neighbouring elements of a row as they lie, and as pieces.
template <Kind KIND>
struct Eight {
    u32x4 v[KIND == kF32 ? 2 : 1];
    uint32_t more;  // kOdd: the word behind
};
// WHOLE: they are in the row; otherwise zeros past its end.  (Where rows begin
// between words, 16 bytes at such an address take more than twice the time: 48
// rows of 2,417 over 17,610 classes 104 us, of 2,418 43.  So whole words are
// loaded, each of which has an element of the row, and moved down.)
template <Kind KIND, bool WHOLE>
__device__ __forceinline__ Eight<KIND> load_eight(uintptr_t row, int c, int cols) {
    Eight<KIND> r;
    if constexpr (KIND == kF32) {
#pragma unroll
        for (int h = 0; h < 2; ++h) r.v[h] = WHOLE ? gld_u<u32x4>(row + c * 4 + h * 16) : load_vec<float, true>(row, c / 4 + h, cols);
    } else if constexpr (KIND == kBf16 || !WHOLE) {
        r.v[0] = WHOLE ? gld_u<u32x4>(row + c * 2) : load_vec<__bf16, true>(row, c / 8, cols);
    } else {
        const uintptr_t at = row + c * 2;
        r.v[0] = gld_u<u32x4>(at & ~uintptr_t{3});
        r.more = gld<uint32_t>((at & ~uintptr_t{3}) + 12 + (at & 2) * 2);
    }
    return r;
}
template <Kind KIND, bool WHOLE>
__device__ __forceinline__ Pieces<KIND == kF32 ? 3 : 1> pieces(const Eight<KIND>& e, uintptr_t row) {
    if constexpr (KIND == kF32) {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(e.v[i / 4][i % 4]);
        return cut<3, true>(f);
    } else if constexpr (KIND == kBf16 || !WHOLE) {
        return {{e.v[0]}};
    } else {
        const uint32_t by = (row & 2) * 8;  // bits
        Pieces<1> r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r.p[0][i] = __builtin_amdgcn_alignbit(i < 3 ? e.v[0][i + 1] : e.more, e.v[0][i], by);
        return r;
    }
}

// Operands of the gradients' products with no value of kSmall or more are taken
// times kLift, factors with none of kSmallFactor times kLiftFactor: their last
// pieces would be under bfloat16's values (2^-133) otherwise.
constexpr float kSmall = 0x1p-90f, kLift = 0x1p100f, kSmallFactor = 0x1p-60f, kLiftFactor = 0x1p64f;

__device__ __forceinline__ bool in_any_lane(bool b) { return __builtin_amdgcn_ballot_w64(b) != 0; }

// The operands of one block of columns from eight rows: one for each of the
// TILES columns that a lane has, 16 bytes of a row (8 of bfloat16, 4 of
// binary32) or 8 (4 of bfloat16).  As right operands: the results' rows are the
// other operand's, and 16 lanes have neighbouring columns of a row.
template <bool BF, int TILES = BF ? 8 : 4>
struct Columns {
    static constexpr int kTiles = TILES, kBlock = 16 * TILES;  // columns of a block
    static constexpr int kWords = TILES * (BF ? 2 : 4) / 4;
    typedef uint32_t Row __attribute__((ext_vector_type(kWords)));
    Row v[8];
    // of a row, at column c; WHOLE: they are in the row; otherwise zeros past its end
    template <bool WHOLE>
    static __device__ __forceinline__ Row load(uintptr_t row, int c, int cols) {
        if constexpr (WHOLE) {
            return gld_u<Row>(row + c * (BF ? 2 : 4));
        } else if constexpr (kWords == 4) {
            return load_vec<std::conditional_t<BF, __bf16, float>, true>(row, c / TILES, cols);
        } else {
            Row r = {};
#pragma unroll
            for (int i = 0; i < TILES; ++i)
                if (c + i < cols) r[i / 2] |= static_cast<uint32_t>(gld<uint16_t>(row + (c + i) * 2)) << i % 2 * 16;
            return r;
        }
    }
    // only rows whose bit is set: the others count as zeros, whatever they hold
    __device__ __forceinline__ void keep(uint32_t rows) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < kWords; ++i) v[j][i] = rows >> j & 1 ? v[j][i] : 0u;
    }
    // binary32: the lane's largest value; all of them times kLift
    __device__ __forceinline__ float largest() const {
        float top = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < kWords; ++i) top = fmaxf(top, fabsf(__uint_as_float(v[j][i])));
        return top;
    }
    __device__ __forceinline__ void lift() {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < kWords; ++i) v[j][i] = __float_as_uint(__uint_as_float(v[j][i]) * kLift);
    }
    // column t of the lane's, over the eight rows
    template <int P>
    __device__ __forceinline__ Pieces<P> get(int t) const {
        if constexpr (BF) {
            Pieces<P> r;
            const uint32_t select = t % 2 ? 0x07060302u : 0x05040100u;
#pragma unroll
            for (int i = 0; i < 4; ++i) r.p[0][i] = __builtin_amdgcn_perm(v[2 * i + 1][t / 2], v[2 * i][t / 2], select);
            return r;
        } else {
            float f[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(v[j][t]);
            return cut<P>(f);
        }
    }
};

// Loads stay on this side: the compiler would move them down to where they are
// needed.
__device__ __forceinline__ void loads_first() { asm volatile("" ::: "memory"); }

// ----------------------------------------------------------------------- logits

struct FewArgs {
    const void* x[kWorkers];
    const void* w[kWorkers];
    const void* bias[kWorkers];
    const int64_t* label[kWorkers];
    float* lse[kWorkers];   // written forward, read backward
    float* loss[kWorkers];  // forward
    const float* dloss[kWorkers];
    void* db[kWorkers];  // dbias
    int64_t rows[kWorkers];
    char* work;
    int64_t stride;            // of the workspace, from worker to worker
    int64_t at_pairs, at_own;  // forward, stream of classes: (largest, sum) [row][workgroup]; the label's logit
    int64_t at_side;           // the side as operands: [32 columns][16 rows][piece][lane]
    int64_t at_g;              // backward, g and f g as operands, one: [32 rows of the stream][16 of the side][piece][lane]
    int64_t at_fg;             // the other: [16 rows of the stream][32 of the side][piece][lane]
    int64_t at_f;              // stream of rows: their factors
    int64_t at_db;             // and partial sums of dbias [workgroup][class]
    int64_t at_z;              // sums over a part of the columns [part][workgroup][row of the side][of the stream]
    int64_t x_ld;              // elements
    int64_t classes;
    int32_t cols, tiles, cuts, w_bf, db_bf, has_dloss, backward;
    int32_t pieces_g, pieces_fg;
    float scale;
};

__device__ __forceinline__ float load_any(const void* p, int64_t i, int bf) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p);
    return bf ? Lane<__bf16>::get(a + i * 2) : Lane<float>::get(a + i * 4);
}
__device__ __forceinline__ void store_any(void* p, int64_t i, int bf, float v) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p);
    if (bf)
        Lane<__bf16>::put(a + i * 2, v);
    else
        Lane<float>::put(a + i * 4, v);
}

// The factor of a row without `scale`: 0 of a row that is left out.
__device__ __forceinline__ float factor_of(const int64_t* label, const float* dloss, int64_t row, int64_t classes) {
    const int64_t l = label[row];
    return l >= 0 && l < classes ? (dloss ? dloss[row] : 1.0f) : 0.0f;
}

__device__ __forceinline__ void join(float& m, float& s, float m2, float s2) {
    const float top = fmaxf(m, m2);
    const float a = m == top ? s : s * __builtin_amdgcn_exp2f((m - top) * kLog2e);
    const float b = m2 == top ? s2 : s2 * __builtin_amdgcn_exp2f((m2 - top) * kLog2e);
    m = top;
    s = a + b;
}

// The side's operands of the logits: a lane's eight elements of one row, in
// pieces, as a wave loads them; zeros where there are no rows or columns.
template <bool TB, bool ROWS>
__global__ void __launch_bounds__(256) few_side_kernel(const FewArgs a, int mt) {
    constexpr int P = TB ? 1 : 3;
    const int k = blockIdx.y, unit = blockIdx.x * 4 + threadIdx.x / 64, lane = threadIdx.x % 64;
    const int steps = (a.cols + 31) / 32, c = unit / mt * 32 + lane / 16 * 8, t = unit % mt * 16 + lane % 16;
    if (unit >= steps * mt) return;
    const int64_t n_t = ROWS ? a.classes : a.rows[k];
    const uintptr_t side = reinterpret_cast<uintptr_t>(ROWS ? a.w[k] : a.x[k]);
    const uintptr_t row = side + t * (ROWS ? a.cols : a.x_ld) * (TB ? 2 : 4);
    constexpr Kind kKind = TB ? kBf16 : kF32;
    Eight<kKind> e{};
    if (t < n_t) e = c + 8 <= a.cols ? load_eight<kKind, true>(row, c, a.cols) : load_eight<kKind, false>(row, c, a.cols);
    const Pieces<P> p = pieces<kKind, false>(e, row);
    u32x4* to = reinterpret_cast<u32x4*>(a.work + k * a.stride + a.at_side) + unit * (P * 64) + lane;
#pragma unroll
    for (int n = 0; n < P; ++n) to[n * 64] = p.p[n];
}

constexpr int kLogitThreads = 512;

// The factors of the rows that a workgroup has (backward), and what f g is held
// times: of the worker's rows, or of each 32 of a stream of rows, for which the
// sum over them finds it from the factors alone.
struct Factors {
    float f[64], lift[2];
};
template <int kS, int MT, bool ROWS>
__device__ __forceinline__ void few_factors(const FewArgs& a, int k, int64_t s0, Factors& factors) {
    constexpr int kT = MT * 16;
    const int tid = threadIdx.x;
    const int64_t rows = a.rows[k];
    const float* dloss = a.has_dloss ? a.dloss[k] : nullptr;
    if (!a.backward || tid >= 64) return;
    auto of = [&](int64_t row) { return row < rows ? factor_of(a.label[k], dloss, row, a.classes) : 0.0f; };
    if (tid < (ROWS ? kS : kT)) factors.f[tid] = of(ROWS ? s0 + tid : tid);
    float top = 1.0f;
    if (dloss) {
        top = fabsf(of(ROWS ? s0 / 32 * 32 + tid : tid));
#pragma unroll
        for (int m = ROWS ? 16 : 32; m > 0; m >>= 1) top = fmaxf(top, __shfl_xor(top, m, 64));
    }
    if (tid % 32 == 0) factors.lift[tid / 32] = top < kSmallFactor ? kLiftFactor : 1.0f;
}

// A class's bias; classes that are none have -infinity.
__device__ __forceinline__ float few_bias(const FewArgs& a, int k, int64_t v) {
    return v >= a.classes ? -INFINITY : a.bias[k] ? load_any(a.bias[k], v, a.w_bf) : 0.0f;
}

// What comes of the logits z [row of the side][of the stream].
template <int kS, int MT, bool ROWS>
__device__ __forceinline__ void few_results(const FewArgs& a, int k, int64_t s0, float* z, const Factors& factors) {
    constexpr int kThreads = kLogitThreads, kT = MT * 16, kPitch = kS + 4;
    const int tid = threadIdx.x;
    const int64_t rows = a.rows[k];
    char* work = a.work + k * a.stride;
    auto at_z = [&](int t, int s) -> float& { return z[t * kPitch + s]; };
    if (!a.backward) {
        // the largest and the sum: of a side's row over the workgroup's classes,
        // or of a stream's row over all of them
        constexpr int kRows = ROWS ? kS : kT, kOver = ROWS ? kT : kS, kLanes = kThreads / kRows < 64 ? kThreads / kRows : 64;
        const int r = tid / kLanes, sub = tid % kLanes;
        auto get = [&](int o) { return ROWS ? at_z(o, r) : at_z(r, o); };
        float top = -INFINITY, sum = 0.0f;
        for (int o = sub; o < kOver; o += kLanes) top = fmaxf(top, get(o));
        const float from = top > -INFINITY ? top : 0.0f;
        for (int o = sub; o < kOver; o += kLanes) sum += __builtin_amdgcn_exp2f((get(o) - from) * kLog2e);
#pragma unroll
        for (int m = kLanes / 2; m > 0; m >>= 1) join(top, sum, __shfl_xor(top, m, 64), __shfl_xor(sum, m, 64));
        const int64_t row = ROWS ? s0 + r : r;
        if (sub || r >= kRows || row >= rows) return;
        const int64_t label = a.label[k][row];
        const bool counts = label >= 0 && label < a.classes;
        if constexpr (ROWS) {
            const float lse = top + log2f(sum) * kLn2;
            a.lse[k][row] = lse;
            a.loss[k][row] = counts ? lse - get(static_cast<int>(label)) : 0.0f;
        } else {
            reinterpret_cast<float2*>(work + a.at_pairs)[row * a.tiles + blockIdx.x] = make_float2(top, sum);
            if (counts && label >= s0 && label < s0 + kS) reinterpret_cast<float*>(work + a.at_own)[row] = get(static_cast<int>(label - s0));
        }
    } else {
        // g with its factor for the gradient that is a sum over the rows, and without
        // for the other one: two elements at a time, as pieces 1,024 bytes from each
        // other
        auto store = [&](char* to, int pieces, float g0, float g1) {
            for (int n = 0; n < pieces; ++n) {
                *reinterpret_cast<uint32_t*>(to + n * 1024) = high_halves(__float_as_uint(g0), __float_as_uint(g1));
                g0 -= __uint_as_float(__float_as_uint(g0) & 0xffff0000u);
                g1 -= __uint_as_float(__float_as_uint(g1) & 0xffff0000u);
            }
        };
        for (int n = tid; n < kT * kS / 2; n += kThreads) {
            const int t = n / (kS / 2), s = n % (kS / 2) * 2;
            float g[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int64_t row = ROWS ? s0 + s + e : t, v = ROWS ? t : s0 + s + e;
                const float f = factors.f[ROWS ? s + e : t];
                g[e] = 0.0f;
                if (f != 0.0f && v < a.classes) {
                    const float p = __builtin_amdgcn_exp2f((at_z(t, s + e) - a.lse[k][row]) * kLog2e);
                    g[e] = a.label[k][row] == v ? p - 1.0f : p;
                }
                at_z(t, s + e) = ROWS ? g[e] : g[e] * f;
                if (ROWS) g[e] *= f * factors.lift[(s0 % 32 + s) / 32];
            }
            const int64_t at = s0 + s;
            store(work + a.at_g + (at / 32 * MT + t / 16) * a.pieces_g * 1024 + ((at % 32 / 8) * 16 + t % 16) * 16 + at % 8 * 2, a.pieces_g, g[0], g[1]);
        }
        if (ROWS && tid < kS) reinterpret_cast<float*>(work + a.at_f)[s0 + tid] = factors.f[tid];
        __syncthreads();
        constexpr int kKs = MT > 2 ? 2 : 1, kSide = kKs * 32;  // rows of the side in f g, with zeros
        for (int n = tid; n < kS * kSide / 2; n += kThreads) {
            const int s = n / (kSide / 2), t = n % (kSide / 2) * 2;
            const bool in = t < kT;
            const float lift = ROWS ? 1.0f : factors.lift[0];
            store(work + a.at_fg + ((s0 + s) / 16 * kKs + t / 32) * a.pieces_fg * 1024 + ((t % 32 / 8) * 16 + s % 16) * 16 + t % 8 * 2,
                  a.pieces_fg, in ? at_z(in ? t : 0, s) * lift : 0.0f, in ? at_z(in ? t + 1 : 0, s) * lift : 0.0f);
        }
        // dbias: sums over the rows
        if (!a.db[k]) return;
        if constexpr (ROWS) {
            if (tid < kT) {
                float sum = 0.0f;
                for (int s = 0; s < kS; ++s) sum += at_z(tid, s) * factors.f[s];
                reinterpret_cast<float*>(work + a.at_db)[static_cast<int64_t>(blockIdx.x) * kShort + tid] = sum;
            }
        } else if (tid < kS && s0 + tid < a.classes) {
            float sum = 0.0f;
            for (int r = 0; r < kT; ++r) sum += at_z(r, tid);
            store_any(a.db[k], s0 + tid, a.db_bf, sum * a.scale);
        }
    }
}

// STREAM, TB: what the stream's rows are, and whether the side is bfloat16.  MT,
// CT: the side's rows, and the stream's of a workgroup, in 16's.  PRE: few_side
// has laid out the side.  ROWS: the stream is the rows, the side the classes.
// Eight waves; W of them have the same rows of the stream, and the sum is cut
// among these, 64 columns at a time, and among a.cuts workgroups.
template <Kind STREAM, bool TB, int MT, int CT, int W, bool PRE, bool ROWS>
__global__ void __launch_bounds__(kLogitThreads) few_logit_kernel(const FewArgs a) {
    constexpr int kS = CT * 16 * (8 / W), kT = MT * 16;  // rows of the stream and the side
    constexpr int kPitch = kS + 4, PT = TB ? 1 : 3;
    __shared__ __attribute__((aligned(16))) float z[W * kT * kPitch];
    __shared__ Factors factors;
    const int k = blockIdx.y, tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const int64_t rows = a.rows[k];
    const int64_t n_s = ROWS ? rows : a.classes;
    const int n_t = static_cast<int>(ROWS ? a.classes : rows);
    const int part = wave % W, group = wave / W * (CT * 16);
    // with the other workgroups of the same rows
    const int parts = W * a.cuts, own_part = static_cast<int>(blockIdx.z) * W + part;
    const int64_t s0 = static_cast<int64_t>(blockIdx.x) * kS;
    if (s0 >= (n_s + 63) / 64 * 64) return;
    const int cols = a.cols;
    constexpr int se = STREAM == kF32 ? 4 : 2, te = TB ? 2 : 4;
    const uintptr_t stream = reinterpret_cast<uintptr_t>(ROWS ? a.x[k] : a.w[k]);
    const uintptr_t side = reinterpret_cast<uintptr_t>(ROWS ? a.w[k] : a.x[k]);
    const int64_t s_ld = (ROWS ? a.x_ld : cols) * se, t_ld = (ROWS ? cols : a.x_ld) * te;
    char* work = a.work + k * a.stride;
    // ---- the logits
    Sums<STREAM == kF32 ? 3 : 1, PT> acc[CT][MT] = {};
    {
        constexpr Kind kSide = TB ? kBf16 : kF32;
        uintptr_t sp[CT], tp[PRE ? 1 : MT];
#pragma unroll
        for (int i = 0; i < CT; ++i) sp[i] = stream + std::min<int64_t>(s0 + group + i * 16 + lane % 16, n_s - 1) * s_ld;
        if constexpr (PRE)
            tp[0] = reinterpret_cast<uintptr_t>(work + a.at_side) + lane * 16;
        else
#pragma unroll
            for (int j = 0; j < MT; ++j) tp[j] = side + std::min(j * 16 + lane % 16, n_t - 1) * t_ld;
        constexpr int kAhead = 2;
        struct Step {
            Eight<STREAM> s[CT];
            Eight<kSide> t[PRE ? 1 : MT];
            Pieces<PT> p[PRE ? MT : 1];
        } st[kAhead];
        const int own = lane / 16 * 8, full = cols / 32 * 32;
        auto fetch = [&](auto whole, Step& q, int c) {
            constexpr bool kWhole = decltype(whole)::value;
#pragma unroll
            for (int i = 0; i < CT; ++i) q.s[i] = load_eight<STREAM, kWhole>(sp[i], c + own, cols);
            if constexpr (PRE) {
#pragma unroll
                for (int j = 0; j < MT; ++j)
#pragma unroll
                    for (int p = 0; p < PT; ++p) q.p[j].p[p] = gld<u32x4>(tp[0] + ((c / 32 * MT + j) * PT + p) * 1024);
            } else {
#pragma unroll
                for (int j = 0; j < MT; ++j) q.t[j] = load_eight<kSide, kWhole>(tp[j], c + own, cols);
            }
        };
        auto step = [&](auto whole, const Step& q) {
            constexpr bool kWhole = decltype(whole)::value;
            Pieces<STREAM == kF32 ? 3 : 1> ps[CT];
#pragma unroll
            for (int i = 0; i < CT; ++i) ps[i] = pieces<STREAM, kWhole>(q.s[i], sp[i]);
#pragma unroll
            for (int j = 0; j < MT; ++j) {
                const Pieces<PT> pt = PRE ? q.p[PRE ? j : 0] : pieces<kSide, kWhole>(q.t[PRE ? 0 : j], tp[PRE ? 0 : j]);
#pragma unroll
                for (int i = 0; i < CT; ++i) acc[i][j].add(ps[i], pt);
            }
        };
        // The wave's step n: its 64 columns of every 64 `parts`, 32 at a time.  The
        // workgroups begin at different ones, or the rows' equal distances would
        // have all of them at the same channels of the memory at a time.
        auto column = [&](int n) { return n / 2 * (64 * parts) + n % 2 * 32 + own_part * 64; };
        const int steps = full / (64 * parts) * 2 + std::clamp((full % (64 * parts) - own_part * 64) / 32, 0, 2);
        // (past the last step it is loaded again: were the loads left out, the
        // counts of loads under way would differ, and all would be waited for)
        int ahead = steps > 0 ? static_cast<int>(blockIdx.x * kTurn % steps) : 0, asked = 0;
        auto next = [&](Step& to) {
            fetch(std::true_type{}, to, column(ahead));
            loads_first();
            if (asked + 1 < steps) {
                ++asked;
                if (++ahead == steps) ahead = 0;
            }
        };
        if (steps > 0) {
#pragma unroll
            for (int q = 0; q < kAhead - 1; ++q) next(st[q]);
            for (int n = 0;;) {
                bool more = true;
#pragma unroll
                for (int q = 0; q < kAhead; ++q) {
                    next(st[(q + kAhead - 1) % kAhead]);
                    step(std::true_type{}, st[q]);
                    if (++n == steps) {
                        more = false;
                        break;
                    }
                }
                if (!more) break;
            }
        }
        if (column(steps) == full && full < cols) {
            fetch(std::false_type{}, st[0], full);
            step(std::false_type{}, st[0]);
        }
    }
#pragma unroll
    for (int i = 0; i < CT; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j)
            *reinterpret_cast<f32x4*>(z + (part * kT + j * 16 + lane % 16) * kPitch + group + i * 16 + lane / 16 * 4) = acc[i][j].sum();
    if (a.cuts == 1) few_factors<kS, MT, ROWS>(a, k, s0, factors);
    __syncthreads();
    // the sum of the waves' parts
    auto sum = [&](int t, int s) {
        float q = 0.0f;
#pragma unroll
        for (int w = 0; w < W; w += 2) q += z[(w * kT + t) * kPitch + s] + z[(w * kT + kT + t) * kPitch + s];
        return q;
    };
    if (a.cuts > 1) {
        float* out = reinterpret_cast<float*>(work + a.at_z) + (static_cast<int64_t>(blockIdx.z) * a.tiles + blockIdx.x) * (kT * kS);
        for (int n = tid; n < kT * kS; n += kLogitThreads) out[n] = sum(n / kS, n % kS);
        return;
    }
    for (int n = tid; n < kT * kS; n += kLogitThreads) {
        const int t = n / kS, s = n % kS;
        z[t * kPitch + s] = sum(t, s) + few_bias(a, k, ROWS ? t : s0 + s);
    }
    __syncthreads();
    few_results<kS, MT, ROWS>(a, k, s0, z, factors);
}

// The same from the sums of the workgroups that shared the columns.
template <int kS, int MT, bool ROWS>
__global__ void __launch_bounds__(kLogitThreads) few_rest_kernel(const FewArgs a) {
    constexpr int kT = MT * 16, kPitch = kS + 4;
    __shared__ __attribute__((aligned(16))) float z[kT * kPitch];
    __shared__ Factors factors;
    const int k = blockIdx.y;
    const int64_t n_s = ROWS ? a.rows[k] : a.classes, s0 = static_cast<int64_t>(blockIdx.x) * kS;
    if (s0 >= (n_s + 63) / 64 * 64) return;
    few_factors<kS, MT, ROWS>(a, k, s0, factors);
    const float* sums = reinterpret_cast<const float*>(a.work + k * a.stride + a.at_z) + static_cast<int64_t>(blockIdx.x) * (kT * kS);
    for (int n = threadIdx.x; n < kT * kS; n += kLogitThreads) {
        const int t = n / kS, s = n % kS;
        float q = few_bias(a, k, ROWS ? t : s0 + s);
#pragma unroll 4
        for (int c = 0; c < a.cuts; ++c) q += sums[static_cast<int64_t>(c) * a.tiles * (kT * kS) + n];
        z[t * kPitch + s] = q;
    }
    __syncthreads();
    few_results<kS, MT, ROWS>(a, k, s0, z, factors);
}

// Joins the workgroups' pairs of a row.
__global__ void __launch_bounds__(1024) few_join_kernel(const FewArgs a) {
    __shared__ float2 lds[16];
    const int k = blockIdx.y;
    const int64_t row = blockIdx.x;
    if (row >= a.rows[k]) return;
    const char* work = a.work + k * a.stride;
    const float2* pairs = reinterpret_cast<const float2*>(work + a.at_pairs) + row * a.tiles;
    float top = -INFINITY, sum = 0.0f;
    for (int t = threadIdx.x; t < a.tiles; t += blockDim.x) join(top, sum, pairs[t].x, pairs[t].y);
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) join(top, sum, __shfl_xor(top, m, 64), __shfl_xor(sum, m, 64));
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = make_float2(top, sum);
    __syncthreads();
    if (threadIdx.x) return;
    for (int w = 1; w < static_cast<int>(blockDim.x / 64); ++w) join(top, sum, lds[w].x, lds[w].y);
    const float lse = top + log2f(sum) * kLn2;
    a.lse[k][row] = lse;
    const int64_t label = a.label[k][row];
    a.loss[k][row] = label >= 0 && label < a.classes ? lse - reinterpret_cast<const float*>(work + a.at_own)[row] : 0.0f;
}

// ------------------------------------------------------- the sum over the stream

struct SumArgs {
    const void* stream[kWorkers];
    const int64_t* label[kWorkers];
    const float* dloss[kWorkers];
    void* out[kWorkers];  // the side's gradient
    void* db[kWorkers];
    int64_t rows[kWorkers];
    char* work;
    int64_t stride, at_g, at_f, at_sums, sums_stride, at_db;
    int64_t ld, out_ld;  // elements
    int64_t classes;
    int32_t cols, cols_p, splits, out_bf, db_bf, has_dloss, groups, is_rows;
    float scale;
};

// Four columns of the side's gradient.
__device__ __forceinline__ void side_gradient(const SumArgs& a, int k, int t, int c, f32x4 v) {
    const float f = a.is_rows ? 1.0f : factor_of(a.label[k], a.has_dloss ? a.dloss[k] : nullptr, t, a.classes);
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (c + e < a.cols) store_any(a.out[k], t * a.out_ld + c + e, a.out_bf, f == 0.0f ? 0.0f : v[e] * (f * a.scale));
}

// A workgroup takes a block of columns and a part of the stream's rows, 32 at a
// time a wave.
template <bool SB, int MT, bool ROWS, int PG>
__global__ void __launch_bounds__(256) few_sum_kernel(const SumArgs a) {
    using Col = Columns<SB, SB && MT < 4 ? 8 : 4>;  // (with more the sums would not fit the registers)
    constexpr int kT = MT * 16, kB = Col::kBlock, kPS = SB ? 1 : 3;
    __shared__ __attribute__((aligned(16))) float lds[2][kT][kB + 4];
    const int k = blockIdx.z, tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const int64_t rows = a.rows[k], n_s = ROWS ? rows : a.classes;
    const int n_t = static_cast<int>(ROWS ? a.classes : rows);
    const int cols = a.cols, c0 = blockIdx.x * kB, c = c0 + lane % 16 * Col::kTiles;
    const int64_t steps = (n_s + 31) / 32;  // of which this workgroup has
    const int64_t from = steps * blockIdx.y / a.splits, to = steps * (blockIdx.y + 1) / a.splits;
    char* work = a.work + k * a.stride;
    const uintptr_t stream = reinterpret_cast<uintptr_t>(a.stream[k]);
    const int64_t ld = a.ld * (SB ? 2 : 4);
    const char* g0 = work + a.at_g + lane * 16;
    const float* f0 = reinterpret_cast<const float*>(work + a.at_f);
    struct Step {
        Col x;
        Pieces<PG> g[MT];
        uint32_t there;
        float top;  // of the lane's rows' factors
    } st[2];
    const bool whole = c0 + kB <= cols;
    auto fetch = [&](Step& q, int64_t step) {
        const int64_t s = step * 32 + lane / 16 * 8;
        auto rows_of = [&](auto whole) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                q.x.v[j] = Col::template load<decltype(whole)::value>(stream + std::min(s + j, n_s - 1) * ld, c, cols);
        };
        if (whole)
            rows_of(std::true_type{});
        else
            rows_of(std::false_type{});
        if (ROWS) {
            // rows that are left out (g is zero there, and the rows may hold anything)
            q.there = 0;
            q.top = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float f = f0[std::min(s + j, n_s - 1)];
                q.there |= f != 0.0f ? 1u << j : 0u;
                q.top = fmaxf(q.top, fabsf(f));
            }
        }
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int p = 0; p < PG; ++p)
                q.g[m].p[p] = *reinterpret_cast<const u32x4*>(g0 + ((step * MT + m) * PG + p) * 1024);
        loads_first();
    };
    f32x4 acc[Col::kTiles][MT] = {};
    auto times = [&](f32x4 (&v)[Col::kTiles][MT], float by) {
#pragma unroll
        for (int t = 0; t < Col::kTiles; ++t)
#pragma unroll
            for (int m = 0; m < MT; ++m) v[t][m] *= by;
    };
    auto add = [&](const Step& q, f32x4 (&v)[Col::kTiles][MT]) {
#pragma unroll
        for (int t = 0; t < Col::kTiles; ++t) {
            const Pieces<kPS> x = q.x.template get<kPS>(t);
#pragma unroll
            for (int m = 0; m < MT; ++m) v[t][m] = multiply(q.g[m], x, v[t][m]);
        }
    };
    // What the sums are times kLift, or kLiftFactor: until a larger value, or a
    // larger factor, comes.
    bool small = !SB, small_factors = ROWS && a.has_dloss;
    auto use = [&](Step& q) {
        if (ROWS) q.x.keep(q.there);
        if constexpr (!SB)
            if (small) {
                if (in_any_lane(q.x.largest() >= kSmall)) {
                    small = false;
                    times(acc, 1.0f / kLift);
                } else {
                    q.x.lift();
                }
            }
        if constexpr (ROWS)
            if (a.has_dloss && in_any_lane(q.there != 0)) {
                const bool lifted = !in_any_lane(q.top >= kSmallFactor);
                if (lifted && !small_factors) {
                    f32x4 own[Col::kTiles][MT] = {};
                    add(q, own);
                    times(own, 1.0f / kLiftFactor);
#pragma unroll
                    for (int t = 0; t < Col::kTiles; ++t)
#pragma unroll
                        for (int m = 0; m < MT; ++m) acc[t][m] += own[t][m];
                    return;
                }
                if (small_factors && !lifted) {
                    small_factors = false;
                    times(acc, 1.0f / kLiftFactor);
                }
            }
        add(q, acc);
    };
    // (past the last step it is loaded again: were the loads left out, the counts
    // of loads under way would differ, and all would be waited for)
    const int64_t last = to - 1 - (to - 1 - from - wave) % 4;
    int64_t at = from + wave;
    if (at < to) {
        fetch(st[0], at);
        for (;;) {
            fetch(st[1], std::min(at + 4, last));
            use(st[0]);
            if (at == last) break;
            fetch(st[0], std::min(at + 8, last));
            use(st[1]);
            if (at + 4 == last) break;
            at += 8;
        }
    }
    if (small) times(acc, 1.0f / kLift);
    if (small_factors) times(acc, 1.0f / kLiftFactor);
    // the four waves' sums, two at a time
    auto place = [&](int half, int m, int e) -> float* { return &lds[half][m * 16 + lane / 16 * 4 + e][lane % 16 * Col::kTiles]; };
#pragma unroll
    for (int turn = 0; turn < 2; ++turn) {
        if (wave / 2 == 1 - turn)
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float* p = place(wave % 2, m, e);
#pragma unroll
                    for (int t = 0; t < Col::kTiles; ++t) p[t] = turn ? p[t] + acc[t][m][e] : acc[t][m][e];
                }
        __syncthreads();
    }
    for (int n = tid; n < kT * kB / 4; n += 256) {
        const int t = n / (kB / 4), q = n % (kB / 4) * 4;
        if (t >= n_t) break;
        const f32x4 v = *reinterpret_cast<const f32x4*>(&lds[0][t][q]) + *reinterpret_cast<const f32x4*>(&lds[1][t][q]);
        if (a.splits > 1)
            *reinterpret_cast<f32x4*>(work + a.at_sums + blockIdx.y * a.sums_stride + (static_cast<int64_t>(t) * a.cols_p + c0 + q) * 4) = v;
        else
            side_gradient(a, k, t, c0 + q, v);
    }
}

// The side's gradient from the workgroups' sums; dbias where the side is the
// classes.
__global__ void __launch_bounds__(256) few_finish_kernel(const SumArgs a) {
    const int k = blockIdx.z, t = blockIdx.y;
    const int64_t rows = a.rows[k];
    const int n_t = static_cast<int>(a.is_rows ? a.classes : rows);
    if (t >= n_t) return;
    const char* work = a.work + k * a.stride;
    if (blockIdx.x == gridDim.x - 1) {  // the last one has no columns
        if (!a.is_rows || !a.db[k]) return;
        __shared__ float lds[256];
        float s = 0.0f;
        const int64_t groups = (rows + a.groups - 1) / a.groups;
        for (int64_t g = threadIdx.x; g < groups; g += 256) s += reinterpret_cast<const float*>(work + a.at_db)[g * kShort + t];
        lds[threadIdx.x] = s;
        __syncthreads();
        for (int m = 128; m > 0; m >>= 1) {
            if (threadIdx.x < m) lds[threadIdx.x] += lds[threadIdx.x + m];
            __syncthreads();
        }
        if (threadIdx.x == 0) store_any(a.db[k], t, a.db_bf, lds[0] * a.scale);
        return;
    }
    if (a.splits == 1) return;
    // 64 lanes of four columns; the waves take the parts in turn
    __shared__ f32x4 sums[4][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, c = (blockIdx.x * 64 + lane) * 4;
    const char* from = work + a.at_sums + (static_cast<int64_t>(t) * a.cols_p + c) * 4;
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (c < a.cols)
#pragma unroll 4
        for (int s = wave; s < a.splits; s += 4) v += *reinterpret_cast<const f32x4*>(from + s * a.sums_stride);
    sums[wave][lane] = v;
    __syncthreads();
    if (wave || c >= a.cols) return;
    side_gradient(a, k, t, c, (v + sums[1][lane]) + (sums[2][lane] + sums[3][lane]));
}

// ----------------------------------------------------------- the stream's gradient

struct OuterArgs {
    const void* side[kWorkers];
    const int64_t* label[kWorkers];
    const float* dloss[kWorkers];
    void* out[kWorkers];
    int64_t rows[kWorkers];
    char* work;
    int64_t stride, at_fg, at_f;
    int64_t ld, out_ld;  // elements
    int64_t classes;
    int32_t cols, out_bf, has_dloss, chunk;  // rows of the stream of a workgroup
    float scale;
};

// A wave holds its block of columns of the side as pieces, and takes its rows of
// the stream 16 at a time.  Its stores pass the caches by, which hold the stream
// (16 rows of 4,096 over 32,000 classes in bfloat16, the whole gradient: 194 us,
// so 149; 3 x 13 rows of 4,224 over 5,426 in float 213 and 168).
template <bool TB, int KS, bool ROWS, int PG>
__global__ void __launch_bounds__(256) few_outer_kernel(const OuterArgs a) {
    using Col = Columns<TB>;
    constexpr int kPT = TB ? 1 : 3;
    const int k = blockIdx.z, lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int64_t rows = a.rows[k], n_s = ROWS ? rows : a.classes;
    const int n_t = static_cast<int>(ROWS ? a.classes : rows);
    const int cols = a.cols, c0 = (blockIdx.x * 4 + wave) * Col::kBlock;
    if (c0 >= cols) return;
    const int c = c0 + lane % 16 * Col::kTiles;
    const uintptr_t side = reinterpret_cast<uintptr_t>(a.side[k]);
    const int64_t t_ld = a.ld * (TB ? 2 : 4);
    Pieces<kPT> x[KS][Col::kTiles];
    Col block[KS];
    float top = 0.0f;  // of the factors
#pragma unroll
    for (int h = 0; h < KS; ++h) {
        Col& v = block[h];
        auto fetch = [&](auto whole) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                v.v[j] = Col::template load<decltype(whole)::value>(side + std::min(h * 32 + lane / 16 * 8 + j, n_t - 1) * t_ld, c, cols);
        };
        if (c0 + Col::kBlock <= cols)
            fetch(std::true_type{});
        else
            fetch(std::false_type{});
        if constexpr (!ROWS) {
            uint32_t there = 0;  // the rows that are not left out
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int r = h * 32 + lane / 16 * 8 + j;
                const float f = r < n_t ? factor_of(a.label[k], a.has_dloss ? a.dloss[k] : nullptr, r, a.classes) : 0.0f;
                if (f != 0.0f) there |= 1u << j;
                top = fmaxf(top, fabsf(f));
            }
            v.keep(there);
        }
    }
    // what the results are times
    bool small = false;
    if constexpr (!TB) {
        float largest = 0.0f;
#pragma unroll
        for (int h = 0; h < KS; ++h) largest = fmaxf(largest, block[h].largest());
        small = !in_any_lane(largest >= kSmall);
        if (small)
#pragma unroll
            for (int h = 0; h < KS; ++h) block[h].lift();
    }
    const bool small_factors = !ROWS && a.has_dloss && !in_any_lane(top >= kSmallFactor);
#pragma unroll
    for (int h = 0; h < KS; ++h)
#pragma unroll
        for (int q = 0; q < Col::kTiles; ++q) x[h][q] = block[h].template get<kPT>(q);
    const char* fg = a.work + k * a.stride + a.at_fg + lane * 16;
    const int64_t first = static_cast<int64_t>(blockIdx.y) * a.chunk, end = std::min<int64_t>(first + a.chunk, n_s);
    const char* f0 = a.work + k * a.stride + a.at_f + lane / 16 * 16;
    struct Operands {
        Pieces<PG> b[KS];
        f32x4 f;  // of the lane's rows of a stream of rows
    } now, next;
    auto fetch = [&](Operands& f, int64_t s) {
#pragma unroll
        for (int h = 0; h < KS; ++h)
#pragma unroll
            for (int p = 0; p < PG; ++p) f.b[h].p[p] = *reinterpret_cast<const u32x4*>(fg + ((s / 16 * KS + h) * PG + p) * 1024);
        if (ROWS) f.f = *reinterpret_cast<const f32x4*>(f0 + s * 4);
        loads_first();
    };
    if (first >= end) return;
    const int64_t last = first + (end - 1 - first) / 16 * 16;
    fetch(now, first);
    for (int64_t s0 = first; s0 < end; s0 += 16) {
        fetch(next, std::min(s0 + 16, last));
        f32x4 d[Col::kTiles] = {};
#pragma unroll
        for (int q = 0; q < Col::kTiles; ++q)
#pragma unroll
            for (int h = 0; h < KS; ++h) d[q] = multiply(now.b[h], x[h][q], d[q]);
        if (small || small_factors)
#pragma unroll
            for (int q = 0; q < Col::kTiles; ++q) d[q] = d[q] * (small ? 1.0f / kLift : 1.0f) * (small_factors ? 1.0f / kLiftFactor : 1.0f);
        const f32x4 f = now.f;
        now = next;
        // lane: rows lane / 16 * 4 + e of the stream, its columns of the side
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t s = s0 + lane / 16 * 4 + e;
            if (s >= n_s) continue;
            const uintptr_t out = reinterpret_cast<uintptr_t>(a.out[k]) + s * a.out_ld * (a.out_bf ? 2 : 4);
            const int at = c;
            float v[8] = {};
#pragma unroll
            for (int q = 0; q < Col::kTiles; ++q) v[q] = !ROWS ? d[q][e] * a.scale : f[e] == 0.0f ? 0.0f : d[q][e] * (f[e] * a.scale);
            if (a.out_bf) {
                if constexpr (TB) {
                    store_vec<__bf16, true, true>(out, at / 8, cols, v);
                } else if (at + 4 <= cols) {
                    const u32x4 h = Lane<__bf16>::narrow(v);
                    gst_u_nt(out + at * 2, u32x2{h[0], h[1]});
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (at + q < cols) Lane<__bf16>::put(out + (at + q) * 2, v[q]);
                }
            } else {
#pragma unroll
                for (int h = 0; h < Col::kTiles / 4; ++h) store_vec<float, true, true>(out, at / 4 + h, cols, v + 4 * h);
            }
        }
    }
}

// --------------------------------------------------------------------- dispatch

// What a call takes, from its sizes and types alone.
struct FewPlan {
    bool rows_stream;  // the stream is the rows
    bool pre;          // the side is laid out for the logits
    int mt, ct, waves, groups, batch, tiles, cuts, splits, cols_p, blocks, pieces, pieces_fg;
    int64_t n_s, stride, at_pairs, at_own, at_side, at_g, at_fg, at_f, at_db, at_z, at_sums, sums_stride;
};

FewPlan few_plan(int K, const int64_t* rows, int64_t cols, int64_t classes, int dtype, int w_dtype, bool backward, int dw_dtype) {
    FewPlan p{};
    int64_t most = 0;
    int with = 0;
    for (int k = 0; k < K; ++k) {
        most = std::max(most, rows[k]);
        with += rows[k] > 0;
    }
    p.rows_stream = classes < most;
    const int64_t n_t = p.rows_stream ? classes : most;
    p.n_s = p.rows_stream ? most : classes;
    p.mt = n_t <= 16 ? 1 : n_t <= 32 ? 2 : 4;
    p.batch = std::max(1, std::min(with, kWorkers));
    const bool side_bf = (p.rows_stream ? w_dtype : dtype) == TC_BF16, stream_bf = (p.rows_stream ? dtype : w_dtype) == TC_BF16;
    // A side of more than 32 rows (or 16, if the stream is long) is laid out: it is
    // read by every workgroup.  (4 x 64 rows of 4,096 over 1,000 classes, the
    // logits: 50 us as it lies, 32 + 5 laid out; 8 x 32 rows of 2,048, 20.5 and
    // 21.7 + 5.)  Smaller calls save the launch.
    const int64_t size = p.n_s * cols * p.batch;
    // Of short rows (up to 256 columns) two waves cut the sum, not eight.
    p.waves = cols <= 256 ? 2 : 8;
    p.pre = p.waves == 8 && ((p.mt == 4 && size > (1 << 21)) || (p.mt == 2 && size > (1 << 26)));
    // Rows of the stream of a workgroup: 64 or 32 where that leaves workgroups
    // enough (8 rows of 4,096 over 131,072 classes in bfloat16: 280 us with 16, 245,
    // 224; in float, whose sums take three times the registers, 5 over 32,000 101 us
    // with 32 and 120 with 64, of 1,024 38 and 31)
    p.ct = p.mt == 1 && (stream_bf || cols < 2048) && (p.n_s + 63) / 64 * p.batch >= 384 ? 4 : (p.pre || p.mt < 4) && (p.n_s + 31) / 32 * p.batch >= (p.pre ? 512 : 256) ? 2 : 1;
    if (p.waves == 2) p.ct = 1;
    // 32 also where the columns can be cut (below) and the side is three pieces,
    // which every workgroup reads from L2 (60 rows of 8,192 over 4,000 classes in
    // float: 55 us with 16, 48)
    if (p.pre && !side_bf && (p.n_s + 31) / 32 * p.batch * std::min<int64_t>(8, cols / 1024) >= 256) p.ct = 2;
    const int64_t padded = (p.n_s + 63) / 64 * 64;
    p.groups = p.ct * 16 * (8 / p.waves);
    p.tiles = static_cast<int>(padded / p.groups);
    // Where workgroups are too few for the chip, several share the columns, 1,024
    // and more each, and another kernel adds their sums up (one worker: 32 rows of
    // 4,096 over 1,000 classes in float, forward, 29 us, 16.5 with four; 60 of
    // 8,192 52 and 28).  Up to 16 rows are small calls, which two do not pay for
    // (2 x 1 row of 4,096 16 and 19 us).
    p.cuts = static_cast<int>(std::min<int64_t>({256 / (static_cast<int64_t>(p.tiles) * p.batch), cols / 1024, 8}));
    if (p.cuts < (p.mt == 1 ? 3 : 2)) p.cuts = 1;
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    if (p.cuts > 1) p.at_z = take(static_cast<int64_t>(p.cuts) * p.tiles * (p.mt * 16) * p.groups * 4);
    if (p.pre) p.at_side = take((cols + 31) / 32 * p.mt * (side_bf ? 1 : 3) * 1024);
    if (!backward) {
        if (!p.rows_stream) {
            p.at_pairs = take(n_t * p.tiles * 8);
            p.at_own = take(n_t * 4);
        }
    } else {
        p.pieces = (p.rows_stream ? dw_dtype : dtype) == TC_BF16 ? 2 : 3;
        p.pieces_fg = (p.rows_stream ? dtype : dw_dtype) == TC_BF16 ? 2 : 3;
        p.at_g = take(padded / 32 * p.mt * p.pieces * 1024);
        p.at_fg = take(padded / 16 * (p.mt > 2 ? 2 : 1) * p.pieces_fg * 1024);
        const int block = stream_bf && p.mt < 4 ? 128 : 64;
        p.blocks = static_cast<int>((cols + block - 1) / block);
        p.cols_p = p.blocks * block;
        // workgroups enough to fill the chip, of at least 128 rows of the stream
        p.splits = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(256 / (p.blocks * p.batch), (p.n_s + 127) / 128)));
        p.sums_stride = n_t * p.cols_p * 4;
        if (p.splits > 1) p.at_sums = take(p.splits * p.sums_stride);
        if (p.rows_stream) {
            p.at_f = take(padded * 4);
            p.at_db = take(static_cast<int64_t>(p.tiles) * kShort * 4);
        }
    }
    p.stride = std::max<int64_t>(at, 256);
    return p;
}

template <Kind STREAM, bool TB, int MT, bool ROWS>
void run_logit(const FewArgs& a, const FewPlan& p, dim3 grid, hipStream_t s) {
    if (p.waves == 2) {
        few_logit_kernel<STREAM, TB, MT, 1, 2, false, ROWS><<<grid, 512, 0, s>>>(a);
    } else if (MT > 1 && p.pre) {
        if (p.ct == 1)
            few_logit_kernel<STREAM, TB, MT, 1, 8, MT != 1, ROWS><<<grid, 512, 0, s>>>(a);
        else
            few_logit_kernel<STREAM, TB, MT, 2, 8, MT != 1, ROWS><<<grid, 512, 0, s>>>(a);
    } else if (MT == 4 || p.ct == 1) {
        few_logit_kernel<STREAM, TB, MT, 1, 8, false, ROWS><<<grid, 512, 0, s>>>(a);
    } else if (MT == 1 && p.ct == 4) {
        few_logit_kernel<STREAM, TB, MT, MT == 1 ? 4 : 1, 8, false, ROWS><<<grid, 512, 0, s>>>(a);
    } else {
        few_logit_kernel<STREAM, TB, MT, MT < 4 ? 2 : 1, 8, false, ROWS><<<grid, 512, 0, s>>>(a);
    }
}
template <Kind STREAM, bool TB, bool ROWS>
void run_logit(const FewArgs& a, const FewPlan& p, dim3 grid, hipStream_t s) {
    if (p.mt == 1)
        run_logit<STREAM, TB, 1, ROWS>(a, p, grid, s);
    else if (p.mt == 2)
        run_logit<STREAM, TB, 2, ROWS>(a, p, grid, s);
    else
        run_logit<STREAM, TB, 4, ROWS>(a, p, grid, s);
}
template <int MT, bool ROWS>
void run_rest(const FewArgs& a, const FewPlan& p, dim3 grid, hipStream_t s) {
    if (p.ct == 1)
        few_rest_kernel<16, MT, ROWS><<<grid, kLogitThreads, 0, s>>>(a);
    else if (MT > 1 || p.ct == 2)
        few_rest_kernel<32, MT, ROWS><<<grid, kLogitThreads, 0, s>>>(a);
    else
        few_rest_kernel<64, MT, ROWS><<<grid, kLogitThreads, 0, s>>>(a);
}
template <bool TB, bool ROWS>
hipError_t run_logit(const FewArgs& a, const FewPlan& p, Kind stream, int n, hipStream_t s) {
    if (p.pre) {
        const int units = (a.cols + 31) / 32 * p.mt;
        few_side_kernel<TB, ROWS><<<dim3((units + 3) / 4, n), 256, 0, s>>>(a, p.mt);
        if (hipError_t e = hipGetLastError()) return e;
    }
    const dim3 grid(p.tiles, n, p.cuts);
    if (stream == kF32)
        run_logit<kF32, TB, ROWS>(a, p, grid, s);
    else if (stream == kBf16)
        run_logit<kBf16, TB, ROWS>(a, p, grid, s);
    else
        run_logit<kOdd, TB, ROWS>(a, p, grid, s);
    if (p.cuts == 1) return hipGetLastError();
    if (hipError_t e = hipGetLastError()) return e;
    const dim3 rest(p.tiles, n);
    if (p.mt == 1)
        run_rest<1, ROWS>(a, p, rest, s);
    else if (p.mt == 2)
        run_rest<2, ROWS>(a, p, rest, s);
    else
        run_rest<4, ROWS>(a, p, rest, s);
    return hipGetLastError();
}
template <bool TB, bool ROWS>
void run_outer(const OuterArgs& a, int mt, int pieces, dim3 grid, hipStream_t s) {
    if (mt > 2)
        pieces == 3 ? few_outer_kernel<TB, 2, ROWS, 3><<<grid, 256, 0, s>>>(a) : few_outer_kernel<TB, 2, ROWS, 2><<<grid, 256, 0, s>>>(a);
    else
        pieces == 3 ? few_outer_kernel<TB, 1, ROWS, 3><<<grid, 256, 0, s>>>(a) : few_outer_kernel<TB, 1, ROWS, 2><<<grid, 256, 0, s>>>(a);
}
template <bool SB, bool ROWS, int PG>
void run_sum(const SumArgs& a, int mt, dim3 grid, hipStream_t s) {
    if (mt == 1)
        few_sum_kernel<SB, 1, ROWS, PG><<<grid, 256, 0, s>>>(a);
    else if (mt == 2)
        few_sum_kernel<SB, 2, ROWS, PG><<<grid, 256, 0, s>>>(a);
    else
        few_sum_kernel<SB, 4, ROWS, PG><<<grid, 256, 0, s>>>(a);
}

}  // namespace

bool few_fits(int K, const int64_t* rows, int64_t classes) {
    int64_t most = 0;
    for (int k = 0; k < K; ++k) most = std::max(most, rows[k]);
    return most <= kShort || classes <= kShort;
}

int64_t few_workspace(int K, const int64_t* rows, int64_t cols, int64_t classes, int dtype, int w_dtype, bool backward, int dw_dtype) {
    const FewPlan p = few_plan(K, rows, cols, classes, dtype, w_dtype, backward, dw_dtype);
    return p.batch * p.stride;
}

hipError_t launch_few(const LossCall& c, const int* list, int count, hipStream_t s) {
    const FewPlan p = few_plan(c.K, c.rows, c.cols, c.classes, c.dtype, c.w_dtype, c.backward, c.dw_dtype);
    const bool x_bf = c.dtype == TC_BF16, w_bf = c.w_dtype == TC_BF16, dw_bf = c.dw_dtype == TC_BF16;
    const bool sb = p.rows_stream ? x_bf : w_bf, tb = p.rows_stream ? w_bf : x_bf;
    const int32_t cols = static_cast<int32_t>(c.cols), has_dloss = c.dloss != nullptr;
    for (int k0 = 0; k0 < count; k0 += p.batch) {
        const int n = std::min(p.batch, count - k0);
        FewArgs a{};
        SumArgs m{};
        OuterArgs o{};
        for (int i = 0; i < n; ++i) {
            const int k = list[k0 + i];
            a.x[i] = c.x[k];
            a.w[i] = c.weight[k];
            a.bias[i] = c.bias ? c.bias[k] : nullptr;
            a.label[i] = m.label[i] = o.label[i] = c.label[k];
            a.rows[i] = m.rows[i] = o.rows[i] = c.rows[k];
            if (c.backward) {
                a.lse[i] = const_cast<float*>(c.lse_in[k]);
                a.dloss[i] = m.dloss[i] = o.dloss[i] = c.dloss ? c.dloss[k] : nullptr;
                a.db[i] = m.db[i] = c.dbias ? c.dbias[k] : nullptr;
                o.side[i] = p.rows_stream ? c.weight[k] : c.x[k];
                o.out[i] = p.rows_stream ? c.dx[k] : c.dweight[k];
                m.stream[i] = p.rows_stream ? c.x[k] : c.weight[k];
                m.out[i] = p.rows_stream ? c.dweight[k] : c.dx[k];
            } else {
                a.lse[i] = c.lse[k];
                a.loss[i] = c.loss[k];
            }
        }
        a.work = m.work = o.work = static_cast<char*>(c.workspace);
        a.stride = m.stride = o.stride = p.stride;
        a.at_pairs = p.at_pairs;
        a.at_own = p.at_own;
        a.at_side = p.at_side;
        a.at_g = m.at_g = p.at_g;
        a.at_fg = o.at_fg = p.at_fg;
        a.at_f = m.at_f = o.at_f = p.at_f;
        a.at_db = m.at_db = p.at_db;
        a.x_ld = c.x_ld;
        a.classes = m.classes = o.classes = c.classes;
        a.cols = m.cols = o.cols = cols;
        a.tiles = p.tiles;
        a.cuts = p.cuts;
        a.at_z = p.at_z;
        a.w_bf = w_bf;
        a.db_bf = m.db_bf = dw_bf;
        a.has_dloss = m.has_dloss = o.has_dloss = has_dloss;
        a.pieces_g = p.pieces;
        a.pieces_fg = p.pieces_fg;
        a.scale = m.scale = o.scale = c.scale;
        a.backward = c.backward;
        // rows of the stream that begin between words
        bool odd = sb && p.n_s > 1 && (p.rows_stream ? c.x_ld : c.cols) % 2;
        for (int i = 0; sb && i < n; ++i) odd = odd || reinterpret_cast<uintptr_t>(p.rows_stream ? a.x[i] : a.w[i]) % 4;
        const Kind stream = !sb ? kF32 : odd ? kOdd : kBf16;
        hipError_t e = p.rows_stream ? (tb ? run_logit<true, true>(a, p, stream, n, s) : run_logit<false, true>(a, p, stream, n, s))
                                     : (tb ? run_logit<true, false>(a, p, stream, n, s) : run_logit<false, false>(a, p, stream, n, s));
        if (e != hipSuccess) return e;
        if (!c.backward) {
            if (!p.rows_stream) few_join_kernel<<<dim3(static_cast<uint32_t>(p.mt * 16), n), p.tiles > 512 ? 1024 : 256, 0, s>>>(a);
            if (hipError_t e = hipGetLastError()) return e;
            continue;
        }
        m.at_sums = p.at_sums;
        m.sums_stride = p.sums_stride;
        m.ld = p.rows_stream ? c.x_ld : c.cols;
        m.out_ld = p.rows_stream ? c.cols : c.dx_ld;
        m.cols_p = p.cols_p;
        m.splits = p.splits;
        m.out_bf = p.rows_stream ? dw_bf : x_bf;
        m.groups = p.groups;
        m.is_rows = p.rows_stream;
        auto sum = [&] {
            const dim3 grid(p.blocks, p.splits, n);
            const bool three = p.pieces == 3;
            if (p.rows_stream)
                sb ? (three ? run_sum<true, true, 3>(m, p.mt, grid, s) : run_sum<true, true, 2>(m, p.mt, grid, s))
                   : (three ? run_sum<false, true, 3>(m, p.mt, grid, s) : run_sum<false, true, 2>(m, p.mt, grid, s));
            else
                sb ? (three ? run_sum<true, false, 3>(m, p.mt, grid, s) : run_sum<true, false, 2>(m, p.mt, grid, s))
                   : (three ? run_sum<false, false, 3>(m, p.mt, grid, s) : run_sum<false, false, 2>(m, p.mt, grid, s));
            return hipGetLastError();
        };
        o.ld = p.rows_stream ? c.cols : c.x_ld;
        o.out_ld = p.rows_stream ? c.dx_ld : c.cols;
        o.out_bf = p.rows_stream ? x_bf : dw_bf;
        const int64_t across = (c.cols + (tb ? 512 : 256) - 1) / (tb ? 512 : 256);
        // rows of a workgroup: 256, or as many as leave 256 workgroups (4 x 64 rows of
        // 4,096 over 1,000 classes, all: 84 us, with 1,024 89, 2,048 93)
        int64_t chunk = p.n_s * across * n / 256 / 16 * 16;
        o.chunk = static_cast<int32_t>(std::max<int64_t>(32, std::min<int64_t>(256, chunk)));
        if ((p.n_s + o.chunk - 1) / o.chunk > 65535) o.chunk = static_cast<int32_t>((p.n_s / 65535 + 16) / 16 * 16);
        auto outer = [&] {
            const dim3 grid(static_cast<uint32_t>(across), static_cast<uint32_t>((p.n_s + o.chunk - 1) / o.chunk), n);
            if (p.rows_stream)
                tb ? run_outer<true, true>(o, p.mt, p.pieces_fg, grid, s) : run_outer<false, true>(o, p.mt, p.pieces_fg, grid, s);
            else
                tb ? run_outer<true, false>(o, p.mt, p.pieces_fg, grid, s) : run_outer<false, false>(o, p.mt, p.pieces_fg, grid, s);
            return hipGetLastError();
        };
        // dweight, which reads the rows, and then dx, which may take their place
        if (p.rows_stream) {
            if (hipError_t e = sum()) return e;
            if (hipError_t e = outer()) return e;
        } else {
            if (hipError_t e = outer()) return e;
            if (hipError_t e = sum()) return e;
        }
        const int64_t n_t = p.rows_stream ? c.classes : p.mt * 16;
        if (p.splits == 1 && !(p.rows_stream && c.dbias)) continue;
        few_finish_kernel<<<dim3(static_cast<uint32_t>((c.cols + 255) / 256 + 1), static_cast<uint32_t>(n_t), n), 256, 0, s>>>(m);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

}  // namespace tc
