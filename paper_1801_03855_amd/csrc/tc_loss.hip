// Softmax cross entropy of K workers' rows over a large vocabulary, and its
// backward pass, without keeping the logits.
//
//     z = x W^T + b;   lse = log sum exp z;   loss = lse - z[label]
// and with f = scale * dloss of a row (0 of a row that is left out)
//     g = exp(z - lse) - [class = label]
//     dx = f g W;   dW = (f g)^T x;   db = sum of f g over the rows
//
// The forward pass is one product whose tiles leave, instead of the logits,
// their largest and the sum of the exponentials next to it for every row; a
// second kernel joins the tiles' pairs.  The backward pass takes the classes in
// pieces: it makes a piece's logits again, writes g of the piece, in binary16,
// both ways, and takes both products from it.
//
// Every product is of rows that run along the summed axis, 16 bits an element,
// on the matrix cores with binary32 sums.  bfloat16 rows and weights are
// multiplied as they are.  A binary32 operand is the sum of two binary16 values
// (hi = the nearest, lo = the nearest to the rest) times a power of two that
// puts its largest value under 2^15: lo hi + hi lo + hi hi leaves out only lo
// lo, 2^-22 of a term, at a third of the rate (binary32 matrix instructions run
// at a sixteenth).  g is within [-1, 1] and is held times 2^14 (f g for dweight
// alike, next to the largest |f|).  Where the result is bfloat16 it is one binary16
// value, 11 bits: half a step of those is an eighth of half a step of the result,
// and to either side from term to term (8,192 rows of 4,096 over 131,072 classes:
// 2.0% of dx's values are another bfloat16 value than with binary32 products, and
// 7.4e-4 of its size where the result's own rounding is 1.7e-3; with two values
// 0.1% and 1.7e-4, in 42.2 ms for 24.9).  Where it is binary32 it is hi and lo, in
// steps of 2^-38: 22 bits from 2^-16 on, 11 at 2^-28, nothing under 2^-39.  (Finer
// ones need a unit of lo's own, so that all sums are multiplied once between two
// runs over them, for which this loop has no registers: two workers' 901 rows of
// 1,003 over 30,011 classes 965 us, 2,880 so.)
//
// Layout.  An operand in the workspace is a panel: for every 32 elements of the
// summed axis, one line of 64 bytes a row, all rows next to each other, so that a
// stage of a tile is one block of memory.  (Loaded from where they lie instead,
// rows of 8 KB have a stage's lines at a few of the memory's channels: 8,192 rows
// of 4,096 over 131,072 classes in bfloat16 16.5 ms.)  The summed axis is padded
// with zeros to 64 elements.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "tc_grid.h"
#include "tc_lane.h"

namespace tc {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(1))) const char global_char;

constexpr int kBatch = 8;      // workers of one launch
constexpr int kLine = 64;      // bytes of a panel's row: 32 elements of the summed axis
constexpr int kParts = 512;    // partial maxima of an operand
constexpr int kUnitBits = 14;  // g is held times 2^14
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

__host__ __device__ constexpr int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

__device__ __forceinline__ float load_as(const void* p, int64_t i, int bf) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p);
    return bf ? Lane<__bf16>::get(a + i * 2) : Lane<float>::get(a + i * 4);
}

// ------------------------------------------------------------ scales of operands

// The exponent that puts a largest value `top` under 2^15, in [2^14, 2^15).
__device__ __forceinline__ int exponent_for(float top) { return top > 0.0f ? 14 - ilogbf(top) : 0; }

// |v| where it is finite: what is not makes its own sums NaN, whatever the scale.
__device__ __forceinline__ float finite_abs(float v) {
    const float a = fabsf(v);
    return a <= 3.402823466e+38f ? a : 0.0f;
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) v = fmaxf(v, __shfl_xor(v, m, 64));
    return v;
}

struct TopArgs {
    const void* x[kBatch];
    const void* w[kBatch];
    const int64_t* label[kBatch];
    const float* dloss[kBatch];
    int64_t rows[kBatch];
    char* ws;
    int64_t ws_stride;          // from worker to worker
    int64_t x_ld;               // elements
    int64_t w_size;             // elements
    int64_t at_rows, at_parts;  // in a worker's workspace
    int64_t classes;
    int32_t cols, x_bf, w_bf, has_dloss, backward;
};

// Partial maxima of one worker's operands: of x over the rows that count, of
// their factors, of the weight.
struct Parts {
    float x[kParts], f[kParts], w[kParts];
};

// One read of x (and of the weight): the exponent of every row of x, each row's
// factor (0 of a row that is left out), the partial maxima.
__global__ void __launch_bounds__(256) loss_top_kernel(const TopArgs a) {
    __shared__ float lds[2][4];
    const int k = blockIdx.y, wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    char* ws = a.ws + k * a.ws_stride;
    Parts* parts = reinterpret_cast<Parts*>(ws + a.at_parts);
    const int part = blockIdx.x % kParts;
    if (blockIdx.x >= kParts) {
        // the weight, in vectors of eight elements
        float top = 0.0f;
        const int64_t n = a.w_size / 8;
        const uintptr_t w = reinterpret_cast<uintptr_t>(a.w[k]);
        // four at a time: with one the loads' latency is what bounds it (131,072 x
        // 4,096 bfloat16 560 us)
        constexpr int kAhead = 4;
        for (int64_t v = part * 256 + threadIdx.x; v < n; v += kAhead * kParts * 256) {
            u32x4 q[kAhead][2];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int64_t at = std::min(v + i * kParts * 256, n - 1);
                q[i][0] = gld_u<u32x4>(w + at * (a.w_bf ? 16 : 32));
                if (!a.w_bf) q[i][1] = gld_u<u32x4>(w + at * 32 + 16);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                float f[8];
                if (a.w_bf) {
                    Lane<__bf16>::widen(q[i][0], f);
                } else {
                    Lane<float>::widen(q[i][0], f);
                    Lane<float>::widen(q[i][1], f + 4);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) top = fmaxf(top, finite_abs(f[e]));
            }
        }
        if (part == 0 && threadIdx.x < a.w_size - n * 8) top = fmaxf(top, finite_abs(load_as(a.w[k], n * 8 + threadIdx.x, a.w_bf)));
        top = wave_max(top);
        if (lane == 0) lds[0][wave] = top;
        __syncthreads();
        if (threadIdx.x == 0) parts->w[part] = fmaxf(fmaxf(lds[0][0], lds[0][1]), fmaxf(lds[0][2], lds[0][3]));
        return;
    }
    int32_t* exponents = reinterpret_cast<int32_t*>(ws + a.at_rows);
    const int64_t rows = a.rows[k], padded = round_up(rows, 256);
    float* factors = reinterpret_cast<float*>(exponents + padded);
    float top = 0.0f, top_f = 0.0f;
    for (int64_t r = part * 4 + wave; r < padded; r += kParts * 4) {
        float m = 0.0f, f = 0.0f;
        if (r < rows) {
            const uintptr_t x = reinterpret_cast<uintptr_t>(a.x[k]) + r * a.x_ld * (a.x_bf ? 2 : 4);
            for (int c = lane * 8; c < a.cols; c += 512) {
                float v[8];
                if (a.x_bf) {
                    Lane<__bf16>::widen(load_vec<__bf16, true>(x, c / 8, a.cols), v);
                } else {
                    Lane<float>::widen(load_vec<float, true>(x, c / 4, a.cols), v);
                    Lane<float>::widen(load_vec<float, true>(x, c / 4 + 1, a.cols), v + 4);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) m = fmaxf(m, finite_abs(v[e]));
            }
            m = wave_max(m);
            if (a.backward) {
                const int64_t label = a.label[k][r];
                if (label >= 0 && label < a.classes) {
                    f = a.has_dloss ? a.dloss[k][r] : 1.0f;
                    if (f != 0.0f) top = fmaxf(top, m);
                    top_f = fmaxf(top_f, finite_abs(f));
                }
            }
        }
        if (lane == 0) {
            exponents[r] = exponent_for(m);
            factors[r] = f;
        }
    }
    if (lane == 0) {
        lds[0][wave] = top;
        lds[1][wave] = top_f;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        parts->x[part] = fmaxf(fmaxf(lds[0][0], lds[0][1]), fmaxf(lds[0][2], lds[0][3]));
        parts->f[part] = fmaxf(fmaxf(lds[1][0], lds[1][1]), fmaxf(lds[1][2], lds[1][3]));
    }
}

// The exponent of a whole operand from its partial maxima, the same in every lane.
__device__ __forceinline__ int exponent_of(const float* parts) {
    float m = 0.0f;
    for (int i = threadIdx.x % 64; i < kParts; i += 64) m = fmaxf(m, parts[i]);
    return __builtin_amdgcn_readfirstlane(exponent_for(wave_max(m)));
}

// ------------------------------------------------------------------------ panels

// The panels of one operand, of every worker: as it lies (rows the operand's
// rows) and transposed (rows its columns), each in one or two planes.
struct Panels {
    const void* p[kBatch];
    int64_t rows[kBatch];      // of the operand, from `first` on
    int64_t at, at_t;          // of the panels in a worker's workspace; at_t -1: not wanted
    int64_t plane, plane_t;    // from hi to lo
    int64_t padded, padded_t;  // rows of the panels
    int64_t ld;                // elements
    int32_t planes, planes_t;
    int32_t bf;                // of the operand
    int32_t raw;               // as it lies: bfloat16 as it is
    int32_t by_rows;           // as it lies: every row with its own exponent
    int32_t tiles_r, tiles_c;  // of 64 x 64
    int32_t first;             // block of the launch
};

struct PanelArgs {
    Panels x, w;
    char* ws;
    int64_t ws_stride, at_rows, at_parts;
    int32_t cols;
};

__device__ __forceinline__ void split(const float* v, int e, u16x8& hi, u16x8& lo) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float s = ldexpf(v[i], e);
        const _Float16 h = static_cast<_Float16>(s);
        hi[i] = __builtin_bit_cast(uint16_t, h);
        lo[i] = __builtin_bit_cast(uint16_t, static_cast<_Float16>(s - static_cast<float>(h)));
    }
}

// A workgroup takes 64 x 64 elements of one operand; bound by memory.  2^36
// elements of each are more workgroups than one dimension takes, so they go on
// along z (those behind the last tile find no rows).
__global__ void __launch_bounds__(256) loss_panel_kernel(const PanelArgs a) {
    __shared__ float lds[64][65];
    const int k = blockIdx.y, b = blockIdx.z * gridDim.x + blockIdx.x, tid = threadIdx.x;
    const bool weight = b >= a.w.first;
    const Panels& o = weight ? a.w : a.x;
    char* ws = a.ws + k * a.ws_stride;
    const int64_t rows = o.rows[k];
    const int t = b - o.first;
    const int64_t r0 = static_cast<int64_t>(t / o.tiles_c) * 64;
    const int c0 = t % o.tiles_c * 64;
    if (r0 >= rows) return;
    const Parts* parts = reinterpret_cast<const Parts*>(ws + a.at_parts);
    const int32_t* exponents = reinterpret_cast<const int32_t*>(ws + a.at_rows);
    const float* factors = reinterpret_cast<const float*>(exponents + round_up(rows, 256));
    const int whole = o.raw && o.at_t < 0 ? 0 : exponent_of(weight ? parts->w : parts->x);
    const int es = o.bf ? 2 : 4;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int r = tid / 8 + 32 * h, piece = tid % 8, c = c0 + piece * 8;
        const int64_t row = r0 + r;
        float v[8] = {};
        if (row < rows && c < a.cols) {
            const uintptr_t at = reinterpret_cast<uintptr_t>(o.p[k]) + row * o.ld * es;
            if (o.bf) {
                Lane<__bf16>::widen(load_vec<__bf16, true>(at, c / 8, a.cols), v);
            } else {
                Lane<float>::widen(load_vec<float, true>(at, c / 4, a.cols), v);
                Lane<float>::widen(load_vec<float, true>(at, c / 4 + 1, a.cols), v + 4);
            }
        }
        {
            char* to = ws + o.at + ((c0 / 32 + piece / 4) * o.padded + row) * kLine + piece % 4 * 16;
            if (o.raw) {
                *reinterpret_cast<u32x4*>(to) = Lane<__bf16>::narrow(v);
            } else {
                u16x8 hi, lo;
                split(v, o.by_rows ? exponents[row] : whole, hi, lo);
                *reinterpret_cast<u16x8*>(to) = hi;
                if (o.planes > 1) *reinterpret_cast<u16x8*>(to + o.plane) = lo;
            }
        }
        if (o.at_t >= 0) {
            // a row that is left out, whatever it holds, is zeros here
            const bool there = weight || (row < rows && factors[row] != 0.0f);
#pragma unroll
            for (int e = 0; e < 8; ++e) lds[r][piece * 8 + e] = there ? v[e] : 0.0f;
        }
    }
    if (o.at_t < 0) return;
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int c = tid / 8 + 32 * h, piece = tid % 8;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = lds[piece * 8 + e][c];
        u16x8 hi, lo;
        split(v, whole, hi, lo);
        char* to = ws + o.at_t + ((r0 / 32 + piece / 4) * o.padded_t + c0 + c) * kLine + piece % 4 * 16;
        *reinterpret_cast<u16x8*>(to) = hi;
        if (o.planes_t > 1) *reinterpret_cast<u16x8*>(to + o.plane_t) = lo;
    }
}

// ---------------------------------------------------------------------- products

// Rows of one operand of a product.
struct Side {
    int64_t step;     // bytes from one 32 elements of the sum to the next
    int64_t plane;    // from hi to lo
    uint32_t planes;  // bit n: plane of the n-th run over the sum
};

template <bool BF>
__device__ __forceinline__ f32x16 multiply(u32x4 a, u32x4 b, f32x16 c) {
    if constexpr (BF)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// One tile of left right^T, TILE x TILE, of four waves with a quarter each, as
// 32 x 32 x 16 products.  A stage is 32 elements (64 bytes) of each of the 2 TILE
// rows; kStages of them are in LDS, loaded straight from memory while others are
// multiplied.  A row's 64 bytes are four 16-byte pieces; piece p of row r lies at
// p ^ (r / 4 % 4), so that 16 lanes reading one piece each of 16 rows touch all
// 64 banks once.  Left and right: the tile's first rows, of which there are
// `rows` (the last one stands for those behind it).  The sum runs over the steps
// [first, end) of 32 elements `runs` times, over other planes each time.
//
// A SIMD has one wave (or two), so nothing but the order of the instructions
// covers for what is not a product: every product is followed by at most one
// read from LDS or load.  8,192 rows of 4,096 over 131,072 classes in bfloat16:
// the logits run at 1,180 TFLOP/s, their ends included, the gradients' products at
// 1,160, the matrix cores busy 58% of the time at 1.92 GHz (the library's 8,192^3
// product: 1,420).  With stages of 64 elements, loads and reads asked for between
// groups of products, it was 970 and 1,125.
//
// Stages of tiles of 256: with two the forward pass takes 9.3 ms, with three, four
// or five 7.6.  Of 128: with three a CU has room for three workgroups (206 rows of
// 2,585 over 7,511 classes, backward: 204 us with four, 193).
//
// acc[i][j], lane l, element e: row i * 32 + e / 4 * 8 + l / 32 * 4 + e % 4 of
// the wave's quarter of left, row j * 32 + l % 32 of its quarter of right.
template <int TILE>
constexpr int kStages = TILE == 256 ? 4 : 3;

template <int TILE, bool BF>
__device__ __forceinline__ void product(char* lds, const char* left, const Side& ls, int left_rows, const char* right,
                                        const Side& rs, int right_rows, int first, int end, int runs,
                                        f32x16 (&acc)[TILE / 64][TILE / 64]) {
    constexpr int kHalf = TILE * kLine, kStage = 2 * kHalf, kSide = TILE / 64, kLoads = TILE / 64;
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const int wr = wave / 2 * (TILE / 2), wc = wave % 2 * (TILE / 2);
    // this wave's 1,024-byte pieces of a stage: sixteen rows each
    uint32_t off_l[kLoads], off_r[kLoads];
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
        const int r = (wave * kLoads + q) * 16 + lane / 4, p = (lane % 4) ^ (r / 4 % 4);
        off_l[q] = static_cast<uint32_t>(min(r, left_rows - 1) * kLine + p * 16);
        off_r[q] = static_cast<uint32_t>(min(r, right_rows - 1) * kLine + p * 16);
    }
    // the stage that is loaded next, and the one behind the last
    const int stages = (end - first) * runs;
    int asked = 0, at = first, run = 0;
    const char *pl, *pr;
    auto seek = [&] {
        pl = left + first * ls.step + (ls.planes >> run & 1) * ls.plane;
        pr = right + first * rs.step + (rs.planes >> run & 1) * rs.plane;
    };
    seek();
    // load n of a stage's 2 kLoads
    auto load = [&](int buf, int n) {
        char* dst = lds + buf * kStage + wave * kLoads * 1024;
        const int q = n / 2;
        if (n % 2 == 0)
            __builtin_amdgcn_global_load_lds((global_char*)(pl + off_l[q]), (lds_char*)(dst + q * 1024), 16, 0, 0);
        else
            __builtin_amdgcn_global_load_lds((global_char*)(pr + off_r[q]), (lds_char*)(dst + kHalf + q * 1024), 16, 0, 0);
    };
    auto advance = [&] {
        ++asked;
        pl += ls.step;
        pr += rs.step;
        if (++at == end) {
            at = first;
            ++run;
            seek();
        }
    };
    struct Operands {
        u32x4 a[kSide], b[kSide];
    } now, next;
    const int ra = (wr + lane % 32) * kLine, rb = kHalf + (wc + lane % 32) * kLine, turn = lane / 4 % 4;
    const int piece[2] = {((lane / 32) ^ turn) * 16, ((2 + lane / 32) ^ turn) * 16};
    // operand n of 2 kSide: those of the first products first
    auto read = [&](Operands& f, int buf, int step, int n) {
        const char* p = lds + buf * kStage + piece[step];
        if (n == 0)
            f.a[0] = *reinterpret_cast<const u32x4*>(p + ra);
        else if (n <= kSide)
            f.b[n - 1] = *reinterpret_cast<const u32x4*>(p + rb + (n - 1) * 32 * kLine);
        else
            f.a[n - kSide] = *reinterpret_cast<const u32x4*>(p + ra + (n - kSide) * 32 * kLine);
    };
    constexpr int kAll = kSide * kSide, kReads = 2 * kSide, kAsks = 2 * kLoads;
    auto one = [&](const Operands& f, int n) {
        acc[n / kSide][n % kSide] = multiply<BF>(f.a[n / kSide], f.b[n % kSide], acc[n / kSide][n % kSide]);
    };
    for (int n = 0; n < kStages<TILE> - 1 && n < stages; ++n) {
#pragma unroll
        for (int q = 0; q < kAsks; ++q) load(n, q);
        advance();
    }
    // The stage after the one under way is there, in every wave, and every wave
    // has its operands of the one under way, whose buffer is loaded next.
    // `full`: the stages after it are all asked for.
    auto arrive = [&](bool full) {
        if (full)
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((kStages<TILE> - 2) * kAsks) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    arrive(stages >= kStages<TILE> - 1);
#pragma unroll
    for (int q = 0; q < kReads; ++q) read(now, 0, 0, q);
    int buf = 0;
    for (int st = 0; st < stages; ++st) {
        const int then = buf + 1 == kStages<TILE> ? 0 : buf + 1, before = buf == 0 ? kStages<TILE> - 1 : buf - 1;
        const bool more = asked < stages;
        // the first 16 elements; the next 16 are read, a stage is asked for
#pragma unroll
        for (int n = 0; n < kAll; ++n) {
            one(now, n);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int q = n * kReads / kAll; q < (n + 1) * kReads / kAll; ++q) read(next, buf, 1, q);
#pragma unroll
            for (int q = n * kAsks / kAll; q < (n + 1) * kAsks / kAll; ++q)
                if (more) load(before, q);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (more) advance();
        constexpr int kFirst = kAll / 4;
#pragma unroll
        for (int n = 0; n < kFirst; ++n) one(next, n);
        __builtin_amdgcn_sched_barrier(0);
        const bool last = st + 1 == stages;
        if (!last) arrive(more);
#pragma unroll
        for (int n = kFirst; n < kAll; ++n) {
            // (past the end of the last stage they are operands of nothing)
#pragma unroll
            for (int q = (n - kFirst) * kReads / (kAll - kFirst); q < (n - kFirst + 1) * kReads / (kAll - kFirst); ++q)
                read(now, then, 0, q);
            __builtin_amdgcn_sched_barrier(0);
            one(next, n);
            __builtin_amdgcn_sched_barrier(0);
        }
        buf = then;
    }
}

// Tile t of `down` x `across` tiles, in an order that keeps the tiles under way
// on one XCD (workgroup b runs on XCD b % 8) in a compact part of the result.
struct Place {
    int i, j;
};
__device__ __forceinline__ Place place_of(uint32_t b, uint32_t n, int down, int across) {
    const uint32_t per = n / 8, rest = n % 8, xcd = b % 8;
    const uint32_t t = xcd * per + min(xcd, rest) + b / 8;
    constexpr uint32_t kGroup = 8;
    const uint32_t group = t / (kGroup * across), in = t % (kGroup * across);
    const uint32_t height = min(kGroup, static_cast<uint32_t>(down) - group * kGroup);
    return {static_cast<int>(group * kGroup + in % height), static_cast<int>(in / height)};
}

// The logits of one piece of the classes.
struct LogitArgs {
    const void* bias[kBatch];
    const int64_t* label[kBatch];
    const float* lse[kBatch];
    int64_t rows[kBatch];
    Side ws, xs;
    char* work;
    int64_t stride;                 // of the workspace, from worker to worker
    int64_t at_rows, at_parts;
    int64_t at_w, at_x;             // panels
    int64_t at_g, at_gt;            // g as [row][class] and [class][row]
    int64_t plane_g, plane_gt;
    int64_t at_pairs, at_own;       // (largest, sum) of every tile and row; the label's logit
    int64_t padded;                 // classes of the panel of g
    int64_t padded_r;               // rows of the panels
    int64_t first;                  // class of the piece
    int64_t pair_tile;              // and its first tile among those that are joined with it
    int32_t classes, count;         // in all, of the piece
    int32_t tiles_v, tiles_r, steps, runs;
    int32_t scaled;                 // operands have exponents
    int32_t w_bf;                   // of the bias
    int32_t planes_g, planes_gt, has_dloss;
    int64_t at_db;                  // sums of f g over a wave's rows [wave][class]; -1: not wanted
    int64_t at_acc;                 // sums of a part of the columns [part][tile][register][lane]
    int32_t splits;
};

// Joins (m, s) and (m2, s2): the largest, and the sum of exp(z - largest).  A
// largest value of -infinity has no sum to scale.
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2) {
    const float top = fmaxf(m, m2);
    const float a = m == top ? s : s * __builtin_amdgcn_exp2f((m - top) * kLog2e), b = m2 == top ? s2 : s2 * __builtin_amdgcn_exp2f((m2 - top) * kLog2e);
    m = top;
    s = a + b;
}

// What a launch does of a tile: all; where tiles are few, the sums over parts of
// the columns; what comes after them.
enum Part { kWhole, kSums, kRest };

// Rows of left are classes, rows of right are workers' rows: a lane has one row's
// logits of 16 classes of each 32 x 32 product.
template <int TILE, bool BF, bool GRAD, Part PART>
__global__ void __launch_bounds__(256, TILE == 256 ? 1 : 2) loss_logit_kernel(const LogitArgs a) {
    constexpr int kSide = TILE / 64;
    // (the stages of the product; then a tile of g)
    constexpr int kLds = kStages<TILE> * 2 * TILE * kLine, kTileG = TILE * TILE * 2;
    __shared__ __attribute__((aligned(16))) char lds[GRAD && kTileG > kLds ? kTileG : kLds];
    float* const extra = reinterpret_cast<float*>(lds);  // after the product: biases; forward, pairs of the upper waves
    const int k = blockIdx.y;
    const int64_t rows = a.rows[k];
    // (workers with fewer rows leave the tiles behind them)
    const Place at = place_of(blockIdx.x, gridDim.x, a.tiles_v, a.tiles_r);
    const int v0 = at.i * TILE;
    const int64_t r0 = static_cast<int64_t>(at.j) * TILE;
    if (r0 >= rows) return;
    char* work = a.work + k * a.stride;
    f32x16 acc[kSide][kSide] = {};
    // (in the order of the registers, 16 bytes a lane)
    f32x4* sums = reinterpret_cast<f32x4*>(work + a.at_acc) + (static_cast<int64_t>(at.i) * a.tiles_r + at.j) * (TILE * TILE / 4) + threadIdx.x;
    const int64_t all = static_cast<int64_t>(a.tiles_v) * a.tiles_r * (TILE * TILE / 4);
    if constexpr (PART != kRest) {
        const int from = PART == kSums ? a.steps * static_cast<int>(blockIdx.z) / a.splits : 0;
        const int to = PART == kSums ? a.steps * (static_cast<int>(blockIdx.z) + 1) / a.splits : a.steps;
        product<TILE, BF>(lds, work + a.at_w + static_cast<int64_t>(v0) * kLine, a.ws, a.count - v0, work + a.at_x + r0 * kLine, a.xs,
                          static_cast<int>(min(static_cast<int64_t>(TILE), rows - r0)), from, to, a.runs, acc);
    }
    // What the lane's rows have, asked for at once.
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
    const int wr = wave / 2 * (TILE / 2), wc = wave % 2 * (TILE / 2);
    const int32_t* exponents = reinterpret_cast<const int32_t*>(work + a.at_rows);
    const float* factors = reinterpret_cast<const float*>(exponents + round_up(rows, 256));
    const Parts* parts = reinterpret_cast<const Parts*>(work + a.at_parts);
    int64_t label[kSide];
    float lses[kSide], factor[kSide];
    int exponent[kSide];
    int ew = 0;
    auto ask = [&] {
#pragma unroll
        for (int j = 0; j < kSide; ++j) {
            const int64_t row = std::min<int64_t>(r0 + wc + j * 32 + lane % 32, rows - 1);
            label[j] = a.label[k][row];
            lses[j] = GRAD ? a.lse[k][row] : 0.0f;
            factor[j] = GRAD ? factors[row] : 1.0f;
            exponent[j] = a.scaled ? exponents[row] : 0;
        }
        if (a.scaled) ew = exponent_of(parts->w);
    };
    if constexpr (PART == kRest) ask();
    if constexpr (PART != kWhole)
        for (int p = 0; p < (PART == kSums ? 1 : a.splits); ++p)
#pragma unroll
            for (int i = 0; i < kSide; ++i)
#pragma unroll
                for (int j = 0; j < kSide; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        f32x4* place = sums + ((i * kSide + j) * 4 + q) * 256 + all * (PART == kSums ? static_cast<int>(blockIdx.z) : p);
                        if constexpr (PART == kSums) {
                            *place = {acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2], acc[i][j][q * 4 + 3]};
                        } else {
                            const f32x4 v = *place;
#pragma unroll
                            for (int n = 0; n < 4; ++n) acc[i][j][q * 4 + n] += v[n];
                        }
                    }
    if constexpr (PART == kSums) return;
    if constexpr (PART == kWhole) ask();
    // the tile's biases; classes behind the last one have -infinity
    __syncthreads();
    for (int v = tid; v < TILE; v += 256)
        extra[v] = v0 + v < a.count ? (a.bias[k] ? load_as(a.bias[k], a.first + v0 + v, a.w_bf) : 0.0f) : -INFINITY;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kSide; ++j) {
        const int64_t row = r0 + wc + j * 32 + lane % 32;
        // (backward, a factor of 0 leaves a row out as well)
        const bool counts = row < rows && label[j] >= 0 && label[j] < a.classes && (!GRAD || factor[j] != 0.0f);
        const int own = counts && label[j] >= a.first + v0 && label[j] < a.first + v0 + TILE ? static_cast<int>(label[j] - a.first) - v0 : -1;
        const int e = -(ew + exponent[j]);
        const float lse = lses[j];
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < kSide; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int v = wr + i * 32 + q * 8 + lane / 32 * 4;
                const f32x4 b = *reinterpret_cast<const f32x4*>(extra + v);
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    float z = acc[i][j][q * 4 + n];
                    if (!BF) z = ldexpf(z, e);
                    z += b[n];
                    if constexpr (GRAD) {
                        const float p = __builtin_amdgcn_exp2f((z - lse) * kLog2e);
                        z = counts ? (v + n == own ? p - 1.0f : p) : 0.0f;
                    } else {
                        if (v + n == own) reinterpret_cast<float*>(work + a.at_own)[row] = z;
                        top = fmaxf(top, z);
                    }
                    acc[i][j][q * 4 + n] = z;
                }
            }
        if constexpr (!GRAD) {
            float sum = 0.0f;
            const float from = top > -INFINITY ? top : 0.0f;
#pragma unroll
            for (int i = 0; i < kSide; ++i)
#pragma unroll
                for (int q = 0; q < 16; ++q) sum += __builtin_amdgcn_exp2f((acc[i][j][q] - from) * kLog2e);
            join(top, sum, __shfl_xor(top, 32, 64), __shfl_xor(sum, 32, 64));
            float* pairs = extra + TILE;  // of the upper waves
            const int at_pair = (wc + j * 32 + lane % 32) * 2;
            if (wr && lane < 32) {
                pairs[at_pair] = top;
                pairs[at_pair + 1] = sum;
            }
            acc[0][j][0] = top;
            acc[0][j][1] = sum;
        }
    }
    if constexpr (!GRAD) {
        __syncthreads();
        if (wr || lane >= 32) return;
        float2* out = reinterpret_cast<float2*>(work + a.at_pairs) + (a.pair_tile + at.i) * a.padded_r + r0;
#pragma unroll
        for (int j = 0; j < kSide; ++j) {
            const int r = wc + j * 32 + lane;
            float top = acc[0][j][0], sum = acc[0][j][1];
            join(top, sum, extra[TILE + r * 2], extra[TILE + r * 2 + 1]);
            out[r] = make_float2(top, sum);
        }
    } else {
        if (a.at_db >= 0) {
            // f g summed over the wave's rows: in the lane, then over 32 lanes, of which
            // each step leaves half of the classes to either half
            float sum[16 * kSide] = {};
#pragma unroll
            for (int j = 0; j < kSide; ++j) {
                const float f = factor[j];
#pragma unroll
                for (int i = 0; i < kSide; ++i)
#pragma unroll
                    for (int q = 0; q < 16; ++q) sum[i * 16 + q] = acc[i][j][q] == 0.0f ? sum[i * 16 + q] : fmaf(acc[i][j][q], f, sum[i * 16 + q]);
            }
#pragma unroll
            for (int m = 16; m > 0; m >>= 1) {
                const bool upper = lane & m;
                const int half = 8 * kSide * m / 16;
#pragma unroll
                for (int h = 0; h < half; ++h) {
                    const float keep = upper ? sum[h + half] : sum[h], send = upper ? sum[h] : sum[h + half];
                    sum[h] = keep + __shfl_xor(send, m, 64);
                }
            }
            float* out = reinterpret_cast<float*>(work + a.at_db) + (at.j * 2 + wave % 2) * a.padded + v0;
#pragma unroll
            for (int h = 0; h < kSide / 2; ++h) {
                const int n = lane % 32 * (kSide / 2) + h;  // i, e / 4, e % 4
                out[wr + n / 16 * 32 + n / 4 % 4 * 8 + lane / 32 * 4 + n % 4] = sum[h];
            }
        }
        // g leaves through LDS, as [row][class] with 16-byte pieces turned, a
        // plane at a time, in both orders.
        constexpr int kPieces = TILE / 8;
        auto piece_at = [&](int r, int p) { return lds + r * TILE * 2 + (p ^ (r % kPieces)) * 16; };
        const int64_t left_k = round_up(rows, 64);  // of the sum over rows
        const int ef = a.has_dloss ? exponent_of(parts->f) - 14 : 0;  // a factor's largest value under 2
        const int bits = kUnitBits - (a.has_dloss ? 1 : 0);
        // (one body for every plane; `turn` keeps the places of a pass from being
        // held in registers next to the sums)
        auto fill = [&](int plane, bool factored, int turn) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kSide; ++j) {
                const int r = wc + j * 32 + lane % 32 + turn;
                const float unit = factored ? ldexpf(factor[j], ef + bits) : static_cast<float>(1 << kUnitBits);
#pragma unroll
                for (int i = 0; i < kSide; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        f16x4 h;
#pragma unroll
                        for (int n = 0; n < 4; ++n) {
                            // (0 of a row that is left out, whatever its factor)
                            const float g = acc[i][j][q * 4 + n], s = g == 0.0f ? 0.0f : g * unit;
                            h[n] = static_cast<_Float16>(s);
                            if (plane) h[n] = static_cast<_Float16>(s - static_cast<float>(h[n]));
                        }
                        const int v = wr + i * 32 + q * 8 + lane / 32 * 4;
                        *reinterpret_cast<f16x4*>(piece_at(r, v / 8) + v % 8 * 2) = h;
                    }
            }
            __syncthreads();
        };
        // (a SIMD has one wave, which waits for what it reads: several at a time)
        constexpr int kAtOnce = 8;
        auto put_g = [&](int plane) {
            char* g = work + a.at_g + plane * a.plane_g;
            for (int n0 = tid; n0 < TILE * kPieces; n0 += 256 * kAtOnce) {
                u32x4 h[kAtOnce];
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    const int n = n0 + u * 256, block = n / (TILE * 4), r = n / 4 % TILE, p = n % 4;  // of 32 classes
                    h[u] = *reinterpret_cast<const u32x4*>(piece_at(r, block * 4 + p));
                }
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    const int n = n0 + u * 256, block = n / (TILE * 4), r = n / 4 % TILE, p = n % 4;
                    *reinterpret_cast<u32x4*>(g + ((v0 / 32 + block) * a.padded_r + r0 + r) * kLine + p * 16) = h[u];
                }
            }
        };
        // two classes of eight rows
        auto put_gt = [&](int plane) {
            char* g = work + a.at_gt + plane * a.plane_gt;
            constexpr int kPairs = kAtOnce / 2;
            for (int n0 = tid; n0 < TILE * kPieces / 2; n0 += 256 * kPairs) {
                uint32_t h[kPairs][8];
#pragma unroll
                for (int u = 0; u < kPairs; ++u) {
                    const int n = n0 + u * 256, block = n / (TILE * 2), v = n / 4 % (TILE / 2) * 2, p = n % 4;  // of 32 rows
#pragma unroll
                    for (int e = 0; e < 8; ++e) h[u][e] = *reinterpret_cast<const uint32_t*>(piece_at(block * 32 + p * 8 + e, v / 8) + v % 8 * 2);
                }
#pragma unroll
                for (int u = 0; u < kPairs; ++u) {
                    const int n = n0 + u * 256, block = n / (TILE * 2), v = n / 4 % (TILE / 2) * 2, p = n % 4;
                    if (r0 + block * 32 >= left_k) continue;
                    char* to = g + ((r0 / 32 + block) * a.padded + v0 + v) * kLine + p * 16;
                    u32x4 first, second;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        first[i] = __builtin_amdgcn_perm(h[u][2 * i + 1], h[u][2 * i], 0x05040100u);
                        second[i] = __builtin_amdgcn_perm(h[u][2 * i + 1], h[u][2 * i], 0x07060302u);
                    }
                    *reinterpret_cast<u32x4*>(to) = first;
                    *reinterpret_cast<u32x4*>(to + kLine) = second;
                }
            }
        };
        for (int pass = 0; pass < 4; ++pass) {
            const int plane = pass / 2;
            const bool factored = pass % 2;
            const bool g = !factored && plane < a.planes_g, gt = plane < a.planes_gt && factored == (a.has_dloss != 0);
            if (!g && !gt) continue;
            int turn = 0;
            asm volatile("" : "+v"(turn));
            fill(plane, factored, turn);
            if (g) put_g(plane);
            if (gt) put_gt(plane);
        }
    }
}

struct LossArgs {
    const int64_t* label[kBatch];
    float* loss[kBatch];
    float* lse[kBatch];
    int64_t rows[kBatch];
    char* work;
    int64_t stride, at_pairs, at_own;
    int64_t at_run;     // the pairs of the classes before these
    int64_t padded_r;
    int32_t tiles, classes;
    int32_t first, last;
};

// Joins the tiles' pairs of every row: 64 rows a workgroup, whose 16 waves take
// the tiles in turn.  Where the pairs of all classes would not fit their place
// they are joined several times, each time with what came of those before.
__global__ void __launch_bounds__(1024) loss_join_kernel(const LossArgs a) {
    __shared__ float2 lds[16][64];
    const int k = blockIdx.y, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t rows = a.rows[k], row = static_cast<int64_t>(blockIdx.x) * 64 + lane;
    if (static_cast<int64_t>(blockIdx.x) * 64 >= rows) return;
    char* work = a.work + k * a.stride;
    float top = -INFINITY, sum = 0.0f;
    if (row < rows)
        for (int t = wave; t < a.tiles; t += 16) {
            const float2 p = reinterpret_cast<const float2*>(work + a.at_pairs)[t * a.padded_r + row];
            join(top, sum, p.x, p.y);
        }
    lds[wave][lane] = make_float2(top, sum);
    __syncthreads();
    if (wave || row >= rows) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) join(top, sum, lds[w][lane].x, lds[w][lane].y);
    float2* run = reinterpret_cast<float2*>(work + a.at_run) + row;
    if (!a.first) join(top, sum, run->x, run->y);
    if (!a.last) {
        *run = make_float2(top, sum);
        return;
    }
    const float lse = top + log2f(sum) * kLn2;
    a.lse[k][row] = lse;
    const int64_t label = a.label[k][row];
    a.loss[k][row] = label >= 0 && label < a.classes ? lse - reinterpret_cast<const float*>(work + a.at_own)[row] : 0.0f;
}

// One of the backward pass's two products: rows of left are columns of x.
struct GradJob {
    int64_t at_left, at_right;
    Side left, right;
    int64_t at_sums, sums_stride;  // partial sums [split][row of right][column], or
    void* out[kBatch];             // (at_sums < 0) results of `bf` with rows of cols
    int64_t rows[kBatch];          // of right
    int64_t out_ld;                // elements
    int32_t down, across, splits, steps, runs;
    int32_t padded;                // columns of the partial sums
    int32_t add;                   // to the sums that are there
    int32_t bf;
    int32_t first;                 // block of the launch
    int32_t by_rows;               // the summed axis is the worker's rows
};

struct GradArgs {
    GradJob job[2];
    char* work;
    int64_t stride, at_rows, at_parts;
    int64_t x_rows[kBatch];
    float scale;
    int32_t cols, has_dloss;
};

template <int TILE>
__global__ void __launch_bounds__(256, TILE == 256 ? 1 : 2) loss_grad_kernel(const GradArgs a) {
    constexpr int kSide = TILE / 64;
    __shared__ __attribute__((aligned(16))) char lds[kStages<TILE> * 2 * TILE * kLine];
    const int k = blockIdx.y;
    const bool second = static_cast<int>(blockIdx.x) >= a.job[1].first;
    const GradJob& o = a.job[second];
    const int tiles = o.down * o.across, b = blockIdx.x - o.first;
    const Place at = place_of(b % tiles, tiles, o.down, o.across);
    const int part = b / tiles;
    const int64_t rows = o.rows[k], n0 = static_cast<int64_t>(at.j) * TILE;
    if (n0 >= rows) return;
    const int m0 = at.i * TILE;
    const int steps = o.by_rows ? static_cast<int>(round_up(a.x_rows[k], 64) / 32) : o.steps;
    const int from = static_cast<int>(static_cast<int64_t>(steps) * part / o.splits);
    const int to = static_cast<int>(static_cast<int64_t>(steps) * (part + 1) / o.splits);
    char* work = a.work + k * a.stride;
    f32x16 acc[kSide][kSide] = {};
    if (to > from)
        product<TILE, false>(lds, work + o.at_left + static_cast<int64_t>(m0) * kLine, o.left, TILE,
                             work + o.at_right + n0 * kLine, o.right, TILE, from, to, o.runs, acc);
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int wr = wave / 2 * (TILE / 2), wc = wave % 2 * (TILE / 2);
    const Parts* parts = reinterpret_cast<const Parts*>(work + a.at_parts);
    const int e = o.at_sums >= 0 ? 0
                  : o.by_rows    ? -(exponent_of(parts->x) + kUnitBits + (a.has_dloss ? exponent_of(parts->f) - 15 : 0))
                                 : -(exponent_of(parts->w) + kUnitBits);
    const float* factors = reinterpret_cast<const float*>(work + a.at_rows) + round_up(a.x_rows[k], 256);
    if (o.at_sums >= 0) {
#pragma unroll
        for (int j = 0; j < kSide; ++j) {
            const int64_t row = n0 + wc + j * 32 + lane % 32;
            if (row >= rows) continue;
#pragma unroll
            for (int i = 0; i < kSide; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = m0 + wr + i * 32 + q * 8 + lane / 32 * 4;
                    f32x4 v = {acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2], acc[i][j][q * 4 + 3]};
                    f32x4* sums = reinterpret_cast<f32x4*>(work + o.at_sums + part * o.sums_stride + (row * o.padded + c) * 4);
                    if (o.add) v += *sums;
                    *sums = v;
                }
        }
        return;
    }
    // The result leaves through LDS in two halves of the tile's rows, so that
    // whole lines are stored, past the caches: a row's columns as 16-byte pieces,
    // piece p of row r at p ^ (r % 32).  (2 x 206 rows of 2,585 over 7,511 classes,
    // the whole gradient, 222 us from the registers, 220 so, 203 past the caches.)
    constexpr int kHalfRows = TILE / 2, kPieces = TILE / 4, kRowsAtOnce = 256 / kPieces, kAtOnce = 8;
    static_assert(kHalfRows * TILE * 4 <= kStages<TILE> * 2 * TILE * kLine, "half a tile fits");
    const int tid = threadIdx.x, p = tid % kPieces, c = m0 + p * 4;
    auto piece_at = [&](int r, int at) { return reinterpret_cast<f32x4*>(lds + (r * kPieces + (at ^ (r % 32))) * 16); };
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        __syncthreads();
        if (wave % 2 == half)
#pragma unroll
            for (int j = 0; j < kSide; ++j)
#pragma unroll
                for (int i = 0; i < kSide; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *piece_at(j * 32 + lane % 32, (wr + i * 32 + q * 8) / 4 + lane / 32) =
                            f32x4{acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2], acc[i][j][q * 4 + 3]};
        __syncthreads();
        for (int first = tid / kPieces; first < kHalfRows; first += kRowsAtOnce * kAtOnce) {
            f32x4 v[kAtOnce];
            float f[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const int64_t row = n0 + half * kHalfRows + first + u * kRowsAtOnce;
                v[u] = *piece_at(first + u * kRowsAtOnce, p);
                // (dx: a row that is left out is 0, whatever the sums hold)
                f[u] = o.by_rows ? 1.0f : factors[std::min<int64_t>(row, rows - 1)];
            }
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const int64_t row = n0 + half * kHalfRows + first + u * kRowsAtOnce;
                if (row >= rows || c >= a.cols) break;
#pragma unroll
                for (int x = 0; x < 4; ++x) v[u][x] = f[u] == 0.0f ? 0.0f : ldexpf(v[u][x], e) * (f[u] * a.scale);
                const uintptr_t out = reinterpret_cast<uintptr_t>(o.out[k]) + (row * o.out_ld + c) * (o.bf ? 2 : 4);
                if (c + 4 <= a.cols) {
                    if (o.bf) {
                        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
                        bf16x4 h;
#pragma unroll
                        for (int x = 0; x < 4; ++x) h[x] = static_cast<__bf16>(v[u][x]);
                        gst_u_nt(out, __builtin_bit_cast(u32x2, h));
                    } else {
                        gst_u_nt(out, v[u]);
                    }
                } else {
#pragma unroll
                    for (int x = 0; x < 3; ++x)
                        if (c + x < a.cols) {
                            if (o.bf)
                                Lane<__bf16>::put(out + x * 2, v[u][x]);
                            else
                                Lane<float>::put(out + x * 4, v[u][x]);
                        }
                }
            }
        }
    }
}

struct FinishArgs {
    void* out[kBatch];
    int64_t rows[kBatch];
    int64_t x_rows[kBatch];
    char* work;
    int64_t stride, at_sums, sums_stride, at_rows, at_parts;
    int64_t ld;  // elements
    int32_t padded, splits, cols, bf, has_dloss;
    int32_t weight;  // dweight, or dx
    float scale;
};

// dx (or dweight) from the partial sums, in a fixed order: four columns a lane.
__global__ void __launch_bounds__(256) loss_finish_kernel(const FinishArgs a) {
    const int k = blockIdx.y;
    const int64_t rows = a.rows[k];
    const int per = (a.cols + 3) / 4;
    const char* work = a.work + k * a.stride;
    const Parts* parts = reinterpret_cast<const Parts*>(work + a.at_parts);
    const int e = -(a.weight ? exponent_of(parts->x) + kUnitBits + (a.has_dloss ? exponent_of(parts->f) - 15 : 0)
                             : exponent_of(parts->w) + kUnitBits);
    const float* factors = reinterpret_cast<const float*>(work + a.at_rows) + round_up(a.x_rows[k], 256);
    const int64_t n = rows * per;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * 256) {
        const int64_t row = i / per;
        const int c = static_cast<int>(i - row * per) * 4;
        const char* from = work + a.at_sums + (row * a.padded + c) * 4;
        f32x4 v = *reinterpret_cast<const f32x4*>(from);
        for (int s = 1; s < a.splits; ++s) v += *reinterpret_cast<const f32x4*>(from + s * a.sums_stride);
        const float f = a.weight ? 1.0f : factors[row];
        const uintptr_t out = reinterpret_cast<uintptr_t>(a.out[k]) + (row * a.ld + c) * (a.bf ? 2 : 4);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            // (a row that is left out is 0, whatever the sums hold)
            const float y = f == 0.0f ? 0.0f : ldexpf(v[x], e) * (a.weight ? a.scale : a.scale * f);
            if (c + x < a.cols) {
                if (a.bf)
                    Lane<__bf16>::put(out + x * 2, y);
                else
                    Lane<float>::put(out + x * 4, y);
            }
        }
    }
}

struct BiasArgs {
    void* out[kBatch];
    int64_t rows[kBatch];
    char* work;
    int64_t stride, at_db;
    int64_t padded, first;  // classes of a part; first class of the piece
    int32_t count, tile, bf;
    float scale;
};

// dbias of a piece's classes from the waves' sums, in a fixed order.
__global__ void __launch_bounds__(256) loss_bias_kernel(const BiasArgs a) {
    const int k = blockIdx.y, v = blockIdx.x * 256 + threadIdx.x;
    if (v >= a.count) return;
    const float* parts = reinterpret_cast<const float*>(a.work + k * a.stride + a.at_db) + v;
    const int n = static_cast<int>((a.rows[k] + a.tile - 1) / a.tile * 2);
    float s = 0.0f;
#pragma unroll 4
    for (int p = 0; p < n; ++p) s += parts[p * a.padded];
    const uintptr_t out = reinterpret_cast<uintptr_t>(a.out[k]) + (a.first + v) * (a.bf ? 2 : 4);
    if (a.bf)
        Lane<__bf16>::put(out, s * a.scale);
    else
        Lane<float>::put(out, s * a.scale);
}

// A worker without rows has gradients of zero.
__global__ void __launch_bounds__(256) loss_zero_kernel(void* out, int64_t n, int bf) {
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * 256) {
        if (bf)
            Lane<__bf16>::put(reinterpret_cast<uintptr_t>(out) + i * 2, 0.0f);
        else
            Lane<float>::put(reinterpret_cast<uintptr_t>(out) + i * 4, 0.0f);
    }
}

// -------------------------------------------------------------------- the plan

// What a call takes, from its sizes and types alone.
struct Plan {
    bool bf;                   // bfloat16 rows and weight
    int planes_x, planes_w;    // of the logits' operands
    int planes_g, planes_wt;   // of dx's
    int planes_gt, planes_xt;  // of dweight's
    int64_t rows, rows_p, cols_p, steps;  // most rows of a worker, padded to 256, columns to 256, 32's
    int64_t piece, pieces;     // classes at a time
    int64_t joined;            // pieces whose pairs are joined at a time
    int batch;                 // workers at a time
    int tile, cuts;            // of the logits; parts of their sum
    int tile_g;                // of the gradients' products
    int splits;                // of the sum of dx
    bool sums_dx;              // which is added up before it is rounded
    int splits_w;              // and of dweight; 0: it is written as it is computed
    // offsets in a worker's part of the workspace
    int64_t at_rows, at_parts, at_own, at_pairs, at_run, at_xz, at_wz, at_xt, at_wt, at_g, at_gt, at_sums, at_sums_w, at_acc, at_db, stride;
};

// Workspace of a batch of workers: enough for a piece whose products fill the
// chip many times over.
constexpr int64_t kRoom = int64_t{2} << 30;
constexpr int kTilesPair = 128;  // classes of the smallest tile of pairs
// And a worker's of pairs, which would grow with the rows and the classes (2^20
// rows over 2^18: 16 GiB).  A piece's fit it, so that it has 2^18 tiles at most:
// HIP takes fewer than 2^24 workgroups of 256 along x.
constexpr int64_t kPairs = int64_t{256} << 20;
constexpr int64_t kChunk = 64;   // rows that count as few
constexpr int kMostChunks = 8;   // of a worker's rows

Plan plan_of(int K, const int64_t* rows, int64_t cols, int64_t classes, int dtype, int w_dtype, bool backward, int dw_dtype) {
    Plan p{};
    p.bf = dtype == TC_BF16 && w_dtype == TC_BF16;
    p.planes_x = dtype == TC_BF16 ? 1 : 2;
    p.planes_w = w_dtype == TC_BF16 ? 1 : 2;
    p.planes_g = dtype == TC_BF16 ? 1 : 2;
    // (an operand has its 22 bits whatever the result is rounded to: where the sums
    // cancel, the weight's common part in dx, its lower half is all that is left)
    p.planes_wt = p.planes_w;
    p.planes_gt = dw_dtype == TC_BF16 ? 1 : 2;
    p.planes_xt = p.planes_x;
    for (int k = 0; k < K; ++k) p.rows = std::max(p.rows, rows[k]);
    p.rows_p = round_up(p.rows, 256);
    p.cols_p = round_up(cols, 256);
    p.steps = round_up(cols, 64) / 32;
    // classes of a piece by the bytes that one takes, most of them the panels of
    // g and of the weight
    const int64_t all = round_up(classes, 256);
    int64_t each = p.steps * kLine * p.planes_w;
    if (backward) each += 2 * p.rows_p * (p.planes_g + p.planes_gt) + 2 * p.cols_p * p.planes_wt;
    // forward, what stays in the last-level cache, unless that is too few tiles
    int64_t room = kRoom;
    if (!backward) room = std::min(kRoom, std::max(kRoom / 16, each * 256 * (1024 / std::max<int64_t>(1, p.rows_p / 256))));
    p.piece = std::min(all, std::max<int64_t>(1024, room / each / 256 * 256));
    const int64_t tile_pairs = std::max<int64_t>(256, p.rows_p) * 8;  // bytes
    if (!backward) p.piece = std::min(p.piece, kPairs / tile_pairs * kTilesPair / 256 * 256);
    p.pieces = (all + p.piece - 1) / p.piece;
    p.piece = round_up((all + p.pieces - 1) / p.pieces, 256);
    // Tiles of 256 or 128.  A CU makes about as much of two small ones (0.9) as of
    // a large one, whose operands are read less often, but the padding of the
    // sides differs; and two workgroups cover for each other's beginnings and
    // ends, which count where sums are short (stages: 8,192 rows of 4,096 over
    // 131,072 classes, 128 of them, 7.65 ms with 256 and 8.6 with 128; 7,158 of 307
    // over 12,827, 20, 1,055 us and 1,020; backward, where ends are longer, 901 of
    // 1,003 over 30,011, 64, 974 and 951).  128 also where larger ones would leave
    // CUs idle; and where tiles are few their sums are cut, so that every CU has
    // two.
    int64_t with = 0;
    for (int k = 0; k < K; ++k) with += rows[k] > 0;
    with = std::max<int64_t>(1, std::min<int64_t>(with, kBatch));
    auto tiles = [](int64_t t, int64_t down, int64_t across) { return (down + t - 1) / t * ((across + t - 1) / t); };
    const int64_t here = std::min(p.piece, classes);
    const int64_t large = tiles(256, here, p.rows), small = tiles(128, here, p.rows);
    const int64_t stages = p.steps * (p.planes_w + p.planes_x - 1);
    p.tile = large * with >= 256 && large * 4 * 0.9 <= small && stages >= (backward ? 100 : 32) ? 256 : 128;
    // A part's sums are 64 KB of a tile, which the rest reads at about the time of
    // three stages: as many parts as leave both alike.
    p.cuts = 1;
    if (p.tile == 128)
        p.cuts = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({512 / (small * with), static_cast<int64_t>(std::sqrt(0.3 * stages)), p.steps, 16})));
    if (backward) {
        const int64_t sx = round_up(here, 64) / 32 * (p.planes_g + p.planes_wt - 1), sw = round_up(p.rows, 64) / 32 * (p.planes_gt + p.planes_xt - 1);
        auto work = [&](int64_t t) { return tiles(t, p.rows, cols) * sx + tiles(t, here, cols) * sw; };
        const int64_t most = tiles(256, p.rows, cols) + tiles(256, here, cols);
        // (206 rows of 2,585 over 7,511 classes, 14 stages on average, 269 us with 256
        // and 226 with 128; 531 of 1,088 over 16,853, 55, 288 and 246; 901 of 1,003
        // over 30,011, 86, the products alone, 369 and 407)
        p.tile_g = most * with >= 256 && work(256) >= 80 * most && work(256) * 4 * 0.9 <= work(128) ? 256 : 128;
        const int64_t each = std::max<int64_t>(16, work(p.tile_g) * with / (p.tile_g == 256 ? 512 : 1024));
        p.splits = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({(sx + each - 1) / each, round_up(here, 64) / 64, 32})));
        // (sums of dweight that are cut are written and read once more)
        p.splits_w = static_cast<int>(std::min<int64_t>({sw / (2 * each), round_up(p.rows, 64) / 64, 32}));
        if (p.splits_w < 2) p.splits_w = 0;
        p.sums_dx = p.splits > 1 || p.pieces > 1;
    }
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += round_up(bytes, 256);
        return here;
    };
    p.at_parts = take(sizeof(Parts));
    p.at_rows = take(p.rows_p * 8);
    if (!backward) {
        p.at_own = take(p.rows_p * 4);
        p.joined = std::min(p.pieces, kPairs / (p.piece / kTilesPair * tile_pairs));
        p.at_pairs = take(p.joined * (p.piece / kTilesPair) * tile_pairs);
        if (p.joined < p.pieces) p.at_run = take(p.rows_p * 8);
    }
    if (p.cuts > 1) p.at_acc = take(p.cuts * small * 128 * 128 * 4);
    p.at_xz = take(p.steps * p.rows_p * kLine * p.planes_x);
    p.at_wz = take(p.steps * p.piece * kLine * p.planes_w);
    if (backward) {
        const int64_t rows_k = round_up(p.rows, 64) / 32;
        p.at_db = take(p.rows_p / 128 * 2 * p.piece * 4);
        p.at_xt = take(rows_k * p.cols_p * kLine * p.planes_xt);
        p.at_wt = take(p.piece / 32 * p.cols_p * kLine * p.planes_wt);
        p.at_g = take(p.piece / 32 * p.rows_p * kLine * p.planes_g);
        p.at_gt = take(rows_k * p.piece * kLine * p.planes_gt);
        if (p.sums_dx) p.at_sums = take(p.splits * p.rows_p * p.cols_p * 4);
        if (p.splits_w) p.at_sums_w = take(p.splits_w * p.piece * p.cols_p * 4);
    }
    p.stride = round_up(at, 4096);
    p.batch = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({K, kBatch, 2 * kRoom / p.stride})));
    return p;
}

// Runs over the sum, and each one's planes: lo hi, hi lo, hi hi.
int runs_of(int left, int right, Side& l, Side& r) {
    int n = 0;
    l.planes = r.planes = 0;
    if (left > 1) l.planes |= 1u << n++;
    if (right > 1) r.planes |= 1u << n++;
    return n + 1;
}

}  // namespace

namespace {

// Forward, rows have nothing to do with each other, so somewhat more than few of
// them are taken as several workers that share their weight, which is read again
// for each, mostly from the caches.  One worker, 128 rows of 4,096 over 32,000
// classes in bfloat16 113 us (in tiles 170), in float 350 (472), over 1,000 20
// (31) and 26 (53); 256 over 1,000 21 (33) and 37 (55), over 32,000 212 (192) and
// 680 (529); 500 over 1,000 31 (34) and 49 (65); 500 of 1,024 over 8,000 43 (39)
// and 104 (75); four workers, 256 of 4,096 over 1,000 42 (48) and 87 (109), 500
// 82 (59) and 168 (140).
struct Chunks {
    int K = 0;  // 0: they are not
    int64_t rows[TC_MAX_K * kMostChunks];
    int of[TC_MAX_K * kMostChunks];
};

void chunks_of(Chunks& c, int K, const int64_t* rows, int64_t cols, int64_t classes, bool backward) {
    if (backward) return;
    int64_t most = 0, all = 0, count = 0;
    for (int k = 0; k < K; ++k) {
        most = std::max(most, rows[k]);
        all += rows[k];
        count += (rows[k] + kChunk - 1) / kChunk;
    }
    // (more than 32 would be many launches)
    const double work = static_cast<double>(all) * classes * cols;
    if (most > 2 * kChunk && (count > 32 || most > kMostChunks * kChunk || work > (most <= 4 * kChunk ? 0x1p32 : 0x1p31))) return;
    for (int k = 0; k < K; ++k)
        for (int64_t r = 0; r < rows[k]; r += kChunk) {
            c.rows[c.K] = std::min(kChunk, rows[k] - r);
            c.of[c.K++] = k;
        }
}

}  // namespace

int64_t cross_entropy_workspace(int K, const int64_t* rows, int64_t cols, int64_t classes, int dtype, int w_dtype,
                                bool backward, int dw_dtype) {
    if (few_fits(K, rows, classes)) return few_workspace(K, rows, cols, classes, dtype, w_dtype, backward, dw_dtype);
    Chunks chunks;
    chunks_of(chunks, K, rows, cols, classes, backward);
    if (chunks.K) return few_workspace(chunks.K, chunks.rows, cols, classes, dtype, w_dtype, backward, dw_dtype);
    const Plan p = plan_of(K, rows, cols, classes, dtype, w_dtype, backward, dw_dtype);
    return p.batch * p.stride;
}

namespace {

template <int TILE, bool GRAD, Part PART>
void run_logits(const LogitArgs& a, bool bf, int n, hipStream_t s) {
    const dim3 grid(static_cast<uint32_t>(a.tiles_v) * a.tiles_r, n, PART == kSums ? a.splits : 1);
    if (bf)
        loss_logit_kernel<TILE, true, GRAD, PART><<<grid, 256, 0, s>>>(a);
    else
        loss_logit_kernel<TILE, false, GRAD, PART><<<grid, 256, 0, s>>>(a);
}
template <bool GRAD>
hipError_t run_logits(const LogitArgs& a, int tile, bool bf, int n, hipStream_t s) {
    if (tile == 256) {
        run_logits<256, GRAD, kWhole>(a, bf, n, s);
    } else if (a.splits == 1) {
        run_logits<128, GRAD, kWhole>(a, bf, n, s);
    } else {
        run_logits<128, false, kSums>(a, bf, n, s);
        if (hipError_t e = hipGetLastError()) return e;
        run_logits<128, GRAD, kRest>(a, bf, n, s);
    }
    return hipGetLastError();
}

hipError_t launch_chunks(const LossCall& c, const Chunks& chunks, hipStream_t s) {
    constexpr int kMost = TC_MAX_K * kMostChunks;
    const void *x[kMost], *weight[kMost], *bias[kMost];
    const int64_t* label[kMost];
    float *loss[kMost], *lse[kMost];
    int list[kMost];
    int64_t r = 0;
    for (int i = 0; i < chunks.K; ++i) {
        const int k = chunks.of[i];
        r = i && chunks.of[i - 1] == k ? r + kChunk : 0;
        x[i] = static_cast<const char*>(c.x[k]) + r * c.x_ld * (c.dtype == TC_BF16 ? 2 : 4);
        weight[i] = c.weight[k];
        bias[i] = c.bias ? c.bias[k] : nullptr;
        label[i] = c.label[k] + r;
        loss[i] = c.loss[k] + r;
        lse[i] = c.lse[k] + r;
        list[i] = i;
    }
    LossCall d = c;
    d.K = chunks.K;
    d.rows = chunks.rows;
    d.x = x;
    d.weight = weight;
    if (c.bias) d.bias = bias;
    d.label = label;
    d.loss = loss;
    d.lse = lse;
    return launch_few(d, list, chunks.K, s);
}

}  // namespace

hipError_t launch_cross_entropy(const LossCall& c, hipStream_t s) {
    const bool back = c.backward;
    const int x_bf = c.dtype == TC_BF16, w_bf = c.w_dtype == TC_BF16, dw_bf = c.dw_dtype == TC_BF16;
    const int we = w_bf ? 2 : 4, dwe = dw_bf ? 2 : 4;
    const int64_t cols = c.cols, classes = c.classes;
    const int32_t has_dloss = c.dloss != nullptr;
    char* const work = static_cast<char*>(c.workspace);
    // workers with rows; those without have gradients of zero
    int list[TC_MAX_K], count = 0;
    for (int k = 0; k < c.K; ++k) {
        if (c.rows[k]) {
            list[count++] = k;
        } else if (back) {
            loss_zero_kernel<<<1024, 256, 0, s>>>(c.dweight[k], classes * cols, dw_bf);
            if (c.dbias) loss_zero_kernel<<<64, 256, 0, s>>>(c.dbias[k], classes, dw_bf);
            if (hipError_t e = hipGetLastError()) return e;
        }
    }
    if (few_fits(c.K, c.rows, classes)) return launch_few(c, list, count, s);
    Chunks chunks;
    chunks_of(chunks, c.K, c.rows, cols, classes, back);
    if (chunks.K) return launch_chunks(c, chunks, s);
    const Plan p = plan_of(c.K, c.rows, cols, classes, c.dtype, c.w_dtype, back, c.dw_dtype);
    for (int k0 = 0; k0 < count; k0 += p.batch) {
        const int n = std::min(p.batch, count - k0);
        const int* who = list + k0;
        int64_t most = 0;
        for (int i = 0; i < n; ++i) most = std::max(most, c.rows[who[i]]);
        const int64_t piece = p.piece;
        if (back || !p.bf) {
            TopArgs t{};
            for (int i = 0; i < n; ++i) {
                t.x[i] = c.x[who[i]];
                t.w[i] = c.weight[who[i]];
                t.label[i] = c.label[who[i]];
                t.dloss[i] = c.dloss ? c.dloss[who[i]] : nullptr;
                t.rows[i] = c.rows[who[i]];
            }
            t.ws = work;
            t.ws_stride = p.stride;
            t.x_ld = c.x_ld;
            t.w_size = classes * cols;
            t.at_rows = p.at_rows;
            t.at_parts = p.at_parts;
            t.classes = classes;
            t.cols = static_cast<int32_t>(cols);
            t.x_bf = x_bf;
            t.w_bf = w_bf;
            t.has_dloss = has_dloss;
            t.backward = back;
            loss_top_kernel<<<dim3(2 * kParts, n), 256, 0, s>>>(t);
            if (hipError_t e = hipGetLastError()) return e;
        }
        for (int64_t v0 = 0; v0 < classes; v0 += piece) {
            const int64_t here = std::min(piece, classes - v0);
            // the panels: x's once, the weight's of this piece
            PanelArgs a{};
            Panels &x = a.x, &w = a.w;
            for (int i = 0; i < n; ++i) {
                x.p[i] = c.x[who[i]];
                x.rows[i] = c.rows[who[i]];
                w.p[i] = static_cast<const char*>(c.weight[who[i]]) + v0 * cols * we;
                w.rows[i] = here;
            }
            a.ws = work;
            a.ws_stride = p.stride;
            a.at_rows = p.at_rows;
            a.at_parts = p.at_parts;
            a.cols = static_cast<int32_t>(cols);
            const int32_t tiles_c = static_cast<int32_t>(p.steps / 2);
            x.at = p.at_xz;
            x.at_t = back ? p.at_xt : -1;
            x.plane = p.steps * p.rows_p * kLine;
            x.plane_t = round_up(p.rows, 64) / 32 * p.cols_p * kLine;
            x.padded = p.rows_p;
            x.ld = c.x_ld;
            x.planes = p.planes_x;
            x.planes_t = p.planes_xt;
            x.bf = x_bf;
            x.by_rows = 1;
            w.at = p.at_wz;
            w.at_t = back ? p.at_wt : -1;
            w.plane = p.steps * p.piece * kLine;
            w.plane_t = p.piece / 32 * p.cols_p * kLine;
            w.padded = p.piece;
            w.ld = cols;
            w.planes = p.planes_w;
            w.planes_t = p.planes_wt;
            w.bf = w_bf;
            x.raw = w.raw = p.bf;
            x.padded_t = w.padded_t = p.cols_p;
            x.tiles_c = w.tiles_c = tiles_c;
            w.first = v0 == 0 ? static_cast<int32_t>((most + 63) / 64) * tiles_c : 0;
            const GridXY panels = grid_of(w.first + (here + 63) / 64 * tiles_c, 256);
            loss_panel_kernel<<<dim3(panels.x, n, panels.y), 256, 0, s>>>(a);
            if (hipError_t e = hipGetLastError()) return e;
            // the logits
            LogitArgs l{};
            for (int i = 0; i < n; ++i) {
                const int k = who[i];
                l.bias[i] = c.bias ? c.bias[k] : nullptr;
                l.label[i] = c.label[k];
                l.lse[i] = back ? c.lse_in[k] : nullptr;
                l.rows[i] = c.rows[k];
            }
            l.at_w = p.at_wz;
            l.at_x = p.at_xz;
            l.ws = {p.piece * kLine, w.plane, 0};
            l.xs = {p.rows_p * kLine, x.plane, 0};
            l.runs = runs_of(p.planes_w, p.planes_x, l.ws, l.xs);
            l.work = work;
            l.stride = p.stride;
            l.at_rows = p.at_rows;
            l.at_parts = p.at_parts;
            l.at_g = p.at_g;
            l.at_gt = p.at_gt;
            const int64_t plane_g = p.piece / 32 * p.rows_p * kLine, plane_gt = round_up(p.rows, 64) / 32 * p.piece * kLine;
            l.plane_g = plane_g;
            l.plane_gt = plane_gt;
            l.at_pairs = p.at_pairs;
            l.at_own = p.at_own;
            l.padded = p.piece;
            l.padded_r = p.rows_p;
            l.first = v0;
            l.classes = static_cast<int32_t>(classes);
            l.count = static_cast<int32_t>(here);
            l.steps = static_cast<int32_t>(p.steps);
            l.scaled = !p.bf;
            l.w_bf = w_bf;
            l.planes_g = p.planes_g;
            l.planes_gt = p.planes_gt;
            l.has_dloss = has_dloss;
            const int tile = p.tile;
            const int64_t index = v0 / piece;
            const bool last = v0 + piece >= classes;
            if (!back) l.pair_tile = index % p.joined * (piece / tile);
            l.tiles_v = static_cast<int32_t>((here + tile - 1) / tile);
            l.tiles_r = static_cast<int32_t>((most + tile - 1) / tile);
            l.at_acc = p.at_acc;
            l.at_db = c.dbias ? p.at_db : -1;
            l.splits = p.cuts;
            if (hipError_t e = back ? run_logits<true>(l, tile, p.bf, n, s) : run_logits<false>(l, tile, p.bf, n, s)) return e;
            if (!back) {
                if (!last && (index + 1) % p.joined) continue;
                LossArgs o{};
                for (int i = 0; i < n; ++i) {
                    o.label[i] = c.label[who[i]];
                    o.loss[i] = c.loss[who[i]];
                    o.lse[i] = c.lse[who[i]];
                    o.rows[i] = c.rows[who[i]];
                }
                o.work = work;
                o.stride = p.stride;
                o.at_pairs = p.at_pairs;
                o.at_own = p.at_own;
                o.at_run = p.at_run;
                o.first = index < p.joined;
                o.last = last;
                o.padded_r = p.rows_p;
                o.tiles = static_cast<int32_t>(l.pair_tile) + l.tiles_v;
                o.classes = l.classes;
                loss_join_kernel<<<dim3(static_cast<uint32_t>((most + 63) / 64), n), 1024, 0, s>>>(o);
                if (hipError_t e = hipGetLastError()) return e;
                continue;
            }
            if (c.dbias) {
                BiasArgs b{};
                for (int i = 0; i < n; ++i) {
                    b.out[i] = c.dbias[who[i]];
                    b.rows[i] = c.rows[who[i]];
                }
                b.work = work;
                b.stride = p.stride;
                b.at_db = p.at_db;
                b.padded = p.piece;
                b.first = v0;
                b.count = l.count;
                b.tile = tile;
                b.bf = dw_bf;
                b.scale = c.scale;
                loss_bias_kernel<<<dim3(static_cast<uint32_t>((here + 255) / 256), n), 256, 0, s>>>(b);
                if (hipError_t e = hipGetLastError()) return e;
            }
            // both products of g: dx adds the pieces up, dweight is the piece's own
            GradArgs g{};
            GradJob &dx = g.job[0], &dw = g.job[1];
            const int tile2 = p.tile_g;
            const int32_t down = static_cast<int32_t>((cols + tile2 - 1) / tile2);
            dx.at_left = p.at_wt;
            dx.at_right = p.at_g;
            dx.left = {p.cols_p * kLine, w.plane_t, 0};
            dx.right = {p.rows_p * kLine, plane_g, 0};
            dx.runs = runs_of(p.planes_wt, p.planes_g, dx.left, dx.right);
            dx.at_sums = p.sums_dx ? p.at_sums : -1;
            dx.bf = x_bf;
            dx.out_ld = c.dx_ld;
            dw.out_ld = cols;
            dx.sums_stride = p.rows_p * p.cols_p * 4;
            dx.across = static_cast<int32_t>((most + tile2 - 1) / tile2);
            dx.splits = p.splits;
            dx.steps = static_cast<int32_t>((here + 63) / 64 * 2);
            dx.add = v0 > 0;
            dw.at_left = p.at_xt;
            dw.at_right = p.at_gt;
            dw.left = {p.cols_p * kLine, x.plane_t, 0};
            dw.right = {p.piece * kLine, plane_gt, 0};
            dw.runs = runs_of(p.planes_xt, p.planes_gt, dw.left, dw.right);
            dw.at_sums = p.splits_w ? p.at_sums_w : -1;
            dw.sums_stride = p.piece * p.cols_p * 4;
            dw.across = static_cast<int32_t>((here + tile2 - 1) / tile2);
            dw.splits = std::max(1, p.splits_w);
            dw.by_rows = 1;
            dw.bf = dw_bf;
            for (int i = 0; i < n; ++i) {
                g.x_rows[i] = dx.rows[i] = c.rows[who[i]];
                dx.out[i] = c.dx[who[i]];
                dw.out[i] = static_cast<char*>(c.dweight[who[i]]) + v0 * cols * dwe;
                dw.rows[i] = here;
            }
            dx.down = dw.down = down;
            dx.padded = dw.padded = static_cast<int32_t>(p.cols_p);
            dw.first = dx.down * dx.across * dx.splits;
            g.work = work;
            g.stride = p.stride;
            g.at_parts = p.at_parts;
            g.at_rows = p.at_rows;
            g.scale = c.scale;
            g.cols = static_cast<int32_t>(cols);
            g.has_dloss = has_dloss;
            const dim3 grid(dw.first + dw.down * dw.across * dw.splits, n);
            if (tile2 == 256)
                loss_grad_kernel<256><<<grid, 256, 0, s>>>(g);
            else
                loss_grad_kernel<128><<<grid, 256, 0, s>>>(g);
            if (hipError_t e = hipGetLastError()) return e;
            // results from the partial sums
            for (int which = 0; which < 2; ++which) {
                if (which ? !last || !p.sums_dx : !p.splits_w) continue;
                FinishArgs f{};
                for (int i = 0; i < n; ++i) {
                    f.out[i] = which ? c.dx[who[i]] : dw.out[i];
                    f.rows[i] = which ? c.rows[who[i]] : here;
                    f.x_rows[i] = c.rows[who[i]];
                }
                f.work = work;
                f.stride = p.stride;
                f.at_sums = which ? dx.at_sums : dw.at_sums;
                f.sums_stride = which ? dx.sums_stride : dw.sums_stride;
                f.at_rows = p.at_rows;
                f.at_parts = p.at_parts;
                f.ld = which ? c.dx_ld : cols;
                f.padded = dx.padded;
                f.splits = which ? dx.splits : dw.splits;
                f.cols = g.cols;
                f.bf = which ? x_bf : dw_bf;
                f.has_dloss = has_dloss;
                f.weight = !which;
                f.scale = c.scale;
                const int64_t vectors = (which ? most : here) * ((cols + 3) / 4);
                loss_finish_kernel<<<dim3(static_cast<uint32_t>(std::min<int64_t>((vectors + 255) / 256, 4096)), n), 256, 0, s>>>(f);
                if (hipError_t e = hipGetLastError()) return e;
            }
        }
    }
    return hipSuccess;
}

}  // namespace tc
