// The momentum update of K copies of a group with its matrices orthogonalised
// by Newton-Schulz steps.
//
// For a matrix of the group, u its gradient or momentum update and S its
// scale:  X = u / (|u| + eps), then per step, with A = X X^T (of the shorter
// side),
//     X <- a X + b A X + c A^2 X = P X,    P = a I + b A + c A^2,
// and out = S X.  Two steps take one product of the long side: every
// polynomial in A commutes with A, so the next Gram matrix is P A P, and
//     A1 = P (P A),   P1 = a I + b A1 + c A1^2,   X <- (P1 P) X.
// An m x n matrix, m <= n, takes 3 m^2 n + 5 m^3 operations for two steps this
// way (products with a symmetric result at half: only the tiles on and below
// the diagonal are computed, and stored twice) where one at a time takes
// 6 m^2 n + 2 m^3.  A third step from the same Gram matrix would not hold: the
// rounding of A grows by a^2 a step relative to the small eigenvalues, and
// turns them negative.
//
// Arithmetic.  The products run on the matrix cores in binary16 with binary32
// sums, each operand held as the sum of two binary16 values (hi = the nearest,
// lo = the nearest to the rest): hi hi + hi lo + lo hi leaves out only lo lo,
// 2^-22 of a term, which is binary32's accuracy at a third of binary16's rate
// (binary32 matrix instructions run at a sixteenth).  Binary16's range is
// enough because the iteration bounds its values: |X| and X X^T are held times
// 2^12 (up to 16, smallest step 2^-36), P and products of P times 2^8 (up to
// 255); coefficients that leave these ranges are refused on the host.
//
// Layout.  A matrix in the workspace is rows of blocks of 32 elements, 64
// bytes of hi followed by 64 bytes of lo, padded with zeros to multiples of a
// tile, so the products have no edges.  X is held both ways, [m][n] for X X^T
// and [n][m] for P X: in both products the operands' rows then run along the
// summed axis.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "tc_internal.h"

namespace tc {

// One tensor of the group.  Offsets in the workspace are in bytes from the
// copy's start.
struct OrthoMat {
    int64_t at;          // first element in a flat buffer
    int64_t size;        // elements
    int32_t rows, cols;  // as stored
    int32_t m, n;        // m <= n: X is rows x cols, or its transpose (flip)
    int32_t mp, np;      // padded
    int32_t flip;
    float scale;
    int64_t x, xt[2];    // X [mp][np], its transpose [np][mp] (two, in turn)
    int64_t s[3];        // symmetric [mp][mp] matrices
    int32_t chunk0, chunks;  // partial sums of |u|^2
    int32_t index;           // of the matrix among the matrices
};

struct OrthoTile {
    int32_t mat, i, j;
};

}  // namespace tc

struct tc_ortho {
    const tc_group* g = nullptr;
    int32_t K = 0;
    int32_t matrices = 0;
    int64_t copy_bytes = 0;  // of the workspace
    int64_t sums = 0;        // offset of the partial sums in a copy's workspace
    int64_t norms = 0;       // and of the matrices' factors
    std::vector<tc::OrthoMat> mats;
    std::vector<int32_t> of;  // tensor of each matrix
    // chunks of the flat buffer; 64 x 64 tiles of X; tiles on and below the
    // diagonal, longest sums along n first, and along m first; tiles of P X
    int32_t nchunks = 0, nsplit = 0, nsym = 0, napply = 0;
    void* d_blob = nullptr;
    const tc::OrthoMat* d_mats = nullptr;
    const int32_t* d_of = nullptr;
    const tc::OrthoTile* d_chunks = nullptr;  // mat, first element / kChunk, -
    const tc::OrthoTile* d_split = nullptr;
    const tc::OrthoTile* d_gram = nullptr;
    const tc::OrthoTile* d_sym = nullptr;
    const tc::OrthoTile* d_apply = nullptr;
};

namespace tc {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kChunk = 4096;  // elements of a workgroup of the first pass
constexpr int kTile = 128;    // rows and columns of a product's tile
constexpr int kBlock = 32;    // elements of a block of hi and lo
constexpr float kScaleX = 4096.0f, kScaleP = 256.0f;
constexpr int kCopies = TC_MAX_K;

// ------------------------------------------------ momentum and the matrix norm

struct UpdateArgs {
    const void* g[kCopies];
    float* m[kCopies];
    void* out[kCopies];
    const OrthoMat* mats;
    const OrthoTile* chunks;
    char* ws;
    int64_t copy_bytes, sums;
    float mu;
    int32_t nesterov, g_dtype, out_dtype, momentum;
};

__device__ __forceinline__ float load_any(uintptr_t p, int dtype, int64_t i) {
    return dtype == TC_BF16 ? __uint_as_float(static_cast<uint32_t>(gld<uint16_t>(p + i * 2)) << 16) : gld<float>(p + i * 4);
}

__device__ __forceinline__ void store_any(uintptr_t p, int dtype, int64_t i, float v) {
    if (dtype == TC_BF16)
        gst<__bf16>(p + i * 2, static_cast<__bf16>(v));
    else
        gst<float>(p + i * 4, v);
}

// The update from a gradient and a momentum that has it in already.
__device__ __forceinline__ float update_of(float g, float m, float mu, int nesterov) { return nesterov ? fmaf(mu, m, g) : m; }

// m <- mu m + g; of matrices the sum of u^2 over the chunk, in binary64 (so
// that no binary32 gradient over- or underflows); of other tensors out = S u.
__global__ void __launch_bounds__(256) ortho_update_kernel(const UpdateArgs a) {
    __shared__ double lds[4];
    const OrthoTile c = a.chunks[blockIdx.x];
    const OrthoMat& t = a.mats[c.mat];
    const int k = blockIdx.y;
    const int64_t first = t.at + static_cast<int64_t>(c.i) * kChunk;
    const int64_t end = min(first + kChunk, t.at + t.size);
    const uintptr_t g = reinterpret_cast<uintptr_t>(a.g[k]), m = reinterpret_cast<uintptr_t>(a.m[k]);
    double sum = 0.0;
    for (int64_t e = first + threadIdx.x; e < end; e += 256) {
        float u = load_any(g, a.g_dtype, e);
        if (a.momentum) {
            const float v = fmaf(a.mu, gld<float>(m + e * 4), u);
            gst<float>(m + e * 4, v);
            u = update_of(u, v, a.mu, a.nesterov);
        }
        if (t.m == 0)
            store_any(reinterpret_cast<uintptr_t>(a.out[k]), a.out_dtype, e, t.scale * u);
        else
            sum = fma(static_cast<double>(u), static_cast<double>(u), sum);
    }
    if (t.m == 0) return;
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) sum += __shfl_xor(sum, s, 64);
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = sum;
    __syncthreads();
    if (threadIdx.x == 0)
        *reinterpret_cast<double*>(a.ws + k * a.copy_bytes + a.sums + (t.chunk0 + c.i) * 8) = (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// The factor kScaleX / (|u| + eps) of every matrix.
__global__ void __launch_bounds__(256) ortho_norm_kernel(const OrthoMat* mats, const int32_t* of, char* ws, int64_t copy_bytes,
                                                         int64_t sums, int64_t norms, float eps) {
    __shared__ double lds[4];
    const OrthoMat& t = mats[of[blockIdx.x]];
    char* base = ws + blockIdx.y * copy_bytes;
    const double* part = reinterpret_cast<const double*>(base + sums) + t.chunk0;
    double sum = 0.0;
    for (int i = threadIdx.x; i < t.chunks; i += 256) sum += part[i];
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) sum += __shfl_xor(sum, s, 64);
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = sum;
    __syncthreads();
    if (threadIdx.x == 0)
        reinterpret_cast<double*>(base + norms)[blockIdx.x] =
            static_cast<double>(kScaleX) / (sqrt((lds[0] + lds[1]) + (lds[2] + lds[3])) + static_cast<double>(eps));
}

// ------------------------------------------------------------------- splitting

struct Split {
    _Float16 hi, lo;
};

__device__ __forceinline__ Split split(float v) {
    const _Float16 hi = static_cast<_Float16>(v);
    return {hi, static_cast<_Float16>(v - static_cast<float>(hi))};
}

// X and its transpose from u: 64 x 64 tiles through LDS.
__global__ void __launch_bounds__(256) ortho_split_kernel(const UpdateArgs a, const OrthoTile* tiles, int64_t norms) {
    __shared__ uint32_t lds[64][65];
    const OrthoTile c = tiles[blockIdx.x];
    const OrthoMat& t = a.mats[c.mat];
    const int k = blockIdx.y;
    char* base = a.ws + k * a.copy_bytes;
    const double inv = reinterpret_cast<const double*>(base + norms)[t.index];
    const uintptr_t g = reinterpret_cast<uintptr_t>(a.g[k]), m = reinterpret_cast<uintptr_t>(a.m[k]);
    // the tile in the order of the source: its rows are X's, or X^T's
    const int r0 = (t.flip ? c.j : c.i) * 64, c0 = (t.flip ? c.i : c.j) * 64;
    for (int q = threadIdx.x; q < 64 * 64; q += 256) {
        const int r = q / 64, e = q % 64;
        float v = 0.0f;
        if (r0 + r < t.rows && c0 + e < t.cols) {
            const int64_t i = t.at + static_cast<int64_t>(r0 + r) * t.cols + c0 + e;
            float u = load_any(g, a.g_dtype, i);
            if (a.momentum) u = update_of(u, gld<float>(m + i * 4), a.mu, a.nesterov);
            v = static_cast<float>(static_cast<double>(u) * inv);
        }
        const Split s = split(v);
        lds[r][e] = __builtin_bit_cast(uint16_t, s.hi) | static_cast<uint32_t>(__builtin_bit_cast(uint16_t, s.lo)) << 16;
    }
    __syncthreads();
    // 16 elements a lane, in both orders
    const int r = threadIdx.x / 4, e0 = threadIdx.x % 4 * 16;
#pragma unroll
    for (int turned = 0; turned < 2; ++turned) {
        uint32_t hi[8], lo[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const uint32_t v0 = turned ? lds[e0 + 2 * q][r] : lds[r][e0 + 2 * q];
            const uint32_t v1 = turned ? lds[e0 + 2 * q + 1][r] : lds[r][e0 + 2 * q + 1];
            hi[q] = (v0 & 0xffffu) | v1 << 16;
            lo[q] = v0 >> 16 | (v1 & 0xffff0000u);
        }
        // rows of the source are rows of X unless flipped
        const bool to_x = (turned != 0) == (t.flip != 0);
        const int row = (to_x ? c.i : c.j) * 64 + r, col = (to_x ? c.j : c.i) * 64 + e0;
        const int64_t ld = static_cast<int64_t>(to_x ? t.np : t.mp) * 4;
        char* p = base + (to_x ? t.x : t.xt[0]) + row * ld + col / kBlock * 128 + col % kBlock * 2;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            *reinterpret_cast<u32x4*>(p + q * 16) = u32x4{hi[4 * q], hi[4 * q + 1], hi[4 * q + 2], hi[4 * q + 3]};
            *reinterpret_cast<u32x4*>(p + 64 + q * 16) = u32x4{lo[4 * q], lo[4 * q + 1], lo[4 * q + 2], lo[4 * q + 3]};
        }
    }
}

// -------------------------------------------------------------------- products

enum Kind {
    kGram,   // A = X X^T
    kPoly,   // P = a I + b A + c A A
    kMul,    // symmetric product of two commuting matrices
    kApply,  // X <- Q X, both ways
    kFinal   // out = S Q X
};

struct GemmArgs {
    const OrthoMat* mats;
    const OrthoTile* tiles;
    char* ws;
    int64_t copy_bytes;
    int32_t left, right, dst;  // which symmetric matrix, or which transpose of X
    int32_t out_dtype;
    float a, b, c;             // kPoly
    float factor;              // of the sum, to the scale of the result
};

struct Outs {
    void* out[kCopies];
};

// Four values as two halves each, along a row of a matrix: element e and the
// next three, e a multiple of 4.
__device__ __forceinline__ void put4(char* row, int e, const float* v) {
    f16x4 hi, lo;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const Split s = split(v[i]);
        hi[i] = s.hi;
        lo[i] = s.lo;
    }
    char* p = row + e / kBlock * 128 + e % kBlock * 2;
    *reinterpret_cast<f16x4*>(p) = hi;
    *reinterpret_cast<f16x4*>(p + 64) = lo;
}

__device__ __forceinline__ void put1(char* row, int e, float v) {
    const Split s = split(v);
    char* p = row + e / kBlock * 128 + e % kBlock * 2;
    *reinterpret_cast<_Float16*>(p) = s.hi;
    *reinterpret_cast<_Float16*>(p + 64) = s.lo;
}

// One 128 x 128 tile of left right^T, both with rows along the summed axis:
// four waves with 64 x 64 each, as 2 x 2 of 32 x 32 x 16 products.  32 elements
// of the summed axis at a time, hi and lo, in two buffers of LDS: while one is
// multiplied the next block's loads are under way in registers.  A row's 128
// bytes are eight 16-byte pieces; piece p of row r lies at p ^ (r / 2 % 8), so
// that 16 lanes reading one piece each of 16 rows touch all 64 banks once.
template <int KIND>
__global__ void __launch_bounds__(256, 2) ortho_gemm_kernel(const GemmArgs a, const Outs outs) {
    __shared__ __attribute__((aligned(16))) char lds[2][2][kTile * 128];
    const OrthoTile tile = a.tiles[blockIdx.x];
    const OrthoMat& t = a.mats[tile.mat];
    const int k = blockIdx.y;
    char* base = a.ws + k * a.copy_bytes;
    const int ti = tile.i * kTile, tj = tile.j * kTile;
    // rows of the tile come from left (index in m), columns from right
    constexpr bool kLong = KIND == kApply || KIND == kFinal;
    const int len = KIND == kGram ? t.np : t.mp;  // of the summed axis
    const int64_t ld = static_cast<int64_t>(len) * 4;
    const char* left = base + (KIND == kGram ? t.x : t.s[a.left]) + ti * ld;
    const char* right = base + (KIND == kGram ? t.x : kLong ? t.xt[a.right] : t.s[a.right]) + tj * ld;
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
    const int wr = wave / 2 * 64, wc = wave % 2 * 64;
    const int row = tid / 8, piece = tid % 8;
    const int64_t src = row * ld + piece * 16;
    u32x4 ra[4], rb[4];
    auto fetch = [&](int kb) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            ra[q] = gld<u32x4>(reinterpret_cast<uintptr_t>(left + src + q * 32 * ld + static_cast<int64_t>(kb) * 128));
            rb[q] = gld<u32x4>(reinterpret_cast<uintptr_t>(right + src + q * 32 * ld + static_cast<int64_t>(kb) * 128));
        }
    };
    auto stage = [&](int buf) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int r = row + q * 32, at = r * 128 + (piece ^ (r / 2 % 8)) * 16;
            *reinterpret_cast<u32x4*>(lds[buf][0] + at) = ra[q];
            *reinterpret_cast<u32x4*>(lds[buf][1] + at) = rb[q];
        }
    };
    f32x16 acc[2][2] = {};
    const int blocks = len / kBlock;
    fetch(0);
    stage(0);
    __syncthreads();
    for (int kb = 0; kb < blocks; ++kb) {
        if (kb + 1 < blocks) fetch(kb + 1);
        const char* la = lds[kb & 1][0];
        const char* lb = lds[kb & 1][1];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            f16x8 ah[2], al[2], bh[2], bl[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = wr + i * 32 + lane % 32, q = wc + i * 32 + lane % 32, p = s * 2 + lane / 32;
                ah[i] = *reinterpret_cast<const f16x8*>(la + r * 128 + (p ^ (r / 2 % 8)) * 16);
                al[i] = *reinterpret_cast<const f16x8*>(la + r * 128 + ((p + 4) ^ (r / 2 % 8)) * 16);
                bh[i] = *reinterpret_cast<const f16x8*>(lb + q * 128 + (p ^ (q / 2 % 8)) * 16);
                bl[i] = *reinterpret_cast<const f16x8*>(lb + q * 128 + ((p + 4) ^ (q / 2 % 8)) * 16);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah[i], bl[j], acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(al[i], bh[j], acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah[i], bh[j], acc[i][j], 0, 0, 0);
                }
        }
        if (kb + 1 < blocks) stage((kb + 1) & 1);
        __syncthreads();
    }
    const int64_t ld_s = static_cast<int64_t>(t.mp) * 4;
    // a lane has rows r .. r + 3 of one column in four consecutive registers
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int r = ti + wr + i * 32 + q * 8 + lane / 32 * 4, c = tj + wc + j * 32 + lane % 32;
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = acc[i][j][q * 4 + e] * a.factor;
                if constexpr (KIND == kFinal) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (r + e < t.m && c < t.n) {
                            const int64_t at = t.flip ? static_cast<int64_t>(c) * t.cols + r + e : static_cast<int64_t>(r + e) * t.cols + c;
                            store_any(reinterpret_cast<uintptr_t>(outs.out[k]), a.out_dtype, t.at + at, v[e] * t.scale);
                        }
                } else if constexpr (KIND == kApply) {
                    put4(base + t.xt[a.dst] + static_cast<int64_t>(c) * t.mp * 4, r, v);
#pragma unroll
                    for (int e = 0; e < 4; ++e) put1(base + t.x + static_cast<int64_t>(r + e) * t.np * 4, c, v[e]);
                } else {
                    if constexpr (KIND == kPoly) {
                        // b A + a I, at the scale of P; A is symmetric
                        const char* p = base + t.s[a.left] + c * ld_s + r / kBlock * 128 + r % kBlock * 2;
                        const f16x4 hi = *reinterpret_cast<const f16x4*>(p), lo = *reinterpret_cast<const f16x4*>(p + 64);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            v[e] = fmaf(a.b, static_cast<float>(hi[e]) + static_cast<float>(lo[e]), v[e]);
                            if (r + e == c) v[e] += a.a;
                        }
                    }
                    char* d = base + t.s[a.dst];
                    put4(d + c * ld_s, r, v);
                    if (tile.i != tile.j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) put1(d + (r + e) * ld_s, c, v[e]);
                }
            }
}

// Appended to a list of tiles in the order they are launched.
void order_by(std::vector<OrthoTile>& v, const std::vector<OrthoMat>& mats, bool along_n) {
    std::stable_sort(v.begin(), v.end(), [&](const OrthoTile& x, const OrthoTile& y) {
        const OrthoMat &a = mats[x.mat], &b = mats[y.mat];
        return (along_n ? a.np : a.mp) > (along_n ? b.np : b.mp);
    });
}

int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

}  // namespace

tc_ortho* make_ortho(const tc_group* g, int32_t K, const int64_t* rows, const int64_t* cols, const float* scale, hipError_t* e) {
    *e = hipErrorOutOfMemory;
    auto* o = new (std::nothrow) tc_ortho();
    if (!o) return nullptr;
    o->g = g;
    o->K = K;
    o->mats.resize(g->n);
    std::vector<OrthoTile> chunks, split, gram, sym, apply;
    int64_t bytes = 0, sums = 0;
    auto take = [&](int64_t n) {
        const int64_t at = bytes;
        bytes += round_up(n, 256);
        return at;
    };
    for (int32_t t = 0; t < g->n; ++t) {
        OrthoMat& q = o->mats[t];
        q = OrthoMat{};
        q.at = g->offsets[t];
        q.size = g->sizes[t];
        q.scale = scale ? scale[t] : 1.0f;
        const int64_t nc = (q.size + kChunk - 1) / kChunk;
        q.chunk0 = static_cast<int32_t>(sums);
        q.chunks = static_cast<int32_t>(nc);
        for (int64_t i = 0; i < nc; ++i) chunks.push_back({t, static_cast<int32_t>(i), 0});
        if (q.size == 0 || rows[t] == 0) continue;
        sums += nc;
        q.rows = static_cast<int32_t>(rows[t]);
        q.cols = static_cast<int32_t>(cols[t]);
        q.flip = q.rows > q.cols;
        q.m = std::min(q.rows, q.cols);
        q.n = std::max(q.rows, q.cols);
        q.mp = static_cast<int32_t>(round_up(q.m, kTile));
        q.np = static_cast<int32_t>(round_up(q.n, kTile));
        q.index = o->matrices++;
        o->of.push_back(t);
        const int64_t x = static_cast<int64_t>(q.mp) * q.np * 4, s = static_cast<int64_t>(q.mp) * q.mp * 4;
        q.x = take(x);
        q.xt[0] = take(x);
        q.xt[1] = take(x);
        for (auto& v : q.s) v = take(s);
        for (int32_t i = 0; i < q.mp / 64; ++i)
            for (int32_t j = 0; j < q.np / 64; ++j) split.push_back({t, i, j});
        for (int32_t i = 0; i < q.mp / kTile; ++i)
            for (int32_t j = 0; j <= i; ++j) sym.push_back({t, i, j});
        for (int32_t j = 0; j < q.np / kTile; ++j)
            for (int32_t i = 0; i < q.mp / kTile; ++i) apply.push_back({t, i, j});
    }
    o->sums = take(sums * 8);
    o->norms = take(static_cast<int64_t>(o->matrices) * 8);
    o->copy_bytes = bytes;
    gram = sym;
    order_by(gram, o->mats, true);
    order_by(sym, o->mats, false);
    order_by(apply, o->mats, false);
    o->nchunks = static_cast<int32_t>(chunks.size());
    o->nsplit = static_cast<int32_t>(split.size());
    o->nsym = static_cast<int32_t>(sym.size());
    o->napply = static_cast<int32_t>(apply.size());
    for (const auto* v : {&chunks, &split, &gram, &apply})
        if (v->size() >= (size_t{1} << 32) / 256) {  // workgroups of 256 in one dimension of a grid
            delete o;
            *e = hipErrorInvalidValue;
            return nullptr;
        }
    // one block of device memory for all tables
    std::vector<char> host;
    auto put = [&](const void* p, size_t n) {
        const size_t at = host.size();
        host.resize(at + (n + 255) / 256 * 256);
        if (n) std::memcpy(host.data() + at, p, n);
        return at;
    };
    const size_t at_mats = put(o->mats.data(), o->mats.size() * sizeof(OrthoMat));
    const size_t at_of = put(o->of.data(), o->of.size() * 4);
    const std::vector<OrthoTile>* lists[] = {&chunks, &split, &gram, &sym, &apply};
    size_t at[5];
    for (int i = 0; i < 5; ++i) at[i] = put(lists[i]->data(), lists[i]->size() * sizeof(OrthoTile));
    if ((*e = hipMalloc(&o->d_blob, host.size())) != hipSuccess ||
        (*e = hipMemcpy(o->d_blob, host.data(), host.size(), hipMemcpyHostToDevice)) != hipSuccess) {
        destroy_ortho(o);
        return nullptr;
    }
    const char* d = static_cast<const char*>(o->d_blob);
    o->d_mats = reinterpret_cast<const OrthoMat*>(d + at_mats);
    o->d_of = reinterpret_cast<const int32_t*>(d + at_of);
    const OrthoTile** to[] = {&o->d_chunks, &o->d_split, &o->d_gram, &o->d_sym, &o->d_apply};
    for (int i = 0; i < 5; ++i) *to[i] = reinterpret_cast<const OrthoTile*>(d + at[i]);
    return o;
}

void destroy_ortho(tc_ortho* o) {
    if (o->d_blob) (void)hipFree(o->d_blob);
    delete o;
}

const tc_group* ortho_group(const tc_ortho* o) { return o->g; }
int32_t ortho_copies(const tc_ortho* o) { return o->K; }
int64_t ortho_workspace(const tc_ortho* o) { return o->copy_bytes * o->K; }

// Whether values stay in the ranges the formats hold.  s bounds the singular
// values before a step (1 at first: |X| <= 1), and with x = s^2 the step makes
// them s |q(x)|, q = a + b x + c x^2; both extremes lie at the ends or where a
// derivative is 0.
bool ortho_in_range(int steps, const float* coeff) {
    double s = 1.0, q_before = 1.0;
    for (int i = 0; i < steps; ++i) {
        const double a = coeff[3 * i], b = coeff[3 * i + 1], c = coeff[3 * i + 2], x = s * s;
        auto q = [&](double v) { return std::fabs(a + v * (b + c * v)); };
        auto p = [&](double v) { return std::sqrt(v) * q(v); };
        double qs = std::max(q(0), q(x)), ps = p(x);
        auto at = [&](double v) {
            if (v > 0 && v < x) {
                qs = std::max(qs, q(v));
                ps = std::max(ps, p(v));
            }
        };
        if (c != 0) {
            at(-b / (2 * c));
            const double disc = 9 * b * b - 20 * a * c;
            if (disc >= 0) {
                at((-3 * b + std::sqrt(disc)) / (10 * c));
                at((-3 * b - std::sqrt(disc)) / (10 * c));
            }
        } else if (b != 0) {
            at(-a / (3 * b));
        }
        // what is stored: X X^T (x), P A (s p), P A P (p^2), P (q), P P (q q), X (p); 1/64 for rounding
        const double lim_x = 65504.0 / kScaleX * (63.0 / 64.0), lim_p = 65504.0 / kScaleP * (63.0 / 64.0);
        const bool second = i % 2 == 1;
        if (!(x <= lim_x && s * ps <= lim_x && ps * ps <= lim_x && qs <= lim_p && (!second || qs * q_before <= lim_p))) return false;
        q_before = qs;
        s = ps;
    }
    return true;
}

hipError_t launch_ortho(const tc_ortho* o, const void* const* g, int g_dtype, float* const* m, float mu, int nesterov,
                        void* const* out, int out_dtype, int steps, const float* coeff, float eps, void* workspace,
                        hipStream_t s) {
    UpdateArgs u{};
    Outs outs{};
    for (int k = 0; k < o->K; ++k) {
        u.g[k] = g[k];
        u.m[k] = m ? m[k] : nullptr;
        u.out[k] = outs.out[k] = out[k];
    }
    u.mats = o->d_mats;
    u.chunks = o->d_chunks;
    u.ws = static_cast<char*>(workspace);
    u.copy_bytes = o->copy_bytes;
    u.sums = o->sums;
    u.mu = mu;
    u.nesterov = nesterov;
    u.g_dtype = g_dtype;
    u.out_dtype = out_dtype;
    u.momentum = m != nullptr;
    const uint32_t K = o->K;
    ortho_update_kernel<<<dim3(o->nchunks, K), 256, 0, s>>>(u);
    if (o->matrices == 0) return hipGetLastError();
    ortho_norm_kernel<<<dim3(o->matrices, K), 256, 0, s>>>(o->d_mats, o->d_of, u.ws, o->copy_bytes, o->sums, o->norms, eps);
    ortho_split_kernel<<<dim3(o->nsplit, K), 256, 0, s>>>(u, o->d_split, o->norms);
    GemmArgs a{};
    a.mats = o->d_mats;
    a.ws = u.ws;
    a.copy_bytes = o->copy_bytes;
    a.out_dtype = out_dtype;
    // symmetric matrices: [0] A, then P A P, then P1 P; [1] P; [2] P A, then P1
    auto gram = [&] {
        a.tiles = o->d_gram;
        a.dst = 0;
        a.factor = 1.0f / kScaleX;
        ortho_gemm_kernel<kGram><<<dim3(o->nsym, K), 256, 0, s>>>(a, outs);
    };
    auto poly = [&](const float* c, int dst) {
        a.tiles = o->d_sym;
        a.left = a.right = 0;
        a.dst = dst;
        a.a = c[0] * kScaleP;
        a.b = c[1] * (kScaleP / kScaleX);
        a.factor = c[2] * (kScaleP / kScaleX / kScaleX);
        ortho_gemm_kernel<kPoly><<<dim3(o->nsym, K), 256, 0, s>>>(a, outs);
    };
    auto mul = [&](int left, int right, int dst) {  // left is a P
        a.tiles = o->d_sym;
        a.left = left;
        a.right = right;
        a.dst = dst;
        a.factor = 1.0f / kScaleP;
        ortho_gemm_kernel<kMul><<<dim3(o->nsym, K), 256, 0, s>>>(a, outs);
    };
    int from = 0;
    for (int i = 0; i < steps; i += 2) {
        const bool pair = i + 1 < steps, last = i + 2 >= steps;
        gram();
        poly(coeff + 3 * i, 1);
        int q = 1;
        if (pair) {
            mul(1, 0, 2);
            mul(1, 2, 0);
            poly(coeff + 3 * i + 3, 2);
            mul(2, 1, 0);
            q = 0;
        }
        a.tiles = o->d_apply;
        a.left = q;
        a.right = from;
        a.dst = from = 1 - from;
        a.factor = 1.0f / kScaleP;
        if (last) {
            a.factor /= kScaleX;
            ortho_gemm_kernel<kFinal><<<dim3(o->napply, K), 256, 0, s>>>(a, outs);
        } else {
            ortho_gemm_kernel<kApply><<<dim3(o->napply, K), 256, 0, s>>>(a, outs);
        }
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

}  // namespace tc
