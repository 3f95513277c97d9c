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
// enough because the iteration bounds its values: X and X X^T are held times
// 2^12 (up to 16, smallest step 2^-36), polynomials times 2^10 (up to 63);
// coefficients that leave these ranges are refused on the host.  Two things
// keep the products from losing what the operands hold.  P is held without its
// a I, which is added in binary32 where P is used: along the large singular
// values a I and the rest cancel, and a rounding of P's large diagonal would
// stay.  And X X^T and the symmetric products are summed in the matrix cores
// 128 terms at a time, which are added up in registers of their own: small
// terms are cut off against a large sum there.  Without that the result of
// 512 x 4,608 was 1.7e-5 off, with it 3.5e-6 (a binary32 product's iteration:
// 3.8e-6), of 200 x 20,000, one step at a time, 3.9e-6 and 0.9e-6 (2.8e-6).
// P X, whose sums are the shorter side and which is added to a X, is summed
// whole: 4,096 x 4,096 and 4,096 x 8,192 are 1.8e-6 and 2.0e-6 off so (3.3e-6
// both).  None of this goes by the other matrices of the group, nor
// does the order of a sum, so a matrix over the size that one workgroup takes
// has the same bits whatever its neighbours.
//
// Layout.  A matrix in the workspace is rows of blocks of 32 elements, 64
// bytes of hi followed by 64 bytes of lo, padded with zeros to multiples of a
// tile, so the products have no edges.  X is held both ways, [m][n] for X X^T
// and [n][m] for P X: in both products the operands' rows then run along the
// summed axis.
#include <algorithm>
#include <array>
#include <cmath>
#include <cstring>
#include <memory>
#include <new>

#include "tc_internal.h"

namespace tc {

// One tensor of the group.  Offsets in the workspace are in bytes from the
// copy's start.
struct OrthoMat {
    int64_t at;          // first element in a flat buffer
    int64_t size;        // elements
    int32_t rows, cols;  // as stored
    int32_t m, n;        // m <= n: X is rows x cols, or its transpose (flip); 0: no matrix
    int32_t mp, np;      // padded
    int32_t flip;
    int32_t pair;        // takes two steps to a Gram matrix
    float scale;
    int64_t x, xt;       // X [mp][np]; then its transpose [np][mp] (two, in
                         // turn), then three symmetric [mp][mp] matrices
    int32_t chunk0, chunks;  // partial sums of |u|^2
    int32_t index;           // of the matrix among the matrices
};

struct OrthoTile {
    int32_t mat, i, j;
    // of a product's tile: the copy, and what the product needs of the matrix
    // (a load of its own, after the tile's, would be waited for)
    int16_t copy, pair;
    int32_t mp, np;
    int64_t x;
};

// Tiles of the products of one launch, and their side.
struct OrthoList {
    const OrthoTile* d = nullptr;
    int32_t n = 0;
    int32_t side = 0;
    int32_t short_sums = 0;  // sums of up to 1,024 terms on average
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
    // small matrices, taken whole by a workgroup, in two sizes of LDS
    const int32_t* d_small[2] = {nullptr, nullptr};
    int32_t nsmall[2] = {0, 0};
    // chunks of the flat buffer; 64 x 64 tiles of X
    int32_t nchunks = 0, nsplit = 0;
    void* d_blob = nullptr;
    const tc::OrthoMat* d_mats = nullptr;
    const int32_t* d_of = nullptr;
    const tc::OrthoTile* d_chunks = nullptr;  // mat, first element / kChunk, -
    const tc::OrthoTile* d_split = nullptr;
    tc::OrthoList gram, sym, apply;  // all matrices
    tc::OrthoList sym_pair;          // those that take two steps to a Gram matrix
    tc::OrthoList gram_one, sym_one, apply_one;  // and one
};

namespace tc {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kChunk = 4096;  // elements of a workgroup of the first pass
constexpr int kTile = 128;    // rows and columns of a product's larger tile
constexpr int kBlock = 32;    // elements of a block of hi and lo
constexpr float kScaleX = 4096.0f, kScaleP = 1024.0f;
constexpr int kRun = 4;       // stages summed in the matrix cores at a time in X X^T and symmetric products
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

typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));

// Elements i .. i + n - 1 of a flat buffer, n <= 4, at any alignment.
__device__ __forceinline__ f32x4 load_four(uintptr_t p, int dtype, int64_t i, int n) {
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (n < 4) {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < n) v[e] = load_any(p, dtype, i + e);
    } else if (dtype == TC_BF16) {
        const u16x4 h = gld_u<u16x4>(p + i * 2);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(static_cast<uint32_t>(h[e]) << 16);
    } else {
        v = gld_u<f32x4>(p + i * 4);
    }
    return v;
}

__device__ __forceinline__ void store_four(uintptr_t p, int dtype, int64_t i, int n, f32x4 v) {
    if (n < 4) {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < n) store_any(p, dtype, i + e, v[e]);
    } else if (dtype == TC_BF16) {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        bf16x4 h;
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = static_cast<__bf16>(v[e]);
        gst_u<u16x4>(p + i * 2, __builtin_bit_cast(u16x4, h));
    } else {
        gst_u<f32x4>(p + i * 4, v);
    }
}

// The update from a gradient and a momentum that has it in already.
__device__ __forceinline__ float update_of(float g, float m, float mu, int nesterov) { return nesterov ? fmaf(mu, m, g) : m; }

// m <- mu m + g; of matrices the sum of u^2 over the chunk, in binary64 (so
// that no binary32 gradient over- or underflows); of other tensors out = S u.
// Bound by memory: 12 bytes an element with binary32 gradients, 5.3 TB/s on
// the ResNet-50 group, 8 copies (0.45 ms).
__global__ void __launch_bounds__(256) ortho_update_kernel(const UpdateArgs a) {
    __shared__ double lds[4];
    const OrthoTile c = a.chunks[blockIdx.x];
    const OrthoMat& t = a.mats[c.mat];
    const int k = blockIdx.y;
    const int64_t first = t.at + static_cast<int64_t>(c.i) * kChunk;
    const int left = static_cast<int>(min(static_cast<int64_t>(kChunk), t.at + t.size - first));
    const uintptr_t g = reinterpret_cast<uintptr_t>(a.g[k]), m = reinterpret_cast<uintptr_t>(a.m[k]);
    constexpr int N = kChunk / 1024;  // vectors of four elements a lane
    f32x4 u[N], v[N];
    int n[N];
#pragma unroll
    for (int q = 0; q < N; ++q) {
        const int e = (q * 256 + threadIdx.x) * 4;
        n[q] = min(4, left - e);
        if (n[q] <= 0) continue;
        u[q] = load_four(g, a.g_dtype, first + e, n[q]);
        if (a.momentum) v[q] = load_four(m, TC_F32, first + e, n[q]);
    }
    double sum = 0.0;
#pragma unroll
    for (int q = 0; q < N; ++q) {
        if (n[q] <= 0) continue;
        const int64_t e = first + (q * 256 + threadIdx.x) * 4;
        if (a.momentum) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[q][i] = fmaf(a.mu, v[q][i], u[q][i]);
                u[q][i] = update_of(u[q][i], v[q][i], a.mu, a.nesterov);
            }
            store_four(m, TC_F32, e, n[q], v[q]);
        }
        if (t.m == 0) {
            store_four(reinterpret_cast<uintptr_t>(a.out[k]), a.out_dtype, e, n[q], u[q] * t.scale);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)  // (zeros past the end)
                sum = fma(static_cast<double>(u[q][i]), static_cast<double>(u[q][i]), sum);
        }
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

__device__ __forceinline__ uint32_t pack(float v) {
    const Split s = split(v);
    return __builtin_bit_cast(uint16_t, s.hi) | static_cast<uint32_t>(__builtin_bit_cast(uint16_t, s.lo)) << 16;
}

// Eight packed values to elements e .. e + 7 of a row, e a multiple of 8.
__device__ __forceinline__ void put8(char* row, int e, const uint32_t* v) {
    u32x4 hi, lo;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        hi[i] = (v[2 * i] & 0xffffu) | v[2 * i + 1] << 16;
        lo[i] = v[2 * i] >> 16 | (v[2 * i + 1] & 0xffff0000u);
    }
    char* p = row + e / kBlock * 128 + e % kBlock * 2;
    *reinterpret_cast<u32x4*>(p) = hi;
    *reinterpret_cast<u32x4*>(p + 64) = lo;
}

// Elements e .. e + 7 of a row, and v += f times them.
struct Eight {
    f16x8 hi, lo;
};

__device__ __forceinline__ Eight get8(const char* row, int e) {
    const char* p = row + e / kBlock * 128 + e % kBlock * 2;
    return {*reinterpret_cast<const f16x8*>(p), *reinterpret_cast<const f16x8*>(p + 64)};
}

__device__ __forceinline__ void add8(const Eight& x, float f, float* v) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = fmaf(f, static_cast<float>(x.hi[i]) + static_cast<float>(x.lo[i]), v[i]);
}

// X and its transpose from u: 64 x 64 tiles through LDS, so that both are
// written in whole lines.  The update is formed again from g and m (8 bytes
// an element) rather than written by the first pass and read here (as many).
// Bound by memory: 16 bytes an element, 5.1 TB/s on the ResNet-50 group, 8
// copies (0.64 ms).
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
    f32x4 u[4], v[4];
    int n[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int r = q * 16 + threadIdx.x / 16, e = threadIdx.x % 16 * 4;
        n[q] = r0 + r < t.rows ? max(0, min(4, t.cols - c0 - e)) : 0;
        u[q] = v[q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (n[q] == 0) continue;
        const int64_t i = t.at + static_cast<int64_t>(r0 + r) * t.cols + c0 + e;
        u[q] = load_four(g, a.g_dtype, i, n[q]);
        if (a.momentum) v[q] = load_four(m, TC_F32, i, n[q]);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float w = a.momentum ? update_of(u[q][i], v[q][i], a.mu, a.nesterov) : u[q][i];
            lds[q * 16 + threadIdx.x / 16][threadIdx.x % 16 * 4 + i] = n[q] ? pack(static_cast<float>(static_cast<double>(w) * inv)) : 0;
        }
    __syncthreads();
    // eight elements a lane, in both orders
#pragma unroll
    for (int turned = 0; turned < 2; ++turned) {
        // rows of the source are rows of X unless flipped
        const bool to_x = (turned != 0) == (t.flip != 0);
        const int64_t ld = static_cast<int64_t>(to_x ? t.np : t.mp) * 4;
        for (int q = threadIdx.x; q < 64 * 8; q += 256) {
            const int r = q / 8, e0 = q % 8 * 8;
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = turned ? lds[e0 + i][r] : lds[r][e0 + i];
            const int row = (to_x ? c.i : c.j) * 64 + r, col = (to_x ? c.j : c.i) * 64 + e0;
            put8(base + (to_x ? t.x : t.xt) + row * ld, col, w);
        }
    }
}

// -------------------------------------------------------------------- products

enum Kind {
    kGram,   // X X^T
    kSym,    // product of two symmetric matrices that commute, and multiples of up to two more
    kApply,  // X <- a X + Q X, both ways
    kFinal   // out = S (a X + Q X)
};

// What a product of one kind of matrix takes: left and right are indices of
// symmetric matrices (right of kApply and kFinal: of a transpose of X), and so
// is dst.
struct Operation {
    int32_t left, right, dst;
    int32_t add[2];  // symmetric matrices added to a symmetric product; second -1: none
    float factor;    // of the product, to the scale of the result
    float f[2];      // of what is added
};

struct GemmArgs {
    const OrthoMat* mats;
    const OrthoTile* tiles;
    char* ws;
    int64_t copy_bytes;
    int32_t out_dtype;
    Operation op[2];  // of matrices that take one step to a Gram matrix, and two
};

struct Outs {
    void* out[kCopies];
};

typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(1))) const char global_char;

// Up to eight of the values to a flat buffer, from element `at` on.
__device__ __forceinline__ void put_out(void* out, int dtype, int64_t at, int left, const float* v) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int n = min(4, left - 4 * h);
        if (n > 0) store_four(reinterpret_cast<uintptr_t>(out), dtype, at + 4 * h, n, f32x4{v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]});
    }
}

// One tile of left right^T, both with rows along the summed axis, of four waves
// with a quarter each, as 32 x 32 x 16 products: 128 x 128, or 64 x 64 where
// the larger tiles would be fewer than the CUs.
//
// Measured, in TFLOP/s of binary16 products: X X^T of the VGG-16 group, 2
// copies, 790, its symmetric products 770 to 920, P X 1,000 to 1,110; of the
// ResNet-50 group, 8 copies, whose sums are a tenth as long and whose tiles are
// read and written at 2.5 TB/s meanwhile, 880, 680 and 660 to 720.  On long
// sums the card's power is a part of what bounds it: the same products without
// the loads of their operands run at 1,280 to 1,400, with the clock at 1.3 GHz.
//
// A stage is 128 bytes of each of the 2 TILE rows: a block of 32 elements, hi
// and lo.  64 KB of LDS hold two or four stages, which are loaded straight from
// memory while others are multiplied, so that a CU takes two workgroups; or
// (kOneStage) 32 KB one, nothing is loaded ahead, and four workgroups cover
// for each other.  That pays where sums are short, and beginnings and ends of
// tiles much of the time.  A row's 128 bytes are eight 16-byte pieces; piece p
// of row r lies at p ^ (r / 2 % 8), so that 16 lanes reading one piece each of
// 16 rows touch all 64 banks once.
template <int KIND, int TILE, bool kOneStage>
__global__ void __launch_bounds__(256, kOneStage ? 4 : 2) ortho_gemm_kernel(const GemmArgs a, const Outs outs) {
    constexpr int kHalf = TILE * 128, kStage = 2 * kHalf, STAGES = kOneStage ? 1 : 65536 / kStage;
    constexpr int kSide = TILE / 64, kLoads = TILE / 32;  // 32 x 32 products of a wave each way; loads of each operand
    constexpr int kSteps = kBlock / 16;  // products of 16 elements in a stage
    constexpr bool kLong = KIND == kApply || KIND == kFinal, kApart = !kLong;  // (sums of kRun stages)
    __shared__ __attribute__((aligned(16))) char lds[STAGES * kStage];
    const OrthoTile tile = a.tiles[blockIdx.x];
    const OrthoMat& t = a.mats[tile.mat];  // (read at the end, for the result)
    const Operation& op = a.op[tile.pair];
    const int k = tile.copy;
    const int64_t ld_m = static_cast<int64_t>(tile.mp) * 4, ld_n = static_cast<int64_t>(tile.np) * 4;
    char* const x = a.ws + k * a.copy_bytes + tile.x;
    const int64_t x_bytes = ld_n * tile.mp, s_bytes = ld_m * tile.mp;
    auto xt = [&](int i) { return x + (1 + i) * x_bytes; };
    auto sym = [&](int i) { return x + 3 * x_bytes + i * s_bytes; };
    const int ti = tile.i * TILE, tj = tile.j * TILE;
    // rows of the tile come from left (index in m), columns from right
    const int len = KIND == kGram ? tile.np : tile.mp;  // of the summed axis
    const uint32_t ld = static_cast<uint32_t>(len) * 4;
    const char* left = (KIND == kGram ? x : sym(op.left)) + static_cast<int64_t>(ti) * ld;
    const char* right = (KIND == kGram ? x : kLong ? xt(op.right) : sym(op.right)) + static_cast<int64_t>(tj) * ld;
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const int wr = wave / 2 * (TILE / 2), wc = wave % 2 * (TILE / 2);
    // this wave's 1,024-byte pieces of a stage: eight rows each
    uint32_t off[kLoads];
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
        const int r = (wave * kLoads + q) * 8 + lane / 8, p = (lane % 8) ^ (r / 2 % 8);
        off[q] = static_cast<uint32_t>(r) * ld + static_cast<uint32_t>(p * 16);
    }
    auto fetch = [&](int stage, int buf) {
        const int64_t at = static_cast<int64_t>(stage) * 128;
        char* to = lds + buf * kStage + wave * kLoads * 1024;
#pragma unroll
        for (int q = 0; q < kLoads; ++q)
            __builtin_amdgcn_global_load_lds((global_char*)(left + at + off[q]), (lds_char*)(to + q * 1024), 16, 0, 0);
#pragma unroll
        for (int q = 0; q < kLoads; ++q)
            __builtin_amdgcn_global_load_lds((global_char*)(right + at + off[q]), (lds_char*)(to + kHalf + q * 1024), 16, 0, 0);
    };
    f32x16 acc[kSide][kSide] = {}, sum[kApart ? kSide : 1][kApart ? kSide : 1] = {};
    struct Operands {
        f16x8 ah[kSide], al[kSide], bh[kSide], bl[kSide];
    } now, next;
    const int ra = (wr + lane % 32) * 128, rb = kHalf + (wc + lane % 32) * 128, turn = lane / 2 % 8;
    auto read = [&](Operands& f, int buf, int step) {
        const char* p = lds + buf * kStage;
        const int hi = ((step * 2 + lane / 32) ^ turn) * 16, lo = ((step * 2 + lane / 32 + 4) ^ turn) * 16;
#pragma unroll
        for (int i = 0; i < kSide; ++i) {
            f.ah[i] = *reinterpret_cast<const f16x8*>(p + ra + i * 4096 + hi);
            f.bh[i] = *reinterpret_cast<const f16x8*>(p + rb + i * 4096 + hi);
            f.al[i] = *reinterpret_cast<const f16x8*>(p + ra + i * 4096 + lo);
            f.bl[i] = *reinterpret_cast<const f16x8*>(p + rb + i * 4096 + lo);
        }
    };
    // products `from` to `to` of a step: lo hi, hi lo, hi hi of every place
    auto multiply = [&](const Operands& f, int from, int to) {
#pragma unroll
        for (int n = from; n < to; ++n) {
            constexpr int kOne = kSide * kSide;
            const int w = n / kOne, i = n / kSide % kSide, j = n % kSide;
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(w == 0 ? f.al[i] : f.ah[i], w == 1 ? f.bl[j] : f.bh[j], acc[i][j], 0, 0, 0);
        }
    };
    constexpr int kAll = kSide * kSide * 3, kFirst = (kAll + 2) / 3;
    // The loads of the oldest stage under way are done, in every wave; and
    // every wave has its operands of the stage before: without the wait for
    // them here, products and their wait could be moved past the barrier, and
    // the next loads into the buffer would run against the reads.
    auto arrive = [&] {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((STAGES > 2 ? STAGES - 2 : 0) * 2 * kLoads) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    const int stages = len / kBlock;
    if constexpr (!kOneStage) {
#pragma unroll
        for (int st = 0; st < STAGES - 1; ++st) fetch(min(st, stages - 1), st);
        arrive();
        read(now, 0, 0);
    }
    int buf = 0;
    for (int st = 0; st < stages; ++st) {
        if constexpr (kOneStage) {
            fetch(st, 0);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
#pragma unroll
            for (int step = 0; step < kSteps; ++step) {
                read(now, 0, step);
                multiply(now, 0, kAll);
            }
            // every wave has its operands before the buffer is loaded again
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            continue;
        }
        // The next step's operands are read after the first products of a
        // step, and arrive under the others (asked for before them, the wait
        // for the step's own operands would be for these too).  The buffer
        // that the stage before this one left is loaded with the stage
        // STAGES - 1 ahead (past the end the last one again, so that the count
        // of loads under way stays the same).
        if (STAGES > 2 || st + 1 < stages) fetch(min(st + STAGES - 1, stages - 1), buf == 0 ? STAGES - 1 : buf - 1);
        const int then = buf + 1 == STAGES ? 0 : buf + 1;
        multiply(now, 0, kFirst);
        __builtin_amdgcn_sched_barrier(0);
        read(next, buf, 1);
        __builtin_amdgcn_sched_barrier(0);
        multiply(now, kFirst, kAll);
        __builtin_amdgcn_sched_barrier(0);
        multiply(next, 0, kFirst);
        __builtin_amdgcn_sched_barrier(0);
        if (st + 1 < stages) {
            arrive();
            read(now, then, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        multiply(next, kFirst, kAll);
        __builtin_amdgcn_sched_barrier(0);
        buf = then;
        if constexpr (kApart) {
            if (st % kRun == kRun - 1) {  // stages is a multiple of kRun
#pragma unroll
                for (int i = 0; i < kSide; ++i)
#pragma unroll
                    for (int j = 0; j < kSide; ++j) {
                        sum[i][j] += acc[i][j];
                        acc[i][j] = f32x16{};
                    }
            }
        }
    }
    // The loads past the end are still under way, and the tile is written over
    // their buffers: each wave waits for its own, and all meet at the barrier
    // before the first of those writes.
    if constexpr (STAGES > 2) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    auto& total = [&]() -> auto& {
        if constexpr (kApart) return sum;
        else return acc;
    }();
    // The tile leaves through LDS, in one part or two of its columns, so that
    // both orders leave in whole lines: column c holds its rows as TILE / 4
    // pieces of four, piece p at p ^ (c % (TILE / 4)).  Then a lane takes eight
    // rows of a column, `kTurns` times; what is added to them is loaded while
    // the tile goes through LDS.
    constexpr int kParts = kOneStage ? 2 : 1, kPart = TILE / kParts;
    constexpr int kEights = TILE / 8, kTurns = kPart * kEights / 256;
    const int col0 = tid / kEights, r = tid % kEights * 8;
    const bool natural = kLong ? KIND == kApply || !t.flip : tile.i != tile.j;
    float* tiled = reinterpret_cast<float*>(lds);
    auto piece = [&](int c, int p) { return c * TILE + (p ^ (c % (TILE / 4))) * 4; };
#pragma unroll
    for (int part = 0; part < kParts; ++part) {
        const int tc = tj + part * kPart;  // the part's first column
        Eight extra[KIND == kSym ? 2 : 1][kOneStage ? 1 : kTurns];
        auto more = [&](int n, int to) {
            const int64_t at = (tc + col0 + n * (256 / kEights)) * ld_m;
            if constexpr (kLong) extra[0][to] = get8(xt(op.right) + at, ti + r);
            if constexpr (KIND == kSym) {
                // (a symmetric matrix: its row tc + c)
                extra[0][to] = get8(sym(op.add[0]) + at, ti + r);
                if (op.add[1] >= 0) extra[KIND == kSym][to] = get8(sym(op.add[1]) + at, ti + r);
            }
        };
        if constexpr (!kOneStage)
#pragma unroll
            for (int n = 0; n < kTurns; ++n) more(n, n);
        __syncthreads();
        if (kParts == 1 || wc == part * kPart) {
#pragma unroll
            for (int i = 0; i < kSide; ++i)
#pragma unroll
                for (int j = 0; j < kSide; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        // a lane has four rows of one column in four consecutive registers
                        const int row = wr + i * 32 + q * 8 + lane / 32 * 4, c = wc - part * kPart + j * 32 + lane % 32;
                        f32x4 v;
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = total[i][j][q * 4 + e] * op.factor;
                        *reinterpret_cast<f32x4*>(tiled + piece(c, row / 4)) = v;
                    }
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < kTurns; ++n) {
            const int c = col0 + n * (256 / kEights), own = kOneStage ? 0 : n;
            if constexpr (kOneStage) more(n, 0);
            float v[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const f32x4 w = *reinterpret_cast<const f32x4*>(tiled + piece(c, r / 4 + h));
#pragma unroll
                for (int e = 0; e < 4; ++e) v[4 * h + e] = w[e];
            }
            if constexpr (KIND != kGram) add8(extra[0][own], op.f[0], v);
            if constexpr (KIND == kSym)
                if (op.add[1] >= 0) add8(extra[1][own], op.f[1], v);
            uint32_t u[8];
            if constexpr (KIND == kFinal) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    v[e] *= t.scale;
                    u[e] = __float_as_uint(v[e]);
                }
                if (t.flip && tc + c < t.n)
                    put_out(outs.out[k], a.out_dtype, t.at + static_cast<int64_t>(tc + c) * t.cols + ti + r, t.m - (ti + r), v);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) u[e] = pack(v[e]);
                put8((KIND == kApply ? xt(op.dst) : sym(op.dst)) + (tc + c) * ld_m, ti + r, u);
            }
            if (natural)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    *reinterpret_cast<u32x4*>(tiled + piece(c, r / 4 + h)) = u32x4{u[4 * h], u[4 * h + 1], u[4 * h + 2], u[4 * h + 3]};
        }
        if (!natural) continue;
        __syncthreads();
        // four lanes a row's block of 32 columns, eight each
        for (int q = tid / 4; q < TILE * (kPart / kBlock); q += 64) {
            const int row = q % TILE, c = q / TILE * kBlock + tid % 4 * 8;
            uint32_t u[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) u[e] = reinterpret_cast<uint32_t*>(tiled)[piece(c + e, row / 4) + row % 4];
            if constexpr (KIND == kFinal) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(u[e]);
                if (ti + row < t.m) put_out(outs.out[k], a.out_dtype, t.at + static_cast<int64_t>(ti + row) * t.cols + tc + c, t.n - (tc + c), v);
            } else {
                put8((KIND == kApply ? x : sym(op.dst)) + (ti + row) * (KIND == kApply ? ld_n : ld_m), tc + c, u);
            }
        }
    }
}

// ------------------------------------------------------------ small matrices

constexpr int kSmallSide = 64;
constexpr int kSmallThreads = 512;
constexpr int kSmallLds = 48 * 1024, kMostLds = 160 * 1024;

// LDS of a small matrix: X, X X^T and R, rows of a multiple of 16 elements and
// four more (an odd multiple of four: 16 rows' pieces of 16 bytes touch every
// bank once).
__host__ __device__ inline int64_t small_row(int64_t v) { return (v + 15) / 16 * 16 + 4; }
int64_t small_lds(int64_t m, int64_t n) {
    const int64_t mp = (m + 15) / 16 * 16;
    return (mp * small_row(n) + 2 * mp * small_row(m)) * 4 + 256;
}

struct SmallArgs {
    UpdateArgs u;
    const int32_t* which;  // tensors
    int32_t steps;
    float eps;
    float coeff[3 * TC_MAX_ORTHO_STEPS];
};

// All steps of a matrix of at most 64 rows (or columns) that fits LDS, in one
// workgroup: a group of such matrices is bound by the time of launches and of
// dependent steps, and pays neither memory traffic nor more than one launch
// here (the tiny group, 2 copies: 20 launches 168 us, one 25; 64 x 256: 67 us).
// The products are binary32 ones, 16 x 16 x 4.  In each, a lane holds
// for its row (of the left) and column (of the right) elements 4 q .. 4 q + 3
// of 16 of the summed axis, q = lane / 16, and the four products take one each.
template <int LDS>
__global__ void __launch_bounds__(kSmallThreads) ortho_small_kernel(const SmallArgs a) {
    __shared__ __attribute__((aligned(16))) char lds[LDS];
    const OrthoMat& t = a.u.mats[a.which[blockIdx.x]];
    const int k = blockIdx.y, tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    constexpr int kWaves = kSmallThreads / 64;
    const int mt = (t.m + 15) / 16, nt = (t.n + 15) / 16;  // tiles
    const int lx = nt * 16 + 4, la = mt * 16 + 4;
    double* part = reinterpret_cast<double*>(lds);
    float* x = reinterpret_cast<float*>(lds + 256);
    float* ga = x + mt * 16 * lx;
    float* gr = ga + mt * 16 * la;
    const uintptr_t g = reinterpret_cast<uintptr_t>(a.u.g[k]), m = reinterpret_cast<uintptr_t>(a.u.m[k]);
    const uint32_t cols = t.cols, size = static_cast<uint32_t>(t.size);
    for (int e = tid; e < mt * 16 * lx; e += kSmallThreads) x[e] = 0.0f;
    __syncthreads();
    double sum = 0.0;
    constexpr int N = 8;  // elements of a lane whose loads are under way together
    for (uint32_t e0 = tid; e0 < size; e0 += N * kSmallThreads) {
        float u[N], v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t e = e0 + i * kSmallThreads;
            u[i] = v[i] = 0.0f;
            if (e >= size) continue;
            u[i] = load_any(g, a.u.g_dtype, t.at + e);
            if (a.u.momentum) v[i] = gld<float>(m + (t.at + e) * 4);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t e = e0 + i * kSmallThreads;
            if (e >= size) continue;
            if (a.u.momentum) {
                const float w = fmaf(a.u.mu, v[i], u[i]);
                gst<float>(m + (t.at + e) * 4, w);
                u[i] = update_of(u[i], w, a.u.mu, a.u.nesterov);
            }
            const uint32_t r = e / cols, c = e - r * cols;
            x[t.flip ? c * lx + r : r * lx + c] = u[i];
            sum = fma(static_cast<double>(u[i]), static_cast<double>(u[i]), sum);
        }
    }
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) sum += __shfl_xor(sum, s, 64);
    if (lane == 0) part[wave] = sum;
    __syncthreads();
    sum = part[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) sum += part[w];
    const double inv = 1.0 / (sqrt(sum) + static_cast<double>(a.eps));
    for (int e = tid; e < mt * 16 * lx; e += kSmallThreads) x[e] = static_cast<float>(static_cast<double>(x[e]) * inv);
    __syncthreads();
    const int row = lane % 16, q = lane / 16;
    // tile (i, j) of left right^T over `len` (a multiple of 16), rows of lu and lv elements
    auto product = [&](const float* u, int lu, const float* v, int lv, int len) {
        f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
        const float *pu = u + row * lu + q * 4, *pv = v + row * lv + q * 4;
        for (int e = 0; e < len; e += 16) {
            const f32x4 l = *reinterpret_cast<const f32x4*>(pu + e), r = *reinterpret_cast<const f32x4*>(pv + e);
#pragma unroll
            for (int s = 0; s < 4; ++s) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(l[s], r[s], acc, 0, 0, 0);
        }
        return acc;
    };
    for (int step = 0; step < a.steps; ++step) {
        const float ca = a.coeff[3 * step], cb = a.coeff[3 * step + 1], cc = a.coeff[3 * step + 2];
        // a lane's results: rows 4 q .. 4 q + 3 of column `row`
        for (int w = wave; w < mt * (mt + 1) / 2; w += kWaves) {
            int i = 0;
            while ((i + 1) * (i + 2) / 2 <= w) ++i;
            const int j = w - i * (i + 1) / 2;
            const f32x4 acc = product(x + i * 16 * lx, lx, x + j * 16 * lx, lx, nt * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                ga[(i * 16 + q * 4 + e) * la + j * 16 + row] = acc[e];
                ga[(j * 16 + row) * la + i * 16 + q * 4 + e] = acc[e];
            }
        }
        __syncthreads();
        for (int w = wave; w < mt * mt; w += kWaves) {
            const int i = w / mt, j = w % mt;
            const f32x4 acc = product(ga + i * 16 * la, la, ga + j * 16 * la, la, mt * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int at = (i * 16 + q * 4 + e) * la + j * 16 + row;
                gr[at] = fmaf(cc, acc[e], cb * ga[at]);
            }
        }
        __syncthreads();
        // X <- a X + R X: a wave has 16 columns to itself
        for (int j = wave; j < nt; j += kWaves) {
            float b[kSmallSide / 16][4];
#pragma unroll
            for (int h = 0; h < kSmallSide / 16; ++h)
                if (h < mt)
#pragma unroll
                    for (int s = 0; s < 4; ++s) b[h][s] = x[(h * 16 + q * 4 + s) * lx + j * 16 + row];
            f32x4 out[kSmallSide / 16];
#pragma unroll
            for (int i = 0; i < kSmallSide / 16; ++i)
                if (i < mt) {
                    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int h = 0; h < kSmallSide / 16; ++h)
                        if (h < mt) {
                            const f32x4 l = *reinterpret_cast<const f32x4*>(gr + (i * 16 + row) * la + h * 16 + q * 4);
#pragma unroll
                            for (int s = 0; s < 4; ++s) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(l[s], b[h][s], acc, 0, 0, 0);
                        }
                    // (b[i] has X at just these places)
#pragma unroll
                    for (int e = 0; e < 4; ++e) out[i][e] = fmaf(ca, b[i][e], acc[e]);
                }
#pragma unroll
            for (int i = 0; i < kSmallSide / 16; ++i)
                if (i < mt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[(i * 16 + q * 4 + e) * lx + j * 16 + row] = out[i][e];
        }
        __syncthreads();
    }
    for (uint32_t e = tid; e < size; e += kSmallThreads) {
        const uint32_t r = e / cols, c = e - r * cols;
        store_any(reinterpret_cast<uintptr_t>(a.u.out[k]), a.u.out_dtype, t.at + e, x[t.flip ? c * lx + r : r * lx + c] * t.scale);
    }
}

// The tiles of one product of the given matrices, all copies, in the order they
// are launched.  Workgroup w of a launch runs on XCD w % 8, each with an L2 of
// its own, so tiles that share rows belong on one: squares of up to 8 x 8
// tiles (16 panels of rows for 64 tiles) go to the XCD with the least to do so
// far, those with the longest sums first.  A square is cut where it is more
// than an eighth of an XCD's share.
//
// The tiles are 64 x 64 where 128 x 128 ones would leave the chip waiting for
// the longest: where all tiles' sums, shared by the 256 CUs, are no more than
// the longest sum.  (One copy in binary32, large tiles against small ones:
// 1,024 x 1,024, 36 tiles of symmetric products and 64 of P X, 514 us against
// 211; 2,048 x 2,048, 136 and 256, 920 against 831.)
enum Which { kAlongN, kAlongM, kAcross };  // X X^T, products of symmetric matrices, P X
struct Tiling {
    int side;
    int64_t count, total;  // of the tiles, and of the terms of their sums
    bool short_sums;
};

int32_t length(const OrthoMat& t, Which which) { return which == kAlongN ? t.np : t.mp; }

Tiling tiling_of(const std::vector<OrthoMat>& mats, const std::vector<int32_t>& of, int K, Which which) {
    Tiling r{};
    for (r.side = kTile;; r.side = kTile / 2) {
        int64_t longest = 0;
        r.total = r.count = 0;
        for (int32_t t : of) {
            const int64_t mi = mats[t].mp / r.side, ni = mats[t].np / r.side;
            const int64_t n = which == kAcross ? mi * ni : mi * (mi + 1) / 2;
            r.count += n * K;
            r.total += n * K * length(mats[t], which);
            longest = std::max<int64_t>(longest, length(mats[t], which));
        }
        if (r.side < kTile || r.total > longest * 256) break;
    }
    r.short_sums = r.total <= r.count * 1024;
    return r;
}

std::vector<OrthoTile> tiles_of(const std::vector<OrthoMat>& mats, const std::vector<int32_t>& of, int K, Which which, const Tiling& tiling) {
    struct Chunk {
        int64_t cost;
        int32_t len;
        size_t first, count;  // of the tiles
    };
    const int side = tiling.side;
    const int64_t total = tiling.total, count = tiling.count;
    const int32_t across = 8 * kTile / side;  // tiles of a square
    std::vector<Chunk> chunks;
    std::vector<OrthoTile> tiles;
    tiles.reserve(count);
    for (int32_t t : of) {
        const int32_t mi = mats[t].mp / side, nj = which == kAcross ? mats[t].np / side : mi, len = length(mats[t], which);
        for (int32_t k = 0; k < K; ++k)
            for (int32_t j0 = 0; j0 < nj; j0 += across)
                for (int32_t i0 = 0; i0 < mi; i0 += across) {
                    chunks.push_back({0, len, tiles.size(), 0});
                    for (int32_t j = j0; j < std::min(j0 + across, nj); ++j)
                        for (int32_t i = i0; i < std::min(i0 + across, mi); ++i) {
                            if (which != kAcross && j > i) continue;
                            if (chunks.back().cost + len > total / 64 && chunks.back().cost > 0) chunks.push_back({0, len, tiles.size(), 0});
                            tiles.push_back({t, i, j, static_cast<int16_t>(k), static_cast<int16_t>(mats[t].pair), mats[t].mp, mats[t].np, mats[t].x});
                            ++chunks.back().count;
                            chunks.back().cost += len;
                        }
                }
    }
    std::stable_sort(chunks.begin(), chunks.end(), [](const Chunk& x, const Chunk& y) {
        return x.len != y.len ? x.len > y.len : x.cost > y.cost;
    });
    std::vector<OrthoTile> queue[8], out;
    int64_t load[8] = {};
    for (const Chunk& c : chunks) {
        const int x = static_cast<int>(std::min_element(load, load + 8) - load);
        load[x] += c.cost;
        queue[x].insert(queue[x].end(), tiles.begin() + c.first, tiles.begin() + c.first + c.count);
    }
    out.reserve(count);
    size_t at[8] = {};
    for (int64_t w = 0; w < count; ++w) {
        size_t x = w % 8;
        if (at[x] == queue[x].size())  // the others' are left: from the longest
            for (size_t y = x = 0; y < 8; ++y)
                if (queue[y].size() - at[y] > queue[x].size() - at[x]) x = y;
        out.push_back(queue[x][at[x]++]);
    }
    return out;
}

// Whether a matrix takes two steps to a Gram matrix.  Two steps take
// 3 m^2 n + 5 m^3 operations instead of 6 m^2 n + 2 m^3, and two launches more
// between products of the long side, which on less than twice the length do
// not pay.  P1 P is also larger than P, and the roundings of it and of the one
// X X^T with it: against a binary32 iteration, whose roundings grow with m, it
// is further off below about 450 rows, and below about 1,000 on sums past
// 10,000 terms.  Errors (1e-6) of one step at a time, of two, and in binary32,
// five steps from 1/8 as many directions as rows and noise:
//   256 x 1,024   0.95  2.3  1.5      512 x 16,384    1.7  5.2  6.5
//   300 x 600     1.1   2.4  1.7      512 x 24,576    1.7  6.0  4.4
//   384 x 768     1.4   2.5  2.2      768 x 9,216     1.8  3.8  5.0
//   512 x 1,024   1.5   2.5  2.6      768 x 18,432    1.8  5.0  3.6
//   512 x 8,192   1.6   4.1  4.9      1,024 x 49,152  2.0  4.9  9.6
// (ResNet-50 group, 8 copies: 7.2 ms, with pairs from 256 rows 6.9.)
bool takes_pairs(int64_t m, int64_t n) { return n >= 2 * m && (m >= 8 * kTile || (m >= 4 * kTile && n <= 8192)); }

int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

}  // namespace

tc_ortho* make_ortho(const tc_group* g, int32_t K, const int64_t* rows, const int64_t* cols, const float* scale, hipError_t* e) {
    *e = hipErrorOutOfMemory;
    // (released where the host's memory runs out below, too)
    std::unique_ptr<tc_ortho, void (*)(tc_ortho*)> o(new (std::nothrow) tc_ortho(), destroy_ortho);
    if (!o) return nullptr;
    o->g = g;
    o->K = K;
    o->mats.resize(g->n);
    // Workgroups of 256 in one dimension of a grid are fewer than 2^24: lists
    // that are longer are refused before they are built.
    constexpr int64_t kMostTiles = (int64_t{1} << 32) / 256 - 1;
    auto refuse = [&] {
        *e = hipErrorInvalidValue;
        return nullptr;
    };
    int64_t nchunks = 0, nsplit = 0;
    std::vector<OrthoTile> chunks, split;
    std::vector<int32_t> large[2];  // by OrthoMat::pair
    std::vector<int32_t> small[2];
    int64_t bytes = 0, sums = 0;
    auto take = [&](int64_t n) {
        const int64_t at = bytes;
        bytes += round_up(n, 256);
        return at;
    };
    // what the matrix takes of a workgroup's LDS if it is taken whole
    auto lds_of = [&](int32_t t) {
        const int64_t m = std::min(rows[t], cols[t]), n = std::max(rows[t], cols[t]);
        return m == 0 ? 0 : m <= kSmallSide ? small_lds(m, n) : INT64_MAX;
    };
    // Next to larger matrices only the smallest are: the others' tiles cost
    // the larger ones' launches nothing, and a workgroup of their own up to
    // 70 us.
    int64_t most = kMostLds;
    for (int32_t t = 0; t < g->n; ++t)
        if (lds_of(t) > kMostLds) most = kSmallLds;
    for (int32_t t = 0; t < g->n; ++t) {
        OrthoMat& q = o->mats[t];
        q = OrthoMat{};
        q.at = g->offsets[t];
        q.size = g->sizes[t];
        q.scale = scale ? scale[t] : 1.0f;
        const int64_t nc = (q.size + kChunk - 1) / kChunk;
        q.chunk0 = static_cast<int32_t>(sums);
        q.chunks = static_cast<int32_t>(nc);
        const bool matrix = q.size > 0 && rows[t] > 0;
        const bool whole = matrix && lds_of(t) <= most;
        if (!whole) {
            if ((nchunks += nc) > kMostTiles) return refuse();
            for (int64_t i = 0; i < nc; ++i) chunks.push_back({t, static_cast<int32_t>(i), 0, 0, 0, 0, 0, 0});
        }
        if (!matrix) continue;
        q.rows = static_cast<int32_t>(rows[t]);
        q.cols = static_cast<int32_t>(cols[t]);
        q.flip = q.rows > q.cols;
        q.m = std::min(q.rows, q.cols);
        q.n = std::max(q.rows, q.cols);
        if (whole) {
            small[lds_of(t) > kSmallLds].push_back(t);
            continue;
        }
        sums += nc;
        q.mp = static_cast<int32_t>(round_up(q.m, kTile));
        q.np = static_cast<int32_t>(round_up(q.n, kTile));
        q.pair = takes_pairs(q.m, q.n);
        q.index = o->matrices++;
        o->of.push_back(t);
        const int64_t x = static_cast<int64_t>(q.mp) * q.np * 4, s = static_cast<int64_t>(q.mp) * q.mp * 4;
        q.x = take(3 * x + 3 * s);
        q.xt = q.x + x;
        if ((nsplit += static_cast<int64_t>(q.mp / 64) * (q.np / 64)) > kMostTiles) return refuse();
        for (int32_t i = 0; i < q.mp / 64; ++i)
            for (int32_t j = 0; j < q.np / 64; ++j) split.push_back({t, i, j, 0, 0, 0, 0, 0});
        large[q.pair].push_back(t);
    }
    o->sums = take(sums * 8);
    o->norms = take(static_cast<int64_t>(o->matrices) * 8);  // (nothing if there is no large matrix)
    o->copy_bytes = bytes;
    std::vector<int32_t> all = large[0];
    all.insert(all.end(), large[1].begin(), large[1].end());
    // (without pairs the last lists are the first ones again)
    const std::vector<int32_t> none, &one = large[1].empty() ? none : large[0];
    const struct {
        const std::vector<int32_t>& of;
        Which which;
    } products[] = {{all, kAlongN}, {all, kAlongM}, {all, kAcross}, {large[1], kAlongM}, {one, kAlongN}, {one, kAlongM}, {one, kAcross}};
    constexpr int kProducts = sizeof products / sizeof *products, kLists = 2 + kProducts;
    Tiling tilings[kProducts];
    for (int i = 0; i < kProducts; ++i)
        if ((tilings[i] = tiling_of(o->mats, products[i].of, K, products[i].which)).count > kMostTiles) return refuse();
    std::vector<OrthoTile> lists[kLists] = {std::move(chunks), std::move(split)};
    for (int i = 0; i < kProducts; ++i) lists[2 + i] = tiles_of(o->mats, products[i].of, K, products[i].which, tilings[i]);
    o->nchunks = static_cast<int32_t>(nchunks);
    o->nsplit = static_cast<int32_t>(nsplit);
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
    size_t at_small[2];
    for (int i = 0; i < 2; ++i) at_small[i] = put(small[i].data(), small[i].size() * 4);
    size_t at[kLists];
    for (int i = 0; i < kLists; ++i) at[i] = put(lists[i].data(), lists[i].size() * sizeof(OrthoTile));
    if ((*e = hipMalloc(&o->d_blob, host.size())) != hipSuccess ||
        (*e = hipMemcpy(o->d_blob, host.data(), host.size(), hipMemcpyHostToDevice)) != hipSuccess)
        return nullptr;
    const char* d = static_cast<const char*>(o->d_blob);
    o->d_mats = reinterpret_cast<const OrthoMat*>(d + at_mats);
    o->d_of = reinterpret_cast<const int32_t*>(d + at_of);
    for (int i = 0; i < 2; ++i) {
        o->d_small[i] = reinterpret_cast<const int32_t*>(d + at_small[i]);
        o->nsmall[i] = static_cast<int32_t>(small[i].size());
    }
    o->d_chunks = reinterpret_cast<const OrthoTile*>(d + at[0]);
    o->d_split = reinterpret_cast<const OrthoTile*>(d + at[1]);
    OrthoList* to[] = {&o->gram, &o->sym, &o->apply, &o->sym_pair, &o->gram_one, &o->sym_one, &o->apply_one};
    for (int i = 0; i < kProducts; ++i)
        *to[i] = {reinterpret_cast<const OrthoTile*>(d + at[2 + i]), static_cast<int32_t>(tilings[i].count), tilings[i].side, tilings[i].short_sums};
    if (large[1].empty()) {
        o->gram_one = o->gram;
        o->sym_one = o->sym;
        o->apply_one = o->apply;
    }
    return o.release();
}

void destroy_ortho(tc_ortho* o) {
    if (o->d_blob) (void)hipFree(o->d_blob);
    delete o;
}

const tc_group* ortho_group(const tc_ortho* o) { return o->g; }
int32_t ortho_copies(const tc_ortho* o) { return o->K; }
int64_t ortho_workspace(const tc_ortho* o) { return o->copy_bytes * o->K; }

// The largest |f| over [0, top] of a polynomial of degree 12 at most, and up to
// 0.3% more: |f| is nowhere larger than the largest of its values at N
// Chebyshev points over cos(12 pi / (2 N)) (Ehlich and Zeller 1964).
template <typename F>
double largest(double top, F f) {
    constexpr int kPoints = 256;
    static const std::array<double, kPoints> points = [] {
        std::array<double, kPoints> p;
        for (int i = 0; i < kPoints; ++i) p[i] = 0.5 + 0.5 * std::cos((i + 0.5) * std::acos(-1.0) / kPoints);
        return p;
    }();
    static const double room = std::cos(12 * std::acos(-1.0) / (2 * kPoints));
    double most = 0.0;
    for (double p : points) most = std::max(most, std::fabs(f(top * p)));
    return most / room;
}

// Whether values stay in the ranges the formats hold.  s bounds the singular
// values before a step (1 at first: |X| <= 1), and with x = s^2 the step makes
// them s |q(x)|, q = a + b x + c x^2.  What is stored, by its largest
// eigenvalue or singular value, with 1/64 of the range for rounding: A = X X^T
// (x), P - a I (q - a), X (s q), and of matrices that take two steps to a Gram
// matrix P A (x q), P A P (x q^2), both no more than the bounds of X allow, and
// S = P1 P - a1 a I (q1(x q^2) q - a1 a).
bool ortho_in_range(const tc_ortho* o, int steps, const float* coeff) {
    const double lim_x = 65504.0 / kScaleX * (63.0 / 64.0), lim_p = 65504.0 / kScaleP * (63.0 / 64.0);
    double x = 1.0, before = 1.0;  // largest x of this step and the one before
    for (int i = 0; i < steps; ++i) {
        const double a = coeff[3 * i], b = coeff[3 * i + 1], c = coeff[3 * i + 2];
        // where s q(s^2) has a derivative of 0, as a value of s^2
        double after = x * std::pow(a + x * (b + c * x), 2);
        auto at = [&](double v) {
            if (v > 0 && v < x) after = std::max(after, v * std::pow(a + v * (b + c * v), 2));
        };
        double rest = std::fabs(x * (b + c * x));
        if (c != 0) {
            if (const double v = -b / (2 * c); v > 0 && v < x) rest = std::max(rest, std::fabs(v * (b + c * v)));
            const double disc = 9 * b * b - 20 * a * c;
            if (disc >= 0) {
                at((-3 * b + std::sqrt(disc)) / (10 * c));
                at((-3 * b - std::sqrt(disc)) / (10 * c));
            }
        } else if (b != 0) {
            at(-a / (3 * b));
        }
        if (!(after <= lim_x && rest <= lim_p)) return false;
        if (i % 2 == 1 && o->sym_pair.n) {
            const double a0 = coeff[3 * i - 3], b0 = coeff[3 * i - 2], c0 = coeff[3 * i - 1];
            const double both = largest(before, [&](double v) {
                const double q = a0 + v * (b0 + c0 * v), w = v * q * q;
                return (a + w * (b + c * w)) * q - a * a0;
            });
            if (!(both <= lim_p)) return false;
        }
        before = x;
        x = after;
    }
    return true;
}

namespace {

// The products of the long side take one stage at a time where their sums are
// short (P X of the ResNet-50 group, 8 copies, mostly 256 and 512 terms: 1,145
// us with two stages, 900 with one, the last one with the result; of the
// VGG-16 group, 4,096 terms: 5.5 ms with two, 5.9 with one).
template <int KIND>
void launch_product(GemmArgs& a, const Outs& outs, const OrthoList& list, hipStream_t s) {
    if (list.n == 0) return;
    a.tiles = list.d;
    constexpr bool kLong = KIND == kApply || KIND == kFinal;
    if (list.side != kTile)
        ortho_gemm_kernel<KIND, kTile / 2, false><<<list.n, 256, 0, s>>>(a, outs);
    else if (kLong && list.short_sums)
        ortho_gemm_kernel<KIND, kTile, kLong><<<list.n, 256, 0, s>>>(a, outs);
    else
        ortho_gemm_kernel<KIND, kTile, false><<<list.n, 256, 0, s>>>(a, outs);
}

}  // namespace

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
    if (o->nsmall[0] + o->nsmall[1] > 0) {
        SmallArgs sm{};
        sm.u = u;
        sm.steps = steps;
        sm.eps = eps;
        std::copy(coeff, coeff + 3 * steps, sm.coeff);
        sm.which = o->d_small[1];
        if (o->nsmall[1]) ortho_small_kernel<kMostLds><<<dim3(o->nsmall[1], K), kSmallThreads, 0, s>>>(sm);
        sm.which = o->d_small[0];
        if (o->nsmall[0]) ortho_small_kernel<kSmallLds><<<dim3(o->nsmall[0], K), kSmallThreads, 0, s>>>(sm);
    }
    if (o->nchunks) ortho_update_kernel<<<dim3(o->nchunks, K), 256, 0, s>>>(u);
    if (o->matrices == 0) return hipGetLastError();
    ortho_norm_kernel<<<dim3(o->matrices, K), 256, 0, s>>>(o->d_mats, o->d_of, u.ws, o->copy_bytes, o->sums, o->norms, eps);
    ortho_split_kernel<<<dim3(o->nsplit, K), 256, 0, s>>>(u, o->d_split, o->norms);
    GemmArgs a{};
    a.mats = o->d_mats;
    a.ws = u.ws;
    a.copy_bytes = o->copy_bytes;
    a.out_dtype = out_dtype;
    auto gram = [&](const OrthoList& list) {
        a.op[0] = a.op[1] = {0, 0, 0, {-1, -1}, 1.0f / kScaleX, {0.0f, 0.0f}};
        launch_product<kGram>(a, outs, list, s);
    };
    auto sym = [&](const OrthoList& list, Operation p) {
        a.op[0] = a.op[1] = p;
        launch_product<kSym>(a, outs, list, s);
    };
    // R = P - a I of the Gram matrix in [0]
    constexpr float kXtoP = kScaleP / kScaleX;
    auto rest = [&](const OrthoList& list, const float* c, int dst) {
        sym(list, {0, 0, dst, {0, -1}, c[2] * (kXtoP / kScaleX), {c[1] * kXtoP, 0.0f}});
    };
    int from[2] = {0, 0};  // which transpose of X is the current one
    // X <- (f I + [left]) X: of matrices of one step to a Gram matrix, of two
    struct Factor {
        int32_t left;
        float f;
    };
    auto apply = [&](const OrthoList& list, Factor one, Factor pair, bool last) {
        for (int q = 0; q < 2; ++q) {
            const Factor& p = q ? pair : one;
            const float scale = last ? 1.0f / kScaleX : 1.0f;
            a.op[q] = {p.left, from[q], 1 - from[q], {-1, -1}, scale / kScaleP, {p.f * scale, 0.0f}};
        }
        if (last)
            launch_product<kFinal>(a, outs, list, s);
        else
            launch_product<kApply>(a, outs, list, s);
    };
    // The symmetric matrices, with R = P - a I: [0] A, then P A P, then
    // S = P1 P - a1 a I; [1] R (P1's where one step is taken at a time);
    // [2] P A, then R1.
    for (int i = 0; i < steps; i += 2) {
        const bool two = i + 1 < steps, last = i + 2 >= steps;
        const float *c0 = coeff + 3 * i, *c1 = c0 + 3;
        gram(o->gram);
        rest(o->sym, c0, 1);
        if (two) {
            sym(o->sym_pair, {1, 0, 2, {0, -1}, 1.0f / kScaleP, {c0[0], 0.0f}});   // P A = R A + a A
            sym(o->sym_pair, {1, 2, 0, {2, -1}, 1.0f / kScaleP, {c0[0], 0.0f}});   // P A P = R (P A) + a (P A)
            rest(o->sym_pair, c1, 2);                                              // R1
            sym(o->sym_pair, {2, 1, 0, {1, 2}, 1.0f / kScaleP, {c1[0], c0[0]}});   // S = R1 R + a1 R + a R1
            apply(o->apply_one, {1, c0[0]}, {}, false);
            from[0] = 1 - from[0];
            gram(o->gram_one);
            rest(o->sym_one, c1, 1);
        }
        const Factor one = {1, two ? c1[0] : c0[0]}, pair = two ? Factor{0, c0[0] * c1[0]} : one;
        apply(o->apply, one, pair, last);
        for (int& f : from) f = 1 - f;
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

}  // namespace tc
