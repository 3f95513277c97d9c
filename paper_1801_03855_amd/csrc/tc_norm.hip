// Layer norm of K workers' rows, and its backward pass.
//
// With mu and sigma^2 the mean and the variance of a row's C elements,
// r = 1 / sqrt(sigma^2 + eps) and xh = (x - mu) r:
//     y  = xh w + b
//     h  = dy w;   dx = r (h - mean(h) - xh mean(h xh))
//     dw = sum over rows of dy xh;   db = sum over rows of dy
// Both passes are bound by memory: the forward reads x and writes y, the
// backward reads dy and x and writes dx, each once.  A row is therefore held
// in registers from its only read on, by a group of L lanes (8 to 64 lanes of
// a wave, or a whole workgroup of 256 or 512) that takes NV vectors of 16
// bytes a lane; the variance is summed from the differences to the mean, so it
// loses nothing where the mean is large.  Workgroups stay on one worker and
// take its rows in turn, the next rows' loads under way while one is reduced:
// the scale and shift stay in registers, and in the backward pass so do the
// column sums of dw and db, in binary32, which are written once per workgroup
// and added up by a second kernel in a fixed order (no atomics: the same
// inputs give the same bits).
//
// Eight workers' 4,096 rows of 4,096 bfloat16: forward 0.103 ms, 5.2 TB/s;
// backward 0.173 ms, 4.65 TB/s (the rows' kernel 0.16 to 0.17).  On the same
// machine a copy by ordinary accesses reaches 5.0 to 5.3 TB/s, the library's
// own, whose loads and stores pass the caches by, 6.5.  2,048 rows of 16,384:
// backward 67 us, the rows' kernel 53, 4.4 TB/s with the partial column sums,
// one workgroup of 512 lanes a CU being all that the registers hold (in float,
// past 12,288 columns, not quite: 152 to 208 bytes a lane spill).
//
// Rows are at any alignment of their element: on gfx950 a 16-byte access at
// any address is one instruction.
#include "tc_internal.h"

namespace tc {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Elements of T in 16 bytes, and their conversions.
template <typename T>
struct Lane;
template <>
struct Lane<float> {
    static constexpr int kVec = 4;
    static __device__ __forceinline__ void widen(u32x4 v, float* f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
    }
    static __device__ __forceinline__ u32x4 narrow(const float* f) {
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __float_as_uint(f[i]);
        return v;
    }
    static __device__ __forceinline__ float get(uintptr_t a) { return gld<float>(a); }
    static __device__ __forceinline__ void put(uintptr_t a, float f) { gst<float>(a, f); }
};
// bfloat16: widened exactly, rounded to nearest even once, where a result is
// stored.
template <>
struct Lane<__bf16> {
    static constexpr int kVec = 8;
    static __device__ __forceinline__ void widen(u32x4 v, float* f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(v[i] << 16);
            f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ u32x4 narrow(const float* f) {
        typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            bf2 p = {static_cast<__bf16>(f[2 * i]), static_cast<__bf16>(f[2 * i + 1])};
            v[i] = __builtin_bit_cast(uint32_t, p);
        }
        return v;
    }
    static __device__ __forceinline__ float get(uintptr_t a) {
        return __uint_as_float(static_cast<uint32_t>(gld<uint16_t>(a)) << 16);
    }
    static __device__ __forceinline__ void put(uintptr_t a, float f) { gst<__bf16>(a, static_cast<__bf16>(f)); }
};

// Vector v of a row at address a: whole, or what the row has of it with zeros
// after the row's end.  EDGE: the row may end inside a vector.
template <typename T, bool EDGE>
__device__ __forceinline__ u32x4 load_vec(uintptr_t a, int v, int cols) {
    constexpr int V = Lane<T>::kVec;
    const int left = cols - v * V;
    if (left >= V) return gld_u<u32x4>(a + static_cast<uintptr_t>(v) * 16);
    u32x4 r = {0, 0, 0, 0};
    if (EDGE && left > 0) {
        float f[V];
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = i < left ? Lane<T>::get(a + static_cast<uintptr_t>(v) * 16 + i * sizeof(T)) : 0.0f;
        r = Lane<T>::narrow(f);
    }
    return r;
}

// The same where it is needed only later.  A load of single elements would be
// waited for at once, with all loads before it; so of the vector that the row
// ends inside, the row's last 16 bytes are loaded, which are in the row where
// it has that many, and `settle` moves their elements down to their places
// (12,764 rows of 8,513 bfloat16, forward: 188 us by elements, 109 so; two
// workers' 22,424 rows of 722, backward: 59 and 50).  Not for the long rows'
// kernels, whose lanes may have stored over the elements before by then.
template <typename T, bool EDGE>
__device__ __forceinline__ u32x4 load_ahead(uintptr_t a, int v, int cols) {
    constexpr int V = Lane<T>::kVec;
    if (!EDGE || cols < V) return load_vec<T, EDGE>(a, v, cols);
    const int c = v * V;
    u32x4 r = {0, 0, 0, 0};
    if (c < cols) r = gld_u<u32x4>(a + static_cast<uintptr_t>(c + V <= cols ? c : cols - V) * sizeof(T));
    return r;
}
template <typename T, bool EDGE>
__device__ __forceinline__ void settle(float* f, int v, int cols) {
    constexpr int V = Lane<T>::kVec;
    if (!EDGE || cols < V || v != cols / V) return;
    const int by = V - cols % V;
#pragma unroll
    for (int m = V / 2; m > 0; m >>= 1)
        if (by & m)
#pragma unroll
            for (int e = 0; e < V; ++e) f[e] = e + m < V ? f[e + m] : 0.0f;
}

template <typename T, bool EDGE>
__device__ __forceinline__ void store_vec(uintptr_t a, int v, int cols, const float* f) {
    constexpr int V = Lane<T>::kVec;
    const int left = cols - v * V;
    if (left >= V) {
        gst_u<u32x4>(a + static_cast<uintptr_t>(v) * 16, Lane<T>::narrow(f));
    } else if (EDGE) {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < left) Lane<T>::put(a + static_cast<uintptr_t>(v) * 16 + i * sizeof(T), f[i]);
    }
}

// V binary32 values (a scale, a shift) for the columns of vector v; `fill`
// past the row's end and where there is no such buffer.
template <int V, bool EDGE>
__device__ __forceinline__ void load_f32(const float* p, int v, int cols, float fill, float* f) {
    const int left = cols - v * V;
    const uintptr_t a = reinterpret_cast<uintptr_t>(p) + static_cast<uintptr_t>(v) * V * 4;
    if (p && left >= V) {
#pragma unroll
        for (int q = 0; q < V / 4; ++q) {
            f32x4 t = gld_u<f32x4>(a + q * 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) f[q * 4 + i] = t[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = EDGE && p && i < left ? gld<float>(a + i * 4) : fill;
    }
}

// Sums of N values over the L lanes of a group, the same in every lane.  For
// L over 64 the group is the workgroup, whose waves meet in LDS: `turn`
// alternates between two halves of it, so one barrier a sum is enough.
template <int L, int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float* lds, int& turn) {
#pragma unroll
    for (int m = (L < 64 ? L : 64) / 2; m > 0; m >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], m, 64);
    if constexpr (L > 64) {
        constexpr int W = L / 64;
        float* half = lds + turn * (W * 2);
        if (threadIdx.x % 64 == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) half[i * W + threadIdx.x / 64] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float s = half[i * W];
#pragma unroll
            for (int w = 1; w < W; ++w) s += half[i * W + w];
            v[i] = s;
        }
        turn ^= 1;
    }
}

// Pointers of the workers of one launch.
constexpr int kWorkers = 32;

struct NormArgs {
    const void* x[kWorkers];
    const float* w[kWorkers];
    const float* b[kWorkers];
    void* y[kWorkers];
    float* mean[kWorkers];
    float* rstd[kWorkers];
    int64_t rows[kWorkers];
    uint32_t wg[kWorkers + 1];  // first workgroup of each worker
    int32_t K;
    int32_t cols;
    int64_t x_ld, y_ld;  // bytes from row to row
    float eps;
};

struct NormGradArgs {
    const void* dy[kWorkers];
    const void* x[kWorkers];
    const float* w[kWorkers];
    const float* mean[kWorkers];
    const float* rstd[kWorkers];
    void* dx[kWorkers];
    void* dw[kWorkers];
    void* db[kWorkers];
    int64_t rows[kWorkers];
    uint32_t wg[kWorkers + 1];
    int32_t K;
    int32_t cols;
    int64_t dy_ld, x_ld, dx_ld;  // bytes from row to row
    float* part;                 // column sums of each workgroup: 2 * cols values
    int32_t w_dtype;             // of dw and db
    int32_t direct;              // one workgroup a worker: it writes dw and db itself
};

template <typename A>
__device__ __forceinline__ int worker_of(const A& a, uint32_t b) {
    int k = 0;
    while (k + 1 < a.K && b >= a.wg[k + 1]) ++k;
    return k;
}

// Whether element e of vector v is in the row.
template <bool EDGE, int V>
__device__ __forceinline__ bool in_row(int v, int e, int cols) {
    return EDGE ? v * V + e < cols : v * V < cols;
}

template <typename T, int L, int NV, bool EDGE>
__global__ void __launch_bounds__(L > 256 ? L : 256) norm_kernel(const NormArgs a) {
    constexpr int V = Lane<T>::kVec;
    constexpr int kThreads = L > 256 ? L : 256;
    constexpr int G = kThreads / L;  // rows at a time
    __shared__ float lds[L > 64 ? 4 * (L / 64) : 1];
    const int k = worker_of(a, blockIdx.x);
    const int lane = threadIdx.x % L, cols = a.cols;
    const int64_t step = static_cast<int64_t>(a.wg[k + 1] - a.wg[k]) * G;
    int64_t row = static_cast<int64_t>(blockIdx.x - a.wg[k]) * G + threadIdx.x / L;
    const int64_t rows = a.rows[k];
    const uintptr_t x0 = reinterpret_cast<uintptr_t>(a.x[k]), y0 = reinterpret_cast<uintptr_t>(a.y[k]);
    int turn = 0;
    u32x4 ahead[2][NV];  // the next two rows
    auto fetch = [&](u32x4 (&to)[NV], int64_t at) {
        if (at < rows)
#pragma unroll
            for (int i = 0; i < NV; ++i) to[i] = load_ahead<T, EDGE>(x0 + at * a.x_ld, lane + i * L, cols);
    };
    fetch(ahead[0], row);
    fetch(ahead[1], row + step);
    float w[NV][V], b[NV][V];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        load_f32<V, EDGE>(a.w[k], lane + i * L, cols, 1.0f, w[i]);
        load_f32<V, EDGE>(a.b[k], lane + i * L, cols, 0.0f, b[i]);
    }
    auto one = [&](u32x4 (&from)[NV]) {
        float x[NV][V];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            Lane<T>::widen(from[i], x[i]);
            settle<T, EDGE>(x[i], lane + i * L, cols);
        }
        fetch(from, row + 2 * step);
        float s[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) s[0] += x[i][e];
        group_sum<L, 1>(s, lds, turn);
        const float mean = s[0] / static_cast<float>(cols);
        float q[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                x[i][e] -= mean;
                q[0] = in_row<EDGE, V>(lane + i * L, e, cols) ? fmaf(x[i][e], x[i][e], q[0]) : q[0];
            }
        group_sum<L, 1>(q, lds, turn);
        const float r = 1.0f / sqrtf(q[0] / static_cast<float>(cols) + a.eps);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int e = 0; e < V; ++e) x[i][e] = fmaf(x[i][e] * r, w[i][e], b[i][e]);
            store_vec<T, EDGE>(y0 + row * a.y_ld, lane + i * L, cols, x[i]);
        }
        if (lane == 0) {
            if (a.mean[k]) a.mean[k][row] = mean;
            if (a.rstd[k]) a.rstd[k][row] = r;
        }
        row += step;
    };
    // (where L > 64 and there are barriers, all of a workgroup have one row)
    while (row < rows) {
        one(ahead[0]);
        if (row < rows) one(ahead[1]);
    }
}

__device__ __forceinline__ void put_weight(void* p, int dtype, int64_t c, float v) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p);
    if (dtype == TC_BF16)
        Lane<__bf16>::put(a + c * 2, v);
    else
        Lane<float>::put(a + c * 4, v);
}

template <typename T, int L, int NV, bool EDGE>
__global__ void __launch_bounds__(L > 256 ? L : 256) norm_grad_kernel(const NormGradArgs a) {
    constexpr int V = Lane<T>::kVec;
    constexpr int kThreads = L > 256 ? L : 256;
    constexpr int G = kThreads / L;
    // rows ahead: two, or one where two do not fit the registers (with 24
    // elements of bfloat16 they do: 12,764 rows of 8,513 183 us, with one 184)
    constexpr int kAhead = NV * V > 16 ? 1 : 2;
    // and there the scale is held in LDS, each lane's own part, which needs no
    // barrier (read from the L2 for every row instead: 2,048 rows of 16,384 in
    // float 171 us, from LDS 149; in bfloat16 65 and 61)
    constexpr int kHeld = NV * V > 16 ? 1 : NV;
    // the sums of a row's waves, and at the end the column sums of the groups
    constexpr int kCols = L * NV * V;
    __shared__ float lds[G > 1 ? G * kCols : 4 * (L / 64)];
    __shared__ __attribute__((aligned(16))) float scale[kHeld < NV ? kCols : 4];
    const int k = worker_of(a, blockIdx.x);
    const int lane = threadIdx.x % L, group = threadIdx.x / L, cols = a.cols;
    const int64_t step = static_cast<int64_t>(a.wg[k + 1] - a.wg[k]) * G;
    int64_t row = static_cast<int64_t>(blockIdx.x - a.wg[k]) * G + group;
    const int64_t rows = a.rows[k];
    const uintptr_t x0 = reinterpret_cast<uintptr_t>(a.x[k]), d0 = reinterpret_cast<uintptr_t>(a.dy[k]);
    const uintptr_t o0 = reinterpret_cast<uintptr_t>(a.dx[k]);
    const float* means = a.mean[k];
    const float* rstds = a.rstd[k];
    const float inv = 1.0f / static_cast<float>(cols);
    int turn = 0;
    struct Row {
        u32x4 x[NV], d[NV];
        float mean, r;
    } ahead[kAhead];
    auto fetch = [&](Row& to, int64_t at) {
        if (at >= rows) return;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            to.x[i] = load_ahead<T, EDGE>(x0 + at * a.x_ld, lane + i * L, cols);
            to.d[i] = load_ahead<T, EDGE>(d0 + at * a.dy_ld, lane + i * L, cols);
        }
        to.mean = means[at];
        to.r = rstds[at];
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) fetch(ahead[i], row + i * step);
    float w[kHeld][V], dw[NV][V], db[NV][V];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        load_f32<V, EDGE>(a.w[k], lane + i * L, cols, 1.0f, w[i % kHeld]);
        if (kHeld < NV)
#pragma unroll
            for (int q = 0; q < V / 4; ++q)
                *reinterpret_cast<f32x4*>(scale + (lane + i * L) * V + q * 4) =
                    f32x4{w[0][q * 4], w[0][q * 4 + 1], w[0][q * 4 + 2], w[0][q * 4 + 3]};
#pragma unroll
        for (int e = 0; e < V; ++e) dw[i][e] = db[i][e] = 0.0f;
    }
    auto one = [&](Row& from) {
        float x[NV][V], d[NV][V];
        const float mean = from.mean, r = from.r;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            Lane<T>::widen(from.x[i], x[i]);
            Lane<T>::widen(from.d[i], d[i]);
            settle<T, EDGE>(x[i], lane + i * L, cols);
            settle<T, EDGE>(d[i], lane + i * L, cols);
        }
        fetch(from, row + kAhead * step);
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (kHeld < NV)
#pragma unroll
                for (int q = 0; q < V / 4; ++q) {
                    const f32x4 t =
                        *reinterpret_cast<const f32x4*>(scale + (lane + i * L) * V + q * 4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[0][q * 4 + e] = t[e];
                }
#pragma unroll
            for (int e = 0; e < V; ++e) {
                // past the row's end dy is 0 and adds nothing, unless the mean
                // or r is infinite: those columns are never stored, but they
                // would put a NaN into the row's sums
                x[i][e] = in_row<EDGE, V>(lane + i * L, e, cols) ? (x[i][e] - mean) * r : 0.0f;
                dw[i][e] = fmaf(d[i][e], x[i][e], dw[i][e]);
                db[i][e] += d[i][e];
                d[i][e] *= w[i % kHeld][e];
                s[0] += d[i][e];
                s[1] = fmaf(d[i][e], x[i][e], s[1]);
            }
        }
        group_sum<L, 2>(s, lds, turn);
        const float c0 = s[0] * inv, c1 = s[1] * inv;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int e = 0; e < V; ++e) x[i][e] = r * (d[i][e] - c0 - x[i][e] * c1);
            store_vec<T, EDGE>(o0 + row * a.dx_ld, lane + i * L, cols, x[i]);
        }
        row += step;
    };
    while (row < rows) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (row < rows) one(ahead[i]);
    }
    // the workgroup's column sums
    float* part = a.part + static_cast<int64_t>(blockIdx.x) * 2 * cols;
    if constexpr (G == 1) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (lane + i * L) * V;
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (c + e < cols) {
                    if (a.direct) {
                        put_weight(a.dw[k], a.w_dtype, c + e, dw[i][e]);
                        put_weight(a.db[k], a.w_dtype, c + e, db[i][e]);
                    } else {
                        part[c + e] = dw[i][e];
                        part[cols + c + e] = db[i][e];
                    }
                }
        }
    } else {
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e)
                    lds[group * kCols + (lane + i * L) * V + e] = which ? db[i][e] : dw[i][e];
            __syncthreads();
            for (int c = threadIdx.x; c < cols; c += kThreads) {
                float t = lds[c];
#pragma unroll 4
                for (int g = 1; g < G; ++g) t += lds[g * kCols + c];
                if (a.direct)
                    put_weight(which ? a.db[k] : a.dw[k], a.w_dtype, c, t);
                else
                    part[which * cols + c] = t;
            }
        }
    }
}

// Rows too long for the registers of a workgroup: three reads of the row,
// the later ones from the caches.
constexpr int kLong = 1024;

template <typename T>
__global__ void __launch_bounds__(kLong) norm_long_kernel(const NormArgs a) {
    constexpr int V = Lane<T>::kVec;
    __shared__ float lds[4 * (kLong / 64)];
    const int k = worker_of(a, blockIdx.x);
    const int cols = a.cols, nv = (cols + V - 1) / V;
    const int64_t step = a.wg[k + 1] - a.wg[k];
    int turn = 0;
    for (int64_t row = blockIdx.x - a.wg[k]; row < a.rows[k]; row += step) {
        const uintptr_t x = reinterpret_cast<uintptr_t>(a.x[k]) + row * a.x_ld;
        const uintptr_t y = reinterpret_cast<uintptr_t>(a.y[k]) + row * a.y_ld;
        float f[V], w[V], b[V], s[1] = {0.0f}, q[1] = {0.0f};
        for (int v = threadIdx.x; v < nv; v += kLong) {
            Lane<T>::widen(load_vec<T, true>(x, v, cols), f);
#pragma unroll
            for (int e = 0; e < V; ++e) s[0] += f[e];
        }
        group_sum<kLong, 1>(s, lds, turn);
        const float mean = s[0] / static_cast<float>(cols);
        for (int v = threadIdx.x; v < nv; v += kLong) {
            Lane<T>::widen(load_vec<T, true>(x, v, cols), f);
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (v * V + e < cols) q[0] = fmaf(f[e] - mean, f[e] - mean, q[0]);
        }
        group_sum<kLong, 1>(q, lds, turn);
        const float r = 1.0f / sqrtf(q[0] / static_cast<float>(cols) + a.eps);
        for (int v = threadIdx.x; v < nv; v += kLong) {
            Lane<T>::widen(load_vec<T, true>(x, v, cols), f);
            load_f32<V, true>(a.w[k], v, cols, 1.0f, w);
            load_f32<V, true>(a.b[k], v, cols, 0.0f, b);
#pragma unroll
            for (int e = 0; e < V; ++e) f[e] = fmaf((f[e] - mean) * r, w[e], b[e]);
            store_vec<T, true>(y, v, cols, f);
        }
        if (threadIdx.x == 0) {
            if (a.mean[k]) a.mean[k][row] = mean;
            if (a.rstd[k]) a.rstd[k][row] = r;
        }
    }
}

// The column sums of long rows: a workgroup takes 256 columns of a run of
// rows.  Launched before norm_grad_long_kernel, which may overwrite dy or x.
template <typename T>
__global__ void __launch_bounds__(256) norm_columns_kernel(const NormGradArgs a, int runs) {
    const int k = blockIdx.z;
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= a.cols) return;
    float dw = 0.0f, db = 0.0f;
    for (int64_t row = blockIdx.y; row < a.rows[k]; row += runs) {
        const float d = Lane<T>::get(reinterpret_cast<uintptr_t>(a.dy[k]) + row * a.dy_ld + static_cast<uintptr_t>(c) * sizeof(T));
        const float x = Lane<T>::get(reinterpret_cast<uintptr_t>(a.x[k]) + row * a.x_ld + static_cast<uintptr_t>(c) * sizeof(T));
        dw = fmaf(d, (x - a.mean[k][row]) * a.rstd[k][row], dw);
        db += d;
    }
    float* part = a.part + (static_cast<int64_t>(k) * runs + blockIdx.y) * 2 * a.cols;
    part[c] = dw;
    part[a.cols + c] = db;
}

template <typename T>
__global__ void __launch_bounds__(kLong) norm_grad_long_kernel(const NormGradArgs a) {
    constexpr int V = Lane<T>::kVec;
    __shared__ float lds[4 * (kLong / 64)];
    const int k = worker_of(a, blockIdx.x);
    const int cols = a.cols, nv = (cols + V - 1) / V;
    const int64_t step = a.wg[k + 1] - a.wg[k];
    const float inv = 1.0f / static_cast<float>(cols);
    int turn = 0;
    for (int64_t row = blockIdx.x - a.wg[k]; row < a.rows[k]; row += step) {
        const uintptr_t x = reinterpret_cast<uintptr_t>(a.x[k]) + row * a.x_ld;
        const uintptr_t dy = reinterpret_cast<uintptr_t>(a.dy[k]) + row * a.dy_ld;
        const uintptr_t dx = reinterpret_cast<uintptr_t>(a.dx[k]) + row * a.dx_ld;
        const float mean = a.mean[k][row], r = a.rstd[k][row];
        float f[V], d[V], w[V], s[2] = {0.0f, 0.0f};
        for (int v = threadIdx.x; v < nv; v += kLong) {
            Lane<T>::widen(load_vec<T, true>(x, v, cols), f);
            Lane<T>::widen(load_vec<T, true>(dy, v, cols), d);
            load_f32<V, true>(a.w[k], v, cols, 1.0f, w);
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (v * V + e < cols) {
                    s[0] = fmaf(d[e], w[e], s[0]);
                    s[1] = fmaf(d[e] * w[e], (f[e] - mean) * r, s[1]);
                }
        }
        group_sum<kLong, 2>(s, lds, turn);
        const float c0 = s[0] * inv, c1 = s[1] * inv;
        for (int v = threadIdx.x; v < nv; v += kLong) {
            Lane<T>::widen(load_vec<T, true>(x, v, cols), f);
            Lane<T>::widen(load_vec<T, true>(dy, v, cols), d);
            load_f32<V, true>(a.w[k], v, cols, 1.0f, w);
#pragma unroll
            for (int e = 0; e < V; ++e) f[e] = r * (d[e] * w[e] - c0 - (f[e] - mean) * r * c1);
            store_vec<T, true>(dx, v, cols, f);
        }
    }
}

// dw and db of every worker from its workgroups' column sums: 64 columns a
// workgroup, whose 16 waves take the partial sums in turn.
__global__ void __launch_bounds__(1024) norm_finish_kernel(const NormGradArgs a) {
    __shared__ float lds[16][64];
    const int k = blockIdx.z, which = blockIdx.y, cols = a.cols;
    const int c = blockIdx.x * 64 + threadIdx.x % 64, wave = threadIdx.x / 64;
    float s = 0.0f;
    if (c < cols)
        for (uint32_t b = a.wg[k] + wave; b < a.wg[k + 1]; b += 16) s += a.part[static_cast<int64_t>(b) * 2 * cols + which * cols + c];
    lds[wave][threadIdx.x % 64] = s;
    __syncthreads();
    if (wave == 0 && c < cols) {
#pragma unroll
        for (int q = 1; q < 16; ++q) s += lds[q][threadIdx.x];
        put_weight(which ? a.db[k] : a.dw[k], a.w_dtype, c, s);
    }
}

// Lanes of a row and vectors of a lane.
struct Shape {
    int L, NV;  // L = 0: a long row
};

// The fewest lanes that hold a row in one vector each, up to a wave; then a
// wave with up to 16 elements a lane, a workgroup of 256 with 8 or 16, and one
// of 512 with 16, 24 or 32 (more do not fit the registers of so many lanes next
// to the scale and the column sums; two workers' 4,000 rows of 9,000 in float,
// backward: 342 us with 32, which spill, 178 with 24).
Shape shape_of(int64_t cols, int es) {
    const int v = 16 / es;
    for (int l = 8; l <= 64; l *= 2)
        if (cols <= l * v) return {l, 1};
    const struct { int l, e; } more[] = {{64, 8}, {64, 16}, {256, 8}, {256, 16}, {512, 16}, {512, 24}, {512, 32}};
    for (auto m : more)
        if (cols <= static_cast<int64_t>(m.l) * m.e) return {m.l, m.e / v};
    return {0, 0};
}

// Rows that a workgroup takes at a time, and how many workgroups a launch has
// at most.
int rows_at_a_time(Shape s) { return s.L == 0 || s.L >= 256 ? 1 : 256 / s.L; }

// Spreads `most` workgroups over the workers so that each takes about as many
// batches of rows; fills wg[0..K].  Every worker with rows has at least one,
// and with `always` every worker.
void spread(int K, const int64_t* rows, int batch, int64_t most, int64_t least, bool always, uint32_t* wg) {
    int64_t total = 0;
    for (int k = 0; k < K; ++k) total += (rows[k] + batch - 1) / batch;
    int64_t each = (total + most - 1) / most;
    if (each < least) each = least;
    wg[0] = 0;
    for (int k = 0; k < K; ++k) {
        const int64_t b = (rows[k] + batch - 1) / batch;
        int64_t n = (b + each - 1) / each;
        if (n < 1 && always) n = 1;
        wg[k + 1] = wg[k] + static_cast<uint32_t>(n);
    }
}

// Workgroups of a launch at most.  Backward: those that the chip holds at once,
// by the registers that the elements of a lane take (32,768 rows of 4,096
// bfloat16: 768 workgroups 175 us, 1,024, of which the last 256 ran alone,
// 185).  Forward more, of which the next ones start as others end (2,048
// workgroups 107 us, 1,024 112), but of a whole row to 512 lanes no more than
// fit.
int64_t most_forward(Shape s, int es) {
    const int e = s.NV * 16 / es;
    if (s.L == 0) return 512;
    if (s.L == 512) return e > 16 ? 256 : 512;
    return 2048;
}
int64_t most_backward(Shape s, int es) {
    if (s.L == 0 || s.L == 512) return 256;
    return s.NV * 16 / es > 8 ? (es == 2 ? 768 : 512) : 1024;
}
// Batches of rows of a workgroup, backward, at least: fewer workgroups leave
// fewer column sums to add up, more of them more of the chip at work.  With 1,
// 2, 4 and 8, in us: 512 x 4,096 bfloat16 32.4, 20.7, 17.3, 19.7; 1,024 x 1,024
// float 14.2, 12.2, 12.4, 15.7; 4,096 x 256 float 29.0, 18.7, 14.0, 13.7; 512 x
// 8,192 float 25.8, 25.5, 24.1, 28.9.  Few rows lose by it: 64 x 1,024 float
// 6.5, 7.4, 9.4, 13.4; 256 x 16,384 float 44.7, 48.6, 65.3, 105 (bfloat16 38.3,
// 31.4, 33.5, 39.7).
constexpr int64_t kLeastBackward = 4;
constexpr int kRuns = 64;              // of rows, for the column sums of long rows

void spread_backward(int K, const int64_t* rows, Shape s, int es, uint32_t* wg) {
    spread(K, rows, rows_at_a_time(s), most_backward(s, es), kLeastBackward, true, wg);
}

template <typename T, int L, int NV>
void run_norm(const NormArgs& a, hipStream_t s) {
    if (a.cols % Lane<T>::kVec)
        norm_kernel<T, L, NV, true><<<a.wg[a.K], L > 256 ? L : 256, 0, s>>>(a);
    else
        norm_kernel<T, L, NV, false><<<a.wg[a.K], L > 256 ? L : 256, 0, s>>>(a);
}
template <typename T, int L, int NV>
void run_norm_grad(const NormGradArgs& a, hipStream_t s) {
    if (a.cols % Lane<T>::kVec)
        norm_grad_kernel<T, L, NV, true><<<a.wg[a.K], L > 256 ? L : 256, 0, s>>>(a);
    else
        norm_grad_kernel<T, L, NV, false><<<a.wg[a.K], L > 256 ? L : 256, 0, s>>>(a);
}

// CALL<T, L, NV> for the shape of the row.
#define TC_NORM_SHAPES(CALL, T)                                               \
    {                                                                         \
        constexpr int V = Lane<T>::kVec;                                      \
        switch (sh.L * 64 + sh.NV * V) {                                      \
            case 8 * 64 + V: CALL<T, 8, 1>(a, s); break;                      \
            case 16 * 64 + V: CALL<T, 16, 1>(a, s); break;                    \
            case 32 * 64 + V: CALL<T, 32, 1>(a, s); break;                    \
            case 64 * 64 + 4: CALL<T, 64, 4 / V + (V > 4)>(a, s); break;      \
            case 64 * 64 + 8: CALL<T, 64, 8 / V>(a, s); break;                \
            case 64 * 64 + 16: CALL<T, 64, 16 / V>(a, s); break;              \
            case 256 * 64 + 8: CALL<T, 256, 8 / V>(a, s); break;              \
            case 256 * 64 + 16: CALL<T, 256, 16 / V>(a, s); break;            \
            case 512 * 64 + 16: CALL<T, 512, 16 / V>(a, s); break;            \
            case 512 * 64 + 24: CALL<T, 512, 24 / V>(a, s); break;            \
            default: CALL<T, 512, 32 / V>(a, s); break;                       \
        }                                                                     \
    }

}  // namespace

hipError_t launch_layernorm(int K, const int64_t* rows, int64_t cols, const void* const* x, int64_t x_ld, int dtype,
                            const float* const* w, const float* const* b, void* const* y, int64_t y_ld,
                            float* const* mean, float* const* rstd, float eps, hipStream_t s) {
    const int es = dtype == TC_BF16 ? 2 : 4;
    const Shape sh = shape_of(cols, es);
    for (int k0 = 0; k0 < K; k0 += kWorkers) {
        NormArgs a{};
        a.K = K - k0 < kWorkers ? K - k0 : kWorkers;
        a.cols = static_cast<int32_t>(cols);
        a.x_ld = x_ld * es;
        a.y_ld = y_ld * es;
        a.eps = eps;
        for (int k = 0; k < a.K; ++k) {
            a.x[k] = x[k0 + k];
            a.w[k] = w ? w[k0 + k] : nullptr;
            a.b[k] = b ? b[k0 + k] : nullptr;
            a.y[k] = y[k0 + k];
            a.mean[k] = mean ? mean[k0 + k] : nullptr;
            a.rstd[k] = rstd ? rstd[k0 + k] : nullptr;
            a.rows[k] = rows[k0 + k];
        }
        spread(a.K, a.rows, rows_at_a_time(sh), most_forward(sh, es), 1, false, a.wg);
        if (a.wg[a.K] == 0) continue;
        if (sh.L == 0) {
            if (dtype == TC_BF16)
                norm_long_kernel<__bf16><<<a.wg[a.K], kLong, 0, s>>>(a);
            else
                norm_long_kernel<float><<<a.wg[a.K], kLong, 0, s>>>(a);
        } else if (dtype == TC_BF16) {
            TC_NORM_SHAPES(run_norm, __bf16)
        } else {
            TC_NORM_SHAPES(run_norm, float)
        }
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

int64_t layernorm_workspace(int K, const int64_t* rows, int64_t cols) {
    // of the type that takes more workgroups
    int64_t most = 0;
    for (int es : {2, 4}) {
        const Shape sh = shape_of(cols, es);
        for (int k0 = 0; k0 < K; k0 += kWorkers) {
            uint32_t wg[kWorkers + 1];
            const int n = K - k0 < kWorkers ? K - k0 : kWorkers;
            spread_backward(n, rows + k0, sh, es, wg);
            const int64_t parts = sh.L == 0 ? static_cast<int64_t>(n) * kRuns : wg[n];
            most = most > parts ? most : parts;
        }
    }
    return most * 2 * cols * 4;
}

hipError_t launch_layernorm_backward(int K, const int64_t* rows, int64_t cols, const void* const* dy, int64_t dy_ld,
                                     const void* const* x, int64_t x_ld, int dtype, const float* const* w,
                                     const float* const* mean, const float* const* rstd, void* const* dx, int64_t dx_ld,
                                     void* const* dw, void* const* db, int w_dtype, void* workspace, hipStream_t s) {
    const int es = dtype == TC_BF16 ? 2 : 4;
    const Shape sh = shape_of(cols, es);
    for (int k0 = 0; k0 < K; k0 += kWorkers) {
        NormGradArgs a{};
        a.K = K - k0 < kWorkers ? K - k0 : kWorkers;
        a.cols = static_cast<int32_t>(cols);
        a.dy_ld = dy_ld * es;
        a.x_ld = x_ld * es;
        a.dx_ld = dx_ld * es;
        a.part = static_cast<float*>(workspace);
        a.w_dtype = w_dtype;
        for (int k = 0; k < a.K; ++k) {
            a.dy[k] = dy[k0 + k];
            a.x[k] = x[k0 + k];
            a.w[k] = w ? w[k0 + k] : nullptr;
            a.mean[k] = mean[k0 + k];
            a.rstd[k] = rstd[k0 + k];
            a.dx[k] = dx[k0 + k];
            a.dw[k] = dw[k0 + k];
            a.db[k] = db[k0 + k];
            a.rows[k] = rows[k0 + k];
        }
        spread_backward(a.K, a.rows, sh, es, a.wg);
        if (sh.L == 0) {
            const dim3 grid(static_cast<uint32_t>((cols + 255) / 256), kRuns, a.K);
            if (dtype == TC_BF16) {
                norm_columns_kernel<__bf16><<<grid, 256, 0, s>>>(a, kRuns);
                norm_grad_long_kernel<__bf16><<<a.wg[a.K], kLong, 0, s>>>(a);
            } else {
                norm_columns_kernel<float><<<grid, 256, 0, s>>>(a, kRuns);
                norm_grad_long_kernel<float><<<a.wg[a.K], kLong, 0, s>>>(a);
            }
            for (int k = 0; k <= a.K; ++k) a.wg[k] = static_cast<uint32_t>(k) * kRuns;
        } else {
            a.direct = a.wg[a.K] == static_cast<uint32_t>(a.K);
            if (dtype == TC_BF16) {
                TC_NORM_SHAPES(run_norm_grad, __bf16)
            } else {
                TC_NORM_SHAPES(run_norm_grad, float)
            }
        }
        if (hipError_t e = hipGetLastError()) return e;
        if (!a.direct) norm_finish_kernel<<<dim3(static_cast<uint32_t>((cols + 63) / 64), 2, a.K), 1024, 0, s>>>(a);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

}  // namespace tc
