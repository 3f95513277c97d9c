// Dropout of K workers' rows, and its backward pass.
//
//     y = keep ? x * 2^16 / (2^16 - T) : 0  (+ residual),   keep = u >= T
// with T = p * 2^16 rounded, and u 16 bits of Philox 4x32 with 10 rounds
// (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2,
// 3", 2011).  The four words of one counter decide eight neighbouring columns,
// so the mask is a function of the seed, the step, the site, the worker and the
// element's row and column alone: the backward pass makes it again, and nothing
// of it is stored.
//
// Bound by memory: x (and the residual) read once, y written once.  A counter's
// 20 products of 32 bits go to the vector units while the loads are under way.
#include "tc_lane.h"

namespace tc {
namespace {

constexpr int kWorkers = 32;
constexpr int kThreads = 256;

struct DropArgs {
    const void* x[kWorkers];
    const void* r[kWorkers];
    void* y[kWorkers];
    int64_t rows[kWorkers];
    uint32_t wg[kWorkers + 1];  // first workgroup of each worker
    const int64_t* random;      // seed and step
    int64_t x_ld, r_ld, y_ld;   // bytes from row to row
    int32_t K, first;           // workers of the launch, and the first one's index
    int32_t cols;
    uint32_t site, threshold;
    float scale;
};

struct Words {
    uint32_t w[4];
};

__device__ __forceinline__ Words philox(Words c, uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = static_cast<uint64_t>(c.w[0]) * 0xD2511F53u, b = static_cast<uint64_t>(c.w[2]) * 0xCD9E8D57u;
        c = {{static_cast<uint32_t>(b >> 32) ^ c.w[1] ^ k0, static_cast<uint32_t>(b),
              static_cast<uint32_t>(a >> 32) ^ c.w[3] ^ k1, static_cast<uint32_t>(a)}};
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return c;
}

// A lane takes vectors of eight columns, `kAhead` at a time.
template <typename T, bool RESIDUAL, bool EDGE>
__global__ void __launch_bounds__(kThreads) dropout_kernel(const DropArgs a) {
    constexpr int V = Lane<T>::kVec, N = 8 / V;  // 16-byte pieces of a vector
    constexpr int kAhead = 2;
    int k = 0;
    while (k + 1 < a.K && blockIdx.x >= a.wg[k + 1]) ++k;
    const uint32_t per = (static_cast<uint32_t>(a.cols) + 7) / 8;  // vectors of a row
    const uint32_t step = (a.wg[k + 1] - a.wg[k]) * kThreads;
    const uint32_t step_rows = step / per, step_cols = step % per;
    const uint32_t begin = (blockIdx.x - a.wg[k]) * kThreads + threadIdx.x;
    const int64_t end = a.rows[k] * per;
    const uintptr_t x0 = reinterpret_cast<uintptr_t>(a.x[k]), y0 = reinterpret_cast<uintptr_t>(a.y[k]);
    const uintptr_t r0 = reinterpret_cast<uintptr_t>(a.r[k]);
    const uint64_t seed = static_cast<uint64_t>(a.random[0]), when = static_cast<uint64_t>(a.random[1]);
    const uint32_t k0 = static_cast<uint32_t>(seed), k1 = static_cast<uint32_t>(seed >> 32);
    const uint32_t c1 = static_cast<uint32_t>(a.first + k) << 16, c2 = static_cast<uint32_t>(when);
    const uint32_t c3 = static_cast<uint32_t>(when >> 32) << 16 | a.site;
    int64_t at = begin, row = begin / per;
    uint32_t col = begin % per;
    while (at < end) {
        u32x4 x[kAhead][N], r[RESIDUAL ? kAhead : 1][N];
        int64_t rows[kAhead], q[kAhead];
        uint32_t cols[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            rows[i] = row;
            cols[i] = col;
            q[i] = at;
            if (at < end) {
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    const int v = static_cast<int>(col) * N + n;
                    x[i][n] = load_ahead<T, EDGE>(x0 + row * a.x_ld, v, a.cols);
                    if (RESIDUAL) r[i][n] = load_ahead<T, EDGE>(r0 + row * a.r_ld, v, a.cols);
                }
            }
            at += step;
            row += step_rows;
            col += step_cols;
            if (col >= per) {
                col -= per;
                ++row;
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (q[i] >= end) break;
            const Words w = philox({{static_cast<uint32_t>(q[i]), static_cast<uint32_t>(q[i] >> 32) | c1, c2, c3}}, k0, k1);
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int v = static_cast<int>(cols[i]) * N + n;
                float f[V], g[V];
                Lane<T>::widen(x[i][n], f);
                settle<T, EDGE>(f, v, a.cols);
                if (RESIDUAL) {
                    Lane<T>::widen(r[i][n], g);
                    settle<T, EDGE>(g, v, a.cols);
                }
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const int b = n * V + e;
                    const uint32_t u = b % 2 ? w.w[b / 2] >> 16 : w.w[b / 2] & 0xffffu;
                    // (selected, not multiplied: what is dropped may be infinite)
                    const float t = f[e] * a.scale;
                    f[e] = u >= a.threshold ? (RESIDUAL ? t + g[e] : t) : (RESIDUAL ? g[e] : 0.0f);
                }
                store_vec<T, EDGE>(y0 + rows[i] * a.y_ld, v, a.cols, f);
            }
        }
    }
}

template <typename T>
void run(const DropArgs& a, bool residual, hipStream_t s) {
    const uint32_t n = a.wg[a.K];
    // whole vectors of eight columns, or a row that may end inside one
    if (a.cols % 8 == 0) {
        if (residual)
            dropout_kernel<T, true, false><<<n, kThreads, 0, s>>>(a);
        else
            dropout_kernel<T, false, false><<<n, kThreads, 0, s>>>(a);
    } else if (residual) {
        dropout_kernel<T, true, true><<<n, kThreads, 0, s>>>(a);
    } else {
        dropout_kernel<T, false, true><<<n, kThreads, 0, s>>>(a);
    }
}

}  // namespace

hipError_t launch_dropout(int K, const int64_t* rows, int64_t cols, const void* const* x, int64_t x_ld, int dtype,
                          const void* const* r, int64_t r_ld, void* const* y, int64_t y_ld, uint32_t threshold,
                          const int64_t* random, uint32_t site, hipStream_t s) {
    const int es = dtype == TC_BF16 ? 2 : 4;
    const int64_t per = (cols + 7) / 8;
    for (int k0 = 0; k0 < K; k0 += kWorkers) {
        DropArgs a{};
        a.K = K - k0 < kWorkers ? K - k0 : kWorkers;
        a.first = k0;
        a.cols = static_cast<int32_t>(cols);
        a.x_ld = x_ld * es;
        a.r_ld = r_ld * es;
        a.y_ld = y_ld * es;
        a.random = random;
        a.site = site;
        a.threshold = threshold;
        a.scale = threshold < 65536 ? 65536.0f / static_cast<float>(65536 - threshold) : 0.0f;
        int64_t total = 0;
        for (int k = 0; k < a.K; ++k) total += rows[k0 + k] * per;
        // two vectors of eight columns a lane, and in long calls as many as
        // leave each of the chip's 256 CUs eight workgroups
        constexpr int64_t kMost = 2048;
        int64_t each = 2 * kThreads;
        if (total > each * kMost) each = (total + kMost - 1) / kMost;
        for (int k = 0; k < a.K; ++k) {
            a.rows[k] = rows[k0 + k];
            a.x[k] = x[k0 + k];
            a.r[k] = r ? r[k0 + k] : nullptr;
            a.y[k] = y[k0 + k];
            a.wg[k + 1] = a.wg[k] + static_cast<uint32_t>((a.rows[k] * per + each - 1) / each);
        }
        if (a.wg[a.K] == 0) continue;
        if (dtype == TC_BF16)
            run<__bf16>(a, r != nullptr, s);
        else
            run<float>(a, r != nullptr, s);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

}  // namespace tc
