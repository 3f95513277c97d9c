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
// Eight workers' 4,096 x 4,096 bfloat16: 82 to 96 us from run to run, 6.5 to 5.6
// TB/s (the library's own copy reaches 6.5); with the residual 143 us, 5.6 TB/s.
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

// A lane makes the mask of a vector of eight columns, `kAhead` at a time.  In
// binary32 a vector is two pieces of 16 bytes; a wave takes its 128 pieces in
// their order, so that each access is of whole lines, and a lane has the bits of
// its piece from the lane that made them.  NT: the caches are passed by.
template <typename T, bool RESIDUAL, bool EDGE, bool NT>
__global__ void __launch_bounds__(kThreads) dropout_kernel(const DropArgs a) {
    constexpr int V = Lane<T>::kVec, N = 8 / V;  // 16-byte pieces of a vector
    constexpr int kAhead = 2;
    int k = 0;
    while (k + 1 < a.K && blockIdx.x >= a.wg[k + 1]) ++k;
    const uint32_t per = (static_cast<uint32_t>(a.cols) + 7) / 8;  // vectors of a row
    const uint32_t step = (a.wg[k + 1] - a.wg[k]) * kThreads;
    const uint32_t step_rows = step / per, step_cols = step % per * N;
    const uint32_t begin = (blockIdx.x - a.wg[k]) * kThreads + threadIdx.x, lane = threadIdx.x % 64;
    const int64_t end = a.rows[k] * per;
    const uintptr_t x0 = reinterpret_cast<uintptr_t>(a.x[k]), y0 = reinterpret_cast<uintptr_t>(a.y[k]);
    const uintptr_t r0 = reinterpret_cast<uintptr_t>(a.r[k]);
    const uint64_t seed = static_cast<uint64_t>(a.random[0]), when = static_cast<uint64_t>(a.random[1]);
    const uint32_t k0 = static_cast<uint32_t>(seed), k1 = static_cast<uint32_t>(seed >> 32);
    const uint32_t c1 = static_cast<uint32_t>(a.first + k) << 16, c2 = static_cast<uint32_t>(when);
    const uint32_t c3 = static_cast<uint32_t>(when >> 32) << 16 | a.site;
    // the lane's pieces: their vectors, rows, and places in the row
    struct Place {
        int64_t q, row;
        uint32_t v;
    } next[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const uint32_t q = begin - lane + (n * 64 + lane) / N;
        next[n] = {q, q / per, q % per * N + lane % N};
    }
    int64_t at = begin;
    while (at - lane < end) {  // (the same in all of a wave)
        u32x4 x[kAhead][N], r[RESIDUAL ? kAhead : 1][N];
        Place p[kAhead][N];
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int n = 0; n < N; ++n) {
                p[i][n] = next[n];
                if (next[n].q < end) {
                    x[i][n] = load_ahead<T, EDGE, NT>(x0 + next[n].row * a.x_ld, static_cast<int>(next[n].v), a.cols);
                    if (RESIDUAL) r[i][n] = load_ahead<T, EDGE, NT>(r0 + next[n].row * a.r_ld, static_cast<int>(next[n].v), a.cols);
                }
                next[n].q += step;
                next[n].row += step_rows;
                next[n].v += step_cols;
                if (next[n].v >= per * N) {
                    next[n].v -= per * N;
                    ++next[n].row;
                }
            }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const Words w = philox({{static_cast<uint32_t>(at), static_cast<uint32_t>(at >> 32) | c1, c2, c3}}, k0, k1);
            at += step;
            uint32_t keep = 0;
#pragma unroll
            for (int b = 0; b < 8; ++b) {
                const uint32_t u = b % 2 ? w.w[b / 2] >> 16 : w.w[b / 2] & 0xffffu;
                keep |= u >= a.threshold ? 1u << b : 0u;
            }
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const uint32_t bits = N == 1 ? keep : __shfl(keep, (n * 64 + lane) / N, 64) >> lane % N * V;
                if (p[i][n].q >= end) continue;
                const int v = static_cast<int>(p[i][n].v);
                float f[V], g[V];
                Lane<T>::widen(x[i][n], f);
                settle<T, EDGE>(f, v, a.cols);
                if (RESIDUAL) {
                    Lane<T>::widen(r[i][n], g);
                    settle<T, EDGE>(g, v, a.cols);
                }
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    // (selected, not multiplied: what is dropped may be infinite)
                    const float t = f[e] * a.scale;
                    f[e] = bits >> e & 1 ? (RESIDUAL ? t + g[e] : t) : (RESIDUAL ? g[e] : 0.0f);
                }
                store_vec<T, EDGE, NT>(y0 + p[i][n].row * a.y_ld, v, a.cols, f);
            }
        }
    }
}

template <typename T, bool RESIDUAL>
void run(const DropArgs& a, bool nt, hipStream_t s) {
    // whole vectors of eight columns, or a row that may end inside one
    if (a.cols % 8)
        dropout_kernel<T, RESIDUAL, true, false><<<a.wg[a.K], kThreads, 0, s>>>(a);
    else if (nt)
        dropout_kernel<T, RESIDUAL, false, true><<<a.wg[a.K], kThreads, 0, s>>>(a);
    else
        dropout_kernel<T, RESIDUAL, false, false><<<a.wg[a.K], kThreads, 0, s>>>(a);
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
        // two vectors of eight columns a lane, and in long calls more
        constexpr int64_t kMost = 8192;
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
        // What the last-level cache (256 MB) does not hold passes it by, if rows
        // are whole 16 bytes (in turn, 8 x 4,096 x 4,096 bfloat16 100 -> 83 us, with
        // the residual 147 -> 143); at other addresses it takes longer (30,000 x 4,003
        // float 182 -> 187).
        bool nt = total * 8 * es * (r ? 3 : 2) > int64_t{256} << 20 && (a.x_ld | a.y_ld | a.r_ld) % 16 == 0;
        for (int k = 0; k < a.K; ++k)
            nt = nt && (reinterpret_cast<uintptr_t>(a.x[k]) | reinterpret_cast<uintptr_t>(a.y[k]) | reinterpret_cast<uintptr_t>(a.r[k])) % 16 == 0;
        if (dtype == TC_BF16)
            r ? run<__bf16, true>(a, nt, s) : run<__bf16, false>(a, nt, s);
        else
            r ? run<float, true>(a, nt, s) : run<float, false>(a, nt, s);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

}  // namespace tc
