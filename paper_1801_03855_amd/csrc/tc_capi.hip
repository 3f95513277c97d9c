// C entry points: argument validation, descriptors, dispatch to launchers.
#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <new>
#include <string>

#include "tc_internal.h"

namespace tc {

static thread_local std::string t_error;

void set_error(const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    t_error = buf;
}

void clear_error() { t_error.clear(); }

namespace {

int32_t fail(int32_t code, const char* what) {
    set_error("%s", what);
    return code;
}

int32_t hip_fail(hipError_t e, const char* where) {
    set_error("%s: %s", where, hipGetErrorString(e));
    return TC_EHIP;
}

int elem_size(int32_t dtype) { return dtype == TC_BF16 ? 2 : dtype == TC_F32 ? 4 : 0; }

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// [p, p + bytes) and [q, q + bytes2) share a byte.
bool overlap(const void* p, int64_t bytes, const void* q, int64_t bytes2) {
    auto a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
    return a < b + static_cast<uintptr_t>(bytes2) && b < a + static_cast<uintptr_t>(bytes);
}

// The group's device must be the current one.
int32_t check_device(const tc_group* g) {
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
    if (dev != g->device) {
        set_error("the group lives on device %d but device %d is current", g->device, dev);
        return TC_EINVAL;
    }
    return TC_OK;
}

}  // namespace
}  // namespace tc

using namespace tc;

TC_API const char* tc_last_error(void) { return t_error.c_str(); }

TC_API int32_t tc_version(void) { return 100; }

// ---------------------------------------------------------------- groups

TC_API tc_group* tc_group_create(const int64_t* sizes, int32_t n) {
    clear_error();
    if (n < 1) { set_error("n must be >= 1 (got %d)", n); return nullptr; }
    if (!sizes) { set_error("sizes is NULL"); return nullptr; }
    auto* g = new (std::nothrow) tc_group();
    if (!g) { set_error("out of host memory"); return nullptr; }
    g->n = n;
    g->sizes.assign(sizes, sizes + n);
    g->offsets.resize(static_cast<size_t>(n) + 1);
    g->offsets[0] = 0;
    for (int32_t t = 0; t < n; ++t) {
        if (sizes[t] < 0) { set_error("sizes[%d] = %lld is negative", t, (long long)sizes[t]); delete g; return nullptr; }
        if (sizes[t] > INT64_MAX / 8 - g->offsets[t]) { set_error("group too large"); delete g; return nullptr; }
        g->offsets[t + 1] = g->offsets[t] + sizes[t];
    }
    g->N = g->offsets[n];
    g->large = g->N / n >= TC_PACK_LARGE_MEAN;
    g->sep.chunk = g->large ? TC_PACK_CHUNK_LARGE : TC_PACK_CHUNK_SMALL;
    g->tpack.chunk = TC_TPACK_CHUNK;
    g->pipe.chunk = TC_PIPE_CHUNK;
    g->pipe_fine.chunk = TC_PIPE_CHUNK_FINE;
    // 2-byte elements on groups of large tensors: chunks of twice the
    // elements, the bytes of a binary32 chunk (measured on MI355X, bfloat16
    // pack and unpack on ResNet-50 at K = 2-16 and VGG-16 at K = 4: 13-17%
    // faster than 2,048 elements; on 10,000 small tensors 8,192 elements
    // against 4,096 measured +12% to -5%, and they keep 4,096)
    g->sep2.chunk = g->large ? 2 * TC_PACK_CHUNK_LARGE : TC_PACK_CHUNK_SMALL;
    // first[b]: the tensor holding flat position b*chunk, i.e. the last
    // tensor whose offset is <= that position (zero-size tensors at the same
    // offset come before the one that holds it).  The final entry is the
    // tensor holding position N-1.
    auto tensor_at = [&](int64_t j) {
        auto it = std::upper_bound(g->offsets.begin(), g->offsets.begin() + n, j);
        return static_cast<int32_t>(it - g->offsets.begin()) - 1;
    };
    for (tc_chunking* c : {&g->sep, &g->tpack, &g->pipe, &g->pipe_fine, &g->sep2}) {
        c->nchunks = (g->N + c->chunk - 1) / c->chunk;
        if (c->nchunks > INT32_MAX / 2) { set_error("group too large"); delete g; return nullptr; }
        c->first.resize(static_cast<size_t>(c->nchunks) + 1);
        for (int64_t b = 0; b < c->nchunks; ++b) c->first[b] = tensor_at(b * c->chunk);
        c->first[c->nchunks] = g->N > 0 ? tensor_at(g->N - 1) : 0;
    }
    g->slot_bounds = true;
    for (int32_t t = 1; t < n; ++t)
        if (g->offsets[t] % 4 != 0 && g->offsets[t] < g->N / 4 * 4) g->slot_bounds = false;

    hipError_t e = hipGetDevice(&g->device);
    if (e != hipSuccess) { hip_fail(e, "hipGetDevice"); delete g; return nullptr; }
    size_t ob = g->offsets.size() * sizeof(int64_t);
    if ((e = hipMalloc(&g->d_offsets, ob)) != hipSuccess ||
        (e = hipMemcpy(g->d_offsets, g->offsets.data(), ob, hipMemcpyHostToDevice)) != hipSuccess) {
        hip_fail(e, "group offset table");
        tc_group_destroy(g);
        return nullptr;
    }
    for (tc_chunking* c : {&g->sep, &g->tpack, &g->pipe, &g->pipe_fine, &g->sep2}) {
        const size_t cb = c->first.size() * sizeof(int32_t);
        if ((e = hipMalloc(&c->d_first, cb)) != hipSuccess ||
            (e = hipMemcpy(c->d_first, c->first.data(), cb, hipMemcpyHostToDevice)) != hipSuccess) {
            hip_fail(e, "group chunk table");
            tc_group_destroy(g);
            return nullptr;
        }
    }
    return g;
}

TC_API void tc_group_destroy(tc_group* g) {
    if (!g) return;
    if (g->d_offsets) (void)hipFree(g->d_offsets);
    for (tc_chunking* c : {&g->sep, &g->tpack, &g->pipe, &g->pipe_fine, &g->sep2})
        if (c->d_first) (void)hipFree(c->d_first);
    delete g;
}

TC_API int64_t tc_group_numel(const tc_group* g) { return g ? g->N : -1; }

TC_API int32_t tc_group_ntensors(const tc_group* g) { return g ? g->n : -1; }

TC_API int32_t tc_group_offsets(const tc_group* g, int64_t* out) {
    clear_error();
    if (!g || !out) return fail(TC_EINVAL, "tc_group_offsets: NULL argument");
    std::memcpy(out, g->offsets.data(), g->offsets.size() * sizeof(int64_t));
    return TC_OK;
}

// ----------------------------------------------------------- tensor lists

TC_API tc_tensorlist* tc_tensorlist_create(const tc_group* g, int32_t K, const void* const* ptrs,
                                           int32_t dtype) {
    clear_error();
    if (!g || !ptrs) { set_error("tc_tensorlist_create: NULL argument"); return nullptr; }
    if (K < 1 || K > TC_MAX_K) { set_error("K = %d outside [1, %d]", K, TC_MAX_K); return nullptr; }
    const int es = elem_size(dtype);
    if (!es) { set_error("unknown dtype %d", dtype); return nullptr; }
    if (check_device(g) != TC_OK) return nullptr;
    for (int32_t k = 0; k < K; ++k)
        for (int32_t t = 0; t < g->n; ++t) {
            const void* p = ptrs[static_cast<int64_t>(k) * g->n + t];
            if (g->sizes[t] == 0) continue;
            if (!p) { set_error("tensor %d of copy %d is NULL", t, k); return nullptr; }
            if (!aligned(p, es)) { set_error("tensor %d of copy %d is not %d-byte aligned", t, k, es); return nullptr; }
        }
    auto* tl = new (std::nothrow) tc_tensorlist();
    if (!tl) { set_error("out of host memory"); return nullptr; }
    tl->g = g;
    tl->K = K;
    tl->dtype = dtype;
    tl->elem = es;
    tl->ptrs.assign(ptrs, ptrs + static_cast<int64_t>(K) * g->n);
    uintptr_t bits = 0;
    for (int64_t q = 0; q < static_cast<int64_t>(tl->ptrs.size()); ++q)
        if (g->sizes[q % g->n] > 0) bits |= reinterpret_cast<uintptr_t>(tl->ptrs[q]);
    tl->slot_aligned = (bits & static_cast<uintptr_t>(4 * es - 1)) == 0;
    const size_t bytes = tl->ptrs.size() * sizeof(void*);
    hipError_t e = hipMalloc(&tl->d_ptrs, bytes);
    if (e != hipSuccess) { hip_fail(e, "hipMalloc (pointer table)"); delete tl; return nullptr; }
    e = hipMemcpy(tl->d_ptrs, tl->ptrs.data(), bytes, hipMemcpyHostToDevice);
    if (e != hipSuccess) { hip_fail(e, "hipMemcpy (pointer table)"); tc_tensorlist_destroy(tl); return nullptr; }
    return tl;
}

TC_API void tc_tensorlist_destroy(tc_tensorlist* tl) {
    if (!tl) return;
    if (tl->d_ptrs) (void)hipFree(tl->d_ptrs);
    delete tl;
}

// ------------------------------------------------------------ pack/unpack

static int32_t pack_common(const tc_tensorlist* tl, void* const* flat, bool unpack, void* stream) {
    clear_error();
    if (!tl || !flat) return fail(TC_EINVAL, "NULL argument");
    const tc_group* g = tl->g;
    if (int32_t r = check_device(g)) return r;
    if (g->N == 0) return TC_OK;
    const int64_t bytes = g->N * tl->elem;
    for (int32_t k = 0; k < tl->K; ++k) {
        if (!flat[k]) { set_error("flat[%d] is NULL", k); return TC_EINVAL; }
        if (!aligned(flat[k], tl->elem)) { set_error("flat[%d] is not element-aligned", k); return TC_EINVAL; }
        for (int32_t q = 0; q < k; ++q)
            if (overlap(flat[k], bytes, flat[q], bytes)) { set_error("flat[%d] overlaps flat[%d]", k, q); return TC_EINVAL; }
    }
    hipError_t e = launch_pack(tl, flat, unpack, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, unpack ? "tc_unpack launch" : "tc_pack launch");
    return TC_OK;
}

TC_API int32_t tc_pack(const tc_tensorlist* tl, void* const* flat, void* stream) {
    return pack_common(tl, flat, false, stream);
}

TC_API int32_t tc_unpack(const tc_tensorlist* tl, const void* const* flat, void* stream) {
    return pack_common(tl, const_cast<void* const*>(flat), true, stream);
}

// ----------------------------------------------------------------- reduce

TC_API int32_t tc_reduce_ex(const tc_group* g, int32_t K, const void* const* in, int32_t in_dtype,
                            float* out, int32_t op, void* stream) {
    clear_error();
    if (!g) return fail(TC_EINVAL, "group is NULL");
    if (K < 1 || K > TC_MAX_K) { set_error("K = %d outside [1, %d]", K, TC_MAX_K); return TC_EINVAL; }
    if (op != TC_SUM && op != TC_AVG) { set_error("unknown op %d", op); return TC_EINVAL; }
    const int es = elem_size(in_dtype);
    if (!es) { set_error("unknown dtype %d", in_dtype); return TC_EINVAL; }
    if (int32_t r = check_device(g)) return r;
    if (g->N == 0) return TC_OK;
    if (!in || !out) return fail(TC_EINVAL, "NULL buffer");
    bool vec = aligned(out, 16);
    if (!aligned(out, 4)) return fail(TC_EINVAL, "out is not 4-byte aligned");
    for (int32_t i = 0; i < K; ++i) {
        if (!in[i]) { set_error("in[%d] is NULL", i); return TC_EINVAL; }
        if (!aligned(in[i], es)) { set_error("in[%d] is not element-aligned", i); return TC_EINVAL; }
        vec = vec && aligned(in[i], es == 4 ? 16 : 8);
        // in place is allowed only as exact identity with a binary32 input:
        // a binary32 output slot covers two bfloat16 input slots, which
        // other lanes read
        if (overlap(in[i], g->N * es, out, g->N * 4) && (in[i] != out || in_dtype != TC_F32)) {
            set_error(in_dtype == TC_F32 ? "out partially overlaps in[%d]"
                                         : "out overlaps in[%d] (no in-place reduction of bfloat16 inputs)", i);
            return TC_EINVAL;
        }
    }
    hipError_t e = launch_reduce(K, in, in_dtype, out, op, g->N, vec, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "tc_reduce launch");
    return TC_OK;
}

TC_API int32_t tc_reduce(const tc_group* g, int32_t K, const float* const* in, float* out, int32_t op,
                         void* stream) {
    return tc_reduce_ex(g, K, reinterpret_cast<const void* const*>(in), TC_F32, out, op, stream);
}

// ------------------------------------------------------------------ easgd

// The step alone (fused false; out and op unused), or fused with the
// reduction of the gradients into out.
static int32_t easgd_common(const tc_group* g, int32_t K, float* const* x, const void* const* grad, int32_t g_dtype,
                            float* x_c, bool fused, float* out, int32_t op, float eta, float rho, void* stream,
                            const char* what) {
    clear_error();
    if (!g) return fail(TC_EINVAL, "group is NULL");
    if (K < 1 || K > TC_MAX_K) { set_error("K = %d outside [1, %d]", K, TC_MAX_K); return TC_EINVAL; }
    const int es = elem_size(g_dtype);
    if (!es) { set_error("unknown dtype %d", g_dtype); return TC_EINVAL; }
    if (fused && op != TC_SUM && op != TC_AVG) { set_error("unknown op %d", op); return TC_EINVAL; }
    if (!std::isfinite(eta) || !std::isfinite(rho)) return fail(TC_EINVAL, "eta and rho must be finite");
    if (int32_t r = check_device(g)) return r;
    if (g->N == 0) return TC_OK;
    if (!x || !grad || !x_c || (fused && !out)) return fail(TC_EINVAL, "NULL buffer");
    const int64_t xb = g->N * 4, gb = g->N * es;
    if (!aligned(x_c, 4)) return fail(TC_EINVAL, "x_c is not 4-byte aligned");
    bool vec = aligned(x_c, 16);
    if (out) {
        if (!aligned(out, 4)) return fail(TC_EINVAL, "out is not 4-byte aligned");
        if (overlap(out, xb, x_c, xb)) return fail(TC_EINVAL, "out overlaps x_c");
        vec = vec && aligned(out, 16);
    }
    for (int32_t i = 0; i < K; ++i) {
        if (!x[i] || !grad[i]) { set_error("x[%d] or grad[%d] is NULL", i, i); return TC_EINVAL; }
        if (!aligned(x[i], 4) || !aligned(grad[i], es)) { set_error("x[%d] or grad[%d] misaligned", i, i); return TC_EINVAL; }
        vec = vec && aligned(x[i], 16) && aligned(grad[i], es == 4 ? 16 : 8);
        if (overlap(x[i], xb, x_c, xb)) { set_error("x[%d] overlaps x_c", i); return TC_EINVAL; }
        if (overlap(grad[i], gb, x_c, xb)) { set_error("grad[%d] overlaps x_c", i); return TC_EINVAL; }
        if (out && overlap(out, xb, x[i], xb)) { set_error("out overlaps x[%d]", i); return TC_EINVAL; }
        if (out && overlap(out, xb, grad[i], gb)) { set_error("out overlaps grad[%d]", i); return TC_EINVAL; }
        for (int32_t q = 0; q < K; ++q) {
            if (q < i && overlap(x[i], xb, x[q], xb)) { set_error("x[%d] overlaps x[%d]", i, q); return TC_EINVAL; }
            if (overlap(grad[q], gb, x[i], xb)) { set_error("grad[%d] overlaps x[%d]", q, i); return TC_EINVAL; }
        }
    }
    hipError_t e = launch_easgd(K, x, grad, g_dtype, x_c, out, op, eta, rho, g->N, vec,
                                static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, what);
    return TC_OK;
}

TC_API int32_t easgd_step_ex(const tc_group* g, int32_t K, float* const* x, const void* const* grad,
                             int32_t g_dtype, float* x_c, float eta, float rho, void* stream) {
    return easgd_common(g, K, x, grad, g_dtype, x_c, false, nullptr, TC_SUM, eta, rho, stream, "easgd_step launch");
}

TC_API int32_t reduce_easgd_step(const tc_group* g, int32_t K, float* const* x, const void* const* grad,
                                 int32_t g_dtype, float* x_c, float* out, int32_t op, float eta, float rho,
                                 void* stream) {
    return easgd_common(g, K, x, grad, g_dtype, x_c, true, out, op, eta, rho, stream, "reduce_easgd_step launch");
}

TC_API int32_t easgd_step(const tc_group* g, int32_t K, float* const* x, const float* const* grad, float* x_c,
                          float eta, float rho, void* stream) {
    return easgd_step_ex(g, K, x, reinterpret_cast<const void* const*>(grad), TC_F32, x_c, eta, rho, stream);
}

// ---------------------------------------------------------- tensor layout

TC_API int64_t tc_tensor_numel(const tc_group* g, int32_t K) {
    if (!g || K < 1 || K > TC_MAX_K) return -1;
    return (g->N + 3) / 4 * 4 * K;
}

static int32_t tensor_pack_common(const tc_tensorlist* tl, void* tensor, bool unpack, void* stream) {
    clear_error();
    if (!tl) return fail(TC_EINVAL, "NULL tensor list");
    const tc_group* g = tl->g;
    if (int32_t r = check_device(g)) return r;
    if (g->N == 0) return TC_OK;
    if (!tensor) return fail(TC_EINVAL, "tensor is NULL");
    if (!aligned(tensor, 16)) return fail(TC_EINVAL, "tensor buffers must be 16-byte aligned");
    hipError_t e = launch_tensor_pack(tl, tensor, unpack, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, unpack ? "tc_unpack_tensor launch" : "tc_pack_tensor launch");
    return TC_OK;
}

TC_API int32_t tc_pack_tensor(const tc_tensorlist* tl, void* tensor, void* stream) {
    return tensor_pack_common(tl, tensor, false, stream);
}

TC_API int32_t tc_unpack_tensor(const tc_tensorlist* tl, const void* tensor, void* stream) {
    return tensor_pack_common(tl, const_cast<void*>(tensor), true, stream);
}

TC_API int32_t tc_reduce_tensor(const tc_group* g, int32_t K, const void* in, int32_t in_dtype, float* out,
                                int32_t op, void* stream) {
    clear_error();
    if (!g) return fail(TC_EINVAL, "group is NULL");
    if (K < 1 || K > TC_MAX_K) { set_error("K = %d outside [1, %d]", K, TC_MAX_K); return TC_EINVAL; }
    if (op != TC_SUM && op != TC_AVG) { set_error("unknown op %d", op); return TC_EINVAL; }
    const int es = elem_size(in_dtype);
    if (!es) { set_error("unknown dtype %d", in_dtype); return TC_EINVAL; }
    if (int32_t r = check_device(g)) return r;
    if (g->N == 0) return TC_OK;
    if (!in || !out) return fail(TC_EINVAL, "NULL buffer");
    if (!aligned(in, 16) || !aligned(out, 16)) return fail(TC_EINVAL, "tensor-layout calls need 16-byte aligned buffers");
    if (overlap(in, tc_tensor_numel(g, K) * es, out, g->N * 4)) return fail(TC_EINVAL, "out overlaps the input tensor");
    hipError_t e = launch_tensor_reduce(K, in, in_dtype, out, op, g->N, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "tc_reduce_tensor launch");
    return TC_OK;
}

// As easgd_common, on tensor-layout buffers.
static int32_t tensor_easgd_common(const tc_group* g, int32_t K, float* x, const void* grad, int32_t g_dtype,
                                   float* x_c, bool fused, float* out, int32_t op, float eta, float rho,
                                   void* stream, const char* what) {
    clear_error();
    if (!g) return fail(TC_EINVAL, "group is NULL");
    if (K < 1 || K > TC_MAX_K) { set_error("K = %d outside [1, %d]", K, TC_MAX_K); return TC_EINVAL; }
    const int es = elem_size(g_dtype);
    if (!es) { set_error("unknown dtype %d", g_dtype); return TC_EINVAL; }
    if (fused && op != TC_SUM && op != TC_AVG) { set_error("unknown op %d", op); return TC_EINVAL; }
    if (!std::isfinite(eta) || !std::isfinite(rho)) return fail(TC_EINVAL, "eta and rho must be finite");
    if (int32_t r = check_device(g)) return r;
    if (g->N == 0) return TC_OK;
    if (!x || !grad || !x_c || (fused && !out)) return fail(TC_EINVAL, "NULL buffer");
    if (!aligned(x, 16) || !aligned(grad, 16) || !aligned(x_c, 16) || (out && !aligned(out, 16)))
        return fail(TC_EINVAL, "tensor-layout calls need 16-byte aligned buffers");
    const int64_t tn = tc_tensor_numel(g, K);
    if (overlap(x, tn * 4, grad, tn * es)) return fail(TC_EINVAL, "x overlaps grad");
    if (overlap(x, tn * 4, x_c, g->N * 4)) return fail(TC_EINVAL, "x overlaps x_c");
    if (overlap(grad, tn * es, x_c, g->N * 4)) return fail(TC_EINVAL, "grad overlaps x_c");
    if (out && (overlap(out, g->N * 4, x, tn * 4) || overlap(out, g->N * 4, grad, tn * es) ||
                overlap(out, g->N * 4, x_c, g->N * 4)))
        return fail(TC_EINVAL, "out overlaps x, grad or x_c");
    hipError_t e = launch_tensor_easgd(K, x, grad, g_dtype, x_c, out, op, eta, rho, g->N,
                                       static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, what);
    return TC_OK;
}

TC_API int32_t easgd_step_tensor(const tc_group* g, int32_t K, float* x, const void* grad, int32_t g_dtype,
                                 float* x_c, float eta, float rho, void* stream) {
    return tensor_easgd_common(g, K, x, grad, g_dtype, x_c, false, nullptr, TC_SUM, eta, rho, stream,
                               "easgd_step_tensor launch");
}

TC_API int32_t reduce_easgd_step_tensor(const tc_group* g, int32_t K, float* x, const void* grad, int32_t g_dtype,
                                        float* x_c, float* out, int32_t op, float eta, float rho, void* stream) {
    return tensor_easgd_common(g, K, x, grad, g_dtype, x_c, true, out, op, eta, rho, stream,
                               "reduce_easgd_step_tensor launch");
}

// ------------------------------------------- schedules and synchronous SGD

namespace {

// Shared checks of the separate-buffer step calls: K, finite scalars, the
// device; returns TC_OK or an error (N == 0 is reported as TC_OK by the
// caller before buffers are inspected).
int32_t check_step(const tc_group* g, int32_t K, int32_t g_dtype, float s0, float s1) {
    if (!g) return fail(TC_EINVAL, "group is NULL");
    if (K < 1 || K > TC_MAX_K) { set_error("K = %d outside [1, %d]", K, TC_MAX_K); return TC_EINVAL; }
    if (!elem_size(g_dtype)) { set_error("unknown dtype %d", g_dtype); return TC_EINVAL; }
    if (!std::isfinite(s0) || !std::isfinite(s1)) return fail(TC_EINVAL, "step sizes must be finite");
    return check_device(g);
}

// x[0..K) pairwise disjoint, each 4-byte aligned; *vec &= 16-byte aligned.
int32_t check_workers(const tc_group* g, int32_t K, float* const* x, bool* vec) {
    if (!x) return fail(TC_EINVAL, "NULL buffer array");
    const int64_t xb = g->N * 4;
    for (int32_t i = 0; i < K; ++i) {
        if (!x[i]) { set_error("x[%d] is NULL", i); return TC_EINVAL; }
        if (!aligned(x[i], 4)) { set_error("x[%d] misaligned", i); return TC_EINVAL; }
        *vec = *vec && aligned(x[i], 16);
        for (int32_t q = 0; q < i; ++q)
            if (overlap(x[i], xb, x[q], xb)) { set_error("x[%d] overlaps x[%d]", i, q); return TC_EINVAL; }
    }
    return TC_OK;
}

// grad[0..K) element-aligned and disjoint from every x (and from each other
// when `writable`).
int32_t check_grads(const tc_group* g, int32_t K, const void* const* grad, int es, float* const* x, bool writable,
                    bool* vec) {
    if (!grad) return fail(TC_EINVAL, "NULL buffer array");
    const int64_t gb = g->N * es, xb = g->N * 4;
    for (int32_t i = 0; i < K; ++i) {
        if (!grad[i]) { set_error("grad[%d] is NULL", i); return TC_EINVAL; }
        if (!aligned(grad[i], es)) { set_error("grad[%d] misaligned", i); return TC_EINVAL; }
        *vec = *vec && aligned(grad[i], es == 4 ? 16 : 8);
        for (int32_t q = 0; q < K; ++q) {
            if (overlap(grad[i], gb, x[q], xb)) { set_error("grad[%d] overlaps x[%d]", i, q); return TC_EINVAL; }
            if (writable && q < i && overlap(grad[i], gb, grad[q], gb)) {
                set_error("grad[%d] overlaps grad[%d]", i, q);
                return TC_EINVAL;
            }
        }
    }
    return TC_OK;
}

int32_t launched(hipError_t e, const char* what) { return e == hipSuccess ? TC_OK : hip_fail(e, what); }

int32_t check_tensor_step(const tc_group* g, const void* x, int64_t xbytes, const void* grad, int64_t gbytes) {
    if (!x || (gbytes && !grad)) return fail(TC_EINVAL, "NULL buffer");
    if (!aligned(x, 16) || (gbytes && !aligned(grad, 16)))
        return fail(TC_EINVAL, "tensor-layout calls need 16-byte aligned buffers");
    if (gbytes && overlap(x, xbytes, grad, gbytes)) return fail(TC_EINVAL, "x overlaps grad");
    (void)g;
    return TC_OK;
}

int32_t check_order(int32_t K, const int32_t* order, int32_t R) {
    if (R < 0 || R > K) { set_error("R = %d outside [0, K = %d]", R, K); return TC_EINVAL; }
    if (R && !order) return fail(TC_EINVAL, "order is NULL");
    bool seen[TC_MAX_K] = {};
    for (int32_t r = 0; r < R; ++r) {
        if (order[r] < 0 || order[r] >= K) { set_error("order[%d] = %d outside [0, K)", r, order[r]); return TC_EINVAL; }
        if (seen[order[r]]) { set_error("worker %d exchanges twice", order[r]); return TC_EINVAL; }
        seen[order[r]] = true;
    }
    return TC_OK;
}

}  // namespace

TC_API int32_t sgd_step(const tc_group* g, int32_t K, float* const* x, const void* const* grad, int32_t g_dtype,
                        float eta, void* stream) {
    clear_error();
    if (int32_t r = check_step(g, K, g_dtype, eta, 0.0f)) return r;
    if (g->N == 0) return TC_OK;
    bool vec = true;
    if (int32_t r = check_workers(g, K, x, &vec)) return r;
    if (int32_t r = check_grads(g, K, grad, elem_size(g_dtype), x, false, &vec)) return r;
    return launched(launch_sgd(K, x, grad, g_dtype, eta, g->N, vec, static_cast<hipStream_t>(stream)), "sgd_step launch");
}

TC_API int32_t sgd_step_tensor(const tc_group* g, int32_t K, float* x, const void* grad, int32_t g_dtype, float eta,
                               void* stream) {
    clear_error();
    if (int32_t r = check_step(g, K, g_dtype, eta, 0.0f)) return r;
    if (g->N == 0) return TC_OK;
    const int64_t tn = tc_tensor_numel(g, K);
    if (int32_t r = check_tensor_step(g, x, tn * 4, grad, tn * elem_size(g_dtype))) return r;
    return launched(launch_tensor_sgd(K, x, grad, g_dtype, eta, g->N, static_cast<hipStream_t>(stream)),
                    "sgd_step_tensor launch");
}

TC_API int32_t easgd_period_step(const tc_group* g, int32_t K, float* const* x, const void* const* grad,
                                 int32_t g_dtype, float* x_c, float eta, float rho, int64_t iteration, int32_t tau,
                                 void* stream) {
    clear_error();
    if (tau < 1 || iteration < 0) { set_error("need tau >= 1 and iteration >= 0"); return TC_EINVAL; }
    if (iteration % tau == 0) return easgd_step_ex(g, K, x, grad, g_dtype, x_c, eta, rho, stream);
    return sgd_step(g, K, x, grad, g_dtype, eta, stream);
}

TC_API int32_t easgd_period_step_tensor(const tc_group* g, int32_t K, float* x, const void* grad, int32_t g_dtype,
                                        float* x_c, float eta, float rho, int64_t iteration, int32_t tau,
                                        void* stream) {
    clear_error();
    if (tau < 1 || iteration < 0) { set_error("need tau >= 1 and iteration >= 0"); return TC_EINVAL; }
    if (iteration % tau == 0) return easgd_step_tensor(g, K, x, grad, g_dtype, x_c, eta, rho, stream);
    return sgd_step_tensor(g, K, x, grad, g_dtype, eta, stream);
}

TC_API int32_t elastic_async(const tc_group* g, int32_t K, float* const* x, float* x_c, const int32_t* order,
                             int32_t R, float alpha, void* stream) {
    clear_error();
    if (int32_t r = check_step(g, K, TC_F32, alpha, 0.0f)) return r;
    if (int32_t r = check_order(K, order, R)) return r;
    if (g->N == 0 || R == 0) return TC_OK;
    bool vec = true;
    if (int32_t r = check_workers(g, K, x, &vec)) return r;
    if (!x_c || !aligned(x_c, 4)) return fail(TC_EINVAL, "x_c is NULL or misaligned");
    vec = vec && aligned(x_c, 16);
    for (int32_t i = 0; i < K; ++i)
        if (overlap(x[i], g->N * 4, x_c, g->N * 4)) { set_error("x[%d] overlaps x_c", i); return TC_EINVAL; }
    return launched(launch_elastic_async(K, x, x_c, order, R, alpha, g->N, vec, static_cast<hipStream_t>(stream)),
                    "elastic_async launch");
}

TC_API int32_t elastic_async_tensor(const tc_group* g, int32_t K, float* x, float* x_c, const int32_t* order,
                                    int32_t R, float alpha, void* stream) {
    clear_error();
    if (int32_t r = check_step(g, K, TC_F32, alpha, 0.0f)) return r;
    if (int32_t r = check_order(K, order, R)) return r;
    if (g->N == 0 || R == 0) return TC_OK;
    const int64_t tn = tc_tensor_numel(g, K);
    if (int32_t r = check_tensor_step(g, x, tn * 4, x_c, g->N * 4)) return r;
    return launched(launch_tensor_elastic_async(K, x, x_c, order, R, alpha, g->N, static_cast<hipStream_t>(stream)),
                    "elastic_async_tensor launch");
}

TC_API int32_t sync_sgd_step(const tc_group* g, int32_t K, float* const* x, void* const* grad, int32_t g_dtype,
                             float eta, float rescale, int32_t broadcast, void* stream) {
    clear_error();
    if (int32_t r = check_step(g, K, g_dtype, eta, rescale)) return r;
    if (broadcast && g_dtype != TC_F32)
        return fail(TC_EUNSUPPORTED, "broadcasting the summed gradient needs binary32 gradients");
    if (g->N == 0) return TC_OK;
    bool vec = true;
    if (int32_t r = check_workers(g, K, x, &vec)) return r;
    if (int32_t r = check_grads(g, K, const_cast<const void* const*>(grad), elem_size(g_dtype), x, broadcast != 0, &vec))
        return r;
    return launched(launch_sync_sgd(K, x, grad, g_dtype, eta, rescale, broadcast, g->N, vec,
                                    static_cast<hipStream_t>(stream)),
                    "sync_sgd_step launch");
}

TC_API int32_t sync_sgd_step_tensor(const tc_group* g, int32_t K, float* x, void* grad, int32_t g_dtype, float eta,
                                    float rescale, int32_t broadcast, void* stream) {
    clear_error();
    if (int32_t r = check_step(g, K, g_dtype, eta, rescale)) return r;
    if (broadcast && g_dtype != TC_F32)
        return fail(TC_EUNSUPPORTED, "broadcasting the summed gradient needs binary32 gradients");
    if (g->N == 0) return TC_OK;
    const int64_t tn = tc_tensor_numel(g, K);
    if (int32_t r = check_tensor_step(g, x, tn * 4, grad, tn * elem_size(g_dtype))) return r;
    return launched(launch_tensor_sync_sgd(K, x, grad, g_dtype, eta, rescale, broadcast, g->N,
                                           static_cast<hipStream_t>(stream)),
                    "sync_sgd_step_tensor launch");
}

TC_API int32_t tc_broadcast(const tc_group* g, int32_t K, const void* src, void* const* dst, int32_t dtype,
                            void* stream) {
    clear_error();
    if (int32_t r = check_step(g, K, dtype, 0.0f, 0.0f)) return r;
    if (g->N == 0) return TC_OK;
    const int es = elem_size(dtype);
    const int64_t b = g->N * es;
    if (!src || !dst) return fail(TC_EINVAL, "NULL buffer");
    if (!aligned(src, es)) return fail(TC_EINVAL, "src misaligned");
    bool vec = aligned(src, 16);
    for (int32_t i = 0; i < K; ++i) {
        if (!dst[i] || !aligned(dst[i], es)) { set_error("dst[%d] is NULL or misaligned", i); return TC_EINVAL; }
        vec = vec && aligned(dst[i], 16);
        if (overlap(dst[i], b, src, b)) { set_error("dst[%d] overlaps src", i); return TC_EINVAL; }
        for (int32_t q = 0; q < i; ++q)
            if (overlap(dst[i], b, dst[q], b)) { set_error("dst[%d] overlaps dst[%d]", i, q); return TC_EINVAL; }
    }
    return launched(launch_broadcast(K, src, dst, es, g->N, vec, static_cast<hipStream_t>(stream)), "tc_broadcast launch");
}

TC_API int32_t tc_broadcast_tensor(const tc_group* g, int32_t K, const void* src, void* dst, int32_t dtype,
                                   void* stream) {
    clear_error();
    if (int32_t r = check_step(g, K, dtype, 0.0f, 0.0f)) return r;
    if (g->N == 0) return TC_OK;
    const int es = elem_size(dtype);
    if (!src || !dst) return fail(TC_EINVAL, "NULL buffer");
    if (!aligned(src, 16) || !aligned(dst, 16)) return fail(TC_EINVAL, "tensor-layout calls need 16-byte aligned buffers");
    if (overlap(dst, tc_tensor_numel(g, K) * es, src, g->N * es)) return fail(TC_EINVAL, "dst overlaps src");
    return launched(launch_tensor_broadcast(K, src, dst, es, g->N, static_cast<hipStream_t>(stream)),
                    "tc_broadcast_tensor launch");
}

// ------------------------------------------------------------ pipeline

TC_API int32_t easgd_pipeline_tensor(const tc_tensorlist* grads, const tc_tensorlist* params, void* g_tensor,
                                     float* gbar, float* x, float* x_c, float eta, float rho, void* stream) {
    clear_error();
    if (!grads || !params) return fail(TC_EINVAL, "NULL tensor list");
    const tc_group* g = grads->g;
    if (params->g != g) return fail(TC_EINVAL, "the gradient and parameter lists belong to different groups");
    if (params->K != grads->K) return fail(TC_EINVAL, "the gradient and parameter lists have different K");
    if (params->dtype != TC_F32) return fail(TC_EINVAL, "parameter tensors must be binary32");
    if (!std::isfinite(eta) || !std::isfinite(rho)) return fail(TC_EINVAL, "eta and rho must be finite");
    if (int32_t r = check_device(g)) return r;
    if (g->N == 0) return TC_OK;
    if (!gbar || !x || !x_c) return fail(TC_EINVAL, "NULL buffer");
    if (!aligned(gbar, 16) || !aligned(x, 16) || !aligned(x_c, 16) || (g_tensor && !aligned(g_tensor, 16)))
        return fail(TC_EINVAL, "tensor-layout calls need 16-byte aligned buffers");
    const int K = grads->K;
    const int64_t tn = tc_tensor_numel(g, K), nb = g->N * 4;
    const int64_t gtb = g_tensor ? tn * grads->elem : 0;
    if (overlap(x, tn * 4, x_c, nb)) return fail(TC_EINVAL, "x overlaps x_c");
    if (overlap(x, tn * 4, gbar, nb)) return fail(TC_EINVAL, "x overlaps gbar");
    if (overlap(x_c, nb, gbar, nb)) return fail(TC_EINVAL, "x_c overlaps gbar");
    if (gtb && (overlap(g_tensor, gtb, x, tn * 4) || overlap(g_tensor, gtb, x_c, nb) || overlap(g_tensor, gtb, gbar, nb)))
        return fail(TC_EINVAL, "g_tensor overlaps another buffer");
    return launched(launch_tensor_pipeline(grads, params, g_tensor, gbar, x, x_c, eta, rho,
                                           static_cast<hipStream_t>(stream)),
                    "easgd_pipeline_tensor launch");
}

// -------------------------------------------------------------- layer norm

namespace {

// K workers' rows of one buffer argument: `cols` elements every `ld`.
struct Rows {
    const void* const* p;
    int64_t ld;
    int es;
    const char* name;
};

// Memory that a call reads or writes: one block, or `width` bytes every `line`
// (line > 0).
struct Span {
    uintptr_t lo, hi;
    int64_t line, width;
    const char* name;
    int32_t k;
    bool rows, written;
};

// A block shares a byte with rows.
bool block_in_rows(const Span& block, const Span& rows) {
    if (block.lo < rows.lo) return block.hi > rows.lo;
    const int64_t at = static_cast<int64_t>(block.lo - rows.lo) % rows.line;
    // the row it starts in or behind; the next one, if there is one
    return at < rows.width || static_cast<uintptr_t>(rows.line - at) < std::min(block.hi, rows.hi) - block.lo;
}

// Two spans share a byte.  Views of one wider buffer (equal strides) may
// interleave without sharing any.
bool share(const Span& a, const Span& b) {
    if (a.lo >= b.hi || b.lo >= a.hi) return false;
    if (!a.line) return !b.line || block_in_rows(a, b);
    if (!b.line) return block_in_rows(b, a);
    if (a.line != b.line) return true;
    int64_t at = static_cast<int64_t>(b.lo - a.lo) % a.line;
    if (at < 0) at += a.line;
    return at < a.width || at + b.width > a.line;
}

// What one call reads and writes, every worker's.
struct Spans {
    Span s[10 * TC_MAX_K + 1];
    int n = 0;

    void add(const void* p, int64_t bytes, const char* name, int32_t k, bool written) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        if (p && bytes > 0) s[n++] = {at, at + bytes, 0, 0, name, k, false, written};
    }
    void add(const Rows& r, int32_t k, int64_t rows, int64_t cols, bool written) {
        if (rows == 0) return;
        add(r.p[k], ((rows - 1) * r.ld + cols) * r.es, r.name, k, written);
        s[n - 1].rows = true;
        if (rows > 1) {
            s[n - 1].line = r.ld * r.es;
            s[n - 1].width = cols * r.es;
        }
    }
    // What is written shares nothing with what else is written or read, except
    // that a worker's rows may take the place of its own, element for element.
    int32_t check() {
        std::sort(s, s + n, [](const Span& a, const Span& b) { return a.lo < b.lo; });
        for (int i = 0; i < n; ++i)
            for (int j = i + 1; j < n && s[j].lo < s[i].hi; ++j) {
                const Span &a = s[i], &b = s[j];
                if ((!a.written && !b.written) || !share(a, b)) continue;
                if (a.rows && b.rows && a.written != b.written && a.k == b.k && a.lo == b.lo && a.line == b.line) continue;
                set_error("%s[%d] overlaps %s[%d]", a.name, a.k, b.name, b.k);
                return TC_EINVAL;
            }
        return TC_OK;
    }
};

int32_t check_rows(int32_t K, const int64_t* rows, int64_t cols, const Rows& r) {
    if (!r.p) { set_error("%s is NULL", r.name); return TC_EINVAL; }
    int64_t most = 0;
    for (int32_t k = 0; k < K; ++k) {
        most = rows[k] > most ? rows[k] : most;
        if (rows[k] == 0) continue;
        if (!r.p[k]) { set_error("%s[%d] is NULL", r.name, k); return TC_EINVAL; }
        if (!aligned(r.p[k], r.es)) { set_error("%s[%d] is not element-aligned", r.name, k); return TC_EINVAL; }
    }
    if (r.ld < cols) {
        set_error("%s: a row stride of %lld is less than the %lld columns", r.name, (long long)r.ld, (long long)cols);
        return TC_EINVAL;
    }
    if (most > 0 && r.ld > INT64_MAX / 8 / most) { set_error("%s is too large", r.name); return TC_EINVAL; }
    return TC_OK;
}

// Optional per-worker arrays of `n` elements of es bytes each; `rows` given:
// a worker without rows needs none.
int32_t check_vectors(int32_t K, const int64_t* rows, const void* const* p, int es, const char* name) {
    for (int32_t k = 0; k < K; ++k) {
        if (rows && rows[k] == 0) continue;
        if (!p[k]) { set_error("%s[%d] is NULL", name, k); return TC_EINVAL; }
        if (!aligned(p[k], es)) { set_error("%s[%d] is not element-aligned", name, k); return TC_EINVAL; }
    }
    return TC_OK;
}

// The rows' memory belongs to the current device, whose stream the call's work
// goes to (calls without a group have no device of their own to compare).
// dweight: what is written of workers without rows, if anything is.
int32_t check_row_device(int32_t K, const int64_t* rows, const void* const* p, const char* name,
                         const void* const* dweight = nullptr) {
    int dev = -1;
    if (hipError_t e = hipGetDevice(&dev)) return hip_fail(e, "hipGetDevice");
    for (const bool with : {true, false}) {
        const void* const* at_k = with ? p : dweight;
        for (int32_t k = 0; k < K && at_k; ++k) {
            if ((rows[k] > 0) != with) continue;
            hipPointerAttribute_t at{};
            if (hipPointerGetAttributes(&at, at_k[k]) != hipSuccess) {
                (void)hipGetLastError();  // not the runtime's memory: nothing is known of it
            } else if (at.type == hipMemoryTypeDevice && at.device != dev) {
                set_error("%s[%d] is on device %d but device %d is current", with ? name : "dweight", k, at.device, dev);
                return TC_EINVAL;
            }
        }
    }
    return TC_OK;
}

int32_t check_norm(int32_t K, const int64_t* rows, int64_t cols, int32_t dtype) {
    if (K < 1 || K > TC_MAX_K) { set_error("K = %d outside [1, %d]", K, TC_MAX_K); return TC_EINVAL; }
    if (!rows) return fail(TC_EINVAL, "rows is NULL");
    if (cols < 1 || cols > TC_MAX_NORM_COLS) {
        set_error("cols = %lld outside [1, %d]", (long long)cols, TC_MAX_NORM_COLS);
        return TC_EINVAL;
    }
    for (int32_t k = 0; k < K; ++k)
        if (rows[k] < 0) { set_error("rows[%d] = %lld is negative", k, (long long)rows[k]); return TC_EINVAL; }
    if (!elem_size(dtype)) { set_error("unknown dtype %d", dtype); return TC_EINVAL; }
    return TC_OK;
}

}  // namespace

TC_API int32_t tc_layernorm(int32_t K, const int64_t* rows, int64_t cols, const void* const* x, int64_t x_ld,
                            int32_t dtype, const float* const* weight, const float* const* bias, void* const* y,
                            int64_t y_ld, float* const* mean, float* const* rstd, float eps, void* stream) {
    clear_error();
    if (int32_t r = check_norm(K, rows, cols, dtype)) return r;
    if (!std::isfinite(eps) || eps < 0.0f) return fail(TC_EINVAL, "eps must be finite and not negative");
    const int es = elem_size(dtype);
    const Rows in{x, x_ld, es, "x"}, out{y, y_ld, es, "y"};
    if (int32_t r = check_rows(K, rows, cols, in)) return r;
    if (int32_t r = check_rows(K, rows, cols, out)) return r;
    const struct { const void* const* p; const char* name; } vectors[] = {
        {reinterpret_cast<const void* const*>(weight), "weight"}, {reinterpret_cast<const void* const*>(bias), "bias"},
        {reinterpret_cast<const void* const*>(mean), "mean"}, {reinterpret_cast<const void* const*>(rstd), "rstd"}};
    for (auto& v : vectors)
        if (v.p)
            if (int32_t r = check_vectors(K, rows, v.p, 4, v.name)) return r;
    Spans spans;
    for (int32_t k = 0; k < K; ++k) {
        if (rows[k] == 0) continue;
        spans.add(in, k, rows[k], cols, false);
        spans.add(out, k, rows[k], cols, true);
        if (weight) spans.add(weight[k], cols * 4, "weight", k, false);
        if (bias) spans.add(bias[k], cols * 4, "bias", k, false);
        if (mean) spans.add(mean[k], rows[k] * 4, "mean", k, true);
        if (rstd) spans.add(rstd[k], rows[k] * 4, "rstd", k, true);
    }
    if (int32_t r = spans.check()) return r;
    if (int32_t r = check_row_device(K, rows, x, "x")) return r;
    hipError_t e = launch_layernorm(K, rows, cols, x, x_ld, dtype, weight, bias, y, y_ld, mean, rstd, eps,
                                    static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "tc_layernorm launch");
    return TC_OK;
}

TC_API int64_t tc_layernorm_workspace(int32_t K, const int64_t* rows, int64_t cols) {
    clear_error();
    if (check_norm(K, rows, cols, TC_F32) != TC_OK) return -1;
    return layernorm_workspace(K, rows, cols);
}

TC_API int32_t tc_layernorm_backward(int32_t K, const int64_t* rows, int64_t cols, const void* const* dy, int64_t dy_ld,
                                     const void* const* x, int64_t x_ld, int32_t dtype, const float* const* weight,
                                     const float* const* mean, const float* const* rstd, void* const* dx, int64_t dx_ld,
                                     void* const* dweight, void* const* dbias, int32_t w_dtype, void* workspace,
                                     int64_t workspace_bytes, void* stream) {
    clear_error();
    if (int32_t r = check_norm(K, rows, cols, dtype)) return r;
    const int es = elem_size(dtype), ws = elem_size(w_dtype);
    if (!ws) { set_error("unknown dtype %d of dweight and dbias", w_dtype); return TC_EINVAL; }
    const Rows in[2] = {{dy, dy_ld, es, "dy"}, {x, x_ld, es, "x"}}, out{dx, dx_ld, es, "dx"};
    if (int32_t r = check_rows(K, rows, cols, in[0])) return r;
    if (int32_t r = check_rows(K, rows, cols, in[1])) return r;
    if (int32_t r = check_rows(K, rows, cols, out)) return r;
    if (!mean || !rstd || !dweight || !dbias) return fail(TC_EINVAL, "mean, rstd, dweight or dbias is NULL");
    if (weight)
        if (int32_t r = check_vectors(K, rows, reinterpret_cast<const void* const*>(weight), 4, "weight")) return r;
    if (int32_t r = check_vectors(K, rows, reinterpret_cast<const void* const*>(mean), 4, "mean")) return r;
    if (int32_t r = check_vectors(K, rows, reinterpret_cast<const void* const*>(rstd), 4, "rstd")) return r;
    if (int32_t r = check_vectors(K, nullptr, const_cast<const void* const*>(dweight), ws, "dweight")) return r;
    if (int32_t r = check_vectors(K, nullptr, const_cast<const void* const*>(dbias), ws, "dbias")) return r;
    const int64_t need = layernorm_workspace(K, rows, cols);
    if (!workspace || !aligned(workspace, 16)) return fail(TC_EINVAL, "workspace is NULL or not 16-byte aligned");
    if (workspace_bytes < need) {
        set_error("the workspace has %lld bytes, %lld are needed", (long long)workspace_bytes, (long long)need);
        return TC_EINVAL;
    }
    Spans spans;
    for (int32_t k = 0; k < K; ++k) {
        spans.add(dweight[k], cols * ws, "dweight", k, true);
        spans.add(dbias[k], cols * ws, "dbias", k, true);
        if (rows[k] == 0) continue;
        for (const Rows* r : {&in[0], &in[1], &out}) spans.add(*r, k, rows[k], cols, r == &out);
        if (weight) spans.add(weight[k], cols * 4, "weight", k, false);
        spans.add(mean[k], rows[k] * 4, "mean", k, false);
        spans.add(rstd[k], rows[k] * 4, "rstd", k, false);
    }
    spans.add(workspace, need, "workspace", 0, true);
    if (int32_t r = spans.check()) return r;
    if (int32_t r = check_row_device(K, rows, x, "x", const_cast<const void* const*>(dweight))) return r;
    hipError_t e = launch_layernorm_backward(K, rows, cols, dy, dy_ld, x, x_ld, dtype, weight, mean, rstd, dx, dx_ld,
                                             dweight, dbias, w_dtype, workspace, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "tc_layernorm_backward launch");
    return TC_OK;
}

// ---------------------------------------------------------------------- dropout

namespace {

// Both directions: residual only forward, `in` and `out` the names of the rows.
int32_t run_dropout(int32_t K, const int64_t* rows, int64_t cols, const Rows& in, int32_t dtype, const Rows* residual,
                    const Rows& out, float p, const int64_t* random, int64_t site, void* stream) {
    if (!(p >= 0.0f && p <= 1.0f)) return fail(TC_EINVAL, "p must be in [0, 1]");
    if (site < 0 || site > 65535) { set_error("site = %lld outside [0, 65535]", (long long)site); return TC_EINVAL; }
    if (!random || !aligned(random, 8)) return fail(TC_EINVAL, "random is NULL or not 8-byte aligned");
    for (int32_t k = 0; k < K; ++k)
        if (rows[k] > (int64_t{1} << 48) / cols) { set_error("rows[%d] * cols is more than 2^48", k); return TC_EINVAL; }
    if (int32_t r = check_rows(K, rows, cols, in)) return r;
    if (residual)
        if (int32_t r = check_rows(K, rows, cols, *residual)) return r;
    if (int32_t r = check_rows(K, rows, cols, out)) return r;
    Spans spans;
    for (int32_t k = 0; k < K; ++k) {
        spans.add(in, k, rows[k], cols, false);
        if (residual) spans.add(*residual, k, rows[k], cols, false);
        spans.add(out, k, rows[k], cols, true);
    }
    spans.add(random, 16, "random", 0, false);
    if (int32_t r = spans.check()) return r;
    if (int32_t r = check_row_device(K, rows, in.p, in.name)) return r;
    const uint32_t threshold = static_cast<uint32_t>(std::floor(static_cast<double>(p) * 65536.0 + 0.5));
    hipError_t e = launch_dropout(K, rows, cols, in.p, in.ld, dtype, residual ? residual->p : nullptr,
                                  residual ? residual->ld : 0, const_cast<void* const*>(out.p), out.ld, threshold, random,
                                  static_cast<uint32_t>(site), static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "dropout launch");
    return TC_OK;
}

}  // namespace

TC_API int32_t tc_dropout(int32_t K, const int64_t* rows, int64_t cols, const void* const* x, int64_t x_ld, int32_t dtype,
                          const void* const* residual, int64_t r_ld, void* const* y, int64_t y_ld, float p,
                          const int64_t* random, int64_t site, void* stream) {
    clear_error();
    if (int32_t r = check_norm(K, rows, cols, dtype)) return r;
    const int es = elem_size(dtype);
    const Rows add{residual, r_ld, es, "residual"};
    return run_dropout(K, rows, cols, {x, x_ld, es, "x"}, dtype, residual ? &add : nullptr, {y, y_ld, es, "y"}, p, random,
                       site, stream);
}

TC_API int32_t tc_dropout_backward(int32_t K, const int64_t* rows, int64_t cols, const void* const* dy, int64_t dy_ld,
                                   int32_t dtype, void* const* dx, int64_t dx_ld, float p, const int64_t* random,
                                   int64_t site, void* stream) {
    clear_error();
    if (int32_t r = check_norm(K, rows, cols, dtype)) return r;
    const int es = elem_size(dtype);
    return run_dropout(K, rows, cols, {dy, dy_ld, es, "dy"}, dtype, nullptr, {dx, dx_ld, es, "dx"}, p, random, site, stream);
}

// ---------------------------------------------------------------- cross entropy

namespace {

int32_t check_loss(int32_t K, const int64_t* rows, int64_t cols, int64_t classes, int32_t dtype, int32_t w_dtype) {
    if (int32_t r = check_norm(K, rows, cols, dtype)) return r;
    if (cols > TC_MAX_CE_COLS) { set_error("cols = %lld is more than %d", (long long)cols, TC_MAX_CE_COLS); return TC_EINVAL; }
    if (classes < 1 || classes > TC_MAX_CLASSES) {
        set_error("classes = %lld outside [1, %d]", (long long)classes, TC_MAX_CLASSES);
        return TC_EINVAL;
    }
    for (int32_t k = 0; k < K; ++k)
        if (rows[k] > TC_MAX_CE_ROWS) { set_error("rows[%d] = %lld is more than %d", k, (long long)rows[k], TC_MAX_CE_ROWS); return TC_EINVAL; }
    for (int32_t k = -1; k < K; ++k)
        if ((k < 0 ? classes : rows[k]) > TC_MAX_CE_SIZE / cols) {
            set_error(k < 0 ? "the weight has more than 2^36 elements" : "rows[%d] * cols is more than 2^36", k);
            return TC_EINVAL;
        }
    if (!elem_size(w_dtype)) { set_error("unknown dtype %d of weight and bias", w_dtype); return TC_EINVAL; }
    return TC_OK;
}

int32_t run_loss(LossCall& c, int64_t workspace_bytes, void* stream, const char* name) {
    const int32_t K = c.K;
    const int64_t *rows = c.rows, cols = c.cols, classes = c.classes;
    const int es = elem_size(c.dtype), ws = elem_size(c.w_dtype), dws = elem_size(c.dw_dtype);
    const Rows in{c.x, c.x_ld, es, "x"}, out{c.dx, c.dx_ld, es, "dx"};
    if (int32_t r = check_rows(K, rows, cols, in)) return r;
    if (c.backward)
        if (int32_t r = check_rows(K, rows, cols, out)) return r;
    // one vector (or matrix) a worker
    const struct Vector {
        const void* const* p;
        int64_t each;  // elements; 0: one a row
        int es;
        const char* name;
        bool wanted, written, always;
    } vectors[] = {
        {c.weight, classes * cols, ws, "weight", true, false, false},
        {c.bias, classes, ws, "bias", c.bias != nullptr, false, false},
        {reinterpret_cast<const void* const*>(c.label), 0, 8, "label", true, false, false},
        {reinterpret_cast<const void* const*>(c.loss), 0, 4, "loss", !c.backward, true, false},
        {c.backward ? reinterpret_cast<const void* const*>(c.lse_in) : reinterpret_cast<const void* const*>(c.lse), 0, 4,
         "lse", true, !c.backward, false},
        {reinterpret_cast<const void* const*>(c.dloss), 0, 4, "dloss", c.dloss != nullptr, false, false},
        {const_cast<const void* const*>(c.dweight), classes * cols, dws, "dweight", c.backward, true, true},
        {const_cast<const void* const*>(c.dbias), classes, dws, "dbias", c.dbias != nullptr, true, true},
    };
    for (const Vector& v : vectors) {
        if (!v.wanted) continue;
        if (!v.p) { set_error("%s is NULL", v.name); return TC_EINVAL; }
        if (int32_t r = check_vectors(K, v.always ? nullptr : rows, v.p, v.es, v.name)) return r;
    }
    const int64_t need = cross_entropy_workspace(K, rows, cols, classes, c.dtype, c.w_dtype, c.backward, c.dw_dtype);
    if (!c.workspace || !aligned(c.workspace, 256)) return fail(TC_EINVAL, "workspace is NULL or not 256-byte aligned");
    if (workspace_bytes < need) {
        set_error("the workspace has %lld bytes, %lld are needed", (long long)workspace_bytes, (long long)need);
        return TC_EINVAL;
    }
    Spans spans;
    for (int32_t k = 0; k < K; ++k) {
        for (const Vector& v : vectors)
            if (v.wanted && (v.always || rows[k] > 0)) spans.add(v.p[k], (v.each ? v.each : rows[k]) * v.es, v.name, k, v.written);
        spans.add(in, k, rows[k], cols, false);
        if (c.backward) spans.add(out, k, rows[k], cols, true);
    }
    spans.add(c.workspace, need, "workspace", 0, true);
    if (int32_t r = spans.check()) return r;
    if (int32_t r = check_row_device(K, rows, c.x, "x", const_cast<const void* const*>(c.dweight))) return r;
    hipError_t e = launch_cross_entropy(c, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, name);
    return TC_OK;
}

}  // namespace

TC_API int64_t tc_cross_entropy_workspace(int32_t K, const int64_t* rows, int64_t cols, int64_t classes, int32_t dtype,
                                          int32_t w_dtype) {
    clear_error();
    if (check_loss(K, rows, cols, classes, dtype, w_dtype) != TC_OK) return -1;
    return cross_entropy_workspace(K, rows, cols, classes, dtype, w_dtype, false, TC_F32);
}

TC_API int32_t tc_cross_entropy(int32_t K, const int64_t* rows, int64_t cols, int64_t classes, const void* const* x,
                                int64_t x_ld, int32_t dtype, const void* const* weight, const void* const* bias,
                                int32_t w_dtype, const int64_t* const* label, float* const* loss, float* const* lse,
                                void* workspace, int64_t workspace_bytes, void* stream) {
    clear_error();
    if (int32_t r = check_loss(K, rows, cols, classes, dtype, w_dtype)) return r;
    LossCall c;
    c.K = K;
    c.rows = rows;
    c.cols = cols;
    c.classes = classes;
    c.x = x;
    c.x_ld = x_ld;
    c.dtype = dtype;
    c.w_dtype = w_dtype;
    c.weight = weight;
    c.bias = bias;
    c.label = label;
    c.workspace = workspace;
    c.loss = loss;
    c.lse = lse;
    return run_loss(c, workspace_bytes, stream, "tc_cross_entropy launch");
}

TC_API int64_t tc_cross_entropy_backward_workspace(int32_t K, const int64_t* rows, int64_t cols, int64_t classes,
                                                   int32_t dtype, int32_t w_dtype, int32_t dw_dtype) {
    clear_error();
    if (check_loss(K, rows, cols, classes, dtype, w_dtype) != TC_OK) return -1;
    if (!elem_size(dw_dtype)) { set_error("unknown dtype %d of dweight and dbias", dw_dtype); return -1; }
    return cross_entropy_workspace(K, rows, cols, classes, dtype, w_dtype, true, dw_dtype);
}

TC_API int32_t tc_cross_entropy_backward(int32_t K, const int64_t* rows, int64_t cols, int64_t classes,
                                         const void* const* x, int64_t x_ld, int32_t dtype, const void* const* weight,
                                         const void* const* bias, int32_t w_dtype, const int64_t* const* label,
                                         const float* const* lse, const float* const* dloss, float scale, void* const* dx,
                                         int64_t dx_ld, void* const* dweight, void* const* dbias, int32_t dw_dtype,
                                         void* workspace, int64_t workspace_bytes, void* stream) {
    clear_error();
    if (int32_t r = check_loss(K, rows, cols, classes, dtype, w_dtype)) return r;
    if (!elem_size(dw_dtype)) { set_error("unknown dtype %d of dweight and dbias", dw_dtype); return TC_EINVAL; }
    if (!std::isfinite(scale)) return fail(TC_EINVAL, "scale must be finite");
    LossCall c;
    c.K = K;
    c.rows = rows;
    c.cols = cols;
    c.classes = classes;
    c.x = x;
    c.x_ld = x_ld;
    c.dtype = dtype;
    c.w_dtype = w_dtype;
    c.weight = weight;
    c.bias = bias;
    c.label = label;
    c.workspace = workspace;
    c.backward = true;
    c.lse_in = lse;
    c.dloss = dloss;
    c.scale = scale;
    c.dx = dx;
    c.dx_ld = dx_ld;
    c.dweight = dweight;
    c.dbias = dbias;
    c.dw_dtype = dw_dtype;
    return run_loss(c, workspace_bytes, stream, "tc_cross_entropy_backward launch");
}

// ------------------------------------------------------- orthogonalised update

TC_API tc_ortho* tc_ortho_create(const tc_group* g, int32_t K, const int64_t* rows, const int64_t* cols,
                                 const float* scale) {
    clear_error();
    if (!g || !rows || !cols) { set_error("tc_ortho_create: NULL argument"); return nullptr; }
    if (K < 1 || K > TC_MAX_K) { set_error("K = %d outside [1, %d]", K, TC_MAX_K); return nullptr; }
    if (check_device(g) != TC_OK) return nullptr;
    for (int32_t t = 0; t < g->n; ++t) {
        if (scale && !std::isfinite(scale[t])) { set_error("scale[%d] is not finite", t); return nullptr; }
        if (rows[t] == 0 && cols[t] == 0) continue;  // no matrix
        if (rows[t] < 0 || cols[t] < 0 || (rows[t] > 0 && cols[t] != g->sizes[t] / rows[t]) || rows[t] * cols[t] != g->sizes[t]) {
            set_error("tensor %d has %lld elements and is no %lld x %lld matrix", t, (long long)g->sizes[t],
                      (long long)rows[t], (long long)cols[t]);
            return nullptr;
        }
        if (std::min(rows[t], cols[t]) > TC_MAX_ORTHO_SIDE || std::max(rows[t], cols[t]) > TC_MAX_ORTHO_LONG) {
            set_error("tensor %d: a %lld x %lld matrix is too large", t, (long long)rows[t], (long long)cols[t]);
            return nullptr;
        }
    }
    hipError_t e = hipSuccess;
    tc_ortho* o = nullptr;
    try {
        o = make_ortho(g, K, rows, cols, scale, &e);
    } catch (const std::bad_alloc&) {
        set_error("out of host memory");
        return nullptr;
    }
    if (!o) hip_fail(e, "tc_ortho_create (device tables)");
    return o;
}

TC_API void tc_ortho_destroy(tc_ortho* o) {
    if (o) destroy_ortho(o);
}

TC_API int64_t tc_ortho_workspace(const tc_ortho* o) { return o ? ortho_workspace(o) : -1; }

TC_API int32_t tc_orthogonalize(const tc_ortho* o, const void* const* grad, int32_t g_dtype, float* const* momentum,
                                float mu, int32_t nesterov, void* const* out, int32_t out_dtype, int32_t steps,
                                const float* coeff, float eps, void* workspace, int64_t workspace_bytes, void* stream) {
    clear_error();
    if (!o) return fail(TC_EINVAL, "the plan is NULL");
    const tc_group* g = ortho_group(o);
    const int32_t K = ortho_copies(o);
    const int gs = elem_size(g_dtype), os = elem_size(out_dtype);
    if (!gs || !os) { set_error("unknown dtype %d", gs ? out_dtype : g_dtype); return TC_EINVAL; }
    if (steps < 1 || steps > TC_MAX_ORTHO_STEPS) { set_error("steps = %d outside [1, %d]", steps, TC_MAX_ORTHO_STEPS); return TC_EINVAL; }
    if (!coeff) return fail(TC_EINVAL, "coeff is NULL");
    for (int i = 0; i < 3 * steps; ++i)
        if (!std::isfinite(coeff[i])) return fail(TC_EINVAL, "the coefficients must be finite");
    if (!std::isfinite(mu) || !std::isfinite(eps) || eps <= 0.0f) return fail(TC_EINVAL, "mu must be finite, eps finite and positive");
    if (!ortho_in_range(o, steps, coeff)) return fail(TC_EINVAL, "the coefficients let the iteration leave its range");
    if (int32_t r = check_device(g)) return r;
    if (g->N == 0) return TC_OK;
    if (!grad || !out) return fail(TC_EINVAL, "NULL buffer");
    const int64_t gb = g->N * gs, ob = g->N * os, mb = g->N * 4, need = ortho_workspace(o);
    if (need > 0 && (!workspace || !aligned(workspace, 256))) return fail(TC_EINVAL, "workspace is NULL or not 256-byte aligned");
    if (workspace_bytes < need) {
        set_error("the workspace has %lld bytes, %lld are needed", (long long)workspace_bytes, (long long)need);
        return TC_EINVAL;
    }
    for (int32_t k = 0; k < K; ++k) {
        if (!grad[k] || !out[k] || (momentum && !momentum[k])) { set_error("a buffer of copy %d is NULL", k); return TC_EINVAL; }
        if (!aligned(grad[k], gs) || !aligned(out[k], os) || (momentum && !aligned(momentum[k], 4))) {
            set_error("a buffer of copy %d is not element-aligned", k);
            return TC_EINVAL;
        }
        if (need > 0 && (overlap(grad[k], gb, workspace, need) || overlap(out[k], ob, workspace, need) ||
                         (momentum && overlap(momentum[k], mb, workspace, need)))) {
            set_error("a buffer of copy %d overlaps the workspace", k);
            return TC_EINVAL;
        }
    }
    for (int32_t k = 0; k < K; ++k)
        for (int32_t q = 0; q < K; ++q) {
            // a copy's update may take the place of its own gradient
            if (overlap(out[k], ob, grad[q], gb) && !(k == q && out[k] == grad[q] && g_dtype == out_dtype)) {
                set_error("out[%d] overlaps grad[%d]", k, q);
                return TC_EINVAL;
            }
            if (q < k && overlap(out[k], ob, out[q], ob)) { set_error("out[%d] overlaps out[%d]", k, q); return TC_EINVAL; }
            if (!momentum) continue;
            if (overlap(momentum[k], mb, grad[q], gb) || overlap(momentum[k], mb, out[q], ob) ||
                (q < k && overlap(momentum[k], mb, momentum[q], mb))) {
                set_error("momentum[%d] overlaps a buffer of copy %d", k, q);
                return TC_EINVAL;
            }
        }
    hipError_t e = launch_ortho(o, grad, g_dtype, momentum, mu, nesterov != 0, out, out_dtype, steps, coeff, eps, workspace,
                                static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "tc_orthogonalize launch");
    return TC_OK;
}
