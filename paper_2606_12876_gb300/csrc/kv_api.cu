// C entry points of the key-value cache and the RMS norm (include/aq.h): argument validation and
// dispatch to the launchers.
#include <climits>
#include <cmath>
#include <initializer_list>

#include "kv.cuh"

namespace {

inline cudaStream_t as_stream(void* s) { return (cudaStream_t)s; }
inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

aq_status check_cache(const aq_kv_cache* c) {
    if (!c || c->layers < 1 || c->num_pages < 1 || c->page_tokens < 1 || c->kv_heads < 1 || c->head_dim < 1 ||
        c->max_seqs < 1 || c->max_pages < 1)
        return AQ_ERR_INVALID_ARG;
    if (c->dtype != AQ_F16 && c->dtype != AQ_BF16 && c->dtype != AQ_E4M3) return AQ_ERR_INVALID_ARG;
    if (c->page_tokens < 8 || c->page_tokens > 1024 || (c->page_tokens & (c->page_tokens - 1)))
        return AQ_ERR_UNSUPPORTED;
    if (c->head_dim % 16 || c->head_dim > 256) return AQ_ERR_UNSUPPORTED;
    // (token numbers are ints, with room for a chunk past the last one)
    if ((long long)c->max_pages * c->page_tokens > INT_MAX - 1023 || c->kv_heads > 16384) return AQ_ERR_UNSUPPORTED;
    return AQ_OK;
}

aq_status check_pools(const aq_kv_cache* c) {
    if (!c->k || !c->v || (c->dtype == AQ_E4M3 && (!c->k_scales || !c->v_scales))) return AQ_ERR_INVALID_ARG;
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_scales, 16) || !aligned(c->v_scales, 16))
        return AQ_ERR_ALIGNMENT;
    return AQ_OK;
}

aq_status check_books(const aq_kv_cache* c) {
    if (!c->tables || !c->lens || !c->refs) return AQ_ERR_INVALID_ARG;
    if (!aligned(c->tables, 4) || !aligned(c->lens, 4) || !aligned(c->refs, 4)) return AQ_ERR_ALIGNMENT;
    return AQ_OK;
}

// The checks that the calls on a cache share: the cache, its bookkeeping, n, int32 lists (which
// may be NULL) and the workspace.
aq_status check_call(const aq_kv_cache* c, int n, long long most, std::initializer_list<const void*> lists,
                     const void* workspace, size_t bytes, size_t need) {
    if (aq_status st = check_cache(c); st != AQ_OK) return st;
    if (aq_status st = check_books(c); st != AQ_OK) return st;
    if (n < 0 || n > most) return AQ_ERR_INVALID_ARG;
    for (const void* p : lists)
        if (!aligned(p, 4)) return AQ_ERR_ALIGNMENT;
    if (!workspace || bytes < need) return AQ_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return AQ_ERR_ALIGNMENT;
    return AQ_OK;
}

bool is_float(int dt) { return dt == AQ_F16 || dt == AQ_BF16 || dt == AQ_F32; }

}  // namespace

extern "C" {

size_t aq_kv_workspace_bytes(const aq_kv_cache* cache) {
    return check_cache(cache) == AQ_OK ? aq::kv_scratch_bytes(*cache) : 0;
}

aq_status aq_kv_init(const aq_kv_cache* cache, void* stream) {
    if (aq_status st = check_cache(cache); st != AQ_OK) return st;
    if (aq_status st = check_books(cache); st != AQ_OK) return st;
    return aq::launch_kv_init(*cache, as_stream(stream));
}

aq_status aq_kv_reserve(const aq_kv_cache* cache, int n, const int32_t* seqs, const int32_t* counts,
                        void* workspace, size_t workspace_bytes, void* stream) {
    if (aq_status st = check_call(cache, n, cache ? cache->max_seqs : 0, {seqs, counts}, workspace, workspace_bytes,
                                  aq_kv_workspace_bytes(cache));
        st != AQ_OK)
        return st;
    if (n == 0) return AQ_OK;
    return aq::launch_kv_reserve(*cache, n, seqs, counts, workspace, as_stream(stream));
}

aq_status aq_kv_fork(const aq_kv_cache* cache, int n, const int32_t* src, const int32_t* dst, void* workspace,
                     size_t workspace_bytes, void* stream) {
    if (aq_status st = check_call(cache, n, cache ? cache->max_seqs : 0, {src, dst}, workspace, workspace_bytes,
                                  aq_kv_workspace_bytes(cache));
        st != AQ_OK)
        return st;
    if (aq_status st = check_pools(cache); st != AQ_OK) return st;
    if (n == 0) return AQ_OK;
    if (!src || !dst) return AQ_ERR_INVALID_ARG;
    return aq::launch_kv_fork(*cache, n, src, dst, workspace, as_stream(stream));
}

aq_status aq_kv_free(const aq_kv_cache* cache, int n, const int32_t* seqs, void* workspace, size_t workspace_bytes,
                     void* stream) {
    if (aq_status st = check_call(cache, n, INT_MAX, {seqs}, workspace, workspace_bytes, aq_kv_workspace_bytes(cache));
        st != AQ_OK)
        return st;
    if (!seqs && n > cache->max_seqs) return AQ_ERR_INVALID_ARG;
    if (n == 0) return AQ_OK;
    return aq::launch_kv_free(*cache, n, seqs, workspace, as_stream(stream));
}

aq_status aq_kv_compact(const aq_kv_cache* cache, int32_t* used, void* workspace, size_t workspace_bytes,
                        void* stream) {
    if (aq_status st = check_call(cache, 0, 0, {used}, workspace, workspace_bytes, aq_kv_workspace_bytes(cache));
        st != AQ_OK)
        return st;
    if (aq_status st = check_pools(cache); st != AQ_OK) return st;
    return aq::launch_kv_compact(*cache, used, workspace, as_stream(stream));
}

aq_status aq_kv_copy_pages(const aq_kv_cache* cache, int n, const int32_t* src, const int32_t* dst,
                           void* workspace, size_t workspace_bytes, void* stream) {
    if (aq_status st = check_call(cache, n, INT_MAX, {src, dst}, workspace, workspace_bytes,
                                  aq_kv_workspace_bytes(cache));
        st != AQ_OK)
        return st;
    if (aq_status st = check_pools(cache); st != AQ_OK) return st;
    if (n == 0) return AQ_OK;
    if (!src || !dst) return AQ_ERR_INVALID_ARG;
    return aq::launch_kv_copy_pages(*cache, n, src, dst, workspace, as_stream(stream));
}

aq_status aq_kv_write(const aq_kv_cache* cache, int layer, int n, const int32_t* seqs, const int32_t* positions,
                      const void* k, const void* v, int x_dtype, int64_t row_stride, void* workspace,
                      size_t workspace_bytes, void* stream) {
    if (aq_status st = check_call(cache, n, INT_MAX, {seqs, positions}, workspace, workspace_bytes,
                                  aq_kv_workspace_bytes(cache));
        st != AQ_OK)
        return st;
    if (aq_status st = check_pools(cache); st != AQ_OK) return st;
    if (layer < 0 || layer >= cache->layers || !is_float(x_dtype)) return AQ_ERR_INVALID_ARG;
    if (row_stride < (int64_t)cache->kv_heads * cache->head_dim) return AQ_ERR_INVALID_ARG;
    if (!seqs && n > cache->max_seqs) return AQ_ERR_INVALID_ARG;
    if (n == 0) return AQ_OK;
    if (!k || !v) return AQ_ERR_INVALID_ARG;
    if (!aligned(k, 16) || !aligned(v, 16) || row_stride % 8) return AQ_ERR_ALIGNMENT;
    return aq::launch_kv_write(*cache, layer, n, seqs, positions, k, v, x_dtype, row_stride, workspace,
                               as_stream(stream));
}

size_t aq_kv_attend_workspace_bytes(const aq_kv_cache* cache, int n, int q_heads) {
    if (check_cache(cache) != AQ_OK || n < 0 || q_heads < 1 || q_heads % cache->kv_heads) return 0;
    return aq::kv_attend_ws_bytes(*cache, q_heads);
}

aq_status aq_kv_attend(const aq_kv_cache* cache, int layer, int n, const int32_t* seqs, const void* q, int q_dtype,
                       int64_t q_stride, int q_heads, float scale, int window, void* out, float* lse, void* workspace,
                       size_t workspace_bytes, void* stream) {
    if (aq_status st = check_call(cache, n, INT_MAX, {seqs, lse}, workspace, workspace_bytes,
                                  aq_kv_attend_workspace_bytes(cache, 0, q_heads));
        st != AQ_OK)
        return st;
    if (aq_status st = check_pools(cache); st != AQ_OK) return st;
    if (layer < 0 || layer >= cache->layers || q_heads < 1 || q_heads % cache->kv_heads || window < 0 ||
        !std::isfinite(scale))
        return AQ_ERR_INVALID_ARG;
    if (q_dtype != AQ_F16 && q_dtype != AQ_BF16) return AQ_ERR_INVALID_ARG;
    if ((cache->dtype != AQ_E4M3 && q_dtype != cache->dtype) || q_heads > 1 << 20) return AQ_ERR_UNSUPPORTED;
    if (q_stride < (int64_t)q_heads * cache->head_dim) return AQ_ERR_INVALID_ARG;
    if (!seqs && n > cache->max_seqs) return AQ_ERR_INVALID_ARG;
    if (n == 0) return AQ_OK;
    if (!q || !out) return AQ_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(out, 16) || q_stride % 8) return AQ_ERR_ALIGNMENT;
    aq::DeviceInfo di;
    if (aq_status st = aq::device_info(&di); st != AQ_OK) return st;
    return aq::launch_kv_attend(*cache, di, layer, n, seqs, q, q_dtype, q_stride, q_heads, scale, window, out, lse,
                                workspace, as_stream(stream));
}

aq_status aq_rmsnorm(int rows, int cols, const void* x, int x_dtype, int64_t x_stride, const void* residual,
                     void* residual_out, int r_dtype, const void* weight, int w_dtype, float eps, void* y,
                     int y_dtype, void* y_scales, int scale_block, void* stream) {
    if (rows < 0 || cols < 1 || x_stride < cols || !is_float(x_dtype) || !is_float(w_dtype) ||
        (!is_float(y_dtype) && y_dtype != AQ_E4M3) || !(eps >= 0.0f))
        return AQ_ERR_INVALID_ARG;
    if ((residual || residual_out) && !is_float(r_dtype)) return AQ_ERR_INVALID_ARG;
    if (cols % 8 || cols > 65536) return AQ_ERR_UNSUPPORTED;
    if (y_dtype == AQ_E4M3) {
        if (scale_block != 32 && scale_block != cols) return AQ_ERR_INVALID_ARG;
        if (cols % scale_block) return AQ_ERR_UNSUPPORTED;
    }
    if (rows == 0) return AQ_OK;
    if (!x || !weight || !y || (y_dtype == AQ_E4M3 && !y_scales)) return AQ_ERR_INVALID_ARG;
    for (const void* p : {x, residual, (const void*)residual_out, weight, (const void*)y})
        if (!aligned(p, 16)) return AQ_ERR_ALIGNMENT;
    if (x_stride % 8) return AQ_ERR_ALIGNMENT;
    return aq::launch_rmsnorm(rows, cols, x, x_dtype, x_stride, residual, residual_out, r_dtype, weight, w_dtype, eps,
                              y, y_dtype, (uint8_t*)y_scales, scale_block, as_stream(stream));
}

}  // extern "C"
