// C ABI of libfa_mi355.so, continued: rotary positions with several axes, and the pages of a cache.  Argument validation and dispatch;
// include/fa_mi355.h holds the contract of every entry point.
#include "fa_cache_check.h"

namespace {

int rope_axes_any(const void* q, const long long* q_strides, const void* k, const long long* k_strides, void* q_out,
                  const long long* q_out_strides, void* k_out, const long long* k_out_strides, const double* inv_freq,
                  const int* axis, const int* positions, int axes, int B, int H, int H_kv, int N, int d, int rot_dim, float amplitude,
                  int interleaved, int dtype, bool transposed, void* stream) {
    if (!axis || !positions) return FA_ERR_NULL;
    Rotation r;
    const int st = check_rotation(r, q, q_strides, k, k_strides, q_out, q_out_strides, k_out, k_out_strides, inv_freq, positions, B, H, H_kv,
                                  N, d, rot_dim, amplitude, interleaved, dtype);
    if (st != FA_OK) return st;
    if (axes <= 0) return FA_ERR_SHAPE;
    if (!aligned_to(axis, 4)) return FA_ERR_ALIGN;
    forget_stale_hip_error();
    return fa::launch_rope_axes(r.q, r.k, r.q_out, r.k_out, inv_freq, positions, axis, axes, B, H, H_kv, N, d, rot_dim, amplitude,
                                interleaved, transposed, dtype, static_cast<hipStream_t>(stream));
}

// What every call on the pages of a pool has to keep to
int check_pool(int B, int n_pages, int max_pages) {
    if (B <= 0 || n_pages <= 0 || max_pages <= 0 || (double)B * max_pages > 2147483647.0) return FA_ERR_SHAPE;
    return FA_OK;
}
int check_workspace(const void* workspace, size_t bytes, int B, int n_pages) {
    const size_t need = fa::cache_pages_workspace_bytes(B, n_pages);
    if (need == 0) return FA_OK;
    if (!workspace || bytes < need) return FA_ERR_WORKSPACE;
    return aligned16(workspace) ? FA_OK : FA_ERR_ALIGN;
}

}  // namespace

extern "C" {

int fa_rope_axes(const void* q, const long long* q_strides, const void* k, const long long* k_strides, void* q_out,
                 const long long* q_out_strides, void* k_out, const long long* k_out_strides, const double* inv_freq,
                 const int* axis, const int* positions, int axes, int B, int H, int H_kv, int N, int d, int rot_dim,
                 float amplitude, int interleaved, int dtype, void* stream) {
    return rope_axes_any(q, q_strides, k, k_strides, q_out, q_out_strides, k_out, k_out_strides, inv_freq, axis, positions, axes, B, H,
                         H_kv, N, d, rot_dim, amplitude, interleaved, dtype, false, stream);
}

int fa_rope_axes_bwd(const void* dq, const long long* dq_strides, const void* dk, const long long* dk_strides, void* dq_out,
                     const long long* dq_out_strides, void* dk_out, const long long* dk_out_strides, const double* inv_freq,
                     const int* axis, const int* positions, int axes, int B, int H, int H_kv, int N, int d, int rot_dim,
                     float amplitude, int interleaved, int dtype, void* stream) {
    return rope_axes_any(dq, dq_strides, dk, dk_strides, dq_out, dq_out_strides, dk_out, dk_out_strides, inv_freq, axis, positions, axes, B, H,
                         H_kv, N, d, rot_dim, amplitude, interleaved, dtype, true, stream);
}

size_t fa_cache_pages_workspace_bytes(int B, int n_pages) {
    return B <= 0 || n_pages <= 0 ? 0 : fa::cache_pages_workspace_bytes(B, n_pages);
}

int fa_cache_fork(const int* block_table, const int* lens, const int* parents, const int* held, int* new_table, int* new_lens, int* src,
                  int* dst, int* missing, void* workspace, size_t workspace_bytes, int B, int B_new, int page_size, int n_pages,
                  int max_pages, void* stream) {
    if (!block_table || !lens || !parents || !new_table || !new_lens || !src || !dst || !missing) return FA_ERR_NULL;
    int st = check_pool(B, n_pages, max_pages);
    if (st == FA_OK) st = check_pool(B_new, n_pages, max_pages);
    if (st != FA_OK || page_size <= 0 || (long)max_pages * page_size > FA_CACHE_MAX_PLACES || new_table == block_table || new_lens == lens)
        return FA_ERR_SHAPE;  // (in place, some rows would be read after they have been written)
    for (const int* p : {block_table, lens, parents, held, (const int*)new_table, (const int*)new_lens, (const int*)src, (const int*)dst, (const int*)missing})
        if (!aligned_to(p, 4)) return FA_ERR_ALIGN;
    st = check_workspace(workspace, workspace_bytes, B_new, n_pages);
    if (st != FA_OK) return st;
    forget_stale_hip_error();
    return fa::launch_cache_fork(block_table, lens, parents, held, new_table, new_lens, src, dst, missing, workspace, B, B_new, page_size,
                                 n_pages, max_pages, static_cast<hipStream_t>(stream));
}

int fa_cache_extend(int* block_table, const int* lens, const int* counts, const int* held, int* missing, void* workspace,
                    size_t workspace_bytes, int B, int T, int page_size, int n_pages, int max_pages, void* stream) {
    if (!block_table || !lens || !missing) return FA_ERR_NULL;
    int st = check_pool(B, n_pages, max_pages);
    if (st != FA_OK || T <= 0 || (double)B * T > 2147483647.0 || page_size <= 0 || (long)max_pages * page_size > FA_CACHE_MAX_PLACES) return FA_ERR_SHAPE;
    for (const int* p : {(const int*)block_table, lens, counts, held, (const int*)missing})
        if (!aligned_to(p, 4)) return FA_ERR_ALIGN;
    st = check_workspace(workspace, workspace_bytes, B, n_pages);
    if (st != FA_OK) return st;
    forget_stale_hip_error();
    return fa::launch_cache_extend(block_table, lens, counts, held, missing, workspace, B, T, page_size, n_pages, max_pages,
                                   static_cast<hipStream_t>(stream));
}

int fa_cache_compact(const int* block_table, const int* held, int* new_table, int* src, int* dst, int* top, void* workspace,
                     size_t workspace_bytes, int B, int moves, int n_pages, int max_pages, void* stream) {
    if (!block_table || !new_table || !src || !dst || !top) return FA_ERR_NULL;
    int st = check_pool(B, n_pages, max_pages);
    if (st != FA_OK || moves <= 0) return FA_ERR_SHAPE;
    for (const int* p : {block_table, held, (const int*)new_table, (const int*)src, (const int*)dst, (const int*)top})
        if (!aligned_to(p, 4)) return FA_ERR_ALIGN;
    st = check_workspace(workspace, workspace_bytes, B, n_pages);
    if (st != FA_OK) return st;
    forget_stale_hip_error();
    return fa::launch_cache_compact(block_table, held, new_table, src, dst, top, workspace, B, moves, n_pages, max_pages,
                                    static_cast<hipStream_t>(stream));
}

int fa_cache_copy(void* k_pages, void* v_pages, void* k_scales, void* v_scales, const int* src, const int* dst, int n, int H_kv, int d,
                  int page_size, int n_pages, int cache_dtype, void* stream) {
    // (a cache without a table or lengths)
    const fa::Cache cache = {k_pages, v_pages, k_scales, v_scales, src, dst, H_kv, page_size, n_pages, 1, cache_dtype};
    const int st = check_cache(cache, 1, d);
    if (st != FA_OK) return st;
    if (n <= 0) return FA_ERR_SHAPE;
    forget_stale_hip_error();
    return fa::launch_cache_copy(cache, src, dst, n, d, static_cast<hipStream_t>(stream));
}

}  // extern "C"
