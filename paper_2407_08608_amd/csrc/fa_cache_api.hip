// C ABI of libfa_mi355.so, continued: rotary positions, the paged cache and attention over it.  Argument validation and
// dispatch; include/fa_mi355.h holds the contract of every entry point.
#include <math.h>
#include <stdint.h>

#include "fa_check.h"
#include "fa_launch.h"

namespace {

size_t elem_size(int dtype) { return dtype == FA_F32 ? 4 : dtype == FA_FP8_E4M3 ? 1 : 2; }

bool aligned_to(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// The rows of a tensor [B, heads, tokens, d] with the caller's strides, or of a contiguous one.  The stride of a dimension of
// size 1 leads nowhere and may be anything; two rows of an output may not be one.
int rows_of(fa::Rows& rows, const void* p, const long long* strides, int B, int heads, int tokens, int d, int dtype, bool written) {
    rows = {p, (long)heads * tokens * d, (long)tokens * d, d};
    if (!strides) return FA_OK;
    const long long whole = 16 / (long long)elem_size(dtype);
    const int size[3] = {B, heads, tokens};
    long* const to[3] = {&rows.batch, &rows.head, &rows.token};
    for (int i = 0; i < 3; ++i) {
        const long long stride = size[i] == 1 ? 0 : strides[i];
        if (stride < 0 || (written && size[i] > 1 && stride < d)) return FA_ERR_SHAPE;
        if (stride % whole != 0) return FA_ERR_ALIGN;
        *to[i] = (long)stride;
    }
    return FA_OK;
}

int rope_any(const void* q, const long long* q_strides, const void* k, const long long* k_strides, void* q_out,
             const long long* q_out_strides, void* k_out, const long long* k_out_strides, const double* inv_freq,
             const int* positions, int B, int H, int H_kv, int N, int d, int rot_dim, float amplitude, int interleaved,
             int dtype, bool transposed, void* stream) {
    if (!q || !q_out || !inv_freq || (k && !k_out)) return FA_ERR_NULL;
    if (dtype < FA_F32 || dtype > FA_FP8_E4M3) return FA_ERR_DTYPE;
    if (dtype == FA_FP8_E4M3) return FA_ERR_UNSUPPORTED;
    if (!k) H_kv = 0;
    if (B <= 0 || H <= 0 || N <= 0 || d <= 0 || (k && H_kv <= 0) || rot_dim <= 0 || rot_dim > d) return FA_ERR_SHAPE;
    if (!(amplitude > 0.f) || !isfinite(amplitude) || (interleaved != 0 && interleaved != 1)) return FA_ERR_SHAPE;
    if (H > 0x7fffffff - H_kv || (double)B * ((double)H + H_kv) * N > 2147483647.0) return FA_ERR_SHAPE;
    if (!head_dim_ok(d) || rot_dim % 16 != 0) return FA_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(k) || !aligned16(q_out) || (k && !aligned16(k_out)) || !aligned_to(inv_freq, 8) || !aligned_to(positions, 4))
        return FA_ERR_ALIGN;
    fa::Rows qr, kr = {}, qo, ko = {};
    int st = rows_of(qr, q, q_strides, B, H, N, d, dtype, false);
    if (st == FA_OK) st = rows_of(qo, q_out, q_out_strides, B, H, N, d, dtype, true);
    if (st == FA_OK && k) st = rows_of(kr, k, k_strides, B, H_kv, N, d, dtype, false);
    if (st == FA_OK && k) st = rows_of(ko, k_out, k_out_strides, B, H_kv, N, d, dtype, true);
    if (st != FA_OK) return st;
    forget_stale_hip_error();
    return fa::launch_rope(qr, kr, qo, ko, inv_freq, positions, B, H, H_kv, N, d, rot_dim, amplitude, interleaved, transposed,
                           dtype, static_cast<hipStream_t>(stream));
}

// What every call on a cache has to keep to
int check_cache(const fa::Cache& c, int B, int d) {
    const bool codes = c.dtype == FA_FP8_E4M3;
    if (!c.k || !c.v || !c.block_table || !c.lens || (codes && (!c.k_scales || !c.v_scales))) return FA_ERR_NULL;
    if (c.dtype < FA_F32 || c.dtype > FA_FP8_E4M3 || (!codes && (c.k_scales || c.v_scales))) return FA_ERR_DTYPE;
    if (c.dtype == FA_F32) return FA_ERR_UNSUPPORTED;
    if (B <= 0 || c.H_kv <= 0 || d <= 0 || c.page_size <= 0 || c.n_pages <= 0 || c.max_pages <= 0) return FA_ERR_SHAPE;
    if ((long)c.max_pages * c.page_size > FA_CACHE_MAX_PLACES) return FA_ERR_SHAPE;
    if (!head_dim_ok(d) || c.page_size % 16 != 0 || (long)c.page_size * d * 4 > 0x7ff00000L) return FA_ERR_UNSUPPORTED;
    if (!aligned16(c.k) || !aligned16(c.v) || !aligned_to(c.k_scales, 4) || !aligned_to(c.v_scales, 4) ||
        !aligned_to(c.block_table, 4) || !aligned_to(c.lens, 4))
        return FA_ERR_ALIGN;
    return FA_OK;
}

}  // namespace

extern "C" {

int fa_rope(const void* q, const long long* q_strides, const void* k, const long long* k_strides, void* q_out,
            const long long* q_out_strides, void* k_out, const long long* k_out_strides, const double* inv_freq,
            const int* positions, int B, int H, int H_kv, int N, int d, int rot_dim, float amplitude, int interleaved,
            int dtype, void* stream) {
    return rope_any(q, q_strides, k, k_strides, q_out, q_out_strides, k_out, k_out_strides, inv_freq, positions, B, H, H_kv, N, d,
                    rot_dim, amplitude, interleaved, dtype, false, stream);
}

int fa_rope_bwd(const void* dq, const long long* dq_strides, const void* dk, const long long* dk_strides, void* dq_out,
                const long long* dq_out_strides, void* dk_out, const long long* dk_out_strides, const double* inv_freq,
                const int* positions, int B, int H, int H_kv, int N, int d, int rot_dim, float amplitude, int interleaved,
                int dtype, void* stream) {
    return rope_any(dq, dq_strides, dk, dk_strides, dq_out, dq_out_strides, dk_out, dk_out_strides, inv_freq, positions, B, H, H_kv,
                    N, d, rot_dim, amplitude, interleaved, dtype, true, stream);
}

int fa_rope_frequencies(double* inv_freq, float* amplitude, int rot_dim, double base, int scaling, double factor,
                        double trained_len) {
    if (!inv_freq) return FA_ERR_NULL;
    if (scaling < FA_ROPE_PLAIN || scaling > FA_ROPE_BY_PARTS) return FA_ERR_SHAPE;
    if (rot_dim <= 0 || rot_dim % 2 != 0 || !(base > 1.0) || !isfinite(base)) return FA_ERR_SHAPE;
    if (scaling == FA_ROPE_PLAIN) factor = 1.0;
    if (!(factor >= 1.0) || !isfinite(factor) || (scaling == FA_ROPE_NTK && rot_dim == 2)) return FA_ERR_SHAPE;
    if (scaling == FA_ROPE_BY_PARTS && (!(trained_len > 0.0) || !isfinite(trained_len))) return FA_ERR_SHAPE;
    if (scaling == FA_ROPE_NTK) base *= pow(factor, rot_dim / (rot_dim - 2.0));
    if (!isfinite(base)) return FA_ERR_SHAPE;
    for (int i = 0; i < rot_dim / 2; ++i) {
        double f = pow(base, -2.0 * i / rot_dim);
        if (scaling == FA_ROPE_LINEAR) f /= factor;
        if (scaling == FA_ROPE_BY_PARTS) {
            const double turns = trained_len * f / (2.0 * M_PI), g = fmin(fmax((turns - 1.0) / 31.0, 0.0), 1.0);
            f *= g + (1.0 - g) / factor;
        }
        inv_freq[i] = f;
    }
    if (amplitude) *amplitude = scaling == FA_ROPE_BY_PARTS ? (float)(0.1 * log(factor) + 1.0) : 1.f;
    return FA_OK;
}

int fa_cache_write(const void* k, const long long* k_strides, const void* v, const long long* v_strides, void* k_pages,
                   void* v_pages, float* k_scales, float* v_scales, const int* block_table, const int* lens, const int* counts,
                   int B, int H_kv, int T, int d, int page_size, int n_pages, int max_pages, int in_dtype, int cache_dtype,
                   void* stream) {
    const fa::Cache cache = {k_pages, v_pages, k_scales, v_scales, block_table, lens, H_kv, page_size, n_pages, max_pages, cache_dtype};
    if (!k || !v) return FA_ERR_NULL;
    if (in_dtype < FA_F32 || in_dtype > FA_FP8_E4M3) return FA_ERR_DTYPE;
    int st = check_cache(cache, B, d);
    if (st != FA_OK) return st;
    if (T <= 0 || (double)B * H_kv * T > 2147483647.0) return FA_ERR_SHAPE;
    if (in_dtype == FA_FP8_E4M3 || (cache_dtype != FA_FP8_E4M3 && in_dtype != FA_F32 && in_dtype != cache_dtype)) return FA_ERR_UNSUPPORTED;
    if (!aligned16(k) || !aligned16(v) || !aligned_to(counts, 4)) return FA_ERR_ALIGN;
    fa::Rows kr, vr;
    st = rows_of(kr, k, k_strides, B, H_kv, T, d, in_dtype, false);
    if (st == FA_OK) st = rows_of(vr, v, v_strides, B, H_kv, T, d, in_dtype, false);
    if (st != FA_OK) return st;
    forget_stale_hip_error();
    return fa::launch_cache_write(kr, vr, cache, counts, B, T, d, in_dtype, static_cast<hipStream_t>(stream));
}

int fa_cache_read(const void* k_pages, const void* v_pages, const float* k_scales, const float* v_scales, const int* block_table,
                  const int* lens, void* k, void* v, int B, int H_kv, int N, int d, int page_size, int n_pages, int max_pages,
                  int cache_dtype, int out_dtype, void* stream) {
    const fa::Cache cache = {const_cast<void*>(k_pages), const_cast<void*>(v_pages), const_cast<float*>(k_scales),
                             const_cast<float*>(v_scales), block_table, lens, H_kv, page_size, n_pages, max_pages, cache_dtype};
    if (!k || !v) return FA_ERR_NULL;
    if (out_dtype < FA_F32 || out_dtype > FA_FP8_E4M3) return FA_ERR_DTYPE;
    const int st = check_cache(cache, B, d);
    if (st != FA_OK) return st;
    if (N <= 0 || (double)B * H_kv * N > 2147483647.0) return FA_ERR_SHAPE;
    if (out_dtype == FA_FP8_E4M3 || (cache_dtype != FA_FP8_E4M3 && out_dtype != FA_F32 && out_dtype != cache_dtype)) return FA_ERR_UNSUPPORTED;
    if (!aligned16(k) || !aligned16(v)) return FA_ERR_ALIGN;
    forget_stale_hip_error();
    return fa::launch_cache_read(cache, k, v, B, N, d, out_dtype, static_cast<hipStream_t>(stream));
}

size_t fa_fwd_cache_workspace_bytes(int B, int H, int H_kv, int T, int d, int max_len, int cache_dtype) {
    if (B <= 0 || H <= 0 || H_kv <= 0 || H % H_kv != 0 || T <= 0 || T > FA_CACHE_MAX_TOKENS || max_len <= 0 || !head_dim_ok(d)) return 0;
    if ((double)B * H * T > 2147483647.0) return 0;
    if (cache_dtype != FA_BF16 && cache_dtype != FA_F16 && cache_dtype != FA_FP8_E4M3) return 0;
    return fa::fwd_cache_workspace_bytes(B, H, H_kv, T, d, max_len, cache_dtype);
}

int fa_fwd_cache(const void* q, const long long* q_strides, const void* k_pages, const void* v_pages, const float* k_scales,
                 const float* v_scales, const int* block_table, const int* lens, const int* counts, const int* tree,
                 int tree_batches, void* o, const long long* o_strides, float* lse, void* workspace, size_t workspace_bytes,
                 int B, int H, int H_kv, int T, int d, int page_size, int n_pages, int max_pages, int max_len, float scale,
                 int dtype, int cache_dtype, void* stream) {
    const fa::Cache cache = {const_cast<void*>(k_pages), const_cast<void*>(v_pages), const_cast<float*>(k_scales),
                             const_cast<float*>(v_scales), block_table, lens, H_kv, page_size, n_pages, max_pages, cache_dtype};
    if (!q || !o || !lse) return FA_ERR_NULL;
    if (dtype < FA_F32 || dtype > FA_FP8_E4M3) return FA_ERR_DTYPE;
    int st = check_cache(cache, B, d);
    if (st != FA_OK) return st;
    if (H <= 0 || H % H_kv != 0 || T <= 0 || max_len < 0 || !(scale > 0.f) || !isfinite(scale)) return FA_ERR_SHAPE;
    if (tree && tree_batches != 1 && tree_batches != B) return FA_ERR_SHAPE;
    if ((double)B * H * T > 2147483647.0) return FA_ERR_SHAPE;
    if (T > FA_CACHE_MAX_TOKENS) return FA_ERR_TOO_LARGE;
    if ((dtype != FA_BF16 && dtype != FA_F16) || (cache_dtype != dtype && cache_dtype != FA_FP8_E4M3)) return FA_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(o) || !aligned_to(lse, 4) || !aligned_to(counts, 4) || !aligned_to(tree, 4)) return FA_ERR_ALIGN;
    fa::Rows qr, orows;
    st = rows_of(qr, q, q_strides, B, H, T, d, dtype, false);
    if (st == FA_OK) st = rows_of(orows, o, o_strides, B, H, T, d, dtype, true);
    if (st != FA_OK) return st;
    if (max_len == 0) max_len = max_pages * page_size;
    const size_t need = fa::fwd_cache_workspace_bytes(B, H, H_kv, T, d, max_len, cache_dtype);
    if (need > 0 && (!workspace || workspace_bytes < need)) return FA_ERR_WORKSPACE;
    if (need > 0 && !aligned16(workspace)) return FA_ERR_ALIGN;
    forget_stale_hip_error();
    return fa::launch_fwd_cache(qr, cache, counts, tree, tree_batches, orows, lse, workspace, B, H, T, d, max_len, scale, dtype,
                                static_cast<hipStream_t>(stream));
}

}  // extern "C"
