// Checks of arguments that the entry points on rotary positions, a cache and its pages share.
#pragma once
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

// The arguments of a rotation: Q and K, in and out, by rows
struct Rotation {
    fa::Rows q, k = {}, q_out, k_out = {};
};
int check_rotation(Rotation& r, const void* q, const long long* q_strides, const void* k, const long long* k_strides, void* q_out,
                   const long long* q_out_strides, void* k_out, const long long* k_out_strides, const double* inv_freq,
                   const int* positions, int B, int H, int& H_kv, int N, int d, int rot_dim, float amplitude, int interleaved, int dtype) {
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
    int st = rows_of(r.q, q, q_strides, B, H, N, d, dtype, false);
    if (st == FA_OK) st = rows_of(r.q_out, q_out, q_out_strides, B, H, N, d, dtype, true);
    if (st == FA_OK && k) st = rows_of(r.k, k, k_strides, B, H_kv, N, d, dtype, false);
    if (st == FA_OK && k) st = rows_of(r.k_out, k_out, k_out_strides, B, H_kv, N, d, dtype, true);
    return st;
}

// What every call on a cache has to keep to
int check_cache(const fa::Cache& c, int B, int d) {
    const bool codes = c.dtype == FA_FP8_E4M3 || c.dtype == FA_FP4_E2M1;
    if (!c.k || !c.v || !c.block_table || !c.lens || (codes && (!c.k_scales || !c.v_scales))) return FA_ERR_NULL;
    if (c.dtype < FA_F32 || c.dtype > FA_FP4_E2M1 || (!codes && (c.k_scales || c.v_scales))) return FA_ERR_DTYPE;
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
