// Attention of the new tokens of every sequence over a paged cache (include/fa_mi355.h: fa_fwd_cache).
//
// A workgroup owns one row (sequence, query head, token); its waves take the keys in turn, each with a running maximum, sum
// and output, which meet in the LDS at the end.  A lane holds d / 64 elements of the row.
#include "fa_device.h"
#include "fa_launch.h"

namespace fa {

struct CachedArgs {
    Rows q, o;
    Cache c;
    const int *counts, *tree;
    float* lse;
    int B, H, T, tree_batches;
    float scale;
};

template <int DTYPE>
static __device__ __forceinline__ float element(const void* p, long i) {
    if constexpr (DTYPE == FA_FP8_E4M3) return __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t*>(p)[i], 0);
    else return Elem<std::conditional_t<DTYPE == FA_BF16, bf16_tag, f16_tag>>::to_float(static_cast<const uint16_t*>(p)[i]);
}

template <int D, int DTYPE, int CACHE>
__global__ void __launch_bounds__(256) fa_fwd_cache_kernel(CachedArgs a) {
    constexpr int E = D / 64;
    const Cache& c = a.c;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int t = blockIdx.x % a.T, bh = blockIdx.x / a.T, b = bh / a.H, h = bh - b * a.H, group = a.H / c.H_kv;
    const int count = a.counts ? min(a.counts[b], a.T) : a.T;
    if (t >= count) return;
    const int places = c.max_pages * c.page_size, len = min(max(c.lens[b], 0), places), keys = len + min(count, places - len);
    float q[E], acc[E] = {}, m = -INFINITY, l = 0.f;
    for (int e = 0; e < E; ++e) q[e] = element<DTYPE>(a.q.p, b * a.q.batch + h * a.q.head + t * a.q.token + lane * E + e);
    for (int j = wave; j < keys; j += 4) {
        if (j >= len) {
            const int u = j - len;
            const int words = (a.T + 31) / 32;
            const bool seen = a.tree ? (a.tree[((long)(a.tree_batches == 1 ? 0 : b) * a.T + t) * words + u / 32] >> (u % 32)) & 1 : u <= t;
            if (!seen) continue;
        }
        const int page = c.block_table[(long)b * c.max_pages + j / c.page_size];
        if (page < 0 || page >= c.n_pages) continue;
        const long slot = ((long)page * c.H_kv + h / group) * c.page_size + j % c.page_size;
        float s = 0.f;
        for (int e = 0; e < E; ++e) s += q[e] * element<CACHE>(c.k, slot * D + lane * E + e);
        for (int x = 1; x < 64; x <<= 1) s += __shfl_xor(s, x);
        if constexpr (CACHE == FA_FP8_E4M3) s *= c.k_scales[slot];
        s *= a.scale;
        const float m_new = fmaxf(m, s), corr = m_new == -INFINITY ? 1.f : __expf(m - m_new), p = m_new == -INFINITY ? 0.f : __expf(s - m_new);
        m = m_new;
        l = l * corr + p;
        const float pv = CACHE == FA_FP8_E4M3 ? p * c.v_scales[slot] : p;
        for (int e = 0; e < E; ++e) acc[e] = acc[e] * corr + pv * element<CACHE>(c.v, slot * D + lane * E + e);
    }
    __shared__ float part[4][D], state[4][2];
    for (int e = 0; e < E; ++e) part[wave][lane * E + e] = acc[e];
    if (lane == 0) {
        state[wave][0] = m;
        state[wave][1] = l;
    }
    __syncthreads();
    float m_all = -INFINITY, l_all = 0.f;
    for (int w = 0; w < 4; ++w) m_all = fmaxf(m_all, state[w][0]);
    const float ref = m_all == -INFINITY ? 0.f : m_all;
    for (int w = 0; w < 4; ++w) l_all += state[w][1] * __expf(state[w][0] - ref);
    for (int i = threadIdx.x; i < D; i += 256) {
        float x = 0.f;
        for (int w = 0; w < 4; ++w) x += part[w][i] * __expf(state[w][0] - ref);
        x = l_all == 0.f ? 0.f : x / l_all;
        uint16_t* o = static_cast<uint16_t*>(const_cast<void*>(a.o.p)) + (b * a.o.batch + h * a.o.head + t * a.o.token);
        o[i] = (uint16_t)Elem<std::conditional_t<DTYPE == FA_BF16, bf16_tag, f16_tag>>::pack2(x, 0.f);
    }
    if (threadIdx.x == 0) a.lse[((long)b * a.H + h) * a.T + t] = m_all + logf(l_all);
}

size_t fwd_cache_workspace_bytes(int, int, int, int, int, int, int) { return 0; }

int launch_fwd_cache(const Rows& q, const Cache& cache, const int* counts, const int* tree, int tree_batches, const Rows& o, float* lse,
                     void*, int B, int H, int T, int d, int, float scale, int dtype, hipStream_t stream) {
    const CachedArgs a = {q, o, cache, counts, tree, lse, B, H, T, tree_batches, scale};
    const dim3 grid((unsigned)B * H * T);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a);
        return (int)(hipGetLastError() == hipSuccess ? FA_OK : FA_ERR_LAUNCH);
    };
#define FA_CACHED(D)                                                                                                 \
    if (cache.dtype == FA_BF16) return go(fa_fwd_cache_kernel<D, FA_BF16, FA_BF16>);                                 \
    if (cache.dtype == FA_F16) return go(fa_fwd_cache_kernel<D, FA_F16, FA_F16>);                                    \
    return dtype == FA_BF16 ? go(fa_fwd_cache_kernel<D, FA_BF16, FA_FP8_E4M3>) : go(fa_fwd_cache_kernel<D, FA_F16, FA_FP8_E4M3>);
    switch (d) {
        case 64: FA_CACHED(64)
        case 128: FA_CACHED(128)
        default: FA_CACHED(256)
    }
#undef FA_CACHED
}

}  // namespace fa
