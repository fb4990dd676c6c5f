// The paged cache of keys and values: writing new tokens to their pages, quantised on the way to an e4m3 cache, and reading
// them back as dense tensors.
//
// Every element is read once and written once, and nothing is computed that takes longer: HBM decides, for a token of each
// sequence the launch.  Measured at d = 128: 138 MB written as codes in 29 us (4.7 TB/s), 142 MB read back from codes in 29 us
// (4.8 TB/s; a copy reaches 5.0).  A row (a token of one head) is d / 16 lanes of 16 elements, its K and its V in the same lanes, so twice
// the bytes are in flight; the largest magnitude of a row is found across its lanes by DPP, without the LDS.
#include "fa_device.h"
#include "fa_launch.h"

namespace fa {

constexpr float kE4m3Max = 448.0f;

// The largest of 4, 8 or 16 neighbouring lanes
template <int CTRL>
static __device__ __forceinline__ float max_dpp(float x) {
    return fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true)));
}
template <int LANES>
static __device__ __forceinline__ float max_of_lanes(float x) {
    x = max_dpp<0xB1>(x);
    x = max_dpp<0x4E>(x);
    if constexpr (LANES >= 8) x = max_dpp<0x141>(x);   // row_half_mirror
    if constexpr (LANES >= 16) x = max_dpp<0x140>(x);  // row_mirror
    return x;
}

// 16 consecutive elements of a row
template <int DTYPE> struct Elements {
    static constexpr int ELEM = DTYPE == FA_F32 ? 4 : DTYPE == FA_FP8_E4M3 ? 1 : 2;
    i32x4 w[ELEM];
    // On the cache's side loads and stores are non-temporal: its pages are many, and the dense tensors are what the launch before
    // or after has in hand.  us, plain / so: 4 prompts of up to 4096 tokens written as codes (16 heads, d = 128) 32.2 / 28.6, 4
    // of up to 8192 read (8 heads) 35.0 / 28.7; on both sides 32.4 and 30.1.
    template <bool ONCE>
    __device__ __forceinline__ void load(const char* p) {
#pragma unroll
        for (int i = 0; i < ELEM; ++i) {
            const i32x4* at = reinterpret_cast<const i32x4*>(p + 16 * i);
            w[i] = ONCE ? __builtin_nontemporal_load(at) : *at;
        }
    }
    template <bool ONCE>
    __device__ __forceinline__ void store(char* p) const {
#pragma unroll
        for (int i = 0; i < ELEM; ++i) {
            i32x4* at = reinterpret_cast<i32x4*>(p + 16 * i);
            if constexpr (ONCE) __builtin_nontemporal_store(w[i], at);
            else *at = w[i];
        }
    }
    __device__ __forceinline__ void get(float (&f)[16]) const {
#pragma unroll
        for (int t = 0; t < 16; ++t) {
            if constexpr (DTYPE == FA_F32) {
                f[t] = __builtin_bit_cast(float, (int)w[t >> 2][t & 3]);
            } else if constexpr (DTYPE == FA_FP8_E4M3) {
                const int u = w[0][t >> 2];
                switch (t & 3) {
                    case 0: f[t] = __builtin_amdgcn_cvt_f32_fp8(u, 0); break;
                    case 1: f[t] = __builtin_amdgcn_cvt_f32_fp8(u, 1); break;
                    case 2: f[t] = __builtin_amdgcn_cvt_f32_fp8(u, 2); break;
                    default: f[t] = __builtin_amdgcn_cvt_f32_fp8(u, 3);
                }
            } else {
                const uint32_t u = (uint32_t)w[t >> 3][(t >> 1) & 3];
                if constexpr (DTYPE == FA_BF16) f[t] = __builtin_bit_cast(float, t & 1 ? u & 0xFFFF0000u : u << 16);
                else f[t] = Elem<f16_tag>::to_float((uint16_t)(t & 1 ? u >> 16 : u));
            }
        }
    }
    __device__ __forceinline__ void set(const float (&f)[16]) {
        if constexpr (DTYPE == FA_F32) {
#pragma unroll
            for (int t = 0; t < 16; ++t) w[t >> 2][t & 3] = __builtin_bit_cast(int, f[t]);
        } else if constexpr (DTYPE == FA_FP8_E4M3) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                w[0][g] = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * g], f[4 * g + 1], 0, false);
                w[0][g] = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * g + 2], f[4 * g + 3], w[0][g], true);
            }
        } else {
            using E = Elem<std::conditional_t<DTYPE == FA_BF16, bf16_tag, f16_tag>>;
#pragma unroll
            for (int t = 0; t < 8; ++t) w[t >> 2][t & 3] = E::pack2(f[2 * t], f[2 * t + 1]);
        }
    }
};

// The slot of place `at` of sequence b counted over all pages and heads' rows, or -1 where there is none
static __device__ __forceinline__ long slot_of(const Cache& c, int b, int at, int head) {
    const int entry = (unsigned)at / (unsigned)c.page_size;
    if (entry >= c.max_pages) return -1;
    const int page = c.block_table[(long)b * c.max_pages + entry];
    if (page < 0 || page >= c.n_pages) return -1;
    return ((long)page * c.H_kv + head) * c.page_size + (at - entry * c.page_size);
}

// What lies below its row's largest finite magnitude a: codes, and their scale
template <int LANES>
static __device__ __forceinline__ float quantise(float (&f)[16]) {
    float a = 0.f;
#pragma unroll
    for (int t = 0; t < 16; ++t) a = fmaxf(a, fabsf(f[t]) < INFINITY ? fabsf(f[t]) : 0.f);
    a = max_of_lanes<LANES>(a);
    if (a > 0.f) a = fmaxf(a, 0x1p-100f);  // (448 / a stays finite)
    const float factor = a > 0.f ? kE4m3Max / a : 1.f;
#pragma unroll
    for (int t = 0; t < 16; ++t) {
        const float z = f[t] * factor;
        f[t] = z > kE4m3Max ? kE4m3Max : z < -kE4m3Max ? -kE4m3Max : z;  // a NaN stays one
    }
    return a > 0.f ? a / kE4m3Max : 1.f;
}

template <int D, int IN, int OUT>
__global__ void __launch_bounds__(256) fa_cache_write_kernel(Rows k, Rows v, Cache c, const int* counts, unsigned rows, unsigned T) {
    constexpr int LANES = D / 16;
    const unsigned row = blockIdx.x * (256 / LANES) + threadIdx.x / LANES, lane = threadIdx.x % LANES;
    if (row >= rows) return;
    const unsigned bh = row / T;
    const int t = row - bh * T, b = bh / c.H_kv, h = bh - b * c.H_kv;
    const int len = max(c.lens[b], 0);
    if ((counts && t >= counts[b]) || len > 0x7fffffff - t) return;
    Elements<IN> x[2];  // (on their way while the table is read)
    x[0].template load<false>(static_cast<const char*>(k.p) + (b * k.batch + h * k.head + t * k.token + 16 * lane) * Elements<IN>::ELEM);
    x[1].template load<false>(static_cast<const char*>(v.p) + (b * v.batch + h * v.head + t * v.token + 16 * lane) * Elements<IN>::ELEM);
    const long slot = slot_of(c, b, len + t, h);
    if (slot < 0) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        char* to = static_cast<char*>(i ? c.v : c.k) + (slot * D + 16 * lane) * Elements<OUT>::ELEM;
        if constexpr (IN == OUT) {
            x[i].template store<true>(to);
        } else {
            float f[16];
            x[i].get(f);
            if constexpr (OUT == FA_FP8_E4M3) {
                const float scale = quantise<LANES>(f);
                if (lane == 0) (i ? c.v_scales : c.k_scales)[slot] = scale;
            }
            Elements<OUT> y;
            y.set(f);
            y.template store<true>(to);
        }
    }
}

template <int D, int IN, int OUT>
__global__ void __launch_bounds__(256) fa_cache_read_kernel(Cache c, char* k, char* v, unsigned rows, unsigned N) {
    constexpr int LANES = D / 16;
    const unsigned row = blockIdx.x * (256 / LANES) + threadIdx.x / LANES, lane = threadIdx.x % LANES;
    if (row >= rows) return;
    const unsigned bh = row / N;
    const int n = row - bh * N, b = bh / c.H_kv, h = bh - b * c.H_kv;
    const int len = c.lens[b];
    const long slot = slot_of(c, b, n, h);  // (looked up before the length is known)
    if (n >= len || slot < 0) return;
    Elements<IN> x[2];
    x[0].template load<true>(static_cast<const char*>(c.k) + (slot * D + 16 * lane) * Elements<IN>::ELEM);
    x[1].template load<true>(static_cast<const char*>(c.v) + (slot * D + 16 * lane) * Elements<IN>::ELEM);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        char* to = (i ? v : k) + ((long)row * D + 16 * lane) * Elements<OUT>::ELEM;
        if constexpr (IN == OUT) {
            x[i].template store<false>(to);
        } else {
            float f[16];
            x[i].get(f);
            if constexpr (IN == FA_FP8_E4M3) {
                const float scale = (i ? c.v_scales : c.k_scales)[slot];
#pragma unroll
                for (int t = 0; t < 16; ++t) f[t] *= scale;
            }
            Elements<OUT> y;
            y.set(f);
            y.template store<false>(to);
        }
    }
}

// Calls f(head dimension, type on the dense side, type of the cache) with the three as types
template <typename F>
static int with_types(int d, int dense, int cache, F&& f) {
    auto by_cache = [&](auto D, auto dense_type) {
        constexpr int X = decltype(dense_type)::value;
        if (cache == FA_FP8_E4M3) return f(D, dense_type, std::integral_constant<int, FA_FP8_E4M3>{});
        if constexpr (X != FA_F16)
            if (cache == FA_BF16) return f(D, dense_type, std::integral_constant<int, FA_BF16>{});
        if constexpr (X != FA_BF16)
            if (cache == FA_F16) return f(D, dense_type, std::integral_constant<int, FA_F16>{});
        return (int)FA_ERR_UNSUPPORTED;
    };
    auto by_dense = [&](auto D) {
        switch (dense) {
            case FA_F32: return by_cache(D, std::integral_constant<int, FA_F32>{});
            case FA_BF16: return by_cache(D, std::integral_constant<int, FA_BF16>{});
            default: return by_cache(D, std::integral_constant<int, FA_F16>{});
        }
    };
    switch (d) {
        case 64: return by_dense(std::integral_constant<int, 64>{});
        case 128: return by_dense(std::integral_constant<int, 128>{});
        default: return by_dense(std::integral_constant<int, 256>{});
    }
}

int launch_cache_write(const Rows& k, const Rows& v, const Cache& cache, const int* counts, int B, int T, int d, int in_dtype,
                       hipStream_t stream) {
    const unsigned rows = (unsigned)B * cache.H_kv * T, per = 256 / (d / 16);
    const dim3 grid((unsigned)(((long)rows + per - 1) / per));
    return with_types(d, in_dtype, cache.dtype, [&](auto D, auto in, auto out) {
        hipLaunchKernelGGL((fa_cache_write_kernel<decltype(D)::value, decltype(in)::value, decltype(out)::value>), grid, dim3(256), 0,
                           stream, k, v, cache, counts, rows, T);
        return (int)(hipGetLastError() == hipSuccess ? FA_OK : FA_ERR_LAUNCH);
    });
}

int launch_cache_read(const Cache& cache, void* k, void* v, int B, int N, int d, int out_dtype, hipStream_t stream) {
    const unsigned rows = (unsigned)B * cache.H_kv * N, per = 256 / (d / 16);
    const dim3 grid((unsigned)(((long)rows + per - 1) / per));
    return with_types(d, out_dtype, cache.dtype, [&](auto D, auto out, auto in) {
        hipLaunchKernelGGL((fa_cache_read_kernel<decltype(D)::value, decltype(in)::value, decltype(out)::value>), grid, dim3(256), 0,
                           stream, cache, static_cast<char*>(k), static_cast<char*>(v), rows, N);
        return (int)(hipGetLastError() == hipSuccess ? FA_OK : FA_ERR_LAUNCH);
    });
}

}  // namespace fa
