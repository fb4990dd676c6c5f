// Rotary positions of Q and K in one launch, and their gradients' way back (the same rotation by the opposite angle).
//
// Every element is read once and written once, which is what bounds the launch (HBM); the angles' sines and cosines would
// cost more than that if each row computed its own.  Measured: 16k tokens x 32 heads of 128 in bf16, 268 MB in 45 us, 6.0 TB/s
// (a copy past the Infinity Cache: 5.0); 8 tokens x 20 heads: 3.6 us, the launch's latency.  They belong to a (token, pair) and not to a head: a thread computes
// those of its eight pairs once and walks over heads of Q, then of K, with them in registers.
//   - A thread owns two 16-byte chunks (8 elements each; two loads each in fp32) of a token's row, whose 16 elements make
//     eight whole pairs in either layout: chunks u and u + rot/16 (half layout: element j of one with element j of the other;
//     interleaved: neighbours within each).  So a row's lanes read 16 bytes side by side in both.
//   - Elements past rot_dim go along two chunks to a thread, or are left alone where output and input are one.
//   - phi = position * inv_freq / 2 pi is computed and reduced to [-1/2, 1/2] turns in fp64 (in fp32 a position of 100000
//     would be off by 6e-3 rad); from there on fp32.
#include "fa_device.h"
#include "fa_launch.h"

namespace fa {

struct RopeArgs {
    Rows x[2], y[2];  // Q and K
    const double* inv_freq;
    const int* positions;  // [B][N] or NULL
    int heads_q, heads, B, N, rot_dim, heads_per_group;
    float amplitude, sign;
};

template <int DTYPE> struct RowChunk {  // 8 elements as floats
    static constexpr int ELEM = DTYPE == FA_F32 ? 4 : 2;
    i32x4 w[ELEM / 2];
    template <bool ONCE>
    __device__ __forceinline__ void load(const char* p) {
#pragma unroll
        for (int i = 0; i < ELEM / 2; ++i) {
            const i32x4* at = reinterpret_cast<const i32x4*>(p + 16 * i);
            w[i] = ONCE ? __builtin_nontemporal_load(at) : *at;
        }
    }
    __device__ __forceinline__ void store(char* p) const {
#pragma unroll
        for (int i = 0; i < ELEM / 2; ++i) *reinterpret_cast<i32x4*>(p + 16 * i) = w[i];
    }
    __device__ __forceinline__ void get(float (&f)[8]) const {
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            if constexpr (DTYPE == FA_F32) {
                f[t] = __builtin_bit_cast(float, (int)w[t >> 2][t & 3]);
            } else {
                const uint32_t u = (uint32_t)w[0][t >> 1];
                if constexpr (DTYPE == FA_BF16) f[t] = __builtin_bit_cast(float, t & 1 ? u & 0xFFFF0000u : u << 16);
                else f[t] = Elem<f16_tag>::to_float((uint16_t)(t & 1 ? u >> 16 : u));
            }
        }
    }
    __device__ __forceinline__ void set(const float (&f)[8]) {
        if constexpr (DTYPE == FA_F32) {
#pragma unroll
            for (int t = 0; t < 8; ++t) w[t >> 2][t & 3] = __builtin_bit_cast(int, f[t]);
        } else {
            using E = Elem<std::conditional_t<DTYPE == FA_BF16, bf16_tag, f16_tag>>;
#pragma unroll
            for (int t = 0; t < 4; ++t) w[0][t] = E::pack2(f[2 * t], f[2 * t + 1]);
        }
    }
};

template <int D, int DTYPE, bool INTERLEAVED, bool ONCE>
__global__ void __launch_bounds__(256) fa_rope_kernel(RopeArgs a) {
    constexpr int TPR = D / 16, ELEM = RowChunk<DTYPE>::ELEM;  // threads per token
    const unsigned token = blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
    if (token >= (unsigned)a.B * a.N) return;
    const int unit = threadIdx.x % TPR, b = token / (unsigned)a.N, n = token - (unsigned)b * a.N;
    const int pairs = a.rot_dim / 16;  // chunks of the first half of what is rotated
    const bool turned = unit < pairs;
    const int c0 = turned ? unit : 2 * unit, c1 = turned ? unit + pairs : 2 * unit + 1;
    float co[8], si[8];
    if (turned) {
        const double turns = 0.15915494309189533577 * (double)(a.positions ? a.positions[token] : n);  // of frequency 1
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const int i = INTERLEAVED ? (t < 4 ? 4 * c0 + t : 4 * c1 + t - 4) : 8 * c0 + t;
            double phi = turns * a.inv_freq[i];
            phi -= __builtin_rint(phi);
            float s, c;
            sincospif(2.f * (float)phi, &s, &c);
            co[t] = c * a.amplitude;
            si[t] = s * a.amplitude * a.sign;
        }
    }
    const int first = blockIdx.y * a.heads_per_group, last = min(first + a.heads_per_group, a.heads);
    for (int h = first; h < last; ++h) {
        const bool is_k = h >= a.heads_q;
        const Rows& xr = a.x[is_k];
        const Rows& yr = a.y[is_k];
        const int head = is_k ? h - a.heads_q : h;
        const char* x = static_cast<const char*>(xr.p) + (b * xr.batch + head * xr.head + n * xr.token) * ELEM;
        char* y = static_cast<char*>(const_cast<void*>(yr.p)) + (b * yr.batch + head * yr.head + n * yr.token) * ELEM;
        if (!turned && x == y) continue;
        RowChunk<DTYPE> w0, w1;
        w0.template load<ONCE>(x + c0 * 8 * ELEM);
        w1.template load<ONCE>(x + c1 * 8 * ELEM);
        if (turned) {
            float f0[8], f1[8];
            w0.get(f0);
            w1.get(f1);
            if constexpr (INTERLEAVED) {
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const float p = f0[2 * t], q = f0[2 * t + 1], r = f1[2 * t], s = f1[2 * t + 1];
                    f0[2 * t] = p * co[t] - q * si[t];
                    f0[2 * t + 1] = p * si[t] + q * co[t];
                    f1[2 * t] = r * co[4 + t] - s * si[4 + t];
                    f1[2 * t + 1] = r * si[4 + t] + s * co[4 + t];
                }
            } else {
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    const float p = f0[t], q = f1[t];
                    f0[t] = p * co[t] - q * si[t];
                    f1[t] = p * si[t] + q * co[t];
                }
            }
            w0.set(f0);
            w1.set(f1);
        }
        w0.store(y + c0 * 8 * ELEM);
        w1.store(y + c1 * 8 * ELEM);
    }
}

// Whether the inputs are read past the caches: so many bytes do not stay there until they are read anyway, and push the outputs out,
// which the next call reads.  us, kept / past, MiB of input (bf16, 16 and 16 heads of 128, a projection's layout); after other inputs |
// after a launch that writes them (included):
//   32 16.0 / 17.7 | 26.5 / 26.7;  64 28.1 / 28.2 | 47.0 / 46.2;  80 34.9 / 33.0 | 62.5 / 57.0;  96 44.5 / 39.4 | 80.3 / 69.7;
//   109 50.0 / 41.6 | 90.0 / 78.4;  128 55.6 / 48.1 | 105 / 98;  150 68.2 / 63.6 | 120 / 114;  188 82.4 / 80.9 | 144 / 139;  256 116 / 112 | 199 / 196
constexpr double kReadOnce = 72.0 * 1024 * 1024;

template <int D, int DTYPE>
static int launch_rope_d(const RopeArgs& a, int interleaved, const dim3& grid, hipStream_t stream) {
    const bool once = (double)a.B * a.heads * a.N * D * RowChunk<DTYPE>::ELEM > kReadOnce;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a); };
    if (interleaved) once ? go(fa_rope_kernel<D, DTYPE, true, true>) : go(fa_rope_kernel<D, DTYPE, true, false>);
    else once ? go(fa_rope_kernel<D, DTYPE, false, true>) : go(fa_rope_kernel<D, DTYPE, false, false>);
    return hipGetLastError() == hipSuccess ? FA_OK : FA_ERR_LAUNCH;
}

int launch_rope(const Rows& q, const Rows& k, const Rows& q_out, const Rows& k_out, const double* inv_freq, const int* positions,
                int B, int H, int H_kv, int N, int d, int rot_dim, float amplitude, int interleaved, bool transposed, int dtype,
                hipStream_t stream) {
    RopeArgs a = {{q, k}, {q_out, k_out}, inv_freq, positions, H, H + H_kv, B, N, rot_dim, 0, amplitude, transposed ? -1.f : 1.f};
    const long per = 256 / (d / 16), tiles = ((long)B * N + per - 1) / per;
    a.heads_per_group = (int)((tiles * a.heads + 2047) / 2048);
    if (a.heads_per_group > 16) a.heads_per_group = 16;
    while ((a.heads + a.heads_per_group - 1) / a.heads_per_group > 65535) a.heads_per_group *= 2;  // what a grid's y takes
    const dim3 grid((unsigned)tiles, (unsigned)((a.heads + a.heads_per_group - 1) / a.heads_per_group));
#define FA_ROPE_D(D)                                                                     \
    switch (dtype) {                                                                     \
        case FA_F32: return launch_rope_d<D, FA_F32>(a, interleaved, grid, stream);      \
        case FA_BF16: return launch_rope_d<D, FA_BF16>(a, interleaved, grid, stream);    \
        default: return launch_rope_d<D, FA_F16>(a, interleaved, grid, stream);          \
    }
    switch (d) {
        case 64: FA_ROPE_D(64)
        case 128: FA_ROPE_D(128)
        default: FA_ROPE_D(256)
    }
#undef FA_ROPE_D
}

}  // namespace fa
