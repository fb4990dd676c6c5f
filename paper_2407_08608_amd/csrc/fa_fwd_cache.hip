// Attention of the new tokens of every sequence over a paged cache (include/fa_mi355.h: fa_fwd_cache).
//
// The rows that read one key/value head, (query head of the group) x (new token), are queries of one dense problem: 32 of them
// make a tile (lane column = row), RT tiles a workgroup.  The keys of a sequence are divided into chunks, a workgroup each; the
// NW waves of a workgroup take the chunk's 32-key tiles in turn, each with a softmax state and an output accumulator of its
// own, and meet in the LDS at the end, in a fixed order.  Where a sequence has several chunks the workgroup leaves (sum p v,
// reference, sum p) in the workspace and a second launch joins them, in a fixed order too.
//
// Bound by HBM up to about 300 rows to a key/value head (4 rows d flops for 4 d bytes of a key): the cache is read once per
// row group, straight into the LDS, and as much of it as the LDS holds is on its way at any time.  A wave stages its own tiles
// (no barrier in the loop): a slot for K and one for V, STG deep, refilled as soon as the wave has read them, so requests go
// on while scores, softmax and products are computed.
//   - Pages: 16 consecutive places lie in one page (page_size is a multiple of 16), so a tile has two resources.  Lane i of a
//     wave looks up the two rows of the wave's i-th tile, 64 tiles at a time; what is no page, or past the last key, gets a
//     resource of length 0 and arrives as zeros.
//   - Masks: only tiles that reach the new tokens (or hold a bad page) look at one.  What a lane's row sees of a tile is a 32-bit
//     word: places before the new tokens, the row's window of the tree, the tokens that are there.
//   - e4m3: codes become 16-bit operands in registers (exact): K in the type of Q, with the key's scale on the score; V in
//     fp16, with P~ = p (v scale / F), F a power of two not below the scales so far.  So P~ is at most 2^kLazyLog2 in fp16 whatever
//     the scales are, and eleven bits of each weight reach the product.
#include "fa_device.h"
#include "fa_launch.h"

namespace fa {

struct CachedArgs {
    Rows q, o;
    Cache c;
    const int *counts, *tree;
    float *lse, *part, *state;  // part, state: the workspace, [split][B H T][D] and [split][B H T][2]
    int B, H, T, tree_batches, row_groups, splits, chunk;  // chunk: keys, a multiple of 32
    float scale;
};

namespace {

constexpr float kLazy = 8.0f;  // the reference of a row rises when a tile's maximum exceeds it by more (log2 units)

// What a sequence has: places before the new tokens, new tokens, all keys
struct Extent {
    int len, count, keys;
    // (in scalar registers: the loads and divisions of one sequence's numbers come out in vector ones)
    __device__ __forceinline__ void make_uniform() {
        len = __builtin_amdgcn_readfirstlane(len);
        count = __builtin_amdgcn_readfirstlane(count);
        keys = __builtin_amdgcn_readfirstlane(keys);
    }
    __device__ __forceinline__ Extent(const CachedArgs& a, int b) {
        const int places = a.c.max_pages * a.c.page_size;
        len = min(max(a.c.lens[b], 0), places);
        count = a.counts ? min(max(a.counts[b], 0), a.T) : a.T;
        keys = len + min(count, places - len);
    }
    __device__ __forceinline__ int splits(const CachedArgs& a) const {  // the last chunk takes what is left
        const int n = (keys + a.chunk - 1) / a.chunk;
        return min(max(n, 1), a.splits);
    }
};

// A wave's tiles of 32 keys in the LDS, as they are staged and read: 16-bit elements like WaveTile, or codes.  A tile is
// unpadded; 16-byte chunk c of row r sits at c ^ swizzle(r), applied through the global address that a lane fetches.
template <typename Tag, int D, bool CODES>
struct CacheTile {
    static constexpr int ROWB = D * (CODES ? 1 : 2), TILE_B = 32 * ROWB, CPR = ROWB / 16, RPI = 1024 / ROWB, NI = 32 / RPI;
    static constexpr int KR = CODES ? D / 32 : D / 16, DT = D / 32, TR = CODES ? 1 : 2;
    uint32_t base;
    int src[NI / 2];           // byte offset within 16 rows for a staging instruction
    uint32_t row_at[KR];       // row operands: lane (col, half), chunk 2 k + half of row col
    uint32_t tr_at[DT][TR];    // transposed operands of rows 0..15

    // Codes: row reads take one chunk of 16 rows, transposing reads two neighbouring chunks of rows 4 h .. 4 h + 3 and 8 more; both
    // hit every bank once if bits 0, 1 and 3 of the row, where they do not choose the bank already, move chunk pairs.
    static __device__ __forceinline__ int swizzle(int r) {
        if constexpr (!CODES) return WaveTile<D>::swizzle(r);
        else if constexpr (D == 64) return (r >> 2) & 3;
        else if constexpr (D == 128) return ((r >> 1) & 1) << 1 | ((r >> 3) & 1) << 2 | ((r >> 2) & 1);
        else return (r & 1) << 1 | ((r >> 1) & 1) << 2 | ((r >> 3) & 1) << 3 | ((r >> 2) & 1);
    }
    __device__ __forceinline__ CacheTile(uint32_t at, int lane) : base(at) {
        const int col = lane & 31, half = lane >> 5, in = lane & 15, blk = (lane >> 4) & 1;
#pragma unroll
        for (int i = 0; i < NI / 2; ++i) {
            const int r = i * RPI + lane / CPR;
            src[i] = r * ROWB + ((lane % CPR) ^ swizzle(r)) * 16;
            asm volatile("" : "+v"(src[i]));
        }
#pragma unroll
        for (int k = 0; k < KR; ++k) {
            row_at[k] = at + col * ROWB + (((2 * k + half) ^ swizzle(col)) << 4);
            asm volatile("" : "+v"(row_at[k]));
        }
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int hi = 0; hi < TR; ++hi) {
                if constexpr (CODES) {  // lanes 2 i, 2 i + 1 of 16 point at row i of the group's eight
                    const int i = in >> 1, r = 4 * half + (i & 3) + 8 * (i >> 2);
                    tr_at[dt][hi] = at + r * ROWB + (((2 * dt + blk) ^ swizzle(r)) << 4) + 8 * (in & 1);
                } else {
                    const int quad = in & 3, r = 4 * half + (in >> 2) + 8 * hi;
                    tr_at[dt][hi] = at + r * ROWB + (((4 * dt + 2 * blk + (quad >> 1)) ^ swizzle(r)) << 4) + 8 * (quad & 1);
                }
                asm volatile("" : "+v"(tr_at[dt][hi]));
            }
    }
    // All instructions that bring a tile, 16 rows from each resource
    __device__ __forceinline__ void request(const BufferWords (&rsrc)[2], uint32_t offset) const {
#pragma unroll
        for (int i = 0; i < NI; ++i) global_to_lds_16B(rsrc[i / (NI / 2)], base + offset + i * 1024, src[i % (NI / 2)]);
    }

    // An infinity or a NaN in V of a new token is no business of the rows that do not see it, and a product with P = 0 would
    // make it theirs.  So where a tile has one (not_finite), matrix products of ones count for each row and column what it sees
    // of them (add_not_finite), and it is a zero for the product with P (clear_not_finite).
    using PE = Elem<std::conditional_t<CODES, f16_tag, Tag>>;
    static constexpr int EXPONENT = CODES ? 0x7F7F7F7F : std::is_same_v<Tag, bf16_tag> ? 0x7F807F80 : 0x7C007C00;
    static constexpr int ONE = !CODES && std::is_same_v<Tag, bf16_tag> ? 0x3F803F80 : 0x3C003C00;  // two ones
    // the elements of a word that are not finite, all bits of each
    static __device__ __forceinline__ uint32_t odd_ones(uint32_t w) {
        const uint32_t x = (w & EXPONENT) ^ EXPONENT;  // 0 where the exponent (of a code: all but the sign) is full
        if constexpr (CODES) {
            const uint32_t full = ~x & (0x80808080u - x) & 0x80808080u;  // x < 0x80 in each byte, so nothing is borrowed
            return (full >> 7) * 0xFFu;
        } else {
            const uint32_t full = (0x80008000u - x) & 0x80008000u;
            return (full >> 15) * 0xFFFFu;
        }
    }
    // of a word of 16-bit elements: ones where an element is an infinity of this sign, or a NaN
    static __device__ __forceinline__ uint32_t infinite(uint32_t w, bool negative) {
        const uint32_t sign = ((w & 0x80008000u) >> 15) * 0xFFFFu;
        const uint32_t nan = ((((w & ~(EXPONENT | 0x80008000u)) + 0x7FFF7FFFu) & 0x80008000u) >> 15) * 0xFFFFu;
        return odd_ones(w) & ((negative ? sign : ~sign) | nan) & ONE;
    }
    // the A operand of 16 keys and 32 columns
    __device__ __forceinline__ i32x4 columns(uint32_t offset, int slab, int dt) const {
        const int at = offset + slab * 16 * ROWB;
        if constexpr (CODES) {
            const i32x2 c = lds_read_tr8(tr_at[dt][0] + at);
            return i32x4{c[0], c[1], 0, 0};
        } else {
            const i32x2 lo = lds_read_tr16(tr_at[dt][0] + at), hi = lds_read_tr16(tr_at[dt][1] + at);
            return i32x4{lo[0], lo[1], hi[0], hi[1]};
        }
    }
    __device__ __forceinline__ bool not_finite(uint32_t offset, int lane) const {
        uint32_t any = 0;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const i32x4 w = lds_load_16B(base + offset + i * 1024 + lane * 16);
            any |= odd_ones(w[0]) | odd_ones(w[1]) | odd_ones(w[2]) | odd_ones(w[3]);
        }
        return __builtin_amdgcn_ballot_w64(any != 0) != 0;
    }
    __device__ __forceinline__ void clear_not_finite(uint32_t offset, int lane) const {
        typedef i32x4 __attribute__((address_space(3))) * lds_vec_ptr;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const uint32_t at = base + offset + i * 1024 + lane * 16;
            i32x4 w = lds_load_16B(at);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] &= ~odd_ones(w[e]);
            *(lds_vec_ptr)(uintptr_t)at = w;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    __device__ __forceinline__ void add_not_finite(uint32_t offset, int half, uint32_t vis, f32x16 (&acc)[DT]) const;
};

// Eight codes as eight 16-bit elements
template <typename Tag>
static __device__ __forceinline__ i32x4 from_codes(int lo, int hi) {
    i32x4 w;
    if constexpr (std::is_same_v<Tag, bf16_tag>) {
        w[0] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false));
        w[1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true));
        w[2] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false));
        w[3] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true));
    } else {
        w[0] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false));
        w[1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true));
        w[2] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false));
        w[3] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true));
    }
    return w;
}

template <typename Tag, int D, bool CODES>
__device__ __forceinline__ void CacheTile<Tag, D, CODES>::add_not_finite(uint32_t offset, int half, uint32_t vis, f32x16 (&acc)[DT]) const {
    i32x4 seen[2];
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
        const uint32_t two = vis >> (4 * half + 8 * (r >> 2) + (r & 3));
        seen[r >> 3][(r >> 1) & 3] = (int)((two & 1 ? 0xFFFFu : 0u) | (two & 2 ? 0xFFFF0000u : 0u)) & ONE;
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int negative = 0; negative < (CODES ? 1 : 2); ++negative) {
            f32x16 count = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int slab = 0; slab < 2; ++slab) {
                i32x4 w = columns(offset, slab, dt);
                if constexpr (CODES) {
                    w = from_codes<f16_tag>((int)odd_ones(w[0]) & 0x38383838, (int)odd_ones(w[1]) & 0x38383838);  // 0x38: 1
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = (int)infinite(w[e], negative);
                }
                count = PE::mma(w, seen[slab], count);
            }
            const float what = CODES ? __builtin_nanf("") : negative ? -INFINITY : INFINITY;  // a NaN counts as both
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[dt][r] += count[r] > 0.f ? what : 0.f;
        }
}

// Asynchronous copy of 4 bytes per lane from an address per lane to lds_base + 4 lane
static __device__ __forceinline__ void global_to_lds_4B(const float* p, uint32_t lds_base) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
                 :
                 : "s"(__builtin_amdgcn_readfirstlane(lds_base)), "v"(p)
                 : "memory", "m0");
}

template <int N>
static __device__ __forceinline__ void wait_vmcnt() {
    static_assert(N < 64, "what the counter holds");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

constexpr int kMergeCols = 64, kMergeStride = kMergeCols + 4;

// A row number of lane i's in scalar registers; negative: none.  (Two words: there is no scalar comparison of 64 bits.)
struct UniformRow {
    int lo, hi;
    UniformRow() = default;
    __device__ __forceinline__ UniformRow(long v, int i) : lo(__builtin_amdgcn_readlane((int)v, i)), hi(__builtin_amdgcn_readlane((int)(v >> 32), i)) {
        asm volatile("" : "+s"(lo), "+s"(hi));  // (or the two are compared as one again)
    }
    __device__ __forceinline__ int none() const { return hi >> 31; }  // all bits set, or none
    __device__ __forceinline__ long index() const { return (long)((uint64_t)(uint32_t)(lo & ~none()) | (uint64_t)(uint32_t)(hi & ~none()) << 32); }
};

template <typename Tag, int D, bool CODES, int NW, int STG, int RT>
struct CachedShape {
    using Tile = CacheTile<Tag, D, CODES>;
    static constexpr int SCALE_B = CODES ? 256 : 0;                    // of a tile: 32 scales of K, 32 of V
    static constexpr int STAGE_B = 2 * Tile::TILE_B + SCALE_B, WAVE_B = STG * STAGE_B;
    static constexpr int MERGE_B = NW * 32 * kMergeStride * 4, STATE_B = NW * RT * 32 * 3 * 4;
    static constexpr int LDS = (NW * WAVE_B > MERGE_B ? NW * WAVE_B : MERGE_B) + STATE_B;
};

template <typename Tag, int D, bool CODES, int NW, int STG, int RT>
__global__ void __launch_bounds__(NW * 64, RT == 1 && D < 256 ? 2 : 1)
fa_fwd_cache_kernel(CachedArgs a) {
    using Shape = CachedShape<Tag, D, CODES, NW, STG, RT>;
    using Tile = typename Shape::Tile;
    using E = Elem<Tag>;
    using PE = Elem<std::conditional_t<CODES, f16_tag, Tag>>;  // of the product with V
    constexpr int KS = D / 16, DT = D / 32, NI = Tile::NI, X = CODES ? 1 : 0;
    extern __shared__ __align__(16) char lds[];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int col = lane & 31, half = lane >> 5;

    // which rows and keys: row groups of a chunk side by side on one XCD
    int item = xcd_run(blockIdx.x, gridDim.x);
    const int rg = __builtin_amdgcn_readfirstlane(item % a.row_groups);
    item /= a.row_groups;
    const int split = __builtin_amdgcn_readfirstlane(item % a.splits);
    item /= a.splits;
    const int H_kv = a.c.H_kv, b = __builtin_amdgcn_readfirstlane(item / H_kv), kvh = __builtin_amdgcn_readfirstlane(item - b * H_kv);
    const int group = a.H / H_kv, n_rows = group * a.T;
    Extent ext(a, b);
    ext.make_uniform();
    const int n_splits = __builtin_amdgcn_readfirstlane(ext.splits(a));
    if (split >= n_splits) return;
    const int key0 = split * a.chunk, key1 = split == n_splits - 1 ? ext.keys : key0 + a.chunk;
    const int n_tiles = (max(key1 - key0, 0) + 31) / 32, mine = n_tiles > wave ? (n_tiles - wave + NW - 1) / NW : 0;

    int t[RT];  // the token of the lane's rows (clamped: rows past the end compute a copy of the last, never stored)
    i32x4 qreg[RT][KS];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        const int row = min((rg * RT + i) * 32 + col, n_rows - 1), g = row / a.T;
        t[i] = row - g * a.T;
        const uint16_t* q = static_cast<const uint16_t*>(a.q.p) + (b * a.q.batch + (kvh * group + g) * a.q.head + t[i] * a.q.token);
#pragma unroll
        for (int u = 0; u < KS; ++u)
            qreg[i][u] = *reinterpret_cast<const i32x4*>(q + (CODES ? 32 * (u / 2) + 16 * half + 8 * (u % 2) : 16 * u + 8 * half));
    }

    const Tile tile(lds_address(lds) + wave * Shape::WAVE_B, lane);
    // rows (of all pages' rows, heads included) of the wave's tiles: lane i has tile i of 64, two times 16 places; -1: no page
    long row_lo = -1, row_hi = -1;
    auto look_up = [&](int first) __attribute__((always_inline)) {
        const int key = key0 + 32 * (wave + NW * (first + lane));
        auto of = [&](int k) -> long {
            if (k >= key1 || k < key0) return -1;
            const int entry = k / a.c.page_size, page = a.c.block_table[(long)b * a.c.max_pages + entry];
            if (page < 0 || page >= a.c.n_pages) return -1;
            return ((long)page * H_kv + kvh) * a.c.page_size + (k - entry * a.c.page_size);
        };
        row_lo = of(key);
        row_hi = of(key + 16);
    };
    // requests K of the wave's tile i into stage st, and its V when that stage's V has been read
    UniformRow rows[STG][2];
    auto resources = [&](const void* pages, int i, const UniformRow (&row)[2], BufferWords (&rsrc)[2]) __attribute__((always_inline)) {
        const int left = key1 - (key0 + 32 * (wave + NW * i));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            int n = max(left - 16 * h, 0);
            asm volatile("" : "+s"(n));  // (with the minimum it would be one vector instruction)
            n = min(n, 16) & ~row[h].none();
            rsrc[h] = make_buffer_words(static_cast<const char*>(pages) + (row[h].index() * Tile::ROWB), n * Tile::ROWB);
        }
    };
    auto request_k = [&](int i, auto stage) __attribute__((always_inline)) {
        constexpr int st = decltype(stage)::value;
        if ((i & 63) == 0) look_up(i);
        rows[st][0] = UniformRow(row_lo, i & 63);
        rows[st][1] = UniformRow(row_hi, i & 63);
        BufferWords rsrc[2];
        resources(a.c.k, i, rows[st], rsrc);
        tile.request(rsrc, st * Shape::STAGE_B);
        if constexpr (CODES) {  // lanes 0..31 the scales of K, 32..63 of V; of a place that is none: any
            long row = rows[st][0].index(), upper = rows[st][1].index();
            asm volatile("" : "+v"(row), "+v"(upper));  // (a choice between vector registers, not between places in memory)
            row = lane & 16 ? upper : row;
            const int left = key1 - (key0 + 32 * (wave + NW * i));
            const long at = (lane & 31) >= left ? 0 : row + (lane & 15);
            global_to_lds_4B((half ? a.c.v_scales : a.c.k_scales) + at, tile.base + st * Shape::STAGE_B + 2 * Tile::TILE_B);
        }
    };
    auto request_v = [&](int i, auto stage) __attribute__((always_inline)) {
        constexpr int st = decltype(stage)::value;
        BufferWords rsrc[2];
        resources(a.c.v, i, rows[st], rsrc);
        tile.request(rsrc, st * Shape::STAGE_B + Tile::TILE_B);
    };

    f32x16 acc[RT][DT];
    float m_run[RT], l_run[RT];
    float F = 0.f, inv_F = 0.f;  // codes: the power of two that P~ is divided by
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        m_run[i] = -INFINITY;
        l_run[i] = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][dt][r] = 0.f;
    }
    const float sc = a.scale * kLog2e;

    // the row's view of the 32 places from `key` on
    auto visible = [&](int key, int row_t, int bad_halves) __attribute__((always_inline)) {
        const int u0 = key - ext.len;  // the number of the first place among the new tokens
        uint32_t vis = 0;
        if (a.tree) {
            const int words = (a.T + 31) >> 5;
            const int* row = a.tree + ((long)(a.tree_batches == 1 ? 0 : b) * a.T + row_t) * words;
            const int w = u0 >> 5, s = u0 & 31;
            const uint32_t lo = w >= 0 && w < words ? (uint32_t)row[w] : 0u, hi = w + 1 >= 0 && w + 1 < words ? (uint32_t)row[w + 1] : 0u;
            vis = s ? lo >> s | hi << (32 - s) : lo;
        } else if (u0 <= row_t) {
            vis = row_t - u0 >= 31 ? ~0u : (2u << (row_t - u0)) - 1;
        }
        if (u0 < 0) vis |= u0 <= -32 ? ~0u : (1u << -u0) - 1;  // places before the new tokens
        const int there = min(ext.keys, key1) - key;
        if (there < 32) vis &= there <= 0 ? 0u : (1u << there) - 1;
        if (bad_halves & 1) vis &= 0xFFFF0000u;
        if (bad_halves & 2) vis &= 0x0000FFFFu;
        return vis;
    };

    if (mine > 0)
        static_for<STG>([&](auto st) {
            request_k(st, st);
            request_v(st, st);
        });
    for (int i0 = 0; i0 < mine; i0 += STG) {
        static_for<STG>([&](auto stage) __attribute__((always_inline)) {
            constexpr int st = decltype(stage)::value, kK = st * Shape::STAGE_B, kV = kK + Tile::TILE_B, kScales = kK + 2 * Tile::TILE_B;
            const int i = i0 + st;
            if (i >= mine) return;
            const int key = key0 + 32 * (wave + NW * i);
            wait_vmcnt<NI * STG + (NI + X) * (STG - 1)>();  // K has landed
            f32x16 s[RT];
#pragma unroll
            for (int x = 0; x < RT; ++x) s[x] = f32x16{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < Tile::KR; ++k) {
                const i32x4 w = lds_load_16B(tile.row_at[k] + kK);
                if constexpr (CODES) {
                    const i32x4 lo = from_codes<Tag>(w[0], w[1]), hi = from_codes<Tag>(w[2], w[3]);
#pragma unroll
                    for (int x = 0; x < RT; ++x) s[x] = E::mma(lo, qreg[x][2 * k], s[x]);
#pragma unroll
                    for (int x = 0; x < RT; ++x) s[x] = E::mma(hi, qreg[x][2 * k + 1], s[x]);
                } else {
#pragma unroll
                    for (int x = 0; x < RT; ++x) s[x] = E::mma(w, qreg[x][k], s[x]);
                }
            }
            float vscale[16];
            if constexpr (CODES) {
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x4 ks = lds_load_4f(tile.base + kScales + 32 * g + 16 * half), vs = lds_load_4f(tile.base + kScales + 128 + 32 * g + 16 * half);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        vscale[4 * g + r] = vs[r];
#pragma unroll
                        for (int x = 0; x < RT; ++x) s[x][4 * g + r] *= ks[r];
                    }
                }
            }
            const int bad_now = (rows[st][0].none() & 1) | (rows[st][1].none() & 2);  // the halves that are on no page
            const int next = i + STG;
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // K and the scales have been read: the next ones may come
            request_k(next, stage);

            const bool special = key + 32 > ext.len || bad_now != 0;
            uint32_t vis[RT];
            if (special) {
#pragma unroll
                for (int x = 0; x < RT; ++x) {
                    vis[x] = visible(key, t[x], bad_now);
                    const uint32_t w = vis[x] >> (4 * half);
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        s[x][r] = w >> (8 * (r >> 2) + (r & 3)) & 1 ? s[x][r] : -INFINITY;
                }
            }
            if constexpr (CODES) {
                // the largest finite scale of V in the tile (places that are none have any: they cost accuracy at most where they exceed the others)
                float top = 0.f;
                const int there = (special ? min(ext.keys, key1) - key : 32) - 4 * half;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    if (special && (8 * (r >> 2) + (r & 3) >= there || (bad_now >> (r >> 3) & 1))) vscale[r] = 0.f;
                    top = fmaxf(top, vscale[r] < INFINITY ? vscale[r] : 0.f);
                }
                top = fminf(fmaxf(max_both_halves(top), 0x1p-100f), 0x1p126f);
                const float new_F = __builtin_bit_cast(float, (int)((__builtin_bit_cast(int, top) + 0x7fffff) & 0x7f800000));
                if (__builtin_amdgcn_readfirstlane(new_F > F)) {
                    const float down = F / new_F;
                    F = new_F;
                    inv_F = 1.f / new_F;
#pragma unroll
                    for (int x = 0; x < RT; ++x)
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                            for (int r = 0; r < 16; ++r) acc[x][dt][r] *= down;
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) vscale[r] *= inv_F;
            }
            i32x4 pb[RT][2];  // what V is multiplied by
#pragma unroll
            for (int x = 0; x < RT; ++x) {
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int r = 0; r < 16; ++r) mx[r & 3] = fmaxf(mx[r & 3], s[x][r]);
                const float m_new = max_both_halves(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])));
                const bool raise = (m_new - m_run[x]) * sc > kLazy;
                if (__builtin_amdgcn_ballot_w64(raise) != 0) {
                    const float corr = raise ? fast_exp2((m_run[x] - m_new) * sc) : 1.0f;
                    m_run[x] = raise ? m_new : m_run[x];
                    l_run[x] *= corr;
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc[x][dt][r] *= corr;
                }
                const float mb = m_run[x] == -INFINITY ? 0.f : m_run[x] * sc;  // a row that has seen nothing yet: P = 0
                float ps[4];
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float p = fast_exp2(__builtin_fmaf(s[x][r], sc, -mb));
                    ps[r & 3] = r < 4 ? p : ps[r & 3] + p;
                    s[x][r] = p;
                    if constexpr (CODES) s[x][r] = p * vscale[r];
                }
                if constexpr (CODES) {
                    if (special) {  // a scale that is not finite belongs to those rows only that see it
                        const uint32_t w = vis[x] >> (4 * half);
#pragma unroll
                        for (int r = 0; r < 16; ++r) s[x][r] = w >> (8 * (r >> 2) + (r & 3)) & 1 ? s[x][r] : 0.f;
                    }
                }
                l_run[x] += (ps[0] + ps[1]) + (ps[2] + ps[3]);
#pragma unroll
                for (int r = 0; r < 16; r += 2) pb[x][r >> 3][(r >> 1) & 3] = PE::pack2(s[x][r], s[x][r + 1]);
            }
            wait_vmcnt<(NI + X) * STG + NI * (STG - 1)>();  // V has landed
            if (special && key + 32 > ext.len)
                if (__builtin_expect(tile.not_finite(kV, lane), 0)) {
#pragma unroll
                    for (int x = 0; x < RT; ++x) tile.add_not_finite(kV, half, vis[x], acc[x]);
                    tile.clear_not_finite(kV, lane);
                }
            // O^T += V^T P^T
#pragma unroll
            for (int u = 0; u < 2 * DT; ++u) {
                const int slab = u / DT, dt = u % DT;
                i32x4 w = tile.columns(kV, slab, dt);
                if constexpr (CODES) w = from_codes<f16_tag>(w[0], w[1]);
#pragma unroll
                for (int x = 0; x < RT; ++x) acc[x][dt] = PE::mma(w, pb[x][slab], acc[x][dt]);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            request_v(next, stage);
        });
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the last requests: the LDS is about to be reused

    // The waves' states meet: with M the largest reference and f = 2^(m - M), sum f F acc, M and sum f l
    float* const state = reinterpret_cast<float*>(lds + Shape::LDS - Shape::STATE_B);  // [RT][NW][32][m, l, F]
    float* const part = reinterpret_cast<float*>(lds);                                 // [NW][32][kMergeStride]
#pragma unroll
    for (int x = 0; x < RT; ++x) {
        const float l = sum_both_halves(l_run[x]);
        if (half == 0) {
            float* at = state + ((x * NW + wave) * 32 + col) * 3;
            at[0] = m_run[x] * sc;
            at[1] = l;
            at[2] = CODES ? F : 1.f;
        }
    }
    const bool whole = n_splits == 1;
#pragma unroll
    for (int x = 0; x < RT; ++x)
#pragma unroll
        for (int c0 = 0; c0 < D; c0 += kMergeCols) {
            __syncthreads();
#pragma unroll
            for (int d2 = 0; d2 < 2; ++d2)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x16& y = acc[x][c0 / 32 + d2];
                    const f32x4 w = {y[4 * g], y[4 * g + 1], y[4 * g + 2], y[4 * g + 3]};
                    *reinterpret_cast<f32x4*>(part + (wave * 32 + col) * kMergeStride + d2 * 32 + 8 * g + 4 * half) = w;
                }
            __syncthreads();
            for (int c = tid; c < 32 * kMergeCols / 8; c += NW * 64) {
                const int r = c / (kMergeCols / 8), cc = (c % (kMergeCols / 8)) * 8, row = (rg * RT + x) * 32 + r;
                if (row >= n_rows) continue;
                const int g = row / a.T, tok = row - g * a.T;
                if (tok >= ext.count) continue;
                float m_all = -INFINITY, l_all = 0.f, f[NW];
#pragma unroll
                for (int w = 0; w < NW; ++w) m_all = fmaxf(m_all, state[((x * NW + w) * 32 + r) * 3]);
                const float m_ref = m_all == -INFINITY ? 0.f : m_all;
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    const float* at = state + ((x * NW + w) * 32 + r) * 3;
                    f[w] = fast_exp2(at[0] - m_ref);
                    l_all += f[w] * at[1];
                    f[w] *= at[2];
                }
                float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < NW; ++w)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const f32x4 z = *reinterpret_cast<const f32x4*>(part + (w * 32 + r) * kMergeStride + cc + 4 * h);
#pragma unroll
                        for (int e = 0; e < 4; ++e) y[4 * h + e] = __builtin_fmaf(f[w], z[e], y[4 * h + e]);
                    }
                const int head = kvh * group + g;
                const long out_row = ((long)b * a.H + head) * a.T + tok;
                if (whole) {
                    const float inv = l_all == 0.f ? 0.f : 1.0f / l_all;  // a row that sees nothing: 0
                    uint16_t* o = static_cast<uint16_t*>(const_cast<void*>(a.o.p)) + (b * a.o.batch + head * a.o.head + tok * a.o.token);
                    i32x4 w;
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = E::pack2(y[2 * e] * inv, y[2 * e + 1] * inv);
                    *reinterpret_cast<i32x4*>(o + c0 + cc) = w;
                    if (c0 + cc == 0) a.lse[out_row] = (m_all + log2f(l_all)) * kLn2;
                } else {
                    const long at = (long)split * a.B * a.H * a.T + out_row;
                    float* o = a.part + at * D + c0 + cc;
                    *reinterpret_cast<f32x4*>(o) = f32x4{y[0], y[1], y[2], y[3]};
                    *reinterpret_cast<f32x4*>(o + 4) = f32x4{y[4], y[5], y[6], y[7]};
                    if (c0 + cc == 0) {
                        a.state[2 * at] = m_all;
                        a.state[2 * at + 1] = l_all;
                    }
                }
            }
        }
}

// Joins the chunks of rows whose sequence has several: D / 8 threads to a row, 8 columns each
template <typename Tag, int D>
__global__ void __launch_bounds__(256) fa_join_kernel(CachedArgs a) {
    using E = Elem<Tag>;
    constexpr int TPR = D / 8;
    const long n_rows = (long)a.B * a.H * a.T, row = (long)blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
    if (row >= n_rows) return;
    const int bh = (int)(row / a.T), tok = (int)(row - (long)bh * a.T), b = bh / a.H, head = bh - b * a.H, c = (threadIdx.x % TPR) * 8;
    const Extent ext(a, b);
    const int n = ext.splits(a);
    if (n == 1 || tok >= ext.count) return;
    float m_all = -INFINITY, l_all = 0.f;
    for (int s = 0; s < n; ++s) m_all = fmaxf(m_all, a.state[2 * (s * n_rows + row)]);
    const float m_ref = m_all == -INFINITY ? 0.f : m_all;
    float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = 0; s < n; ++s) {
        const long at = s * n_rows + row;
        const float f = fast_exp2(a.state[2 * at] - m_ref);
        l_all += f * a.state[2 * at + 1];
        const f32x4 lo = *reinterpret_cast<const f32x4*>(a.part + at * D + c), hi = *reinterpret_cast<const f32x4*>(a.part + at * D + c + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            y[e] = __builtin_fmaf(f, lo[e], y[e]);
            y[4 + e] = __builtin_fmaf(f, hi[e], y[4 + e]);
        }
    }
    const float inv = l_all == 0.f ? 0.f : 1.0f / l_all;
    i32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = E::pack2(y[2 * e] * inv, y[2 * e + 1] * inv);
    uint16_t* o = static_cast<uint16_t*>(const_cast<void*>(a.o.p)) + (b * a.o.batch + head * a.o.head + tok * a.o.token);
    *reinterpret_cast<i32x4*>(o + c) = w;
    if (c == 0) a.lse[row] = (m_all + log2f(l_all)) * kLn2;
}

// How a call is divided: row tiles to a wave, row groups, chunks of keys
struct CachedDivision {
    int rt, row_groups, splits, chunk;
    CachedDivision(int B, int H, int H_kv, int T, int d, int max_len) {
        const int rows = H / H_kv * T, tiles = (rows + 31) / 32;
        rt = tiles > 1 && d < 256 ? 2 : 1;
        row_groups = (tiles + rt - 1) / rt;
        const double base = (double)B * H_kv * row_groups;
        // enough workgroups to fill the chip several times, but chunks of 256 keys at least
        double per = max_len * base / 1536.0;
        if (per > max_len) per = max_len;
        chunk = 256;
        if (per > 256) chunk = per > 0x3fffffff ? 0x3fffffff : ((int)per + 127) / 128 * 128;
        splits = (int)(((long)max_len + chunk - 1) / chunk);
        if (splits > 256) {
            chunk = (max_len / 256 + 128) / 128 * 128;
            splits = (int)(((long)max_len + chunk - 1) / chunk);
        }
    }
};

template <typename Tag, int D, bool CODES, int RT>
static int launch_cached(const CachedArgs& a, hipStream_t stream) {
    constexpr int NW = 4, STG = D * (CODES ? 1 : 2) >= 256 ? 1 : 2;
    using Shape = CachedShape<Tag, D, CODES, NW, STG, RT>;
    auto kernel = fa_fwd_cache_kernel<Tag, D, CODES, NW, STG, RT>;
    const double total = (double)a.B * a.c.H_kv * a.row_groups * a.splits;
    if (total * NW * 64 >= 4294967296.0) return FA_ERR_LAUNCH;
    hipLaunchKernelGGL(kernel, dim3((unsigned)total), dim3(NW * 64), Shape::LDS, stream, a);
    if (hipGetLastError() != hipSuccess) return FA_ERR_LAUNCH;
    if (a.splits > 1) {
        const long per = 256 / (D / 8), rows = (long)a.B * a.H * a.T;
        hipLaunchKernelGGL((fa_join_kernel<Tag, D>), dim3((unsigned)((rows + per - 1) / per)), dim3(256), 0, stream, a);
        if (hipGetLastError() != hipSuccess) return FA_ERR_LAUNCH;
    }
    return FA_OK;
}

template <typename Tag, bool CODES>
static int launch_cached_d(const CachedArgs& a, int d, int rt, hipStream_t stream) {
    switch (d) {
        case 64: return rt == 1 ? launch_cached<Tag, 64, CODES, 1>(a, stream) : launch_cached<Tag, 64, CODES, 2>(a, stream);
        case 128: return rt == 1 ? launch_cached<Tag, 128, CODES, 1>(a, stream) : launch_cached<Tag, 128, CODES, 2>(a, stream);
        default: return launch_cached<Tag, 256, CODES, 1>(a, stream);
    }
}

}  // namespace

size_t fwd_cache_workspace_bytes(int B, int H, int H_kv, int T, int d, int max_len, int) {
    const CachedDivision div(B, H, H_kv, T, d, max_len);
    return div.splits == 1 ? 0 : (size_t)div.splits * B * H * T * (d + 2) * sizeof(float);
}

int launch_fwd_cache(const Rows& q, const Cache& cache, const int* counts, const int* tree, int tree_batches, const Rows& o, float* lse,
                     void* workspace, int B, int H, int T, int d, int max_len, float scale, int dtype, hipStream_t stream) {
    const CachedDivision div(B, H, cache.H_kv, T, d, max_len);
    float* part = static_cast<float*>(workspace);
    float* state = div.splits == 1 ? nullptr : part + (size_t)div.splits * B * H * T * d;
    const CachedArgs a = {q, o, cache, counts, tree, lse, part, state, B, H, T, tree_batches, div.row_groups, div.splits, div.chunk, scale};
    const bool codes = cache.dtype == FA_FP8_E4M3;
    if (dtype == FA_BF16) return codes ? launch_cached_d<bf16_tag, true>(a, d, div.rt, stream) : launch_cached_d<bf16_tag, false>(a, d, div.rt, stream);
    return codes ? launch_cached_d<f16_tag, true>(a, d, div.rt, stream) : launch_cached_d<f16_tag, false>(a, d, div.rt, stream);
}

}  // namespace fa
