// Attention of the new tokens of every sequence over a paged cache (include/fa_mi355.h: fa_fwd_cache).
//
// The rows that read one key/value head, (query head of the group) x (new token), are queries of one dense problem: COLS of them
// (16, or 32) make a tile, one to a lane column, RT tiles a workgroup.  The keys go to workgroups in steps of NW tiles of 32 keys,
// a tile for each wave, which has a softmax state and an output accumulator of its own; they meet in the LDS at the end, in a
// fixed order.
//
// The floor is HBM's up to some 250 rows to a key/value head (4 rows d flops for 4 d bytes of a 16-bit key, at 1.2 PFLOP/s of a
// library product and 5 TB/s of a copy): the cache is read once per row group, straight into the LDS.  Measured with the join:
// 32 sequences of 500 to 4096 keys, H = 32 on 8, bf16, T = 1: 268 MB in 51 us, 5.2 TB/s; 2 of up to 65536 keys, H = 16 on 2,
// d = 256, codes: 129 MB in 33 us, of which some 13 are the look-up of pages, the merge and the join; 4 trees of 64 tokens over up to
// 16384 keys, H = 32 on 4, bf16: 50 GFLOP in 91 us, where the matrix pipes are busy a third of the loop.  A wave stages its own tiles (no barrier in the loop): a slot for K and one for V, STG deep,
// refilled as soon as the wave has read them, so requests go on while scores, softmax and products are computed.
//   - Work: the steps of all sequences and heads lie in a row, and each team of workgroups (one for each row group) takes an equal
//     share of it, whatever the lengths are: they are known on the device only.  A share may end inside a sequence; what a team
//     has of such a one, (sum p v, reference, sum p), goes to the workspace, and a second launch joins it with what the teams
//     before and after have, in that order.  Where no sequence can be long a workgroup has a whole one of a head (whole_sequences).
//   - Pages: 16 consecutive places lie in one page (page_size is a multiple of 16), so a tile has two resources.  Lane i of a
//     wave looks up the two rows of the wave's i-th tile, 64 tiles at a time; what is no page, or past the last key, gets a
//     resource of length 0 and arrives as zeros.
//   - Masks: only tiles that reach the new tokens (or hold a bad page) look at one.  What a lane's row sees of a tile is a 32-bit
//     word: places before the new tokens, the row's window of the tree, the tokens that are there.
//   - e4m3: codes become 16-bit operands in registers (exact): K in the type of Q, with the key's scale on the score; V in
//     bf16, with P~ = p v scale as two bf16 numbers, a rounded value and what that leaves out.  Their range is that of the scales, so
//     no weight depends on a scale of another key, seen or not, and sixteen bits of each reach the product.
//   - 16 columns where a group has no more rows (v_mfma_16x16x32 instead of 32x32x16): half the registers, matrix and vector
//     instructions for a tile.
#include "fa_device.h"
#include "fa_launch.h"

namespace fa {

struct CachedArgs {
    Rows q, o;
    Cache c;
    const int *counts, *tree;
    float* lse;
    // the workspace: where the segments of each sequence and head are [B H_kv], then for each workgroup two segments [rows][D] and [rows][2]
    struct Segments {
        int first, count;  // number of its first team's segment (2 team + 0 or 1); its teams.  The others' are their teams' first ones.
    }* segments;
    float *part, *state;
    int B, H, T, tree_batches, row_groups, teams;  // teams 0: a workgroup to a sequence, head and row group
    float scale;
};

namespace {

// Operands from the LDS go to the matrix instructions this many reads at a time, all issued before the first product: left to itself
// the compiler has one or two on the way, and each instruction of 16 or 32 cycles waits for one.  us before / after: 4 trees of 32, 4 heads
// of d = 256 to a key/value head 47.8 / 42.8; 8 trees of 32, 8 heads, codes 53.8 / 51.2; 2 long sequences of codes, d = 256 35.3 / 33.9;
// within the noise where a CU has 8 waves of 32 columns on 16-bit keys.  4, 8 and 16 are alike.  (Codes: with each weight in one fp16 number.)
constexpr int kReadsAhead = 8;
constexpr float kLazy = 8.0f;  // the reference of a row rises when a tile's maximum exceeds it by more (log2 units)

// What a sequence has: places before the new tokens, new tokens, all keys
struct Extent {
    int len, count, keys;
    Extent() = default;
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
    template <int STEP>
    __device__ __forceinline__ int steps() const {  // at least one: rows that see nothing are written too
        return keys <= STEP ? 1 : (int)(((unsigned)keys + STEP - 1) / STEP);
    }
};

// `of` things in order to `among`: the first of % among of them have one more.  (Steps of all sequences are fewer than 2^31.)
struct Shares {
    uint32_t each, rest;
    __device__ __forceinline__ Shares(uint32_t of, uint32_t among) : each(of / among), rest(of - each * among) {}
    __device__ __forceinline__ uint32_t first(uint32_t i) const { return i * each + min(i, rest); }
    __device__ __forceinline__ uint32_t owner(uint32_t thing) const {
        const uint32_t longer = rest * (each + 1);
        return thing < longer ? thing / (each + 1) : rest + (thing - longer) / each;
    }
};

// x summed up to and with this lane
static __device__ __forceinline__ uint32_t sum_upto(uint32_t x, int lane) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    return x;
}

// x of this lane's row of 16 lanes and of the row next to it (rows 0 and 1, 2 and 3)
static __device__ __forceinline__ HalfPair both_rows(float x) {
    uint32_t a = __builtin_bit_cast(uint32_t, x);
    uint32_t b = a;
    asm volatile("" : "+v"(b));
    auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
    uint32_t r0 = r[0], r1 = r[1];
    asm volatile("" : "+v"(r0), "+v"(r1));
    return {__builtin_bit_cast(float, r0), __builtin_bit_cast(float, r1)};
}

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

// The two shapes of the matrix products, by the columns (queries) of a tile.  Lane (col, part): col = lane % COLS.
//   scores      NS values of the lane's query: register r belongs to key (part << SHIFT) + bit(r) of the tile's 32
//   products    NT accumulators; register r of accumulator dt is output column dt WIDTH + column(r, part)
template <typename Tag, int D, int COLS> struct Matrix;
template <typename Tag, int D> struct Matrix<Tag, D, 32> {
    static constexpr int PARTS = 2, NS = 16, SHIFT = 2, NT = D / 32, WIDTH = 32, SLABS = 2, TILES = 1;
    typedef f32x16 Acc;
    static constexpr __device__ int bit(int r) { return 8 * (r >> 2) + (r & 3); }
    static __device__ __forceinline__ Acc mma(i32x4 a, i32x4 b, Acc c) { return Elem<Tag>::mma(a, b, c); }
    static __device__ __forceinline__ float max_parts(float x) { return max_both_halves(x); }
    static __device__ __forceinline__ float sum_parts(float x) { return sum_both_halves(x); }
};
template <typename Tag, int D> struct Matrix<Tag, D, 16> {
    // rows of the two score tiles are dealt so that a part's keys are eight consecutive ones: row i of tile kt is key
    // 8 (i / 4) + 4 kt + i % 4
    static constexpr int PARTS = 4, NS = 8, SHIFT = 3, NT = D / 16, WIDTH = 16, SLABS = 1, TILES = 2;
    typedef f32x4 Acc;
    static constexpr __device__ int bit(int r) { return r; }
    static __device__ __forceinline__ Acc mma(i32x4 a, i32x4 b, Acc c) {
        if constexpr (std::is_same_v<Tag, bf16_tag>)
            return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
        else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ float max_parts(float x) {
        const HalfPair p = both_rows(x);
        return max_both_halves(fmaxf(p.lo, p.hi));
    }
    static __device__ __forceinline__ float sum_parts(float x) {
        const HalfPair p = both_rows(x);
        return sum_both_halves(p.lo + p.hi);
    }
};

// global_to_lds_16B, non-temporal: what nobody else reads.  (But at d = 256 two row groups of 33 to 64 rows read each key, through this
// too: no form there takes more than 32 rows a workgroup and divides the keys.)
static __device__ __forceinline__ void once_to_lds_16B(const BufferWords& rsrc, uint32_t lds_base, int byte_off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds"
                 :
                 : "s"(__builtin_amdgcn_readfirstlane(lds_base)), "v"(byte_off), "s"(rsrc.w)
                 : "memory", "m0");
}

// A wave's tiles of 32 keys in the LDS, as they are staged and read.  A tile is unpadded; 16-byte chunk c of row r sits at
// c ^ swizzle(r), applied through the global address that a lane fetches, so that each 16 lanes of a row read (16 rows, one
// chunk) and each 32 of a transposing read (8 rows, two chunks, or 4 and 4, or 16 and 1) hit every bank once, with rows of 64 to
// 512 bytes.  Everything but the row is a constant that an exclusive or brings in: one address register for each kind of read.
template <typename Tag, int D, bool CODES, int COLS>
struct CacheTile {
    using M = Matrix<Tag, D, COLS>;
    using PE = std::conditional_t<CODES, bf16_tag, Tag>;  // of the product with V
    using PM = Matrix<PE, D, COLS>;
    static constexpr int ROWB = D * (CODES ? 1 : 2), TILE_B = 32 * ROWB, CPR = ROWB / 16, RPI = 1024 / ROWB, NI = 32 / RPI;
    static constexpr int MASK = CPR < 16 ? CPR - 1 : 15;
    static constexpr int KR = CPR / M::PARTS;  // row reads of a lane and score tile
    // KEPT (32 columns, where matrix and vector instructions compete): an address register for each chunk instead, the rest in
    // the instructions' offsets; the 16 rows of the other slab have the same swizzle
    static constexpr bool KEPT = COLS == 32;
    static constexpr int TR = CODES ? 1 : 2;
    uint32_t base, src0, row0, tr0;
    uint32_t row_at[KEPT ? KR : 1], tr_at[KEPT ? M::NT : 1][TR];

    static constexpr __device__ __host__ int swizzle(int r) {
        return ((r & 1) << 3 | (r >> 1 & 1) << 2 | (r >> 3 & 1) << 1 | ((COLS == 16 ? r >> 2 ^ r >> 4 : r >> 2) & 1)) & MASK;
    }
    // what bringing chunk c into an address of row r, or adding row bits that r has not, does to it
    static constexpr __device__ uint32_t flip(int chunk, int more_rows) { return (uint32_t)((chunk & MASK) ^ swizzle(more_rows)) << 4; }
    static constexpr __device__ uint32_t plus(int chunk, int more_rows) { return (uint32_t)(more_rows * ROWB + (chunk & ~MASK) * 16); }

    __device__ __forceinline__ CacheTile(uint32_t at, int lane) : base(at) {
        const int col = lane % COLS, part = lane / COLS, in = lane & 15, blk = (lane >> 4) & 1;
        const int r = lane / CPR;
        src0 = r * ROWB + (((lane % CPR) ^ swizzle(r)) << 4);
        const int kr = COLS == 32 ? col : 8 * (col >> 2) + (col & 3);
        row0 = at + kr * ROWB + ((part ^ swizzle(kr)) << 4);
        if constexpr (CODES) {  // lanes 2 i, 2 i + 1 of 16 point at row i of the group's eight
            const int i = in >> 1, tr = COLS == 32 ? 4 * part + (i & 3) + 8 * (i >> 2) : 8 * part + i;
            tr0 = at + tr * ROWB + (((COLS == 32 ? blk : 0) ^ swizzle(tr)) << 4) + 8 * (in & 1);
        } else {  // lanes 4 i .. 4 i + 3 of 16 point at row i of the group's four
            const int quad = in & 3, tr = (COLS == 32 ? 4 : 8) * part + (in >> 2);
            tr0 = at + tr * ROWB + (((COLS == 32 ? 2 * blk : 0) + (quad >> 1)) ^ swizzle(tr)) * 16 + 8 * (quad & 1);
        }
        asm volatile("" : "+v"(src0), "+v"(row0), "+v"(tr0));
        if constexpr (KEPT) {
            static_for<KR>([&](auto n) __attribute__((always_inline)) {
                constexpr int k = decltype(n)::value;
                row_at[k] = (row0 ^ flip(M::PARTS * k, 0)) + plus(M::PARTS * k, 0);
                asm volatile("" : "+v"(row_at[k]));
            });
            static_for<M::NT>([&](auto n) __attribute__((always_inline)) {
                constexpr int dt = decltype(n)::value, chunk = (CODES ? 2 : 4) * dt;
                tr_at[dt][0] = (tr0 ^ flip(chunk, 0)) + plus(chunk, 0);
                asm volatile("" : "+v"(tr_at[dt][0]));
                if constexpr (!CODES) {
                    tr_at[dt][TR - 1] = (tr0 ^ flip(chunk, 8)) + plus(chunk, 8);
                    asm volatile("" : "+v"(tr_at[dt][TR - 1]));
                }
            });
        }
    }
    // All instructions that bring a tile, 16 rows from each resource
    __device__ __forceinline__ void request(const BufferWords (&rsrc)[2], uint32_t offset) const {
        static_for<NI>([&](auto n) __attribute__((always_inline)) {
            constexpr int i = decltype(n)::value, r = i * RPI;
            once_to_lds_16B(rsrc[i / (NI / 2)], base + offset + i * 1024, (int)((src0 ^ (uint32_t)(swizzle(r) << 4)) + (r % 16) * ROWB));
        });
    }
    // those of 16 rows; `src`: src0, with the swizzle of the second 16 rows where it is these
    __device__ __forceinline__ void request_half(const BufferWords& rsrc, uint32_t offset, uint32_t src) const {
        static_for<NI / 2>([&](auto n) __attribute__((always_inline)) {
            constexpr int i = decltype(n)::value, r = i * RPI;
            global_to_lds_16B(rsrc, base + offset + i * 1024, (int)((src ^ (uint32_t)(swizzle(r) << 4)) + r * ROWB));
        });
    }
    // the lane's 16 bytes k of its row in score tile kt
    template <int K, int KT>
    __device__ __forceinline__ i32x4 row_read(uint32_t offset) const {
        if constexpr (KEPT) return lds_load_16B(row_at[K] + offset);
        else return lds_load_16B((row0 ^ flip(M::PARTS * K, 4 * KT)) + (offset + plus(M::PARTS * K, 4 * KT)));
    }
    // the A operand of V^T: accumulator dt, keys of slab `slab`; codes: their eight bytes
    template <int DT, int SLAB>
    __device__ __forceinline__ i32x4 columns(uint32_t offset) const {
        if constexpr (KEPT && CODES) {
            const i32x2 c = lds_read_tr8(tr_at[DT][0] + (offset + SLAB * 16 * ROWB));
            return i32x4{c[0], c[1], 0, 0};
        } else if constexpr (KEPT) {
            const i32x2 lo = lds_read_tr16(tr_at[DT][0] + (offset + SLAB * 16 * ROWB)), hi = lds_read_tr16(tr_at[DT][TR - 1] + (offset + SLAB * 16 * ROWB));
            return i32x4{lo[0], lo[1], hi[0], hi[1]};
        } else if constexpr (CODES) {
            constexpr int chunk = COLS == 32 ? 2 * DT : DT;
            const i32x2 c = lds_read_tr8((tr0 ^ flip(chunk, 16 * SLAB)) + (offset + plus(chunk, 16 * SLAB)));
            return i32x4{c[0], c[1], 0, 0};
        } else {
            constexpr int chunk = COLS == 32 ? 4 * DT : 2 * DT, more = 16 * SLAB, upper = more + (COLS == 32 ? 8 : 4);
            const i32x2 lo = lds_read_tr16((tr0 ^ flip(chunk, more)) + (offset + plus(chunk, more)));
            const i32x2 hi = lds_read_tr16((tr0 ^ flip(chunk, upper)) + (offset + plus(chunk, upper)));
            return i32x4{lo[0], lo[1], hi[0], hi[1]};
        }
    }

    // An infinity or a NaN in V of a new token is no business of the rows that do not see it, and a product with P = 0 would
    // make it theirs.  So where a tile with new tokens has one (not_finite) it is a zero for the product (clear_not_finite), one of an
    // old token in the tile too, and the rows that see it get it at the end.
    static constexpr int EXPONENT = CODES ? 0x7F7F7F7F : std::is_same_v<Tag, bf16_tag> ? 0x7F807F80 : 0x7C007C00;
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
};

// Asynchronous copy of 4 bytes per lane from an address per lane to lds_base + 4 lane
static __device__ __forceinline__ void global_to_lds_4B(const float* p, uint32_t lds_base) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
                 :
                 : "s"(__builtin_amdgcn_readfirstlane(lds_base)), "v"(p)
                 : "memory", "m0");
}

// The waves of a workgroup meet; what they have asked of the LDS is done
static __device__ __forceinline__ void barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <int N>
static __device__ __forceinline__ void wait_vmcnt() {
    static_assert(N < 64, "what the counter holds");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

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

// FORM: the waves of a workgroup either share its rows and divide the keys (kDivideKeys), or they have RT tiles of rows each and
// share the keys, which they stage together (kShareKeys).
enum Form { kDivideKeys, kShareKeys };
template <typename Tag, int D, bool CODES, int COLS, int RT, int NW, int STG, int FORM>
struct CachedShape {
    using Tile = CacheTile<Tag, D, CODES, COLS>;
    static constexpr bool SHARED = FORM == kShareKeys;
    static constexpr int ROWS = COLS * RT * (SHARED ? NW : 1);  // of a workgroup
    static constexpr int STEP = 32 * NW;                        // keys of a step
    static constexpr int SCALE_B = CODES ? 256 : 0;             // of a tile: 32 scales of K, 32 of V
    static constexpr int STAGE_B = 2 * Tile::TILE_B + SCALE_B, STAGES_B = STG * STAGE_B * (SHARED ? 1 : NW);
    static constexpr int MERGE_COLS = (COLS == 16 || RT == 2) && D > 64 ? 128 : 64, MERGE_STRIDE = MERGE_COLS + 4;
    static constexpr int MERGE_B = NW * COLS * MERGE_STRIDE * 4, STATE_B = NW * COLS * RT * 2 * 4 + NW * 4;
    static constexpr int LDS = (STAGES_B > MERGE_B ? STAGES_B : MERGE_B) + STATE_B;
    // workgroups (of four waves) to a CU, by registers
    static constexpr int WAVES = SHARED ? (D == 64 ? 3 : D == 128 ? 2 : 1) : COLS == 16 || (RT == 1 && D < 256) ? 2 : 1;
    static constexpr int BY_LDS = 163840 / LDS, PER_CU = BY_LDS < WAVES ? BY_LDS : WAVES;
};

template <typename Tag, int D, bool CODES, int COLS, int RT, int NW, int STG, int FORM>
__global__ void __launch_bounds__(NW * 64, (CachedShape<Tag, D, CODES, COLS, RT, NW, STG, FORM>::WAVES))
fa_fwd_cache_kernel(CachedArgs a) {
    using Shape = CachedShape<Tag, D, CODES, COLS, RT, NW, STG, FORM>;
    constexpr bool SHARED = Shape::SHARED;
    constexpr int KW = SHARED ? 1 : NW, RW = SHARED ? NW : 1;  // waves that divide keys, that have rows of their own
    using Tile = typename Shape::Tile;
    using M = typename Tile::M;
    using PM = typename Tile::PM;
    using PE = Elem<typename Tile::PE>;
    using E = Elem<Tag>;
    constexpr int NS = M::NS, NT = M::NT, NI = Tile::NI, X = CODES ? 1 : 0, ACC = sizeof(typename M::Acc) / 4;
    constexpr bool ACCUMULATION = Shape::WAVES == 1;  // more than 256 registers: accumulators in the half for matrix results
    // Few rows leave the matrix pipes idle: P goes in as its rounded value and what that leaves out, so that its rounding does not
    // add to the output's (error against 64 bits, bf16, of the output's rounding alone: 1.4 times / 1.0 times; the time is the same)
    // With codes always: one bf16 number would be eight times as coarse as the fp16 number that a factor common to all keys allows, and
    // no common factor is right where a key of a large scale weighs little, or nothing (8 trees of 32 tokens, 8 heads: 53.0 us, with
    // fp16 and such a factor 51.3; 64 x 500 to 4096 keys, T = 1, d = 64: 26.1 and 27.8).
    constexpr bool TWO_PARTS = COLS == 16 || CODES;
    constexpr int QS = D / (8 * M::PARTS);  // steps of the scores' contraction
    extern __shared__ __align__(256) char lds[];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int col = lane % COLS, part = lane / COLS, kw = SHARED ? 0 : wave, rw = SHARED ? wave : 0;

    // which rows and keys: a team's workgroups side by side on one XCD
    int team = xcd_run(blockIdx.x, gridDim.x);
    const int wg = team, rg = __builtin_amdgcn_readfirstlane(team % a.row_groups);
    team = __builtin_amdgcn_readfirstlane(team / a.row_groups);
    const int H_kv = a.c.H_kv, group = a.H / H_kv;
    int b, kvh, step = 0, left = 0x7fffffff;  // the first segment, and how many steps the team has
    Extent ext;
    uint32_t pos = 0;  // of the team's first step among all
    Shares shares(1, 1);
    int own_parts = 0;  // how many teams have the sequence and head, where each team has one
    if (a.teams == 0) {
        b = __builtin_amdgcn_readfirstlane(team / H_kv);
        kvh = __builtin_amdgcn_readfirstlane(team - b * H_kv);
        ext = Extent(a, b);
        ext.make_uniform();
    } else {
        // Lane i looks at sequences i, i + 64, ...: first for the sum of their steps, then for the one with the team's first
        // step (again, if there are more than 64)
        uint32_t total = 0, before = 0, n = 0, upto = 0;
        Extent mine;
        auto look_at = [&](int b0) __attribute__((always_inline)) {
            n = 0;
            if (b0 + lane < a.B) {
                mine = Extent(a, b0 + lane);
                n = (uint32_t)mine.steps<Shape::STEP>();
            }
            upto = sum_upto(n, lane);
        };
        for (int b0 = 0; b0 < a.B; b0 += 64) {
            look_at(b0);
            total += __builtin_amdgcn_readlane(upto, 63);
        }
        shares = Shares(total * H_kv, a.teams);
        // Where a share of at most one step more lets each team stay with one sequence and head, it does: no second start
        uint32_t parts = 0, parts_upto = 0;
        if (a.B <= 64) {
            parts = (n + shares.each) / (shares.each + 1);
            parts_upto = sum_upto(parts, lane);
        }
        const uint32_t used = __builtin_amdgcn_readlane(parts_upto, 63) * H_kv;
        int i;
        if (a.B <= 64 && used <= (uint32_t)a.teams) {
            if ((uint32_t)team >= used) return;
            i = __builtin_ctzll(__builtin_amdgcn_ballot_w64((uint32_t)team < parts_upto * H_kv));
            b = i;
            const uint32_t k = __builtin_amdgcn_readlane(parts, i), rel = team - (__builtin_amdgcn_readlane(parts_upto, i) - k) * H_kv;
            kvh = __builtin_amdgcn_readfirstlane((int)(rel / k));
            const uint32_t part = __builtin_amdgcn_readfirstlane((int)(rel - rel / k * k));
            const Shares inside(__builtin_amdgcn_readlane(n, i), k);
            step = __builtin_amdgcn_readfirstlane((int)inside.first(part));
            left = __builtin_amdgcn_readfirstlane((int)inside.first(part + 1)) - step;
            own_parts = (int)k;
        } else {
            pos = __builtin_amdgcn_readfirstlane(shares.first(team));
            left = __builtin_amdgcn_readfirstlane((int)(shares.first(team + 1) - pos));
            if (left == 0) return;
            int b0 = 0;
            if (a.B > 64)
                for (;; b0 += 64) {
                    look_at(b0);
                    const uint32_t here = __builtin_amdgcn_readlane(upto, 63) * H_kv;
                    if (pos < before + here) break;
                    before += here;
                }
            i = __builtin_ctzll(__builtin_amdgcn_ballot_w64(pos < before + upto * H_kv));  // (one there is)
            b = b0 + i;
            const uint32_t steps = __builtin_amdgcn_readlane(n, i);
            const uint32_t rel = pos - before - (__builtin_amdgcn_readlane(upto, i) - steps) * H_kv;
            kvh = __builtin_amdgcn_readfirstlane((int)(rel / steps));
            step = __builtin_amdgcn_readfirstlane((int)(rel - rel / steps * steps));
        }
        ext.len = __builtin_amdgcn_readlane(mine.len, i);
        ext.count = __builtin_amdgcn_readlane(mine.count, i);
        ext.keys = __builtin_amdgcn_readlane(mine.keys, i);
    }

    const Tile tile(lds_address(lds) + kw * (STG * Shape::STAGE_B), lane);
    const float sc = a.scale * kLog2e;
    for (int segment = 0;; segment = 1) {
    const int n_steps = ext.steps<Shape::STEP>();
    const int now = min(n_steps - step, left);
    const bool whole = now == n_steps;
    const int key0 = step * Shape::STEP, key1 = step + now == n_steps ? ext.keys : key0 + now * Shape::STEP;
    // rows of the tokens that are there, packed; a team's last workgroups may have none
    const int n_rows = group * ext.count, per = max(ext.count, 1);
    const int n_tiles = rg * Shape::ROWS >= n_rows ? 0 : (int)(((unsigned)max(key1 - key0, 0) + 31) / 32), mine = n_tiles > kw ? (n_tiles - kw + KW - 1) / KW : 0;

    // rows (of all pages' rows, heads included) of the wave's tiles: lane i has tile i of 64, two times 16 places; -1: no page
    long row_lo = -1, row_hi = -1;
    auto look_up = [&](int first) __attribute__((always_inline)) {
        const int key = key0 + 32 * (kw + KW * (first + lane));
        // (both lookups at once, whether or not the second page is the first)
        const int page_size = a.c.page_size, entry = (unsigned)max(key, 0) / (unsigned)page_size, slot = key - entry * page_size;
        const bool next = slot + 16 >= page_size;
        const int entry_hi = entry + next, slot_hi = slot + 16 - (next ? page_size : 0);
        const int* const table = a.c.block_table + (long)b * a.c.max_pages;
        const bool in_lo = key >= key0 && key < key1, in_hi = key >= key0 && key < key1 - 16;
        const int page = in_lo ? table[entry] : -1, page_hi = in_hi ? table[entry_hi] : -1;
        row_lo = page < 0 || page >= a.c.n_pages ? -1 : ((long)page * H_kv + kvh) * page_size + slot;
        row_hi = page_hi < 0 || page_hi >= a.c.n_pages ? -1 : ((long)page_hi * H_kv + kvh) * page_size + slot_hi;
    };
    // requests K of the wave's tile i into stage st, and its V when that stage's V has been read
    UniformRow rows[STG][2];
    auto resources = [&](const void* pages, int i, const UniformRow (&row)[2], BufferWords (&rsrc)[2]) __attribute__((always_inline)) {
        const int there = key1 - (key0 + 32 * (kw + KW * i));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            int n = max(there - 16 * h, 0);
            asm volatile("" : "+s"(n));  // (with the minimum it would be one vector instruction)
            n = min(n, 16) & ~row[h].none();
            rsrc[h] = make_buffer_words(static_cast<const char*>(pages) + (row[h].index() * Tile::ROWB), n * Tile::ROWB);
        }
    };
    auto request_k = [&](int i, auto stage) __attribute__((always_inline)) {
        constexpr int st = decltype(stage)::value;
        if ((i & 63) == 0 && i > 0) look_up(i);
        rows[st][0] = UniformRow(row_lo, i & 63);
        rows[st][1] = UniformRow(row_hi, i & 63);
        BufferWords rsrc[2];
        resources(a.c.k, i, rows[st], rsrc);
        tile.request(rsrc, st * Shape::STAGE_B);
        if constexpr (CODES) {  // lanes 0..31 the scales of K, 32..63 of V; of a place that is none: any
            long row = rows[st][0].index(), upper = rows[st][1].index();
            asm volatile("" : "+v"(row), "+v"(upper));  // (a choice between vector registers, not between places in memory)
            row = lane & 16 ? upper : row;
            const int there = key1 - (key0 + 32 * (kw + KW * i));
            const long at = (lane & 31) >= there ? 0 : row + (lane & 15);
            global_to_lds_4B((lane & 32 ? a.c.v_scales : a.c.k_scales) + at, tile.base + st * Shape::STAGE_B + 2 * Tile::TILE_B);
        }
    };
    auto request_v = [&](int i, auto stage) __attribute__((always_inline)) {
        constexpr int st = decltype(stage)::value;
        BufferWords rsrc[2];
        resources(a.c.v, i, rows[st], rsrc);
        tile.request(rsrc, st * Shape::STAGE_B + Tile::TILE_B);
    };
    // kShareKeys: wave 0 brings the first 16 rows of K of tile i, 1 the others, 2 and 3 those of V, and wave 0 the scales; `pending` takes
    // which halves of it are on no page
    int pending = 0;
    const uint32_t src_shared = tile.src0 ^ (uint32_t)((wave & 1) * (Tile::swizzle(16) << 4));
    auto request_shared = [&](int i, uint32_t offset, int ahead) __attribute__((always_inline)) {
        if ((i & 63) == 0 && i > 0) look_up(i);
        const UniformRow lo(row_lo, i & 63), hi(row_hi, i & 63), row = wave & 1 ? hi : lo;
        pending |= ((lo.none() & 1) | (hi.none() & 2)) << (2 * ahead);
        const int there = key1 - (key0 + 32 * i);
        int n = max(there - 16 * (wave & 1), 0);
        asm volatile("" : "+s"(n));
        n = min(n, 16) & ~row.none();
        const BufferWords rsrc = make_buffer_words(static_cast<const char*>(wave & 2 ? a.c.v : a.c.k) + row.index() * Tile::ROWB, n * Tile::ROWB);
        tile.request_half(rsrc, offset + (wave >> 1) * Tile::TILE_B + (wave & 1) * (Tile::TILE_B / 2), src_shared);
        if constexpr (CODES)
            if (wave == 0) {
                long at_row = lo.index(), upper = hi.index();
                asm volatile("" : "+v"(at_row), "+v"(upper));
                at_row = lane & 16 ? upper : at_row;
                const long at = (lane & 31) >= there ? 0 : at_row + (lane & 15);
                global_to_lds_4B((lane & 32 ? a.c.v_scales : a.c.k_scales) + at, tile.base + offset + 2 * Tile::TILE_B);
            }
    };
    int t[RT];  // the token of the lane's rows (clamped: rows past the end compute a copy of the last, never stored)
    i32x4 qreg[RT][QS];
#pragma unroll
    for (int x = 0; x < RT; ++x) {
        const int row = min(((rg * RW + rw) * RT + x) * COLS + col, max(n_rows - 1, 0)), g = row / per;
        t[x] = row - g * per;
        const uint16_t* q = static_cast<const uint16_t*>(a.q.p) + (b * a.q.batch + (kvh * group + g) * a.q.head + t[x] * a.q.token);
#pragma unroll
        for (int u = 0; u < QS; ++u) {
            const int at = CODES ? 16 * M::PARTS * (u / 2) + 16 * part + 8 * (u % 2) : 8 * M::PARTS * u + 8 * part;
            qreg[x][u] = *reinterpret_cast<const i32x4*>(q + at);
        }
    }
    // Q is on its way while the table is read, and there before the first request: the compiler, which does not see the requests,
    // would wait for Q inside the loop with a count that waits for them all
    look_up(0);
#pragma unroll
    for (int x = 0; x < RT; ++x)
#pragma unroll
        for (int u = 0; u < QS; ++u) asm volatile("" : "+v"(qreg[x][u]));
    if (mine > 0) {
        if constexpr (SHARED) {
#pragma unroll
            for (int i = 0; i < STG - 1; ++i) request_shared(i, i * Shape::STAGE_B, i);
        } else {
            static_for<STG>([&](auto st) {
                request_k(st, st);
                request_v(st, st);
            });
        }
    }

    typename M::Acc acc[RT][NT];
    float m_run[RT], l_run[RT];
#pragma unroll
    for (int x = 0; x < RT; ++x) {
        m_run[x] = -INFINITY;
        l_run[x] = 0.f;
#pragma unroll
        for (int dt = 0; dt < NT; ++dt) acc[x][dt] = typename M::Acc{};
    }

    // the row's view of the 32 places from `key` on
    auto visible = [&](int key, int row_t, uint32_t live) __attribute__((always_inline)) {
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
        return vis & live;
    };

    int odd = 0;  // whether V of a tile with new tokens held a value that is not finite
    // A tile: scores, softmax, products.  `at`: where it is (K, V, scales from OFFSET on); `bad`: the halves that are on no page
    auto work = [&](const Tile& at, auto off, int key, int bad, auto&& after_scores, auto&& before_products, auto&& after_products) __attribute__((always_inline)) {
            constexpr int kK = decltype(off)::value, kV = kK + Tile::TILE_B, kScales = kK + 2 * Tile::TILE_B;
            const bool special = key + 32 > min(ext.len, key1) || bad != 0;
            float s[RT][NS];
            {
                typename M::Acc y[RT][M::TILES];
#pragma unroll
                for (int x = 0; x < RT; ++x)
#pragma unroll
                    for (int kt = 0; kt < M::TILES; ++kt) y[x][kt] = typename M::Acc{};
                constexpr int READS = Tile::KR * M::TILES, AT_ONCE = READS < kReadsAhead ? READS : kReadsAhead;
                static_for<READS / AT_ONCE>([&](auto n) __attribute__((always_inline)) {
                    constexpr int first = decltype(n)::value * AT_ONCE;
                    i32x4 read[AT_ONCE];
                    static_for<AT_ONCE>([&](auto m) __attribute__((always_inline)) {
                        constexpr int j = first + decltype(m)::value;
                        read[j - first] = at.template row_read<j / M::TILES, j % M::TILES>(kK);
                    });
                    __builtin_amdgcn_sched_barrier(0);
                    static_for<AT_ONCE>([&](auto m) __attribute__((always_inline)) {
                        constexpr int j = first + decltype(m)::value, k = j / M::TILES, kt = j % M::TILES;
                        const i32x4 w = read[j - first];
                        if constexpr (CODES) {
                            const i32x4 lo = from_codes<Tag>(w[0], w[1]), hi = from_codes<Tag>(w[2], w[3]);
#pragma unroll
                            for (int x = 0; x < RT; ++x) y[x][kt] = M::mma(lo, qreg[x][2 * k], y[x][kt]);
#pragma unroll
                            for (int x = 0; x < RT; ++x) y[x][kt] = M::mma(hi, qreg[x][2 * k + 1], y[x][kt]);
                        } else {
#pragma unroll
                            for (int x = 0; x < RT; ++x) y[x][kt] = M::mma(w, qreg[x][k], y[x][kt]);
                        }
                    });
                });
#pragma unroll
                for (int x = 0; x < RT; ++x)
#pragma unroll
                    for (int r = 0; r < NS; ++r) s[x][r] = y[x][r / ACC][r % ACC];
            }
            float vscale[NS];
            if constexpr (CODES) {
#pragma unroll
                for (int g = 0; g < NS / 4; ++g) {
                    const uint32_t scales = at.base + kScales + 4 * (M::bit(4 * g) + (part << M::SHIFT));
                    const f32x4 ks = lds_load_4f(scales), vs = lds_load_4f(scales + 128);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        vscale[4 * g + r] = vs[r];
#pragma unroll
                        for (int x = 0; x < RT; ++x) s[x][4 * g + r] *= ks[r];
                    }
                }
            }
            after_scores();

            uint32_t seen[RT];
            if (special) {
                const int there = key1 - key;
                uint32_t live = there >= 32 ? ~0u : (1u << there) - 1;  // (a tile has a key at least)
                if (bad & 1) live &= 0xFFFF0000u;
                if (bad & 2) live &= 0x0000FFFFu;
#pragma unroll
                for (int x = 0; x < RT; ++x) {
                    seen[x] = visible(key, t[x], live) >> (part << M::SHIFT);
#pragma unroll
                    for (int r = 0; r < NS; ++r) s[x][r] = seen[x] >> M::bit(r) & 1 ? s[x][r] : -INFINITY;
                }
            }
            auto see_to_odd_ones = [&]() __attribute__((always_inline)) {
                if (special && key + 32 > ext.len)
                    if (__builtin_expect(at.not_finite(kV, lane), 0)) {
                        odd = 1;
                        if constexpr (SHARED) barrier();  // all waves have seen it; then each clears all
                        at.clear_not_finite(kV, lane);
                    }
            };
            constexpr int COLUMN_READS = M::SLABS * NT, COLUMNS_AT_ONCE = COLUMN_READS < kReadsAhead ? COLUMN_READS : kReadsAhead;
            i32x4 columns[COLUMNS_AT_ONCE];
            auto read_columns = [&](auto n) __attribute__((always_inline)) {
                constexpr int first = decltype(n)::value * COLUMNS_AT_ONCE;
                static_for<COLUMNS_AT_ONCE>([&](auto m) __attribute__((always_inline)) {
                    constexpr int j = first + decltype(m)::value;
                    columns[j - first] = at.template columns<j % NT, j / NT>(kV);
                });
                __builtin_amdgcn_sched_barrier(0);
            };
            if constexpr (SHARED) {  // (V is there: its first operands arrive beside the softmax)
                before_products();
                see_to_odd_ones();
                read_columns(std::integral_constant<int, 0>{});
            }
            i32x4 pb[RT][M::SLABS], rest[RT][M::SLABS];  // what V is multiplied by
#pragma unroll
            for (int x = 0; x < RT; ++x) {
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int r = 0; r < NS; ++r) mx[r & 3] = fmaxf(mx[r & 3], s[x][r]);
                const float m_new = M::max_parts(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])));
                const bool raise = (m_new - m_run[x]) * sc > kLazy;
                if (__builtin_amdgcn_ballot_w64(raise) != 0) {
                    const float corr = raise ? fast_exp2((m_run[x] - m_new) * sc) : 1.0f;
                    m_run[x] = raise ? m_new : m_run[x];
                    l_run[x] *= corr;
#pragma unroll
                    for (int dt = 0; dt < NT; ++dt) {
                        if constexpr (ACCUMULATION) asm volatile("" : "+a"(acc[x][dt]));  // (copied out here, not in every tile)
                        acc[x][dt] *= corr;
                        if constexpr (ACCUMULATION) asm volatile("" : "+a"(acc[x][dt]));
                    }
                }
                const float mb = m_run[x] == -INFINITY ? 0.f : m_run[x] * sc;  // a row that has seen nothing yet: P = 0
                float ps[4];
#pragma unroll
                for (int r = 0; r < NS; ++r) {
                    const float p = fast_exp2(__builtin_fmaf(s[x][r], sc, -mb));
                    ps[r & 3] = r < 4 ? p : ps[r & 3] + p;
                    s[x][r] = p;
                    if constexpr (CODES) s[x][r] = p * vscale[r];
                }
                if constexpr (CODES)
                    if (special)  // (of a place that a row does not see P is 0, but its scale need not be finite)
#pragma unroll
                        for (int r = 0; r < NS; ++r) s[x][r] = seen[x] >> M::bit(r) & 1 ? s[x][r] : 0.f;
                l_run[x] += (ps[0] + ps[1]) + (ps[2] + ps[3]);
#pragma unroll
                for (int r = 0; r < NS; r += 2) {
                    const int w = PE::pack2(s[x][r], s[x][r + 1]);
                    pb[x][r >> 3][(r >> 1) & 3] = w;
                    if constexpr (TWO_PARTS)
                        rest[x][r >> 3][(r >> 1) & 3] =
                            PE::pack2(s[x][r] - PE::to_float((uint16_t)w), s[x][r + 1] - PE::to_float((uint16_t)((uint32_t)w >> 16)));
                }
            }
            if constexpr (!SHARED) {
                before_products();
                see_to_odd_ones();
                read_columns(std::integral_constant<int, 0>{});
            }
            // O^T += V^T P^T
            static_for<COLUMN_READS / COLUMNS_AT_ONCE>([&](auto n) __attribute__((always_inline)) {
                constexpr int first = decltype(n)::value * COLUMNS_AT_ONCE;
                if constexpr (first > 0) read_columns(n);
                static_for<COLUMNS_AT_ONCE>([&](auto m) __attribute__((always_inline)) {
                    constexpr int j = first + decltype(m)::value, slab = j / NT, dt = j % NT;
                    i32x4 w = columns[j - first];
                    if constexpr (CODES) w = from_codes<bf16_tag>(w[0], w[1]);
#pragma unroll
                    for (int x = 0; x < RT; ++x) {
                        acc[x][dt] = PM::mma(w, pb[x][slab], acc[x][dt]);
                        if constexpr (TWO_PARTS) acc[x][dt] = PM::mma(w, rest[x][slab], acc[x][dt]);
                    }
                });
            });
            after_products();
    };
    if constexpr (SHARED) {
        // Tile i + STG - 1 goes where tile i - 1 was, which all waves have left when they meet in tile i
        for (int i0 = 0; i0 < mine; i0 += STG)
            static_for<STG>([&](auto stage) __attribute__((always_inline)) {
                constexpr int st = decltype(stage)::value;
                const int i = i0 + st;
                if (i >= mine) return;
                wait_vmcnt<(STG - 2) * (NI / 2)>();  // what this wave brings of tile i has landed
                barrier();
                request_shared(i + STG - 1, (st + STG - 1) % STG * Shape::STAGE_B, STG - 1);
                work(tile, std::integral_constant<int, st * Shape::STAGE_B>{}, key0 + 32 * i, pending & 3, [] {}, [] {}, [] {});
                pending >>= 2;
            });
    } else {
        for (int i0 = 0; i0 < mine; i0 += STG)
            static_for<STG>([&](auto stage) __attribute__((always_inline)) {
                constexpr int st = decltype(stage)::value;
                const int i = i0 + st;
                if (i >= mine) return;
                const int bad = (rows[st][0].none() & 1) | (rows[st][1].none() & 2);
                wait_vmcnt<NI * STG + (NI + X) * (STG - 1)>();  // K has landed
                work(tile, std::integral_constant<int, st * Shape::STAGE_B>{}, key0 + 32 * (kw + KW * i), bad,
                     [&] {
                         asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // K and the scales have been read: the next ones may come
                         request_k(i + STG, stage);
                     },
                     [&] { wait_vmcnt<(NI + X) * STG + NI * (STG - 1)>(); },  // V has landed
                     [&] {
                         asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                         request_v(i + STG, stage);
                     });
            });
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the last requests: the LDS is about to be reused

    // The states of waves that divided the keys meet: with M the largest reference and f = 2^(m - M), sum f acc, M and sum f l
    float* const state = reinterpret_cast<float*>(lds + Shape::LDS - Shape::STATE_B);  // [RT][NW][COLS][m, l]
    int* const odd_waves = reinterpret_cast<int*>(state + NW * COLS * RT * 2);
    if (lane == 0) odd_waves[wave] = odd;
    float* const merge = reinterpret_cast<float*>(lds);                                // [NW][COLS][MERGE_STRIDE]
#pragma unroll
    for (int x = 0; x < RT; ++x) {
        const float l = M::sum_parts(l_run[x]);
        if (part == 0) {
            float* at = state + ((x * NW + wave) * COLS + col) * 2;
            at[0] = m_run[x] * sc;
            at[1] = l;
        }
    }
    constexpr int MC = Shape::MERGE_COLS, MS = Shape::MERGE_STRIDE;
#pragma unroll
    for (int x = 0; x < RT; ++x)
#pragma unroll
        for (int c0 = 0; c0 < D; c0 += MC) {
            __syncthreads();
#pragma unroll
            for (int dt = c0 / M::WIDTH; dt < (c0 + MC) / M::WIDTH; ++dt)
#pragma unroll
                for (int g = 0; g < ACC / 4; ++g) {
                    const typename M::Acc& y = acc[x][dt];
                    const f32x4 w = {y[4 * g], y[4 * g + 1], y[4 * g + 2], y[4 * g + 3]};
                    *reinterpret_cast<f32x4*>(merge + (wave * COLS + col) * MS + dt * M::WIDTH - c0 + 4 * M::PARTS * g + 4 * part) = w;
                }
            __syncthreads();
            for (int c = SHARED ? lane : tid; c < COLS * MC / 8; c += KW * 64) {
                const int r = c / (MC / 8), cc = (c % (MC / 8)) * 8, row = ((rg * RW + rw) * RT + x) * COLS + r;
                if (row >= n_rows) continue;
                const int g = row / per, tok = row - g * per;
                float m_all = -INFINITY, l_all = 0.f, f[KW];
#pragma unroll
                for (int w = 0; w < KW; ++w) m_all = fmaxf(m_all, state[((x * NW + rw + w) * COLS + r) * 2]);
                const float m_ref = m_all == -INFINITY ? 0.f : m_all;
#pragma unroll
                for (int w = 0; w < KW; ++w) {
                    const float* at = state + ((x * NW + rw + w) * COLS + r) * 2;
                    f[w] = fast_exp2(at[0] - m_ref);
                    l_all += f[w] * at[1];
                }
                float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < KW; ++w)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const f32x4 z = *reinterpret_cast<const f32x4*>(merge + ((rw + w) * COLS + r) * MS + cc + 4 * h);
#pragma unroll
                        for (int e = 0; e < 4; ++e) y[4 * h + e] = __builtin_fmaf(f[w], z[e], y[4 * h + e]);
                    }
                int any_odd = 0;
#pragma unroll
                for (int w = 0; w < KW; ++w) any_odd |= odd_waves[rw + w];
                if (__builtin_expect(any_odd != 0, 0))
                    for (int place = max(key0, ext.len & ~31); place < key1; ++place) {  // from the first tile with a new token on
                        const int u = place - ext.len, entry = place / a.c.page_size, words = (a.T + 31) >> 5;
                        const bool sees = u < 0 ? true : a.tree ? a.tree[((long)(a.tree_batches == 1 ? 0 : b) * a.T + tok) * words + (u >> 5)] >> (u & 31) & 1 : u <= tok;
                        const int page = a.c.block_table[(long)b * a.c.max_pages + entry];
                        if (!sees || page < 0 || page >= a.c.n_pages) continue;
                        const long at = (((long)page * H_kv + kvh) * a.c.page_size + (place - entry * a.c.page_size)) * D + c0 + cc;
                        for (int e = 0; e < 8; ++e) {
                            float v;
                            if constexpr (CODES) v = __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t*>(a.c.v)[at + e], 0);
                            else v = E::to_float(static_cast<const uint16_t*>(a.c.v)[at + e]);
                            if (!(fabsf(v) < INFINITY))
#pragma unroll
                                for (int k = 0; k < 8; ++k) y[k] += k == e ? v : 0.f;
                        }
                    }
                if (whole) {
                    const int head = kvh * group + g;
                    const float inv = l_all == 0.f ? 0.f : 1.0f / l_all;  // a row that sees nothing: 0
                    uint16_t* o = static_cast<uint16_t*>(const_cast<void*>(a.o.p)) + (b * a.o.batch + head * a.o.head + tok * a.o.token);
                    i32x4 w;
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = E::pack2(y[2 * e] * inv, y[2 * e + 1] * inv);
                    *reinterpret_cast<i32x4*>(o + c0 + cc) = w;
                    if (c0 + cc == 0) a.lse[((long)b * a.H + head) * a.T + tok] = (m_all + log2f(l_all)) * kLn2;
                } else {
                    const long at = ((long)wg * 2 + segment) * Shape::ROWS + (rw * RT + x) * COLS + r;
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
    if (a.teams == 0) break;
    if (step == 0 && rg == 0 && tid == 0)
        a.segments[b * H_kv + kvh] = {2 * team + segment, own_parts ? own_parts : whole ? 1 : (int)shares.owner(pos + n_steps - 1) - team + 1};
    left -= now;
    if (left == 0) break;
    pos += now;
    step = 0;
    if (++kvh == H_kv) {
        kvh = 0;
        ++b;
        ext = Extent(a, b);
        ext.make_uniform();
    }
    __syncthreads();  // the merge area is staged into again
    }
}

// Joins the segments of rows whose sequence several teams have.  A workgroup stands on 64 columns (8 to a thread) of 32 / ways
// rows; `ways` (a power of two, at most 32) threads take a row's segments in turn, each with a reference of its own, and meet in
// the LDS.
constexpr int kJoinCols = 64;
template <typename Tag, int D, int ROWS>
__global__ void __launch_bounds__(256) fa_join_kernel(CachedArgs a, int ways) {
    using E = Elem<Tag>;
    constexpr int TPR = kJoinCols / 8, GROUPS = 256 / TPR;
    __shared__ float meet[GROUPS][kJoinCols + 4];  // and the reference and the sum
    const int group = threadIdx.x / TPR, way = group & (ways - 1), c0 = (threadIdx.x % TPR) * 8, c = blockIdx.y * kJoinCols + c0;
    const unsigned n_rows = (unsigned)a.B * a.H * a.T, row = blockIdx.x * (GROUPS / ways) + group / ways;
    const unsigned bh = min(row, n_rows - 1) / a.T;
    const int tok = row - bh * a.T, b = bh / (unsigned)a.H, head = bh - b * a.H;
    const int heads = a.H / a.c.H_kv, kvh = head / heads, count = a.counts ? min(a.counts[b], a.T) : a.T;
    const int in_group = (head - kvh * heads) * count + tok, rg = in_group / ROWS;
    const CachedArgs::Segments of = a.segments[b * a.c.H_kv + kvh];
    const bool there = row < n_rows && of.count > 1 && tok < count;
    float m = -INFINITY, l = 0.f;
    float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (there)
#pragma unroll 4
        for (int s = way; s < of.count; s += ways) {
            const long segment = s == 0 ? of.first : (of.first & ~1) + 2 * s;
            const long at = (((segment >> 1) * a.row_groups + rg) * 2 + (segment & 1)) * ROWS + (in_group - rg * ROWS);
            const float sm = a.state[2 * at], sl = a.state[2 * at + 1];
            const f32x4 lo = *reinterpret_cast<const f32x4*>(a.part + at * D + c), hi = *reinterpret_cast<const f32x4*>(a.part + at * D + c + 4);
            const float top = fmaxf(m, sm), ref = top == -INFINITY ? 0.f : top, f = fast_exp2(m - ref), g = fast_exp2(sm - ref);
            m = top;
            l = l * f + sl * g;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                y[e] = y[e] * f + lo[e] * g;
                y[4 + e] = y[4 + e] * f + hi[e] * g;
            }
        }
    if (ways > 1) {
#pragma unroll
        for (int e = 0; e < 8; ++e) meet[group][c0 + e] = y[e];
        if (c0 == 0) {
            meet[group][kJoinCols] = m;
            meet[group][kJoinCols + 1] = l;
        }
        __syncthreads();
        if (way == 0) {
            const int used = min(ways, of.count);
            float top = m;
            for (int w = 1; w < used; ++w) top = fmaxf(top, meet[group + w][kJoinCols]);
            const float ref = top == -INFINITY ? 0.f : top, f = fast_exp2(m - ref);
            l *= f;
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] *= f;
            for (int w = 1; w < used; ++w) {
                const float g = fast_exp2(meet[group + w][kJoinCols] - ref);
                l += meet[group + w][kJoinCols + 1] * g;
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] += meet[group + w][c0 + e] * g;
            }
            m = top;
        }
    }
    if (!there || way != 0) return;
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    i32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = E::pack2(y[2 * e] * inv, y[2 * e + 1] * inv);
    uint16_t* o = static_cast<uint16_t*>(const_cast<void*>(a.o.p)) + (b * a.o.batch + head * a.o.head + tok * a.o.token);
    *reinterpret_cast<i32x4*>(o + c) = w;
    if (c == 0) a.lse[row] = (m + log2f(l)) * kLn2;
}

// Whether each workgroup has a whole sequence and head: one launch, and nothing is looked for or joined, but the longest sequence
// decides.  So up to a length that goes with the workgroups there are, in keys that take as long as those of 16 rows at d = 128, and
// where they fill the chip up to kAlone keys, whatever these take: there the second start of a team costs more than even shares
// give, until a sequence much longer than the others keeps its workgroups busy when all others are done.  us, whole / teams, by workgroups and the longest of lengths spread over its last third
// (T = 1) or half, bf16:
//   T = 1 d = 64   8: 768 8.9 / 10.5, 1536 12.7 / 10.9;  128: 1536 15.0 / 15.3;  256: 3000 29.5 / 34.2;  512: 4500 79 / 84
//         d = 128  8: 512 9.5 / 11.4, 1024 13.1 / 11.7;  128: 1024 16.1 / 17.5;  256: 3000 55 / 59, but spread from a tenth of it on
//                  4096 55.6 / 51.5;  512: 4500 155 / 160
//   32 rows        32: 1024 16.0 / 16.7;  128: 2048 28 / 29;  256: 4500 77 / 84.   64 rows  64: 768 21.0 / 20.8;  128: 2048 35 / 38
//   256 rows       128: 512 25.9 / 28.3, 768 32 / 30;  256: 1024 41 / 46, 2048 66 / 59;  512: 4500 157 / 166
// and where they fill the chip, lengths alike (the last third) | one so long, the others 500 to 2000 (64 or 32 sequences of 8 heads):
//   T = 1 d = 64   512: 4500 79 / 83, 9000 148 / 149, 16000 264 / 266 | 4500 42 / 37, 9000 70 / 35, 65536 400 / 58
//         d = 128  512: 4500 153 / 160, 9000 296 / 294, 16000 528 / 521 | 4500 75 / 66, 9000 120 / 60, 65536 608 / 104
//         d = 256  512: 4500 305 / 313, 9000 587 / 576 | 4500 132 / 128, 9000 201 / 121, 65536 1174 / 202
//         codes, d = 128  512: 4500 83 / 88, 9000 154 / 156 | 4500 47 / 39, 9000 80 / 37, 65536 476 / 65
//   32 rows, d = 128   256: 4500 81 / 95, 9000 159 / 168 | 4500 57 / 45, 9000 95 / 48, 32768 306 / 72
//   64 rows, d = 128   256: 4500 86 / 109, 9000 163 / 183 | 4500 62 / 61, 9000 101 / 64
//   256 rows, d = 128  512: 4500 170 / 185, 9000 318 / 325 | 4500 123 / 95, 9000 220 / 100
constexpr int kAlone = 4608;
template <typename Form>
static bool whole_sequences(double workgroups, int max_len) {
    constexpr bool shared = Form::FORM == kShareKeys;
    constexpr double d64 = Form::COLS == 16 ? 0.75 : shared ? 1.0 : 0.5, d128 = Form::COLS == 16 ? 1.0 : shared ? 1.5 : 0.75,
                     d256 = Form::COLS == 16 ? (Form::CODES ? 1.5 : 2.0) : shared ? 2.0 : 1.25;
    if (workgroups >= 512 || (workgroups >= 256 && Form::COLS == 32 && !shared)) return max_len <= kAlone;
    const double limit = 8 * workgroups + 256 > 512 ? 8 * workgroups + 256 : 512;
    return max_len * (Form::D == 64 ? d64 : Form::D == 128 ? d128 : d256) <= limit * (Form::NW == 8 ? 1.8 : 1.0);
}

// Calls f with the shape that a call takes, and what its template arguments are.  (The shapes do not depend on the 16-bit type.)
//   rows to a key/value head  up to 16: 16 columns; 17 to 32: 32; 33 to 64: two tiles of 32 to a wave, so that each operand is read once for
//   both; more: four tiles, a wave each, that share what is staged (256 rows 94 us, divided keys 115; 52 rows 27.4 and 25.9).
// Eight waves instead of four halve the chain of a sequence that a workgroup has for itself, where its keys are small enough for two
// such workgroups' worth of LDS to be worth it: us, four / eight, T = 1, 8 heads: d = 64 1024 9.7 / 8.3; codes d = 64 768 9.9 / 8.1,
// d = 128 768 10.5 / 9.3, d = 256 512 12.7 / 11.6; bf16 d = 128 768 11.2 / 10.3 but 2048 22.2 / 21.7, and 300 7.5 / 7.7.
template <int D_, bool CODES_, int COLS_, int RT_, int NW_, int FORM_>
struct CachedForm {
    static constexpr int D = D_, COLS = COLS_, RT = RT_, NW = NW_, FORM = FORM_, STG = FORM == kShareKeys ? 3 : 1;
    static constexpr bool CODES = CODES_;
    template <typename Tag>
    using Shape = CachedShape<Tag, D, CODES, COLS, RT, NW, STG, FORM>;
};
template <typename F>
static auto with_form(int B, int H_kv, int rows, int d, int max_len, bool codes, F&& f) {
    auto by_rows = [&](auto D, auto c) {
        constexpr int d_ = decltype(D)::value;
        constexpr bool c_ = decltype(c)::value;
        if (rows <= 16) {
            if constexpr (d_ == 64 || c_) {
                using Eight = CachedForm<d_, c_, 16, 1, 8, kDivideKeys>;
                if ((double)B * H_kv <= (c_ && d_ == 128 ? 256 : 128) && max_len > 256 && whole_sequences<Eight>((double)B * H_kv, max_len)) return f(Eight{});
            }
            return f(CachedForm<d_, c_, 16, 1, 4, kDivideKeys>{});
        }
        if (rows > 64) return f(CachedForm<d_, c_, 32, 1, 4, kShareKeys>{});
        if constexpr (d_ < 256)
            if (rows > 32) return f(CachedForm<d_, c_, 32, 2, 4, kDivideKeys>{});
        return f(CachedForm<d_, c_, 32, 1, 4, kDivideKeys>{});
    };
    auto by_codes = [&](auto D) { return codes ? by_rows(D, std::true_type{}) : by_rows(D, std::false_type{}); };
    switch (d) {
        case 64: return by_codes(std::integral_constant<int, 64>{});
        case 128: return by_codes(std::integral_constant<int, 128>{});
        default: return by_codes(std::integral_constant<int, 256>{});
    }
}

// How a call is divided.
struct CachedDivision {
    int row_groups, teams;
    size_t table_bytes, rows;  // of the workspace: where segments are; the segments' rows
    template <typename Form>
    CachedDivision(const Form&, int B, int H, int H_kv, int T, int max_len) {
        using Shape = typename Form::template Shape<bf16_tag>;
        row_groups = (H / H_kv * T + Shape::ROWS - 1) / Shape::ROWS;
        const long items = (long)B * H_kv, most = ((long)max_len + Shape::STEP - 1) / Shape::STEP, slots = 256 * Shape::PER_CU;
        long n = slots / row_groups > 1 ? slots / row_groups : 1;
        if ((double)items * most < n) n = items * most;
        teams = whole_sequences<Form>((double)items * row_groups, max_len) ? 0 : (int)n;
        table_bytes = ((size_t)items * sizeof(CachedArgs::Segments) + 15) / 16 * 16;
        rows = (size_t)teams * row_groups * 2 * Shape::ROWS;
    }
    size_t bytes(int d) const { return teams == 0 ? 0 : table_bytes + rows * (d + 2) * sizeof(float); }
};

template <typename Tag, typename Form>
static int launch_cached(CachedArgs a, void* workspace, int max_len, hipStream_t stream) {
    using Shape = typename Form::template Shape<Tag>;
    constexpr int D = Form::D, NW = Form::NW;
    CachedDivision div(Form{}, a.B, a.H, a.c.H_kv, a.T, max_len);
    // (steps are counted in 32 bits, and there may be as many as there are places, whatever was expected)
    if ((double)a.B * a.c.H_kv * ((double)a.c.max_pages * a.c.page_size / Shape::STEP + 1) >= 2147483647.0) div.teams = 0;
    a.row_groups = div.row_groups;
    a.teams = div.teams;
    if (div.teams != 0) {
        a.segments = static_cast<CachedArgs::Segments*>(workspace);
        a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + div.table_bytes);
        a.state = a.part + div.rows * D;
    }
    const double total = (double)(div.teams != 0 ? div.teams : (double)a.B * a.c.H_kv) * a.row_groups;
    if (total * 64 * NW >= 4294967296.0) return FA_ERR_LAUNCH;
    hipLaunchKernelGGL((fa_fwd_cache_kernel<Tag, D, Form::CODES, Form::COLS, Form::RT, NW, Form::STG, Form::FORM>), dim3((unsigned)total), dim3(NW * 64), Shape::LDS, stream, a);
    if (hipGetLastError() != hipSuccess) return FA_ERR_LAUNCH;
    if (div.teams != 0) {
        const long rows = (long)a.B * a.H * a.T;
        int ways = 1;  // the fewer rows there are, the more threads to a row
        while (ways < 32 && ways < div.teams && rows * ways < 32 * 256) ways *= 2;
        hipLaunchKernelGGL((fa_join_kernel<Tag, D, Shape::ROWS>), dim3((unsigned)((rows * ways + 31) / 32), D / kJoinCols), dim3(256), 0, stream, a, ways);
        if (hipGetLastError() != hipSuccess) return FA_ERR_LAUNCH;
    }
    return FA_OK;
}

}  // namespace

size_t fwd_cache_workspace_bytes(int B, int H, int H_kv, int T, int d, int max_len, int cache_dtype) {
    return with_form(B, H_kv, H / H_kv * T, d, max_len, cache_dtype == FA_FP8_E4M3,
                     [&](auto form) { return CachedDivision(form, B, H, H_kv, T, max_len).bytes(d); });
}

int launch_fwd_cache(const Rows& q, const Cache& cache, const int* counts, const int* tree, int tree_batches, const Rows& o, float* lse,
                     void* workspace, int B, int H, int T, int d, int max_len, float scale, int dtype, hipStream_t stream) {
    const CachedArgs a = {q, o, cache, counts, tree, lse, nullptr, nullptr, nullptr, B, H, T, tree_batches, 1, 0, scale};
    return with_form(B, cache.H_kv, H / cache.H_kv * T, d, max_len, cache.dtype == FA_FP8_E4M3, [&](auto form) {
        using Form = decltype(form);
        return dtype == FA_BF16 ? launch_cached<bf16_tag, Form>(a, workspace, max_len, stream) : launch_cached<f16_tag, Form>(a, workspace, max_len, stream);
    });
}

}  // namespace fa
