// Which pages of a pool belong to which sequence (include/fa_mi355.h: fa_cache_fork, fa_cache_extend, fa_cache_compact), and copies of
// pages (fa_cache_copy).
//
// A page is free if no entry of the table names it and the caller does not hold it, so there are no counters that could go wrong: a
// workgroup marks what is in use in a bitmap in the LDS, a window of the pool at a time, and a sum over its words gives the free pages
// in ascending order.  What needs one gets them in its own order, so the result does not depend on the order of any atomic.  This is a
// few kilobytes and a chain of some six dependent reads of memory: latency decides, and for wide tables what one workgroup reads in a
// time.  The copies move whole pages, and HBM decides.
//
// Measured, kernels alone, us: fork 16 rows of 32 entries 7.7, 128 of 257 in 3130 pages 10.1; extend 2.4 where nothing is wanted, the 128 rows
// 7.7, 256 of 2048 in 100 thousand pages 41, of 8192 103; compact 4 rows 8.1, 64 of 128 in 7677 pages 16.7; copies of 115 MB to
// 115 MB 42, 5.5 TB/s.
#include "fa_device.h"
#include "fa_launch.h"

namespace fa {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;  // (numbers that go up by this, or by a window, may pass 2^31 at the end: they have no sign)
constexpr int kWindow = 1 << 18;  // pages whose bits are in the LDS at a time
constexpr int kListed = 1024;     // rows whose numbers are kept in the LDS and not in the workspace
constexpr int kSmallPool = 4096;  // pages whose lists are
constexpr int kHead = 16;
constexpr int kOwnEntries = 4;    // new entries of a sequence that its own thread sees to

constexpr bool small(int B, int n_pages) { return B <= kListed && n_pages <= kSmallPool; }

// In the workspace, or where that is none in the LDS, in ints: a head, three lists of pages, two of rows
struct Lists {
    int *head, *free, *high, *to, *part, *need;
    __device__ Lists(void* at, int B, int n_pages) {
        head = static_cast<int*>(at);
        free = head + kHead;
        high = free + n_pages;
        to = high + n_pages;
        part = to + n_pages;
        need = part + B;
    }
};
constexpr size_t list_ints(int B, int n_pages) { return kHead + 3 * (size_t)n_pages + 2 * (size_t)B; }

struct Pool {
    const int* held;  // [n_pages] or NULL
    int n_pages, max_pages, page_size;
    __device__ __forceinline__ bool has(int page) const { return (unsigned)page < (unsigned)n_pages; }
    __device__ __forceinline__ int places() const { return max_pages * page_size; }
};

struct Shared {
    int sums[kWaves + 1];
    int whole[kListed], seen[kListed];
    uint32_t bits[1];  // kWindow / 32, or as many as the pool has; a compaction: twice.  Behind them the lists, where there is no workspace.
};
constexpr int bitmap_words(int n_pages) { return ((n_pages < kWindow ? n_pages : kWindow) + 31) / 32; }
constexpr size_t shared_bytes(int B, int n_pages, int bitmaps) {
    return sizeof(Shared) + 4 * ((size_t)bitmap_words(n_pages) * bitmaps + (small(B, n_pages) ? list_ints(B, n_pages) : 0));
}
static __device__ __forceinline__ Lists lists_of(Shared& s, void* workspace, int B, int n_pages, int bitmaps) {
    return Lists(small(B, n_pages) ? static_cast<void*>(s.bits + bitmap_words(n_pages) * bitmaps) : workspace, B, n_pages);
}

// The sum of x over the threads before this one, and over all
static __device__ __forceinline__ int sum_before(int x, int& all, int* sums) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int upto = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(upto, d);
        if (lane >= d) upto += y;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const int s = sums[w];
        before += w < wave ? s : 0;
        all += s;
    }
    __syncthreads();
    return before + upto - x;
}

// (a negative number less base is kWindow or more without a sign: base is 2^31 - kWindow at most)
static __device__ __forceinline__ void mark(uint32_t* bits, int page, int base, int n) {
    const unsigned at = (unsigned)page - (unsigned)base;
    if (at < (unsigned)n) atomicOr(&bits[at >> 5], 1u << (at & 31));
}
static __device__ __forceinline__ bool marked(const uint32_t* bits, int page, int base) { return bits[(page - base) >> 5] >> ((page - base) & 31) & 1; }

static __device__ __forceinline__ void clear(uint32_t* bits, int words) {
    for (int i = threadIdx.x; i < words; i += kThreads) bits[i] = 0;
    __syncthreads();
}

// f(number, value) of n ints, 16 of a thread on their way at a time: one workgroup has nothing else to hide a read of memory behind.
// With SKIPS four negative ones in a row may be left out: a look at each takes longer than the reads.  us, all looked at / so: fa_cache_extend
// of 256 rows of 8192 entries, a thirteenth of them pages, 147 / 103,
// of 2048 with a tenth 44 / 41
template <bool SKIPS, typename F>
static __device__ __forceinline__ void for_each_int(const int* p, int n, F&& f) {
    const int skip = min((int)(-(reinterpret_cast<uintptr_t>(p) / 4) & 3), n), whole = (n - skip) / 4;  // to where four ints are aligned
    const i32x4* const x = reinterpret_cast<const i32x4*>(p + skip);
    const int rest = skip + 4 * whole;
    if ((int)threadIdx.x < skip) f((int)threadIdx.x, p[threadIdx.x]);
    if ((int)threadIdx.x < n - rest) f(rest + (int)threadIdx.x, p[rest + threadIdx.x]);
    constexpr int AHEAD = 4;
    for (int i0 = threadIdx.x; i0 < whole; i0 += AHEAD * kThreads) {
        i32x4 v[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) v[j] = x[min(i0 + j * kThreads, whole - 1)];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
            if (i0 + j * kThreads < whole && !(SKIPS && (v[j][0] & v[j][1] & v[j][2] & v[j][3]) < 0))
#pragma unroll
                for (int e = 0; e < 4; ++e) f(skip + 4 * (i0 + j * kThreads) + e, v[j][e]);
    }
}

// What the caller holds, and all entries of a table
static __device__ __forceinline__ void mark_held(uint32_t* bits, const Pool& pool, int base, int n) {
    if (pool.held)
        for_each_int<false>(pool.held + base, n, [&](int page, int held) {
            if (held != 0) mark(bits, page, 0, n);
        });
}
static __device__ __forceinline__ void mark_table(uint32_t* bits, const int* table, int entries, int base, int n) {
    for_each_int<true>(table, entries, [&](int, int page) { mark(bits, page, base, n); });
}

// The pages base .. base + n - 1 whose bit is `value` (and whose bit in `others` is not set) go to list[found ..] in ascending order, up to `most`
static __device__ __forceinline__ void collect(const uint32_t* bits, const uint32_t* others, bool value, int base, int n, int* list, int most, int& found, int* sums) {
    const int words = (n + 31) / 32, each = (words + kThreads - 1) / kThreads, first = threadIdx.x * each, last = min(first + each, words);
    auto word = [&](int w) __attribute__((always_inline)) {
        const uint32_t there = 32 * w + 32 <= n ? ~0u : (1u << (n & 31)) - 1;
        return (value ? bits[w] : ~bits[w]) & (others ? ~others[w] : ~0u) & there;
    };
    int count = 0;
    for (int w = first; w < last; ++w) count += __popc(word(w));
    int all, at = found + sum_before(count, all, sums);
    for (int w = first; w < last && at < most; ++w)
        for (uint32_t x = word(w); x != 0 && at < most; x &= x - 1) list[at++] = base + 32 * w + __builtin_ctz(x);
    found += all;
}

// ------------------------------------------------------------------------------------------

struct ForkArgs {
    const int *table, *lens, *parents;
    int *new_table, *new_lens, *src, *dst, *missing;
    void* workspace;
    int B, B_new;
    Pool pool;
};

// What a new sequence has of the old one that it continues
struct Continued {
    int parent, len, whole;  // whole pages
    bool last;               // a page that is not full, entry `whole`
    __device__ __forceinline__ Continued(const ForkArgs& a, int row) {
        parent = a.parents[row];
        len = 0;
        if ((unsigned)parent < (unsigned)a.B) len = min(max(a.lens[parent], 0), a.pool.places());
        else parent = -1;
        whole = (unsigned)len / (unsigned)a.pool.page_size;
        last = len != whole * a.pool.page_size;
    }
};

// Workgroup 0 decides which pages are copied and where to; the others write the rest of the new table, kPerThread entries a thread.
constexpr int kPerThread = 4;
__global__ void __launch_bounds__(kThreads) fa_cache_fork_kernel(ForkArgs a) {
    const Pool& pool = a.pool;
    const unsigned total = (unsigned)a.B_new * pool.max_pages;
    if (blockIdx.x > 0) {
#pragma unroll
        for (int j = 0; j < kPerThread; ++j) {
            const unsigned i = ((blockIdx.x - 1) * kPerThread + j) * (unsigned)kThreads + threadIdx.x;
            if (i >= total) return;
            const int row = i / (unsigned)pool.max_pages, e = i - row * pool.max_pages;
            const Continued c(a, row);
            if (e == c.whole && c.last) continue;
            a.new_table[i] = e < c.whole ? a.table[(long)c.parent * pool.max_pages + e] : -1;
        }
        return;
    }
    extern __shared__ char raw[];
    Shared& s = *reinterpret_cast<Shared*>(raw);
    const Lists lists = lists_of(s, a.workspace, a.B_new, pool.n_pages, 1);
    int *const part = lists.part, *const need = lists.need, *const list = lists.free;
    const int tid = threadIdx.x;

    // The pages that new sequences would write to, and whether an earlier one does: that keeps it, the others need a copy.  Of a held page
    // all do: who holds it reads it, and may go on from it.
    auto held = [&](int page) __attribute__((always_inline)) { return pool.held && pool.held[page] != 0; };
    const bool once = a.B <= kListed;  // what is whole of each old sequence that is continued is written down here
    if (once) {
        if (tid < a.B) s.whole[tid] = 0;
        __syncthreads();
    }
    for (unsigned i = tid; i < (unsigned)a.B_new; i += kThreads) {
        const Continued c(a, i);
        if (once && c.parent >= 0) s.whole[c.parent] = c.whole;  // (the same from all)
        const int page = c.last ? a.table[(long)c.parent * pool.max_pages + c.whole] : -1;
        part[i] = pool.has(page) ? page : -1;
        if (i < kListed) s.seen[i] = part[i];
    }
    __syncthreads();
    if (a.B_new <= kListed) {
        if (tid < a.B_new) {
            const int page = part[tid];
            bool earlier = false;
            for (int j = 0; j < tid; ++j) earlier |= s.seen[j] == page;
            need[tid] = page >= 0 && (earlier || held(page));
        }
    } else {
        int* const first = lists.high;
        for (unsigned i = tid; i < (unsigned)a.B_new; i += kThreads)
            if (part[i] >= 0) first[part[i]] = 0x7fffffff;
        __threadfence();
        __syncthreads();
        for (unsigned i = tid; i < (unsigned)a.B_new; i += kThreads)
            if (part[i] >= 0) atomicMin(&first[part[i]], (int)i);
        __threadfence();
        __syncthreads();
        for (unsigned i = tid; i < (unsigned)a.B_new; i += kThreads)
            need[i] = part[i] >= 0 && (__hip_atomic_load(&first[part[i]], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != (int)i || held(part[i]));
    }

    int found = 0;
    for (unsigned window = 0; window < (unsigned)pool.n_pages; window += kWindow) {
        const int base = (int)window, n = min(kWindow, pool.n_pages - base);
        clear(s.bits, (n + 31) / 32);
        // The whole pages of old sequences that are continued, each looked at once however many continue it: a wave takes 512 entries of a
        // row, two rows' at a time.  Of more old sequences than are written down, the entries of the new ones, so the work goes by their
        // number: us, 1024 old ones at a time with all new ones looked at for each / so, 1025 rows of 40 entries 67 / 32, 8192 of 33 continued by
        // 1500 728 / 59, 2048 of 257 by parents at random 304 / 340; a million and more of one entry: minutes / below a second.
        if (once) {
            const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), parts = (pool.max_pages + 511) / 512;
            const unsigned units = (unsigned)a.B * parts;
            for (unsigned u0 = wave; u0 < units; u0 += 2 * kWaves) {
                int page[2][8];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const unsigned u = min(u0 + x * kWaves, units - 1);
                    const int row = u / (unsigned)parts, e0 = (u - row * parts) * 512 + lane, whole = s.whole[row];
                    const int* const entries = a.table + (long)row * pool.max_pages;
#pragma unroll
                    for (int j = 0; j < 8; ++j) page[x][j] = e0 + 64 * j < whole ? entries[e0 + 64 * j] : -1;
                }
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int j = 0; j < 8; ++j) mark(s.bits, page[x][j], base, n);
            }
        } else {
            constexpr int AHEAD = 8;
            static_assert(kListed == kThreads);
            const int more_rows = kThreads / (unsigned)pool.max_pages, more = kThreads - more_rows * pool.max_pages;  // from a thread's entry to its next
            for (unsigned r0 = 0; r0 < (unsigned)a.B_new; r0 += kListed) {
                const unsigned rows = min((unsigned)kListed, a.B_new - r0), entries = rows * pool.max_pages;
                if (tid < (int)rows) {
                    const Continued c(a, (int)(r0 + tid));
                    s.seen[tid] = c.parent;
                    s.whole[tid] = c.whole;
                }
                __syncthreads();
                unsigned row = tid / (unsigned)pool.max_pages;
                int e = tid - row * pool.max_pages;
                for (unsigned i0 = tid; i0 < entries; i0 += AHEAD * kThreads) {
                    int page[AHEAD];
#pragma unroll
                    for (int j = 0; j < AHEAD; ++j) {
                        page[j] = i0 + j * kThreads < entries && e < s.whole[row] ? a.table[(long)s.seen[row] * pool.max_pages + e] : -1;
                        row += more_rows;
                        e += more;
                        if (e >= pool.max_pages) {
                            e -= pool.max_pages;
                            ++row;
                        }
                    }
#pragma unroll
                    for (int j = 0; j < AHEAD; ++j) mark(s.bits, page[j], base, n);
                }
                __syncthreads();
            }
        }
        __syncthreads();
        for (unsigned i = tid; i < (unsigned)a.B_new; i += kThreads)
            if (part[i] >= base && part[i] - base < n && marked(s.bits, part[i], base)) need[i] = 1;  // a whole page of another: not to be written to
        __syncthreads();
        for (unsigned i = tid; i < (unsigned)a.B_new; i += kThreads) mark(s.bits, part[i], base, n);
        mark_held(s.bits, pool, base, n);
        __syncthreads();
        collect(s.bits, nullptr, false, base, n, list, a.B_new, found, s.sums);
        __syncthreads();
    }

    int before = 0;
    for (unsigned r0 = 0; r0 < (unsigned)a.B_new; r0 += kThreads) {
        const unsigned i = r0 + tid;
        const int needs = i < (unsigned)a.B_new ? need[i] : 0;
        int all;
        const int at = before + sum_before(needs, all, s.sums);
        before += all;
        if (i >= (unsigned)a.B_new) continue;
        const Continued c(a, i);
        const int page = needs && at < found ? list[at] : -1;
        a.new_lens[i] = c.len;
        a.src[i] = page >= 0 ? part[i] : -1;
        a.dst[i] = page;
        if (c.last) a.new_table[(long)i * pool.max_pages + c.whole] = needs ? page : a.table[(long)c.parent * pool.max_pages + c.whole];
    }
    if (tid == 0) *a.missing = max(before - found, 0);
}

// ------------------------------------------------------------------------------------------

struct ExtendArgs {
    int* table;
    const int *lens, *counts;
    int* missing;
    void* workspace;
    int B, T;
    Pool pool;
};

__global__ void __launch_bounds__(kThreads) fa_cache_extend_kernel(ExtendArgs a) {
    const Pool& pool = a.pool;
    extern __shared__ char raw[];
    Shared& s = *reinterpret_cast<Shared*>(raw);
    const int tid = threadIdx.x;
    // entries first .. last of a sequence are those of its new tokens; `beyond` of them past the table
    auto entries = [&](int b, int& first, int& last) __attribute__((always_inline)) {
        const int len = max(a.lens[b], 0), count = a.counts ? min(a.counts[b], a.T) : a.T;
        first = (unsigned)len / (unsigned)pool.page_size;
        const long end = count > 0 ? ((long)len + count - 1) / pool.page_size : (long)first - 1;
        last = (int)min(end, (long)pool.max_pages - 1);
        return count > 0 ? (int)(end - max((long)first - 1, (long)last)) : 0;
    };
    auto none = [&](const int* entry, int n) __attribute__((always_inline)) {
        int sum = 0;
        for (int e = 0; e < n; ++e) sum += !pool.has(entry[e]);
        return sum;
    };
    auto give = [&](int* entry, int n, int at, const int* list, int most) __attribute__((always_inline)) {
        for (int e = 0; e < n; ++e) {
            if (pool.has(entry[e])) continue;
            entry[e] = at < most ? list[at] : -1;
            ++at;
        }
    };
    // Few entries of a sequence are seen to by its thread.  If any has many, or some past the table, all go one by one over the threads.  us,
    // by sequences / by entries: one prompt of 131072 tokens in pages of 16 2675 / 28.6, four of a quarter of it 731 / 28.4
    constexpr int kMany = 8192;
    static_assert(kMany > kOwnEntries * kThreads);
    int* mine = nullptr;
    int n_mine = 0;
    auto by_sequences = [&](unsigned b0, int& all) __attribute__((always_inline)) {
        const unsigned b = b0 + tid;
        int first = 0, last = -1, past = 0;
        if (b < (unsigned)a.B) past = entries(b, first, last);
        mine = a.table + (long)b * pool.max_pages + first;
        n_mine = max(last - first + 1, 0);
        return sum_before(n_mine <= kOwnEntries && past == 0 ? none(mine, n_mine) : kMany, all, s.sums);
    };
    int all_past = 0;
    auto by_entries = [&](auto&& f) __attribute__((always_inline)) {
        for (unsigned b0 = 0; b0 < (unsigned)a.B; b0 += kThreads) {
            const unsigned b = b0 + tid;
            int first = 0, last = -1, all;
            if (b < (unsigned)a.B) all_past += entries(b, first, last);
            const int before = sum_before(max(last - first + 1, 0), all, s.sums);
            s.seen[tid] = before;
            s.whole[tid] = first;
            __syncthreads();
            for (unsigned i0 = 0; i0 < (unsigned)all; i0 += kThreads) {
                const unsigned i = i0 + tid;
                int row = 0;  // the last that begins with entry i or before
#pragma unroll
                for (int step = kThreads / 2; step > 0; step /= 2) row += (unsigned)s.seen[row + step] <= i ? step : 0;
                f(a.table + (long)(b0 + row) * pool.max_pages + s.whole[row] + i - s.seen[row], i < (unsigned)all ? 1 : 0);
            }
            __syncthreads();
        }
    };
    int wanted = 0, beyond = 0, at = 0;
    bool any_many = false;
    for (unsigned b0 = 0; b0 < (unsigned)a.B; b0 += kThreads) {
        int all;
        at = by_sequences(b0, all);
        wanted += all % kMany;
        any_many |= all >= kMany;
    }
    if (any_many) {
        int sum = 0;
        by_entries([&](const int* entry, int n) __attribute__((always_inline)) { sum += none(entry, n); });
        sum_before(sum, wanted, s.sums);
        sum_before(all_past, beyond, s.sums);
    }
    if (wanted == 0) {  // (as in most steps)
        if (tid == 0) *a.missing = beyond;
        return;
    }
    const int asked = min(wanted, pool.n_pages);
    int* const list = lists_of(s, a.workspace, a.B, pool.n_pages, 1).free;
    int found = 0;
    for (unsigned window = 0; window < (unsigned)pool.n_pages; window += kWindow) {
        const int base = (int)window, n = min(kWindow, pool.n_pages - base);
        clear(s.bits, (n + 31) / 32);
        mark_table(s.bits, a.table, a.B * pool.max_pages, base, n);
        mark_held(s.bits, pool, base, n);
        __syncthreads();
        collect(s.bits, nullptr, false, base, n, list, asked, found, s.sums);
        __syncthreads();
        if (found >= asked) break;
    }
    const int most = min(found, asked);
    int before = 0;
    if (any_many) {
        by_entries([&](int* entry, int n) __attribute__((always_inline)) {
            int all;
            const int from = before + sum_before(none(entry, n), all, s.sums);
            before += all;
            give(entry, n, from, list, most);
        });
    } else {
        for (unsigned b0 = 0; b0 < (unsigned)a.B; b0 += kThreads) {
            if (a.B > kThreads) {
                int all;
                at = before + by_sequences(b0, all);
                before += all;
            }
            give(mine, n_mine, at, list, most);
        }
    }
    if (tid == 0) *a.missing = max(wanted - found, 0) + beyond;
}

// ------------------------------------------------------------------------------------------

struct CompactArgs {
    const int* table;
    int *new_table, *src, *dst, *top;
    void* workspace;
    int B, moves, renumbers;  // whether the one workgroup sees to the table too
    Pool pool;
};

// The highest page in use goes to the lowest free one, the next to the next, while that is lower
__global__ void __launch_bounds__(kThreads) fa_cache_compact_kernel(CompactArgs a) {
    const Pool& pool = a.pool;
    extern __shared__ char raw[];
    Shared& s = *reinterpret_cast<Shared*>(raw);
    const Lists lists = lists_of(s, a.workspace, a.B, pool.n_pages, 2);
    const int tid = threadIdx.x, half = bitmap_words(pool.n_pages);
    uint32_t *const used = s.bits, *const held = s.bits + half;
    int n_free = 0, n_high = 0, top_held = -1;
    for (unsigned window = 0; window < (unsigned)pool.n_pages; window += kWindow) {
        const int base = (int)window, n = min(kWindow, pool.n_pages - base);
        clear(used, half);
        clear(held, half);
        mark_table(used, a.table, a.B * pool.max_pages, base, n);
        mark_held(held, pool, base, n);
        __syncthreads();
        for (int w = (n + 31) / 32 - 1 - tid; w >= 0; w -= kThreads)
            if (held[w] != 0) {
                top_held = max(top_held, base + 32 * w + 31 - __builtin_clz(held[w]));
                break;
            }
        collect(used, held, true, base, n, lists.high, pool.n_pages, n_high, s.sums);
        collect(used, held, false, base, n, lists.free, pool.n_pages, n_free, s.sums);
        __syncthreads();
    }
    const int most = min(min(n_free, n_high), a.moves);
    int mine = 0, moved;
    constexpr int AHEAD = 4;
    for (unsigned k0 = tid; k0 < (unsigned)a.moves; k0 += AHEAD * kThreads) {
        int from[AHEAD], to[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const unsigned k = k0 + j * kThreads;
            from[j] = k < (unsigned)most ? lists.high[n_high - 1 - k] : -1;
            to[j] = k < (unsigned)most ? lists.free[k] : 0;
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const unsigned k = k0 + j * kThreads;
            const bool moves = to[j] < from[j];  // (once one does not, none after it does)
            if (k < (unsigned)a.moves) {
                a.src[k] = moves ? from[j] : -1;
                a.dst[k] = moves ? to[j] : -1;
            }
            if (moves) lists.to[from[j]] = to[j];
            mine += moves;
        }
    }
    sum_before(mine, moved, s.sums);
    int* const tops = s.whole;
#pragma unroll
    for (int d = 32; d > 0; d /= 2) top_held = max(top_held, __shfl_xor(top_held, d));
    if ((tid & 63) == 0) tops[tid >> 6] = top_held;
    __syncthreads();
    const int threshold = moved > 0 ? lists.high[n_high - moved] : 0x7fffffff;  // pages from here on have moved, but for held ones
    if (tid == 0) {
        int top = tops[0];
        for (int w = 1; w < kWaves; ++w) top = max(top, tops[w]);
        if (n_high > moved) top = max(top, lists.high[n_high - 1 - moved]);
        if (moved > 0) top = max(top, lists.free[moved - 1]);
        *a.top = top + 1;
        lists.head[0] = threshold;
    }
    if (!a.renumbers) return;
    const int entries = a.B * pool.max_pages;
    for_each_int<false>(a.table, entries, [&](int i, int page) {
        if (pool.has(page) && page >= threshold && !(pool.held && pool.held[page] != 0)) page = lists.to[page];
        a.new_table[i] = page;
    });
}

__global__ void __launch_bounds__(256) fa_cache_renumber_kernel(CompactArgs a) {
    const Lists lists(a.workspace, a.B, a.pool.n_pages);
    const unsigned i = blockIdx.x * 256u + threadIdx.x;
    if (i >= (unsigned)a.B * a.pool.max_pages) return;
    int page = a.table[i];
    if (a.pool.has(page) && page >= lists.head[0] && !(a.pool.held && a.pool.held[page] != 0)) page = lists.to[page];
    a.new_table[i] = page;
}

// ------------------------------------------------------------------------------------------

// A workgroup brings 4 AT_ONCE KiB of K or V of a pair's page, and the first one of each its scales.  us, 4 / 2: 112 pairs of 64 KiB each 8.4 /
// 6.8, where all workgroups there are start at once; 1700 of 3838 pairs of 32 KiB 41.9 / 45.3
template <int AT_ONCE>
__global__ void __launch_bounds__(256) fa_cache_copy_kernel(Cache c, const int* src, const int* dst, unsigned chunks, long bytes, long scale_bytes) {
    const unsigned part = blockIdx.x % (2 * chunks), pair = blockIdx.x / (2 * chunks);
    const int from = src[pair], to = dst[pair];
    if ((unsigned)from >= (unsigned)c.n_pages || (unsigned)to >= (unsigned)c.n_pages || from == to) return;
    const bool v = part >= chunks;
    char* const pages = static_cast<char*>(v ? c.v : c.k);
    const long first = (long)(v ? part - chunks : part) * (4096 * AT_ONCE) + threadIdx.x * 16;
    const char* x = pages + from * bytes;
    char* y = pages + to * bytes;
    i32x4 w[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i)
        if (first + i * 4096 < bytes) w[i] = __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(x + first + i * 4096));
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i)
        if (first + i * 4096 < bytes) __builtin_nontemporal_store(w[i], reinterpret_cast<i32x4*>(y + first + i * 4096));
    if (scale_bytes > 0 && part % chunks == 0) {
        char* const scales = static_cast<char*>(v ? c.v_scales : c.k_scales);
        for (long i = threadIdx.x * 4; i < scale_bytes; i += 1024)
            *reinterpret_cast<int*>(scales + to * scale_bytes + i) = *reinterpret_cast<const int*>(scales + from * scale_bytes + i);
    }
}

int launched() { return hipGetLastError() == hipSuccess ? FA_OK : FA_ERR_LAUNCH; }

}  // namespace

size_t cache_pages_workspace_bytes(int B, int n_pages) { return small(B, n_pages) ? 0 : sizeof(int) * list_ints(B, n_pages); }

int launch_cache_fork(const int* block_table, const int* lens, const int* parents, const int* held, int* new_table, int* new_lens, int* src,
                      int* dst, int* missing, void* workspace, int B, int B_new, int page_size, int n_pages, int max_pages, hipStream_t stream) {
    const ForkArgs a = {block_table, lens, parents, new_table, new_lens, src, dst, missing, workspace, B, B_new, {held, n_pages, max_pages, page_size}};
    const long total = (long)B_new * max_pages, each = kThreads * kPerThread;
    hipLaunchKernelGGL(fa_cache_fork_kernel, dim3((unsigned)(1 + (total + each - 1) / each)), dim3(kThreads), shared_bytes(B_new, n_pages, 1), stream, a);
    return launched();
}

int launch_cache_extend(int* block_table, const int* lens, const int* counts, const int* held, int* missing, void* workspace, int B, int T,
                        int page_size, int n_pages, int max_pages, hipStream_t stream) {
    const ExtendArgs a = {block_table, lens, counts, missing, workspace, B, T, {held, n_pages, max_pages, page_size}};
    hipLaunchKernelGGL(fa_cache_extend_kernel, dim3(1), dim3(kThreads), shared_bytes(B, n_pages, 1), stream, a);
    return launched();
}

int launch_cache_compact(const int* block_table, const int* held, int* new_table, int* src, int* dst, int* top, void* workspace, int B,
                         int moves, int n_pages, int max_pages, hipStream_t stream) {
    // (a second launch costs 2 to 3 us; one workgroup takes that long for some 16 thousand entries.  It needs the lists in a workspace.)
    const int renumbers = small(B, n_pages) || (long)B * max_pages <= 16384;
    const CompactArgs a = {block_table, new_table, src, dst, top, workspace, B, moves, renumbers, {held, n_pages, max_pages, 0}};
    hipLaunchKernelGGL(fa_cache_compact_kernel, dim3(1), dim3(kThreads), shared_bytes(B, n_pages, 2), stream, a);
    const int st = launched();
    if (st != FA_OK || renumbers) return st;
    const long total = (long)B * max_pages;
    hipLaunchKernelGGL(fa_cache_renumber_kernel, dim3((unsigned)((total + 255) / 256)), dim3(256), 0, stream, a);
    return launched();
}

int launch_cache_copy(const Cache& cache, const int* src, const int* dst, int n, int d, hipStream_t stream) {
    const long rows = (long)cache.H_kv * cache.page_size;
    const long bytes = rows * (cache.dtype == FA_FP4_E2M1 ? d / 2 : cache.dtype == FA_FP8_E4M3 ? d : 2 * d);
    const long scale_bytes = rows * (cache.dtype == FA_FP4_E2M1 ? d / 32 : cache.dtype == FA_FP8_E4M3 ? 4 : 0);
    auto go = [&](auto at_once, auto kernel) {
        const long each = 4096 * decltype(at_once)::value, chunks = (bytes + each - 1) / each;
        const long most = 0xffffffffL / (256 * 2 * chunks);  // pairs of a launch: a grid has fewer than 2^32 threads
        if (most == 0) return (int)FA_ERR_LAUNCH;
        for (long first = 0; first < n; first += most) {
            const long pairs = n - first < most ? n - first : most;
            hipLaunchKernelGGL(kernel, dim3((unsigned)(pairs * 2 * chunks)), dim3(256), 0, stream, cache, src + first, dst + first, (unsigned)chunks, bytes, scale_bytes);
            if (launched() != FA_OK) return (int)FA_ERR_LAUNCH;
        }
        return (int)FA_OK;
    };
    if ((double)n * 2 * bytes > 64.0 * 1024 * 1024) return go(std::integral_constant<int, 4>{}, fa_cache_copy_kernel<4>);
    return go(std::integral_constant<int, 2>{}, fa_cache_copy_kernel<2>);
}

}  // namespace fa
