// Which pages of a pool belong to which sequence (include/fa_mi355.h: fa_cache_fork, fa_cache_extend, fa_cache_compact), and copies of
// pages (fa_cache_copy).
//
// A page is free if no entry of the table names it and the caller does not hold it, so there are no counters that could go wrong: a
// workgroup marks what is in use in a bitmap in the LDS, a window of the pool at a time, and a sum over its words gives the free pages
// in ascending order.  What needs one gets them in its own order, so the result does not depend on the order of any atomic.  This is a
// few kilobytes and a chain of some six dependent reads of memory: latency decides.  The copies move whole pages, and HBM decides.
#include "fa_device.h"
#include "fa_launch.h"

namespace fa {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kWindow = 1 << 18;  // pages whose bits are in the LDS at a time
constexpr int kListed = 1024;     // rows, and free pages, that are kept in the LDS and not in the workspace
constexpr int kHead = 16;

// The workspace, in ints: a head, three lists of pages, two of rows
struct Lists {
    int *head, *free, *high, *to, *part, *need;
    __host__ __device__ Lists(void* workspace, int B, int n_pages) {
        head = static_cast<int*>(workspace);
        free = head + kHead;
        high = free + n_pages;
        to = high + n_pages;
        part = to + n_pages;
        need = part + B;
    }
};

struct Pool {
    const int* held;  // [n_pages] or NULL
    int n_pages, max_pages, page_size;
    __device__ __forceinline__ bool has(int page) const { return (unsigned)page < (unsigned)n_pages; }
    __device__ __forceinline__ int places() const { return max_pages * page_size; }
};

struct Shared {
    int sums[kWaves + 1];
    int part[kListed], need[kListed], list[kListed], parent[kListed], whole[kListed];
    uint32_t bits[1];  // kWindow / 32, or as many as the pool has; a compaction: twice
};
constexpr size_t shared_bytes(int n_pages, int bitmaps) {
    const int n = n_pages < kWindow ? n_pages : kWindow;
    return sizeof(Shared) + (size_t)((n + 31) / 32) * 4 * bitmaps;
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

static __device__ __forceinline__ void mark(uint32_t* bits, int page, int base, int n) {
    const unsigned at = (unsigned)(page - base);
    if (page >= 0 && at < (unsigned)n) atomicOr(&bits[at >> 5], 1u << (at & 31));
}
static __device__ __forceinline__ bool marked(const uint32_t* bits, int page, int base) { return bits[(page - base) >> 5] >> ((page - base) & 31) & 1; }

static __device__ __forceinline__ void clear(uint32_t* bits, int words) {
    for (int i = threadIdx.x; i < words; i += kThreads) bits[i] = 0;
    __syncthreads();
}

// What the caller holds, and all entries of a table
static __device__ __forceinline__ void mark_held(uint32_t* bits, const Pool& pool, int base, int n) {
    if (!pool.held) return;
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += kThreads)
        if (pool.held[base + i] != 0) mark(bits, i, 0, n);
}
static __device__ __forceinline__ void mark_table(uint32_t* bits, const int* table, int entries, int base, int n) {
#pragma unroll 8
    for (int i = threadIdx.x; i < entries; i += kThreads) mark(bits, table[i], base, n);
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
    const Lists lists(a.workspace, a.B_new, pool.n_pages);
    const bool few = a.B_new <= kListed;
    int *const part = few ? s.part : lists.part, *const need = few ? s.need : lists.need, *const list = few ? s.list : lists.free;
    const int tid = threadIdx.x;

    // The pages that new sequences would write to, and whether an earlier one does: that keeps it, the others need a copy
    for (int i = tid; i < a.B_new; i += kThreads) {
        const Continued c(a, i);
        const int page = c.last ? a.table[(long)c.parent * pool.max_pages + c.whole] : -1;
        part[i] = pool.has(page) ? page : -1;
    }
    __syncthreads();
    if (few) {
        if (tid < a.B_new) {
            const int page = s.part[tid];
            bool earlier = false;
            for (int j = 0; j < tid; ++j) earlier |= s.part[j] == page;
            s.need[tid] = page >= 0 && earlier;
        }
    } else {
        int* const first = lists.high;
        for (int i = tid; i < a.B_new; i += kThreads)
            if (part[i] >= 0) first[part[i]] = 0x7fffffff;
        __threadfence();
        __syncthreads();
        for (int i = tid; i < a.B_new; i += kThreads)
            if (part[i] >= 0) atomicMin(&first[part[i]], i);
        __threadfence();
        __syncthreads();
        for (int i = tid; i < a.B_new; i += kThreads)
            need[i] = part[i] >= 0 && __hip_atomic_load(&first[part[i]], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != i;
    }

    int found = 0;
    for (int base = 0; base < pool.n_pages; base += kWindow) {
        const int n = min(kWindow, pool.n_pages - base);
        clear(s.bits, (n + 31) / 32);
        for (int r0 = 0; r0 < a.B_new; r0 += kListed) {
            const int rows = min(kListed, a.B_new - r0);
            for (int i = tid; i < rows; i += kThreads) {
                const Continued c(a, r0 + i);
                s.parent[i] = c.parent;
                s.whole[i] = c.whole;
            }
            __syncthreads();
            const unsigned entries = (unsigned)rows * pool.max_pages;
#pragma unroll 4
            for (unsigned i = tid; i < entries; i += kThreads) {
                const int row = i / (unsigned)pool.max_pages, e = i - row * pool.max_pages;
                if (e < s.whole[row]) mark(s.bits, a.table[(long)s.parent[row] * pool.max_pages + e], base, n);
            }
            __syncthreads();
        }
        for (int i = tid; i < a.B_new; i += kThreads)
            if (part[i] >= base && part[i] - base < n && marked(s.bits, part[i], base)) need[i] = 1;  // a whole page of another: not to be written to
        __syncthreads();
        for (int i = tid; i < a.B_new; i += kThreads) mark(s.bits, part[i], base, n);
        mark_held(s.bits, pool, base, n);
        __syncthreads();
        collect(s.bits, nullptr, false, base, n, list, a.B_new, found, s.sums);
        __syncthreads();
    }

    int before = 0;
    for (int r0 = 0; r0 < a.B_new; r0 += kThreads) {
        const int i = r0 + tid;
        const int needs = i < a.B_new ? need[i] : 0;
        int all;
        const int at = before + sum_before(needs, all, s.sums);
        before += all;
        if (i >= a.B_new) continue;
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
    int wanted = 0, beyond = 0;
    for (int b0 = 0; b0 < a.B; b0 += kThreads) {
        const int b = b0 + tid;
        int n = 0, past = 0;
        if (b < a.B) {
            int first, last;
            past = entries(b, first, last);
            for (int e = first; e <= last; ++e) n += !pool.has(a.table[(long)b * pool.max_pages + e]);
        }
        int all;
        sum_before(n, all, s.sums);
        wanted += all;
        sum_before(past, all, s.sums);
        beyond += all;
    }
    if (wanted == 0) {  // (as in most steps)
        if (tid == 0) *a.missing = beyond;
        return;
    }
    const int most = min(wanted, pool.n_pages);
    int* const list = most <= kListed ? s.list : Lists(a.workspace, a.B, pool.n_pages).free;
    int found = 0;
    for (int base = 0; base < pool.n_pages; base += kWindow) {
        const int n = min(kWindow, pool.n_pages - base);
        clear(s.bits, (n + 31) / 32);
        mark_table(s.bits, a.table, a.B * pool.max_pages, base, n);
        mark_held(s.bits, pool, base, n);
        __syncthreads();
        collect(s.bits, nullptr, false, base, n, list, most, found, s.sums);
        __syncthreads();
        if (found >= most) break;
    }
    int before = 0;
    for (int b0 = 0; b0 < a.B; b0 += kThreads) {
        const int b = b0 + tid;
        int n = 0, first = 0, last = -1, all;
        if (b < a.B) {
            entries(b, first, last);
            for (int e = first; e <= last; ++e) n += !pool.has(a.table[(long)b * pool.max_pages + e]);
        }
        int at = before + sum_before(n, all, s.sums);
        before += all;
        for (int e = first; e <= last; ++e) {
            int* const entry = a.table + (long)b * pool.max_pages + e;
            if (pool.has(*entry)) continue;
            *entry = at < found && at < most ? list[at] : -1;
            ++at;
        }
    }
    if (tid == 0) *a.missing = max(wanted - found, 0) + beyond;
}

// ------------------------------------------------------------------------------------------

struct CompactArgs {
    const int* table;
    int *new_table, *src, *dst, *top;
    void* workspace;
    int B, moves;
    Pool pool;
};

// The highest page in use goes to the lowest free one, the next to the next, while that is lower
__global__ void __launch_bounds__(kThreads) fa_cache_compact_kernel(CompactArgs a) {
    const Pool& pool = a.pool;
    extern __shared__ char raw[];
    Shared& s = *reinterpret_cast<Shared*>(raw);
    const Lists lists(a.workspace, a.B, pool.n_pages);
    const int tid = threadIdx.x, half = (min(kWindow, pool.n_pages) + 31) / 32;
    uint32_t *const used = s.bits, *const held = s.bits + half;
    int n_free = 0, n_high = 0, top_held = -1;
    for (int base = 0; base < pool.n_pages; base += kWindow) {
        const int n = min(kWindow, pool.n_pages - base);
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
    int moved = 0;
    for (int k0 = 0; k0 < a.moves; k0 += kThreads) {
        const int k = k0 + tid;
        int from = -1, to = -1;
        if (k < most) {
            from = lists.high[n_high - 1 - k];
            to = lists.free[k];
            if (to > from) from = to = -1;
        }
        if (k < a.moves) {
            a.src[k] = from;
            a.dst[k] = to;
        }
        if (from >= 0) lists.to[from] = to;
        int all;
        sum_before(from >= 0, all, s.sums);
        moved += all;
    }
    s.list[tid] = top_held;
    __syncthreads();
    for (int d = kThreads / 2; d > 0; d /= 2) {
        if (tid < d) s.list[tid] = max(s.list[tid], s.list[tid + d]);
        __syncthreads();
    }
    if (tid == 0) {
        int top = s.list[0];
        if (n_high > moved) top = max(top, lists.high[n_high - 1 - moved]);
        if (moved > 0) top = max(top, lists.free[moved - 1]);
        *a.top = top + 1;
        lists.head[0] = moved > 0 ? lists.high[n_high - moved] : 0x7fffffff;  // pages from here on have moved, but for held ones
    }
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

// A workgroup brings 16 KiB of K or V of a pair's page, and the first one of each its scales
constexpr int kChunk = 16384;
__global__ void __launch_bounds__(256) fa_cache_copy_kernel(Cache c, const int* src, const int* dst, unsigned chunks, long bytes, long scale_bytes) {
    const unsigned part = blockIdx.x % (2 * chunks), pair = blockIdx.x / (2 * chunks);
    const int from = src[pair], to = dst[pair];
    if ((unsigned)from >= (unsigned)c.n_pages || (unsigned)to >= (unsigned)c.n_pages || from == to) return;
    const bool v = part >= chunks;
    char* const pages = static_cast<char*>(v ? c.v : c.k);
    const long first = (long)(v ? part - chunks : part) * kChunk + threadIdx.x * 16;
    const char* x = pages + from * bytes;
    char* y = pages + to * bytes;
    i32x4 w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (first + i * 4096 < bytes) w[i] = __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(x + first + i * 4096));
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (first + i * 4096 < bytes) __builtin_nontemporal_store(w[i], reinterpret_cast<i32x4*>(y + first + i * 4096));
    if (scale_bytes > 0 && part % chunks == 0) {
        char* const scales = static_cast<char*>(v ? c.v_scales : c.k_scales);
        for (long i = threadIdx.x * 4; i < scale_bytes; i += 1024)
            *reinterpret_cast<int*>(scales + to * scale_bytes + i) = *reinterpret_cast<const int*>(scales + from * scale_bytes + i);
    }
}

int launched() { return hipGetLastError() == hipSuccess ? FA_OK : FA_ERR_LAUNCH; }

}  // namespace

size_t cache_pages_workspace_bytes(int B, int n_pages) { return sizeof(int) * (kHead + 3 * (size_t)n_pages + 2 * (size_t)B); }

int launch_cache_fork(const int* block_table, const int* lens, const int* parents, const int* held, int* new_table, int* new_lens, int* src,
                      int* dst, int* missing, void* workspace, int B, int B_new, int page_size, int n_pages, int max_pages, hipStream_t stream) {
    const ForkArgs a = {block_table, lens, parents, new_table, new_lens, src, dst, missing, workspace, B, B_new, {held, n_pages, max_pages, page_size}};
    const long total = (long)B_new * max_pages, each = kThreads * kPerThread;
    hipLaunchKernelGGL(fa_cache_fork_kernel, dim3((unsigned)(1 + (total + each - 1) / each)), dim3(kThreads), shared_bytes(n_pages, 1), stream, a);
    return launched();
}

int launch_cache_extend(int* block_table, const int* lens, const int* counts, const int* held, int* missing, void* workspace, int B, int T,
                        int page_size, int n_pages, int max_pages, hipStream_t stream) {
    const ExtendArgs a = {block_table, lens, counts, missing, workspace, B, T, {held, n_pages, max_pages, page_size}};
    hipLaunchKernelGGL(fa_cache_extend_kernel, dim3(1), dim3(kThreads), shared_bytes(n_pages, 1), stream, a);
    return launched();
}

int launch_cache_compact(const int* block_table, const int* held, int* new_table, int* src, int* dst, int* top, void* workspace, int B,
                         int moves, int n_pages, int max_pages, hipStream_t stream) {
    const CompactArgs a = {block_table, new_table, src, dst, top, workspace, B, moves, {held, n_pages, max_pages, 0}};
    hipLaunchKernelGGL(fa_cache_compact_kernel, dim3(1), dim3(kThreads), shared_bytes(n_pages, 2), stream, a);
    const int st = launched();
    if (st != FA_OK) return st;
    const long total = (long)B * max_pages;
    hipLaunchKernelGGL(fa_cache_renumber_kernel, dim3((unsigned)((total + 255) / 256)), dim3(256), 0, stream, a);
    return launched();
}

int launch_cache_copy(const Cache& cache, const int* src, const int* dst, int n, int d, hipStream_t stream) {
    const long rows = (long)cache.H_kv * cache.page_size;
    const long bytes = rows * (cache.dtype == FA_FP4_E2M1 ? d / 2 : cache.dtype == FA_FP8_E4M3 ? d : 2 * d);
    const long scale_bytes = rows * (cache.dtype == FA_FP4_E2M1 ? d / 32 : cache.dtype == FA_FP8_E4M3 ? 4 : 0);
    const long chunks = (bytes + kChunk - 1) / kChunk;
    if ((double)n * 2 * chunks * 256 >= 4294967296.0) return FA_ERR_LAUNCH;
    hipLaunchKernelGGL(fa_cache_copy_kernel, dim3((unsigned)(n * 2 * chunks)), dim3(256), 0, stream, cache, src, dst, (unsigned)chunks, bytes, scale_bytes);
    return launched();
}

}  // namespace fa
