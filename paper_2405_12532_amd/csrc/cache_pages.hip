// Pages of the cache: handed out, shared, given back.  The count of a page is how many rows of the table hold it; 0 is a free page, and the
// counts are all the state there is.  Pages are handed out from the lowest, in the order of the rows that ask, so that what a call
// does follows from the state alone; a call that finds too few changes nothing.  Everything a call decides is decided by one workgroup
// (limits: kMaxRows rows a call, kMaxSlots slots), which looks through the counts 16 per lane at a time and stops at the last page it needs.
// Bound: the latency of the launch and of that workgroup's dependent loads.
#include "cache_device.h"

namespace pyr {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kMaxRows = kMaxCacheRows, kMaxSlots = kMaxCacheSlots;

struct Shared {
    int32_t first[kMaxRows + 1];          // pages that the rows before a row ask for
    int32_t entry[kMaxRows];              // where a row's next page goes, as an entry of the table
    uint32_t seen[kMaxSlots / 32];        // slots that a row names
    int32_t waves[kWaves];
    int32_t status;
};

// Exclusive sum over the workgroup; *total: the whole sum.
__device__ __forceinline__ int scan(Shared& s, int x, int* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int sum = x;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int up = __shfl_up(sum, d);
        if (lane >= d) sum += up;
    }
    __syncthreads();                      // (s.waves may still be read)
    if (lane == 63) s.waves[wave] = sum;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) before += s.waves[w];
        all += s.waves[w];
    }
    *total = all;
    return before + sum - x;
}

// A slot that no other row of the call may name.
__device__ __forceinline__ bool claim(Shared& s, int slot) { return (atomicOr(&s.seen[slot >> 5], 1u << (slot & 31)) >> (slot & 31) & 1) == 0; }

__device__ __forceinline__ void clear(Shared& s, const CacheView& c) {
    for (int i = threadIdx.x; i < (c.n_slots + 31) / 32; i += kThreads) s.seen[i] = 0;
    if (threadIdx.x == 0) s.status = 0;
    __syncthreads();
}

__device__ __forceinline__ void refuse(Shared& s, int status) { atomicMin(&s.status, status); }      // (the lowest of a call's codes is kept)

// need(i, entry) -> pages that row i asks for (their sum fits an int: n * max_pages does), the first of them to become that entry of the table.
// Returns the sum.
template <typename Need>
__device__ __forceinline__ int sum_needs(Shared& s, int n, Need need) {
    int all = 0;
    for (int base = 0; base < n; base += kThreads) {
        const int i = base + threadIdx.x;
        int total, entry = 0;
        const int before = scan(s, i < n ? need(i, &entry) : 0, &total);
        if (i < n) {
            s.first[i] = all + before;
            s.entry[i] = entry;
        }
        all += total;
    }
    if (threadIdx.x == 0) s.first[n] = all;
    __syncthreads();
    return all;
}

__device__ __forceinline__ int row_of_rank(const Shared& s, int n, int rank) {      // the row that gets the rank-th page
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s.first[mid] <= rank) lo = mid;
        else hi = mid;
    }
    return lo;
}

// The lowest `need` free pages go to the rows, with a count of one.  Returns how many are lacking; then none is taken.
__device__ __forceinline__ int hand_out(Shared& s, const CacheView& c, int n, int need) {
    constexpr int kEach = 16;
    int found = 0;
    for (int base = 0; base < c.n_pages && found < need; base += kThreads * kEach) {
        const int p0 = base + threadIdx.x * kEach;
        uint32_t free = 0;
        if (p0 + kEach <= c.n_pages && ((uintptr_t)c.refs & 15) == 0) {
            int4 x[kEach / 4];
#pragma unroll
            for (int i = 0; i < kEach / 4; ++i) x[i] = *(const int4*)(c.refs + p0 + 4 * i);
#pragma unroll
            for (int i = 0; i < kEach / 4; ++i)
                free |= (uint32_t)((x[i].x == 0) | (x[i].y == 0) << 1 | (x[i].z == 0) << 2 | (x[i].w == 0) << 3) << (4 * i);
        } else {
            for (int i = 0; i < kEach; ++i)
                if (p0 + i < c.n_pages && c.refs[p0 + i] == 0) free |= 1u << i;
        }
        int total;
        int rank = found + scan(s, __popc(free), &total);
        if (free != 0 && rank < need) {
            int row = row_of_rank(s, n, rank);
            for (; free != 0 && rank < need; free &= free - 1, ++rank) {
                while (s.first[row + 1] <= rank) ++row;
                const int page = p0 + __ffs(free) - 1;
                c.table[s.entry[row] + (rank - s.first[row])] = page;
                c.refs[page] = 1;
            }
        }
        found += total;
    }
    if (found >= need) return 0;
    __syncthreads();
    for (int rank = threadIdx.x; rank < found; rank += kThreads) {
        const int row = row_of_rank(s, n, rank);
        int32_t* at = &c.table[s.entry[row] + (rank - s.first[row])];
        c.refs[*at] = 0;
        *at = -1;
    }
    __syncthreads();
    return need - found;
}

__device__ __forceinline__ int pages_of(const CacheView& c, int tokens) { return (int)(((int64_t)tokens + (1 << c.shift) - 1) >> c.shift); }

__global__ __launch_bounds__(kThreads) void cache_reserve_kernel(CacheView c, const int32_t* __restrict__ slots, const int32_t* __restrict__ n_new, int n,
                                                                 int32_t* __restrict__ start, int32_t* __restrict__ status) {
    __shared__ Shared s;
    clear(s, c);
    const int64_t most = (int64_t)c.max_pages << c.shift;
    auto need = [&](int i, int* entry) -> int {
        const int slot = slots[i];
        if (slot == -1) return 0;
        if (slot < 0 || slot >= c.n_slots) {
            refuse(s, PYR_CACHE_BAD_SLOT);
            return 0;
        }
        if (!claim(s, slot)) refuse(s, PYR_CACHE_BAD_SLOT);
        const int old = cache_len(c, slot), more = n_new[i];
        if (more < 0 || old + (int64_t)more > most) {
            refuse(s, PYR_CACHE_BAD_COUNT);
            return 0;
        }
        *entry = slot * c.max_pages + pages_of(c, old);
        return pages_of(c, old + more) - pages_of(c, old);
    };
    const int all = sum_needs(s, n, need);
    int state = s.status;
    if (state == 0) state = hand_out(s, c, n, all);
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const int slot = slots[i];
        const int old = slot >= 0 && state == 0 ? cache_len(c, slot) : -1;
        start[i] = old;
        if (old >= 0) c.lens[slot] = old + n_new[i];
    }
    if (threadIdx.x == 0) *status = state;
}

// A child's row: the last page of a parent that is not full gets a page of its own here; the rest is cache_fork_copy_kernel's.
__global__ __launch_bounds__(kThreads) void cache_fork_kernel(CacheView c, const int32_t* __restrict__ parents, const int32_t* __restrict__ children, int n,
                                                              int32_t* __restrict__ status) {
    __shared__ Shared s;
    clear(s, c);
    const int part = (1 << c.shift) - 1;
    auto need = [&](int i, int* entry) -> int {
        const int parent = parents[i], child = children[i];
        if (parent == -1 && child == -1) return 0;
        if (parent < 0 || parent >= c.n_slots || child < 0 || child >= c.n_slots || c.lens[child] != 0 || !claim(s, child)) {
            refuse(s, PYR_CACHE_BAD_SLOT);
            return 0;
        }
        const int len = cache_len(c, parent);
        *entry = child * c.max_pages + (len >> c.shift);
        return (len & part) != 0 ? 1 : 0;
    };
    const int all = sum_needs(s, n, need);
    for (int i = threadIdx.x; i < n; i += kThreads)
        if (parents[i] >= 0 && parents[i] < c.n_slots && (s.seen[parents[i] >> 5] >> (parents[i] & 31) & 1) != 0) refuse(s, PYR_CACHE_BAD_SLOT);
    __syncthreads();
    int state = s.status;
    if (state == 0) state = hand_out(s, c, n, all);
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kThreads)
        if (state == 0 && children[i] >= 0) c.lens[children[i]] = cache_len(c, parents[i]);
    if (threadIdx.x == 0) *status = state;
}

// The full pages are shared, the tiles in use of the last one are copied.  grid: (n, parts of a page); the first part does the rows too.
__global__ __launch_bounds__(256) void cache_fork_copy_kernel(CacheView c, const int32_t* __restrict__ parents, const int32_t* __restrict__ children,
                                                              const int32_t* __restrict__ status, int tile_chunks, int heads_of_part) {
    if (*status != 0) return;
    const int parent = parents[blockIdx.x], child = children[blockIdx.x];
    if (parent < 0) return;
    const int len = cache_len(c, parent), full = len >> c.shift;
    const int32_t* from = c.table + (int64_t)parent * c.max_pages;
    int32_t* to = c.table + (int64_t)child * c.max_pages;
    if (blockIdx.y == 0) {
        for (int i = threadIdx.x; i < full; i += 256) {
            const int page = from[i];
            to[i] = page;
            if (page >= 0 && page < c.n_pages) atomicAdd(&c.refs[page], 1);
        }
    }
    const int tiles = ((len & ((1 << c.shift) - 1)) + 31) >> 5;
    if (tiles == 0) return;
    const int src = from[full], dst = to[full];
    if (src < 0 || src >= c.n_pages || dst < 0 || dst >= c.n_pages) return;
    const int head0 = blockIdx.y * heads_of_part, heads = min(heads_of_part, c.n_kv_heads - head0);
    const int chunks = tiles * tile_chunks;                       // 16 bytes each, of a head
    const int64_t head_chunks = (int64_t)tile_chunks << (c.shift - 5);
    const u32x4* a = (const u32x4*)c.pages + ((int64_t)src * c.n_kv_heads + head0) * head_chunks;
    u32x4* b = (u32x4*)c.pages + ((int64_t)dst * c.n_kv_heads + head0) * head_chunks;
    for (int h = 0; h < heads; ++h)
        for (int i = threadIdx.x; i < chunks; i += 256) b[h * head_chunks + i] = a[h * head_chunks + i];
}

// A slot named twice is given back once: a page goes with its entry.
__global__ __launch_bounds__(256) void cache_release_kernel(CacheView c, const int32_t* __restrict__ slots) {
    const int slot = cache_slot(c, slots, blockIdx.x);
    if (slot < 0) return;
    const int pages = pages_of(c, cache_len(c, slot));
    int32_t* row = c.table + (int64_t)slot * c.max_pages;
    for (int i = threadIdx.x; i < pages; i += 256) {
        const int page = atomicExch(&row[i], -1);
        if (page >= 0 && page < c.n_pages) atomicSub(&c.refs[page], 1);
    }
    __syncthreads();
    if (threadIdx.x == 0) c.lens[slot] = 0;
}

// Rows cut to the lengths out_offsets[i + 1] - out_offsets[i], in fresh pages; what they were goes to old_rows [n, 1 + max_pages] (length, pages)
// for cache_move_kernel, and the old pages are given back (after the new ones were handed out, so that the two have none in common).
__global__ __launch_bounds__(kThreads) void cache_cut_kernel(CacheView c, const int32_t* __restrict__ slots, const int32_t* __restrict__ out_offsets, int n,
                                                             int n_list, int max_keep, int32_t* __restrict__ old_rows, int32_t* __restrict__ status) {
    __shared__ Shared s;
    clear(s, c);
    const int64_t most = min((int64_t)max_keep, (int64_t)c.max_pages << c.shift);
    auto need = [&](int i, int* entry) -> int {
        const int slot = slots[i];
        if (slot == -1) return 0;
        if (slot < 0 || slot >= c.n_slots) {
            refuse(s, PYR_CACHE_BAD_SLOT);
            return 0;
        }
        if (!claim(s, slot)) refuse(s, PYR_CACHE_BAD_SLOT);
        const int at = out_offsets[i], to = out_offsets[i + 1];
        if (at < 0 || to < at || to > n_list || to - at > most) {
            refuse(s, PYR_CACHE_BAD_COUNT);
            return 0;
        }
        *entry = slot * c.max_pages;
        return pages_of(c, to - at);
    };
    const int all = sum_needs(s, n, need);
    int state = s.status;
    // the old rows first: the new pages take their place in the table
    if (state == 0) {
        const int stride = 1 + c.max_pages, entries = n * stride;
        for (int x = threadIdx.x; x < entries; x += kThreads) {
            const int i = x / stride, at = x - i * stride, slot = slots[i];
            if (slot < 0) continue;
            const int len = cache_len(c, slot);
            old_rows[x] = at == 0 ? len : at <= pages_of(c, len) ? c.table[(int64_t)slot * c.max_pages + at - 1] : -1;
        }
        __syncthreads();
        state = hand_out(s, c, n, all);
        __syncthreads();
        for (int x = threadIdx.x; x < entries; x += kThreads) {
            const int i = x / stride, at = x - i * stride, slot = slots[i];
            if (slot < 0) continue;
            const int keep = out_offsets[i + 1] - out_offsets[i], old = old_rows[x];
            if (at == 0) {
                if (state == 0) c.lens[slot] = keep;
                continue;
            }
            if (at > pages_of(c, old_rows[x - at])) continue;
            int32_t* entry = c.table + (int64_t)slot * c.max_pages + at - 1;
            if (state != 0) *entry = old;                                  // (as it was)
            else {
                if (old >= 0 && old < c.n_pages) atomicSub(&c.refs[old], 1);
                if (at > pages_of(c, keep)) *entry = -1;
            }
        }
    }
    if (threadIdx.x == 0) *status = state;
}

}  // namespace

int launch_cache_reserve(const CacheView& c, const int32_t* slots, const int32_t* n_new, int32_t n, int32_t* start, int32_t* status, hipStream_t stream) {
    hipLaunchKernelGGL(cache_reserve_kernel, dim3(1), dim3(kThreads), 0, stream, c, slots, n_new, n, start, status);
    return check_launch();
}

int launch_cache_fork(const CacheView& c, int32_t head_dim, const int32_t* parents, const int32_t* children, int32_t n, int32_t* status, hipStream_t stream) {
    hipLaunchKernelGGL(cache_fork_kernel, dim3(1), dim3(kThreads), 0, stream, c, parents, children, n, status);
    int rc = check_launch();
    if (rc != PYR_OK || n == 0) return rc;
    const int heads_of_part = 1;
    hipLaunchKernelGGL(cache_fork_copy_kernel, dim3(n, (c.n_kv_heads + heads_of_part - 1) / heads_of_part), dim3(256), 0, stream, c, parents, children,
                       (const int32_t*)status, 34 * head_dim / 16, heads_of_part);
    return check_launch();
}

int launch_cache_release(const CacheView& c, const int32_t* slots, int32_t n, hipStream_t stream) {
    if (n == 0) return PYR_OK;
    hipLaunchKernelGGL(cache_release_kernel, dim3(n), dim3(256), 0, stream, c, slots);
    return check_launch();
}

int launch_cache_cut(const CacheView& c, const int32_t* slots, const int32_t* out_offsets, int32_t n, int32_t n_list, int32_t max_keep, int32_t* old_rows,
                     int32_t* status, hipStream_t stream) {
    hipLaunchKernelGGL(cache_cut_kernel, dim3(1), dim3(kThreads), 0, stream, c, slots, out_offsets, n, n_list, max_keep, old_rows, status);
    return check_launch();
}

}  // namespace pyr
