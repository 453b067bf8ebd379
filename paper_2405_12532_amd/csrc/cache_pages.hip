// Pages of the cache: handed out, shared, given back.  The count of a page is how many rows of the table hold it; 0 is a free page, and the
// counts are all the state there is.  Pages are handed out from the lowest, in the order of the rows that ask, so that what a call
// does follows from the state alone; a call that finds too few changes nothing.  Everything a call decides is decided by one workgroup
// (limits: kMaxRows rows a call, kMaxSlots slots), which looks through the counts 16 per lane at a time and stops at the last page it needs.
// Bound: the latency of the launch and of that workgroup's dependent loads: room for a token each of 64 sequences 3 us, for 2048 pages 6 us, for 25000 of
// 54000 pages 23 us; a fork 4 to 6 us and its copy 3 to 5 us, a release 2 to 5 us, the table's part of a cut 9 us.
#include "cache_device.h"

namespace pyr {
namespace {

constexpr int kMaxRows = kMaxCacheRows, kMaxSlots = kMaxCacheSlots;
constexpr int kMaxWaves = 16, kEach = 16;   // wavefronts; pages that a lane looks at at a time

struct Shared {
    int32_t first[kMaxRows + 1];          // pages that the rows before a row ask for
    int32_t entry[kMaxRows];              // where a row's next page goes, as an entry of the table
    int32_t slot[kMaxRows], len[kMaxRows];      // of a row, as the call found them; slot -1: skipped
    union {
        uint32_t seen[kMaxSlots / 32];    // slots that a row names; then
        uint16_t free[kMaxWaves * 64 * kEach];      // the free pages of a look, from its first page on
    };
    int32_t waves[kMaxWaves];
    int32_t status;
};

// Exclusive sum over the wavefronts, of a number that is the same in all lanes of one; *total: the whole sum.
template <int kWaves>
__device__ __forceinline__ int scan_waves(Shared& s, int x, int* total) {
    const int wave = threadIdx.x >> 6;
    __syncthreads();                      // (s.waves may still be read)
    s.waves[wave] = x;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) before += s.waves[w];
        all += s.waves[w];
    }
    *total = all;
    return before;
}
template <int kWaves>
__device__ __forceinline__ int scan(Shared& s, int x, int* total) {
    const int sum = scan_wave(x);
    return scan_waves<kWaves>(s, __builtin_amdgcn_readlane(sum, 63), total) + sum - x;
}

// A slot that no other row of the call may name.
__device__ __forceinline__ bool claim(Shared& s, int slot) { return (atomicOr(&s.seen[slot >> 5], 1u << (slot & 31)) >> (slot & 31) & 1) == 0; }

template <int kWaves>
__device__ __forceinline__ void clear(Shared& s, const PoolView& c) {
    for (int i = threadIdx.x; i < (c.n_slots + 31) / 32; i += 64 * kWaves) s.seen[i] = 0;
    if (threadIdx.x == 0) s.status = 0;
    __syncthreads();
}

__device__ __forceinline__ void refuse(Shared& s, int status) { atomicMin(&s.status, status); }      // (the lowest of a call's codes is kept)

// need(i, entry) -> pages that row i asks for (their sum fits an int: n * max_pages does), the first of them to become that entry of the table.
// Returns the sum.
template <int kWaves, typename Need>
__device__ __forceinline__ int sum_needs(Shared& s, int n, Need need) {
    int all = 0;
    for (int base = 0; base < n; base += 64 * kWaves) {
        const int i = base + threadIdx.x;
        int total, entry = 0;
        const int before = scan<kWaves>(s, i < n ? need(i, &entry) : 0, &total);
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

// The counts of a look: a wavefront has 64 * kEach pages of it, a lane four neighbouring ones of each 256.  1 behind the last page.
constexpr int kQuads = kEach / 4;
struct Counts {
    int4 x[kQuads];
};
__device__ __forceinline__ int place_of(int quad) { return (threadIdx.x >> 6) * (64 * kEach) + quad * 256 + (threadIdx.x & 63) * 4; }
__device__ __forceinline__ Counts look(const PoolView& c, int base) {
    Counts y;
    const bool aligned = ((uintptr_t)c.refs & 15) == 0;
#pragma unroll
    for (int i = 0; i < kQuads; ++i) {
        const int p = base + place_of(i);
        y.x[i] = int4{1, 1, 1, 1};
        if (p >= c.n_pages) continue;
        if (aligned && p + 4 <= c.n_pages) y.x[i] = *(const int4*)(c.refs + p);
        else y.x[i] = int4{c.refs[p], p + 1 < c.n_pages ? c.refs[p + 1] : 1, p + 2 < c.n_pages ? c.refs[p + 2] : 1, p + 3 < c.n_pages ? c.refs[p + 3] : 1};
    }
    return y;
}

// The rows that get the ranks first, first + step ...: the last row that begins at or before each (searches of their own, side by side).
template <int kMany>
__device__ __forceinline__ void rows_of_ranks(const Shared& s, int n, int first, int step, int (&row)[kMany]) {
#pragma unroll
    for (int k = 0; k < kMany; ++k) row[k] = 0;
    int stride = 1;
    while (2 * stride < n) stride *= 2;
    for (; stride > 0; stride >>= 1) {
#pragma unroll
        for (int k = 0; k < kMany; ++k) {
            const int mid = row[k] + stride;
            if (mid < n && s.first[mid] <= first + k * step) row[k] = mid;
        }
    }
}

// The lowest `need` free pages go to the rows, with a count of one; counts, ahead: the first two looks, asked for beforehand.  Returns how many are
// lacking; then none is taken.  What a look finds is listed in LDS first, so that neighbouring lanes write neighbouring entries: a wavefront takes a
// row at a time where there are many rows of many pages (25000 pages of 200 rows 41 -> 23 us), else every lane looks for the row of its page
// (25000 of one row 11 us against 26).
template <int kWaves>
__device__ __forceinline__ int hand_out(Shared& s, const PoolView& c, int n, int need, Counts counts, Counts ahead) {
    constexpr int kThreads = 64 * kWaves, kMany = 4;
    const int lane = threadIdx.x & 63;
    int found = 0;
    for (int base = 0; base < c.n_pages && found < need; base += kThreads * kEach) {
        uint32_t free[kQuads];
        int rank[kQuads], of_wave = 0;
#pragma unroll
        for (int i = 0; i < kQuads; ++i) {
            const int4 x = counts.x[i];
            free[i] = (x.x == 0) | (x.y == 0) << 1 | (x.z == 0) << 2 | (x.w == 0) << 3;
            rank[i] = of_wave;
            if (__builtin_amdgcn_ballot_w64(free[i] != 0) == 0) continue;      // (most of a pool is in use)
            const int mine = __popc(free[i]), sum = scan_wave(mine);
            rank[i] += sum - mine;
            of_wave += __builtin_amdgcn_readlane(sum, 63);
        }
        counts = ahead;
        if (base + 2 * kThreads * kEach < c.n_pages) ahead = look(c, base + 2 * kThreads * kEach);
        int total;
        const int before = scan_waves<kWaves>(s, of_wave, &total);
#pragma unroll
        for (int i = 0; i < kQuads; ++i) {
            if (__builtin_amdgcn_ballot_w64(free[i] != 0) == 0) continue;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (free[i] >> k & 1) s.free[before + rank[i]++] = (uint16_t)(place_of(i) + k);
        }
        if (total == 0) continue;
        __syncthreads();
        const int taken = min(total, need - found);
        constexpr int kLong = 24;
        int ends[2] = {0, -1};
        if (taken >= kLong * kWaves) rows_of_ranks(s, n, found, taken - 1, ends);
        const int rows = ends[1] - ends[0] + 1;
        if (rows >= kWaves && taken >= kLong * rows) {
            for (int row = ends[0] + (threadIdx.x >> 6); row <= ends[1]; row += kWaves) {
                const int first = s.first[row], entry = s.entry[row] - first, last = min(s.first[row + 1], found + taken);
                for (int r = max(first, found) + lane; r < last; r += 64) {
                    const int page = base + s.free[r - found];
                    c.table[entry + r] = page;
                    c.refs[page] = 1;
                }
            }
        } else {
            for (int i = threadIdx.x; i < taken; i += kMany * kThreads) {
                int row[kMany];
                rows_of_ranks(s, n, found + i, kThreads, row);
#pragma unroll
                for (int k = 0; k < kMany; ++k) {
                    const int at = i + k * kThreads;
                    if (at < taken) {
                        const int page = base + s.free[at];
                        c.table[s.entry[row[k]] + (found + at - s.first[row[k]])] = page;
                        c.refs[page] = 1;
                    }
                }
            }
        }
        found += total;
    }
    if (found >= need) return 0;
    __syncthreads();
    for (int rank = threadIdx.x; rank < found; rank += kThreads) {
        int row[1];
        rows_of_ranks(s, n, rank, 0, row);
        int32_t* at = &c.table[s.entry[row[0]] + (rank - s.first[row[0]])];
        c.refs[*at] = 0;
        *at = -1;
    }
    __syncthreads();
    return need - found;
}

__device__ __forceinline__ int pages_of(const PoolView& c, int tokens) { return (int)(((int64_t)tokens + (1 << c.shift) - 1) >> c.shift); }

template <int kWaves>
__global__ __launch_bounds__(64 * kWaves) void cache_reserve_kernel(PoolView c, const int32_t* __restrict__ slots, const int32_t* __restrict__ n_new, int n,
                                                                 int32_t* __restrict__ start, int32_t* __restrict__ status) {
    constexpr int kThreads = 64 * kWaves;
    __shared__ Shared s;
    const Counts counts = look(c, 0), ahead = look(c, kThreads * kEach);
    clear<kWaves>(s, c);
    const int64_t most = (int64_t)c.max_pages << c.shift;
    auto need = [&](int i, int* entry) -> int {
        const int slot = slots[i], more = n_new[i];
        s.slot[i] = -1;
        if (slot == -1) return 0;
        if (slot < 0 || slot >= c.n_slots) {
            refuse(s, PYR_CACHE_BAD_SLOT);
            return 0;
        }
        if (!claim(s, slot)) refuse(s, PYR_CACHE_BAD_SLOT);
        const int old = cache_len(c, slot);
        if (more < 0 || old + (int64_t)more > most) {
            refuse(s, PYR_CACHE_BAD_COUNT);
            return 0;
        }
        s.slot[i] = slot;
        s.len[i] = old;
        *entry = slot * c.max_pages + pages_of(c, old);
        return pages_of(c, old + more) - pages_of(c, old);
    };
    const int all = sum_needs<kWaves>(s, n, need);
    int state = s.status;
    if (state == 0) state = hand_out<kWaves>(s, c, n, all, counts, ahead);
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const int slot = s.slot[i];
        start[i] = slot >= 0 && state == 0 ? s.len[i] : -1;
        if (slot >= 0 && state == 0) c.lens[slot] = s.len[i] + n_new[i];
    }
    if (threadIdx.x == 0) *status = state;
}

// A child's row: the last page of a parent that is not full gets a page of its own here; the rest is cache_fork_copy_kernel's.
template <int kWaves>
__global__ __launch_bounds__(64 * kWaves) void cache_fork_kernel(PoolView c, const int32_t* __restrict__ parents, const int32_t* __restrict__ children, int n,
                                                              int32_t* __restrict__ status) {
    constexpr int kThreads = 64 * kWaves;
    __shared__ Shared s;
    const Counts counts = look(c, 0), ahead = look(c, kThreads * kEach);
    clear<kWaves>(s, c);
    const int part = (1 << c.shift) - 1;
    int mine = -1;                        // the parent of this thread's first row
    auto need = [&](int i, int* entry) -> int {
        const int parent = parents[i], child = children[i];
        s.slot[i] = -1;
        if (i == threadIdx.x) mine = parent;
        if (parent == -1 && child == -1) return 0;
        if (parent < 0 || parent >= c.n_slots || child < 0 || child >= c.n_slots) {
            refuse(s, PYR_CACHE_BAD_SLOT);
            return 0;
        }
        const int len = cache_len(c, parent), held = c.lens[child];
        if (held != 0 || !claim(s, child)) {
            refuse(s, PYR_CACHE_BAD_SLOT);
            return 0;
        }
        s.slot[i] = child;
        s.len[i] = len;
        *entry = child * c.max_pages + (len >> c.shift);
        return (len & part) != 0 ? 1 : 0;
    };
    const int all = sum_needs<kWaves>(s, n, need);
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const int parent = i < kThreads ? mine : parents[i];
        if (parent >= 0 && parent < c.n_slots && (s.seen[parent >> 5] >> (parent & 31) & 1) != 0) refuse(s, PYR_CACHE_BAD_SLOT);
    }
    __syncthreads();
    int state = s.status;
    if (state == 0) state = hand_out<kWaves>(s, c, n, all, counts, ahead);
    for (int i = threadIdx.x; i < n; i += kThreads)
        if (state == 0 && s.slot[i] >= 0) c.lens[s.slot[i]] = s.len[i];
    if (threadIdx.x == 0) *status = state;
}

// The full pages are shared, the tiles in use of the last one are copied.  grid: (n, heads); the first head's workgroup does the row too.
__global__ __launch_bounds__(256) void cache_fork_copy_kernel(PoolView c, const int32_t* __restrict__ parents, const int32_t* __restrict__ children,
                                                              const int32_t* __restrict__ status, int tile_chunks) {
    const int state = *status, parent = parents[blockIdx.x], child = children[blockIdx.x];
    if (state != 0 || parent < 0) return;
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
    const int chunks = tiles * tile_chunks;                       // 16 bytes each
    const int64_t head_chunks = (int64_t)tile_chunks << (c.shift - 5);
    const u32x4* a = (const u32x4*)c.pages + ((int64_t)src * c.n_kv_heads + blockIdx.y) * head_chunks;
    u32x4* b = (u32x4*)c.pages + ((int64_t)dst * c.n_kv_heads + blockIdx.y) * head_chunks;
    constexpr int kMany = 4;
    for (int i = threadIdx.x; i < chunks; i += kMany * 256) {
        u32x4 x[kMany];
#pragma unroll
        for (int k = 0; k < kMany; ++k)
            if (i + 256 * k < chunks) x[k] = a[i + 256 * k];
#pragma unroll
        for (int k = 0; k < kMany; ++k)
            if (i + 256 * k < chunks) b[i + 256 * k] = x[k];
    }
}

// A slot named twice is given back once, by the workgroup that takes its length.
__global__ __launch_bounds__(256) void cache_release_kernel(PoolView c, const int32_t* __restrict__ slots) {
    __shared__ int len;
    const int slot = cache_slot(c, slots, blockIdx.x);
    if (slot < 0) return;
    int32_t* row = c.table + (int64_t)slot * c.max_pages;
    int page = threadIdx.x < c.max_pages ? row[threadIdx.x] : -1;      // (asked for together with the length)
    if (threadIdx.x == 0) len = min(max(atomicExch(&c.lens[slot], 0), 0), c.max_pages << c.shift);
    __syncthreads();
    const int pages = pages_of(c, len);
    for (int i = threadIdx.x; i < pages; i += 256) {
        if (i >= 256) page = row[i];
        row[i] = -1;
        if (page >= 0 && page < c.n_pages) atomicSub(&c.refs[page], 1);
    }
}

// Rows cut to the lengths out_offsets[i + 1] - out_offsets[i], in fresh pages; what they were goes to old_rows [n, 1 + max_pages] (length, pages)
// for cache_move_kernel, and the old pages are given back (after the new ones were handed out, so that the two have none in common).
template <int kWaves>
__global__ __launch_bounds__(64 * kWaves) void cache_cut_kernel(PoolView c, const int32_t* __restrict__ slots, const int32_t* __restrict__ out_offsets, int n,
                                                             int n_list, int max_keep, int32_t* __restrict__ old_rows, int32_t* __restrict__ status) {
    constexpr int kThreads = 64 * kWaves;
    __shared__ Shared s;
    const Counts counts = look(c, 0), ahead = look(c, kThreads * kEach);
    clear<kWaves>(s, c);
    const int64_t most = min((int64_t)max_keep, (int64_t)c.max_pages << c.shift);
    auto need = [&](int i, int* entry) -> int {
        const int slot = slots[i], at = out_offsets[i], to = out_offsets[i + 1];
        s.slot[i] = -1;
        if (slot == -1) return 0;
        if (slot < 0 || slot >= c.n_slots) {
            refuse(s, PYR_CACHE_BAD_SLOT);
            return 0;
        }
        if (!claim(s, slot)) refuse(s, PYR_CACHE_BAD_SLOT);
        const int len = cache_len(c, slot);
        if (at < 0 || to < at || to > n_list || to - at > most) {
            refuse(s, PYR_CACHE_BAD_COUNT);
            return 0;
        }
        s.slot[i] = slot;
        s.len[i] = len;
        *entry = slot * c.max_pages;
        return pages_of(c, to - at);
    };
    const int all = sum_needs<kWaves>(s, n, need);
    int state = s.status;
    // the old rows first: the new pages take their place in the table
    if (state == 0) {
        const int stride = 1 + c.max_pages, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        for (int i = wave; i < n; i += kWaves) {
            if (s.slot[i] < 0) continue;
            const int pages = pages_of(c, s.len[i]);
            const int32_t* row = c.table + (int64_t)s.slot[i] * c.max_pages;
            int32_t* old = old_rows + (int64_t)i * stride;
            if (lane == 0) old[0] = s.len[i];
#pragma unroll 4
            for (int x = lane; x < pages; x += 64) old[1 + x] = row[x];
        }
        __syncthreads();
        state = hand_out<kWaves>(s, c, n, all, counts, ahead);
        __syncthreads();
        for (int i = wave; i < n; i += kWaves) {
            const int slot = s.slot[i];
            if (slot < 0) continue;
            const int pages = pages_of(c, s.len[i]), kept = s.first[i + 1] - s.first[i];
            int32_t* row = c.table + (int64_t)slot * c.max_pages;
            const int32_t* old = old_rows + (int64_t)i * stride;
#pragma unroll 4
            for (int x = lane; x < pages; x += 64) {
                const int page = old[1 + x];
                if (state != 0) row[x] = page;                             // (as it was)
                else {
                    if (page >= 0 && page < c.n_pages) atomicSub(&c.refs[page], 1);
                    if (x >= kept) row[x] = -1;
                }
            }
            if (lane == 0 && state == 0) c.lens[slot] = out_offsets[i + 1] - out_offsets[i];
        }
    }
    if (threadIdx.x == 0) *status = state;
}

}  // namespace

// A workgroup of four wavefronts where one look of it takes all counts: its barriers are shorter (a page of 1500 for one of 8 rows 4.3 us, sixteen wavefronts
// 5.3), though it takes longer over many pages (2048 of 4000 7.1 us, 5.9).
static bool few(const PoolView& c, int32_t n) { return n <= 256 && c.n_pages <= 4 * 64 * kEach; }

int launch_cache_reserve(const PoolView& c, const int32_t* slots, const int32_t* n_new, int32_t n, int32_t* start, int32_t* status, hipStream_t stream) {
    if (few(c, n)) hipLaunchKernelGGL(cache_reserve_kernel<4>, dim3(1), dim3(256), 0, stream, c, slots, n_new, n, start, status);
    else hipLaunchKernelGGL(cache_reserve_kernel<16>, dim3(1), dim3(1024), 0, stream, c, slots, n_new, n, start, status);
    return check_launch();
}

int launch_cache_fork(const PoolView& c, int32_t tile_bytes, const int32_t* parents, const int32_t* children, int32_t n, int32_t* status, hipStream_t stream) {
    if (few(c, n)) hipLaunchKernelGGL(cache_fork_kernel<4>, dim3(1), dim3(256), 0, stream, c, parents, children, n, status);
    else hipLaunchKernelGGL(cache_fork_kernel<16>, dim3(1), dim3(1024), 0, stream, c, parents, children, n, status);
    const int rc = check_launch();
    if (rc != PYR_OK || n == 0) return rc;
    // (tile_bytes 0: the first head's workgroup shares the full pages, and the last one is copied by the caller)
    hipLaunchKernelGGL(cache_fork_copy_kernel, dim3(n, tile_bytes > 0 ? c.n_kv_heads : 1), dim3(256), 0, stream, c, parents, children, (const int32_t*)status,
                       tile_bytes / 16);
    return check_launch();
}

int launch_cache_release(const PoolView& c, const int32_t* slots, int32_t n, hipStream_t stream) {
    if (n == 0) return PYR_OK;
    hipLaunchKernelGGL(cache_release_kernel, dim3(n), dim3(256), 0, stream, c, slots);
    return check_launch();
}

int launch_cache_cut(const PoolView& c, const int32_t* slots, const int32_t* out_offsets, int32_t n, int32_t n_list, int32_t max_keep, int32_t* old_rows,
                     int32_t* status, hipStream_t stream) {
    if (few(c, n)) hipLaunchKernelGGL(cache_cut_kernel<4>, dim3(1), dim3(256), 0, stream, c, slots, out_offsets, n, n_list, max_keep, old_rows, status);
    else hipLaunchKernelGGL(cache_cut_kernel<16>, dim3(1), dim3(1024), 0, stream, c, slots, out_offsets, n, n_list, max_keep, old_rows, status);
    return check_launch();
}

}  // namespace pyr
