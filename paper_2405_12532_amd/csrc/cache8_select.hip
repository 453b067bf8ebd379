// The blocks of a cache held in 8 bits that a token attends to, for every KV head: the first ones, the last ones, and those in between whose bounds
// promise the largest logits (Section 3.2's observation, that few tokens carry the attention, used at every step without the others being given up).
//
// The logit of a query with any K between a block's smallest lo and largest hi is at most sum_c max(q_c hi_c, q_c lo_c) = [max(q, 0); min(q, 0)] . [hi; lo],
// one product of twice the channels.  lo and hi are whole numbers times the block's power, and q is rounded to whole numbers from -127 to 127 times a power
// of its own, so that the product is one of 8-bit integers (v_mfma_i32_16x16x64_i8) and a score, a whole number below 2^22 times a power of two,
// is exact in fp32: which blocks are chosen does not depend on the order of a sum.  A block's score is the largest of the group's query heads.
// Bound: reading the bounds where there are many (64 x 2048 tokens on 32 heads: 9.7 us for 34 MB, 3.6 TB/s with a launch's 2 us in it), the latency of dependent
// loads where there are few (1 x 2048 on 8 heads of 64: 3.9 us; 1 x 131072 on 8 heads: 5.1 for the scores, of 9.6 MB, 7.0 for the choice, which eight workgroups make).
#include "cache8_device.h"

namespace pyr {
namespace {

typedef __attribute__((ext_vector_type(4))) int i32x4;

struct SelectArgs {
    CacheView c;
    const uint16_t* q;
    const int32_t* slots;
    int32_t* blocks;
    uint32_t* keys;                               // [units, max_blocks] or NULL: in LDS
    int32_t n_tokens, n_q_heads, max_blocks, n_first, n_recent, n_best, chunk;
};

__device__ __forceinline__ float max_of_groups(float x) {      // over the lanes with the same lane & 15
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Scores as numbers that compare like them.
__device__ __forceinline__ uint32_t key_of(float score) {
    const uint32_t bits = __float_as_uint(score);
    return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}

// A unit: a token of a sequence and a KV head.  What its tokens and blocks are.
struct Unit {
    int32_t slot, len, head, row;                 // as the device has the length; row of q's tokens
    int32_t count, low, high;                     // blocks it sees; candidates low .. high - 1 (low is n_first where there are some)
};
__device__ __forceinline__ Unit unit_of(const SelectArgs& a, int unit) {
    Unit u;
    const int hkv = a.c.n_kv_heads;
    u.row = unit / hkv;
    u.head = unit - u.row * hkv;
    const int b = u.row / a.n_tokens;
    u.slot = cache_slot(a.c, a.slots, b);
    u.len = a.c.lens[max(u.slot, 0)];
    return u;
}
// The rest, for which the length has to be there.
__device__ __forceinline__ void see(const SelectArgs& a, Unit& u) {
    const int token = u.row % a.n_tokens, len = u.slot < 0 ? 0 : min(max(u.len, 0), a.c.max_pages << a.c.shift);
    u.count = (max(len - a.n_tokens + 1 + token, 0) + 31) >> 5;
    u.low = min(a.n_first, u.count);
    u.high = max(u.low, min(u.count - a.n_recent, a.max_blocks));
}

// 16 query heads of the group as operands of the products, lane 16 j + t: bytes 16 j .. of head t's.
template <int D>
struct Queries {
    static constexpr int kHalf = D / 64, kNone = -1000;
    u32x4 words[kHalf][2];
    i32x4 whole[2 * kHalf];                       // max(u, 0), then min(u, 0)
    int power[4];                                 // of heads 4 j + x; kNone: no query head

    __device__ __forceinline__ void load(const uint16_t* q, int head, int g, int lane) {
#pragma unroll
        for (int s = 0; s < kHalf; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                words[s][h] = head + (lane & 15) < g ? *(const u32x4*)(q + (int64_t)(head + (lane & 15)) * D + 64 * s + 16 * (lane >> 4) + 8 * h) : u32x4{};
    }
    __device__ __forceinline__ void round(int head, int g, int lane) {
        uint32_t pair = 0;
#pragma unroll
        for (int s = 0; s < kHalf; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) pair = max_u16(pair, words[s][h][e] & 0x7fff7fffu);
        float top = __uint_as_float(max(pair & 0xffff0000u, pair << 16));
        if (__builtin_amdgcn_ballot_w64(!(top < INFINITY)) != 0) {      // NaN counts as 0, an infinity as what is largest (below); neither as a magnitude
            top = 0.f;
#pragma unroll
            for (int s = 0; s < kHalf; ++s)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint32_t& w = reinterpret_cast<uint32_t*>(&words[s][h])[e];
                        const float x = __uint_as_float(w << 16), y = __uint_as_float(w & 0xffff0000u);
                        if (x != x) w &= 0xffff0000u;
                        if (y != y) w &= 0xffffu;
                        top = fmaxf(top, fmaxf(fabsf(x) < INFINITY ? fabsf(x) : 0.f, fabsf(y) < INFINITY ? fabsf(y) : 0.f));
                    }
        }
        top = max_of_groups(top);
        const uint32_t bits = __float_as_uint(top);
        const int e = min(max((int)(bits >> 23) - 127 - 6 + ((bits & 0x7fffff) > 0x7e0000 ? 1 : 0), -100), 122);
        const float by = __uint_as_float((uint32_t)(127 - e) << 23);
        // adding 1.5 * 2^23 rounds to a whole number (ties to even) and leaves its byte lowest
        auto byte_of = [&](float x) { return __float_as_uint(__builtin_amdgcn_fmed3f(x * by, -127.f, 127.f) + 12582912.f); };
#pragma unroll
        for (int s = 0; s < kHalf; ++s)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t b[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t both = words[s][w >> 1][2 * (w & 1) + (i >> 1)];
                    b[i] = byte_of(__uint_as_float(i & 1 ? both & 0xffff0000u : both << 16));
                }
                const uint32_t bytes = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u), __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), 0x05040100u);
                const uint32_t below = (bytes >> 7 & 0x01010101u) * 255u;      // of numbers below 0
                whole[s][w] = (int)(bytes & ~below);
                whole[kHalf + s][w] = (int)(bytes & below);
            }
#pragma unroll
        for (int x = 0; x < 4; ++x) power[x] = __shfl(head + (lane & 15) < g ? e : kNone, 4 * (lane >> 4) + x);
    }
};

// The page of a block, asked for before it is known whether it is there (0 where the table names none of the pool: the attention makes NaN of it).
__device__ __forceinline__ int page_of(const SelectArgs& a, const int32_t* row_pages, int block) {
    const int page = row_pages[min(block >> (a.c.shift - 5), a.c.max_pages - 1)];
    return page < 0 || page >= a.c.n_pages ? 0 : page;
}

// The keys of 64 blocks, lane l: that of block base + l (of end - 1 from there on); page: of its block.
template <int D>
__device__ __forceinline__ uint32_t keys_of(const SelectArgs& a, const Unit& u, Queries<D>& w, const uint16_t* q, int g, int base, int end, int page) {
    constexpr int kHalf = D / 64;
    const int lane = threadIdx.x & 63, j = lane >> 4, t = lane & 15;
    const int block = min(base + lane, end - 1);
    i32x4 bounds[4][2 * kHalf];
#pragma unroll
    for (int s = 0; s < 4; ++s) {                           // (all loads in flight)
        const int n = __shfl(block, 16 * s + t), p = __shfl(page, 16 * s + t);
        const i32x4* from = (const i32x4*)Page8<D>(a.c, p).bounds(u.head, n) + j;
#pragma unroll
        for (int i = 0; i < 2 * kHalf; ++i) bounds[s][i] = from[4 * i];
    }
    const int block_power = (int)(*Page8<D>(a.c, page).powers(u.head, block) & 255) - 127;
    int of_block[4];
    float best[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        of_block[s] = __shfl(block_power, 16 * s + t) + 2;
        best[s] = -INFINITY;
    }
#pragma unroll 1
    for (int first = 0; first < g; first += 16) {
        if (g > 16) {
            w.load(q, first, g, lane);
            w.round(first, g, lane);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            i32x4 d = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < 2 * kHalf; ++i) d = __builtin_amdgcn_mfma_i32_16x16x64_i8(w.whole[i], bounds[s][i], d, 0, 0, 0);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int e = min(max(w.power[x] + of_block[s], -120), 100);
                const float score = (float)d[x] * __uint_as_float((uint32_t)(127 + e) << 23);
                best[s] = fmaxf(best[s], w.power[x] == Queries<D>::kNone ? -INFINITY : score);
            }
        }
    }
    uint32_t key = 0;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const uint32_t y = key_of(max_of_groups(best[s]));
        if (j == s) key = y;
    }
    return key;
}

// grid: (units, chunks of candidates), a wavefront each: keys to memory
template <int D>
__global__ __launch_bounds__(64) void cache8_score_kernel(SelectArgs a) {
    const int lane = threadIdx.x, g = a.n_q_heads / a.c.n_kv_heads;
    Unit u = unit_of(a, blockIdx.x);
    const int32_t* row_pages = a.c.table + (int64_t)max(u.slot, 0) * a.c.max_pages;
    const uint16_t* q = a.q + ((int64_t)u.row * a.n_q_heads + u.head * g) * D;
    uint32_t* keys = a.keys + (int64_t)blockIdx.x * a.max_blocks;
    const int begin = (int)min((int64_t)a.n_first + (int64_t)blockIdx.y * a.chunk, (int64_t)a.max_blocks);      // (u.low, where there are candidates)
    Queries<D> w;
    int page = page_of(a, row_pages, begin + lane);
    w.load(q, 0, g, lane);
    see(a, u);
    if (u.high - u.low <= a.n_best) return;
    const int end = min(u.high, begin + a.chunk);
    if (begin >= end) return;
    w.round(0, g, lane);
    for (int base = begin; base < end; base += 64) {
        const uint32_t key = keys_of<D>(a, u, w, q, g, base, end, page);
        if (base + 64 < end) page = page_of(a, row_pages, base + 64 + lane);
        if (base + lane < end) keys[base + lane] = key;
    }
}

// What every list has: the first blocks, the last ones, -1 behind them, and all in between where n_best takes them.  true: that is all.
template <int kThreads>
__device__ __forceinline__ bool sure_blocks(const SelectArgs& a, const Unit& u, int32_t* out) {
    const int width = a.n_first + a.n_recent + a.n_best, candidates = u.high - u.low, chosen = min(candidates, a.n_best);
    const int tail = max(u.low, u.count - a.n_recent), all = u.low + chosen + (u.count - tail);
    const bool done = candidates <= a.n_best || a.n_best == 0;
    for (int i = threadIdx.x; i < width; i += kThreads) {
        const int in_between = i - u.low;
        if (in_between < 0) out[i] = i;
        else if (i >= all) out[i] = -1;
        else if (in_between >= chosen) out[i] = tail + in_between - chosen;
        else if (done) out[i] = i;
    }
    return done;
}

__device__ __forceinline__ uint64_t lanes_below() { return (1ull << (threadIdx.x & 63)) - 1; }

// The n_best-th largest of one wavefront's keys (0: none; no score's key is 0): all above limit are taken, and of those equal to it equal_left.
struct Limit {
    uint32_t limit;
    int equal_left;
};
// One key a lane: bit by bit, from counts of the keys that are at least the prefix with the bit set.
__device__ __forceinline__ Limit limit_of(const SelectArgs& a, uint32_t key) {
    auto count = [](bool test) { return __builtin_popcountll(__builtin_amdgcn_ballot_w64(test)); };
    uint32_t prefix = 0;
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t tried = prefix | 1u << bit;
        const int n = count(key >= tried);
        if (n >= a.n_best) prefix = tried;
        if (n == a.n_best) break;                             // (the others are below)
    }
    return {prefix, a.n_best - count(key > prefix)};
}
// Several: from counts of the keys in 256 parts of the range that it lies in (in LDS, the wavefront's own); 8 x 512 blocks 7.7 us, bit by bit 8.6
template <int kPer>
__device__ __forceinline__ Limit limit_of(const SelectArgs& a, const uint32_t (&keys)[kPer], uint32_t* counts) {
    constexpr int kBits = 8;
    const int lane = threadIdx.x & 63;
    auto meet = [] {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    uint32_t low = 0xffffffffu, high = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        low = min(low, keys[i] - 1);                          // (what is none is the largest)
        high = max(high, keys[i]);
    }
    low = within_wave(low, [](uint32_t x, uint32_t y) { return min(x, y); }) + 1;
    high = within_wave(high, [](uint32_t x, uint32_t y) { return max(x, y); });
    int wanted = a.n_best;                                    // so many of the keys from low to high, and all above
    for (int round = 0;; ++round) {
        const int shift = max(0, 32 - __clz((int)(high - low)) - kBits);
        *(u32x4*)&counts[4 * lane] = u32x4{};
        meet();
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (keys[i] >= low && keys[i] <= high) atomicAdd(&counts[(keys[i] - low) >> shift], 1u);
        meet();
        // lane l: keys in the four parts from 4 (63 - l) on, and above
        const u32x4 own = *(const u32x4*)&counts[4 * (63 - lane)];
        const int all = (int)(own[0] + own[1] + own[2] + own[3]), sum = scan_wave(all);
        const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(sum >= wanted));
        int above = __builtin_amdgcn_readlane(sum - all, at), n = 0, part = 4;
#pragma unroll
        for (int i = 3; i >= 0; --i) {
            if (above + n >= wanted) break;
            above += n;
            n = __builtin_amdgcn_readlane((int)own[i], at);
            part = i;
        }
        low += (uint32_t)(4 * (63 - at) + part) << shift;
        wanted -= above;
        if (shift == 0) return {low, wanted};
        if (n == wanted || round == 3) return {low - 1, 0};   // (32 bits are four rounds at most)
        high = min(high, low + ((1u << shift) - 1));
        meet();
    }
}

// The candidates of a unit that a list takes, by one wavefront that holds all keys: candidate low + 64 i + lane is key i of a lane.  In order: all above the n-th largest,
// and of those equal to it the first.
template <int kPer>
__device__ __forceinline__ void take_alone(const SelectArgs& a, const Unit& u, const uint32_t (&keys)[kPer], Limit l, int32_t* out) {
    int at = u.low;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const uint64_t equals = __builtin_amdgcn_ballot_w64(keys[i] == l.limit), aboves = __builtin_amdgcn_ballot_w64(keys[i] > l.limit);
        const int rank = __builtin_popcountll(equals & lanes_below());
        if (keys[i] > l.limit || (keys[i] == l.limit && rank < l.equal_left))
            out[at + __builtin_popcountll(aboves & lanes_below()) + min(rank, l.equal_left)] = u.low + 64 * i + (threadIdx.x & 63);
        const int taken = min(__builtin_popcountll(equals), l.equal_left);
        at += __builtin_popcountll(aboves) + taken;
        l.equal_left -= taken;
    }
}

// One workgroup a unit, a wavefront for 64 candidates; their keys meet in LDS, and the first wavefront takes.
template <int D, int kWaves>
__global__ __launch_bounds__(64 * kWaves, 4) void cache8_select_kernel(SelectArgs a) {
    __shared__ uint32_t held[kWaves == 1 ? 1 : kWaves][64];
    __shared__ __align__(16) uint32_t counts[kWaves == 1 ? 1 : 256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = a.n_q_heads / a.c.n_kv_heads;
    Unit u = unit_of(a, blockIdx.x);
    int32_t* out = a.blocks + (int64_t)blockIdx.x * (a.n_first + a.n_recent + a.n_best);
    const int32_t* row_pages = a.c.table + (int64_t)max(u.slot, 0) * a.c.max_pages;
    const uint16_t* q = a.q + ((int64_t)u.row * a.n_q_heads + u.head * g) * D;
    const int first = min(a.n_first, a.max_blocks) + 64 * wave;      // (u.low, where there are candidates)
    Queries<D> w;
    const int page = page_of(a, row_pages, first + lane);
    w.load(q, 0, g, lane);
    see(a, u);
    if (sure_blocks<64 * kWaves>(a, u, out)) return;
    uint32_t keys[kWaves] = {};
    if (first < u.high) {
        w.round(0, g, lane);
        keys[0] = keys_of<D>(a, u, w, q, g, first, u.high, page);
        if (first + lane >= u.high) keys[0] = 0;
    }
    if constexpr (kWaves > 1) {
        held[wave][lane] = keys[0];
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int i = 1; i < kWaves; ++i) keys[i] = held[i][lane];
        take_alone<kWaves>(a, u, keys, limit_of<kWaves>(a, keys, counts), out);
    } else {
        take_alone<kWaves>(a, u, keys, limit_of(a, keys[0]), out);
    }
}

// For many candidates, 4096 at a time: candidate low + 64 (wave + kWaves i) + lane is key i of a lane.  kScored: their keys are in memory, else they are worked out
// here, and there are no more than 4096.
// The n-th largest key is found from counts of the keys in as many equal parts of the range that it lies in as there are threads: scores are spread widely
// enough that two rounds mostly do, and few keys ask for the same counter.
template <int D, int kWaves, bool kScored>
__global__ __launch_bounds__(64 * kWaves) void cache8_select_many_kernel(SelectArgs a) {
    constexpr int kThreads = 64 * kWaves, kPer = 4096 / kThreads, kBits = kWaves == 16 ? 10 : 9;
    static_assert(kThreads == 1 << kBits && kPer * kWaves == 64, "");
    __shared__ uint32_t counts[kThreads], ends[2][kWaves], sums[kWaves], found[3], parts[2][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = a.n_q_heads / a.c.n_kv_heads;
    Unit u = unit_of(a, blockIdx.x);
    int32_t* out = a.blocks + (int64_t)blockIdx.x * (a.n_first + a.n_recent + a.n_best);
    const int first = min(a.n_first, a.max_blocks) + 64 * wave;
    uint32_t keys[kPer];                                      // of a pass over the candidates; 0: none
    const uint32_t* from = kScored ? a.keys + (int64_t)blockIdx.x * a.max_blocks : nullptr;
    auto fetch = [&](int base) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int n = base + first + kThreads * i + lane;
            keys[i] = n < u.high ? from[n] : 0;
        }
    };
    if constexpr (kScored) {
        see(a, u);
        fetch(0);
        if (sure_blocks<kThreads>(a, u, out)) return;
    } else {
        const int32_t* row_pages = a.c.table + (int64_t)max(u.slot, 0) * a.c.max_pages;
        const uint16_t* q = a.q + ((int64_t)u.row * a.n_q_heads + u.head * g) * D;
        Queries<D> w;
        int page = page_of(a, row_pages, first + lane);
        w.load(q, 0, g, lane);
        see(a, u);
        if (sure_blocks<kThreads>(a, u, out)) return;
        w.round(0, g, lane);
        // (through LDS, so that the code for a block is there once)
        __shared__ uint32_t held[kPer][kThreads];
#pragma unroll 1
        for (int i = 0; i < kPer; ++i) {
            const int base = first + kThreads * i, next = base + kThreads;
            uint32_t key = 0;
            if (base < u.high) {
                key = keys_of<D>(a, u, w, q, g, base, u.high, page);
                if (base + lane >= u.high) key = 0;
                if (i + 1 < kPer && next < u.high) page = page_of(a, row_pages, next + lane);
            }
            held[i][threadIdx.x] = key;
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) keys[i] = held[i][threadIdx.x];
    }
    const int passes = kScored ? (u.high - u.low + 4095) / 4096 : 1;
    auto each = [&](auto f) {                                 // over all keys that there are
        for (int pass = 0; pass < passes; ++pass) {
            if (passes > 1) fetch(4096 * pass);
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (keys[i] != 0) f(keys[i]);
        }
    };
    uint32_t low = 0xffffffffu, high = 0;
    each([&](uint32_t key) {
        low = min(low, key);
        high = max(high, key);
    });
    low = within_wave(low, [](uint32_t x, uint32_t y) { return min(x, y); });
    high = within_wave(high, [](uint32_t x, uint32_t y) { return max(x, y); });
    if (lane == 0) {
        ends[0][wave] = low;
        ends[1][wave] = high;
    }
    counts[threadIdx.x] = 0;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
        low = min(low, ends[0][v]);
        high = max(high, ends[1][v]);
    }
    uint32_t wanted = a.n_best, limit;                        // so many of the keys from low to high, and all above; all above limit are taken
    int equal_left;                                           // of those equal to it, so many
    for (int round = 0;; ++round) {
        const uint32_t range = high - low;
        const int shift = max(0, 32 - __clz((int)range) - kBits);      // (range 0: 32 leading zeros)
        each([&](uint32_t key) {
            if (key >= low && key <= high) atomicAdd(&counts[(key - low) >> shift], 1u);
        });
        __syncthreads();
        // thread i: keys in its part, the i-th from the top, and above
        const uint32_t own = counts[kThreads - 1 - threadIdx.x];
        uint32_t sum = scan_wave((int)own);
        if (lane == 63) sums[wave] = sum;
        __syncthreads();
#pragma unroll
        for (int v = 0; v < kWaves; ++v) sum += v < wave ? sums[v] : 0;
        if (sum >= wanted && sum - own < wanted) {
            found[0] = kThreads - 1 - threadIdx.x;
            found[1] = sum - own;
            found[2] = own;
        }
        counts[threadIdx.x] = 0;
        __syncthreads();
        low += found[0] << shift;
        wanted -= found[1];
        // (found is not written again before two more barriers; 32 bits are four rounds at most)
        if (shift == 0 || found[2] == wanted || round == 3) {
            limit = shift == 0 ? low : low - 1;
            equal_left = shift == 0 ? (int)wanted : 0;
            break;
        }
        high = min(high, low + ((1u << shift) - 1));
    }
    // in order: all above the limit, and of those equal to it the first
    int at = u.low;
    for (int pass = 0; pass < passes; ++pass) {
        if (passes > 1) fetch(4096 * pass);
        uint32_t* const s = parts[pass & 1];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const uint32_t n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(keys[i] == limit)) | __builtin_popcountll(__builtin_amdgcn_ballot_w64(keys[i] > limit)) << 16;
            if (lane == 0) s[kWaves * i + wave] = n;
        }
        __syncthreads();
        const uint32_t mine = s[lane];
        const uint32_t sum = scan_wave((int)mine);            // (4096 at most in either half)
        const uint32_t all = (uint32_t)__builtin_amdgcn_readlane((int)sum, 63);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const uint32_t before = (uint32_t)__builtin_amdgcn_readlane((int)(sum - mine), kWaves * i + wave);
            const uint64_t equals = __builtin_amdgcn_ballot_w64(keys[i] == limit), aboves = __builtin_amdgcn_ballot_w64(keys[i] > limit);
            const int rank = (int)(before & 0xffff) + __builtin_popcountll(equals & lanes_below());
            const int place = at + (int)(before >> 16) + __builtin_popcountll(aboves & lanes_below()) + min(rank, equal_left);
            if ((keys[i] > limit || (keys[i] == limit && rank < equal_left)) && place < u.low + a.n_best) out[place] = 4096 * pass + first + kThreads * i + lane;
        }
        const int taken = min((int)(all & 0xffff), equal_left);
        at += (int)(all >> 16) + taken;
        equal_left -= taken;
    }
}

constexpr int kAtOnce = 4096;                    // candidates whose keys a workgroup holds

template <int D>
void launch(const CacheSelect& x, const SelectArgs& a, unsigned units, hipStream_t stream) {
    const dim3 threads(64 * x.waves);
    if (x.chunks > 0) hipLaunchKernelGGL((cache8_select_many_kernel<D, 16, true>), dim3(units), threads, 0, stream, a);
    else if (x.max_blocks > 64 * x.waves) hipLaunchKernelGGL((cache8_select_many_kernel<D, 8, false>), dim3(units), threads, 0, stream, a);
    else if (x.waves == 1) hipLaunchKernelGGL((cache8_select_kernel<D, 1>), dim3(units), threads, 0, stream, a);
    else if (x.waves == 4) hipLaunchKernelGGL((cache8_select_kernel<D, 4>), dim3(units), threads, 0, stream, a);
    else if (x.waves == 8) hipLaunchKernelGGL((cache8_select_kernel<D, 8>), dim3(units), threads, 0, stream, a);
    else hipLaunchKernelGGL((cache8_select_kernel<D, 16>), dim3(units), threads, 0, stream, a);
}

}  // namespace

CacheSelect plan_cache8_select(int32_t n_seqs, int32_t n_tokens, int32_t n_kv_heads, int64_t max_len) {
    CacheSelect x{};
    const int64_t units = (int64_t)n_seqs * n_tokens * n_kv_heads, blocks = (max_len + 31) / 32;
    x.max_blocks = (int32_t)blocks;
    x.chunks = 0;
    // A wavefront for 64 blocks; more than 512 (1024 of few units) by eight in parts.  Measured, us, 1024 at once and by parts: 128 x 1024 blocks 13.4 and 15.1; 256 x 640 at 64
    // channels 8.8 and 10.8, but 768 x 640 29.6 and 27.8, 1600 x 750 52 and 43.
    x.waves = blocks <= 64 ? 1 : blocks <= 256 ? 4 : blocks > 512 && blocks <= 1024 && units <= 256 ? 16 : 8;
    // A unit's workgroup scores its blocks by itself unless they are many and the units leave compute units idle.  Measured, us, alone and with a launch for the scores,
    // units x blocks: 8 x 512 7.7 and 10.0, 8 x 1024 12.9 and 9.6, 64 x 640 10.4 and 11.3, 64 x 1024 13.6 and 12.2, 64 x 4096 38.2 and 23.5, 128 x 1024 13.4 and 14.3,
    // 128 x 2048 23.1 and 21.9, 128 x 4096 39.2 and 33.4, 256 x 1024 18.5 and 21.9, 768 x 640 27.9 and 32.8
    if (blocks > (units < 96 ? 512 : units < 192 ? 1536 : kAtOnce)) {
        // 64 candidates a wavefront; 256 (the same time there, 23.7 us for 64 x 4096) where the grid would grow large
        x.chunk = units * blocks <= 64 * 16384 ? 64 : 256;
        while ((blocks + x.chunk - 1) / x.chunk > 32768) x.chunk *= 2;
        x.chunks = (int32_t)((blocks + x.chunk - 1) / x.chunk);
        x.key_bytes = (size_t)units * blocks * sizeof(uint32_t);
        x.waves = 16;
    }
    return x;
}

int launch_cache8_select(const CacheSelect& x, const CacheView& c, int32_t head_dim, const void* q, const int32_t* slots, int32_t n_seqs, int32_t n_tokens,
                         int32_t n_q_heads, int32_t n_first, int32_t n_recent, int32_t n_best, int32_t* blocks, void* keys, hipStream_t stream) {
    const SelectArgs a{c, (const uint16_t*)q, slots, blocks, (uint32_t*)keys, n_tokens, n_q_heads, x.max_blocks, n_first, n_recent, n_best, x.chunk};
    const unsigned units = (unsigned)((int64_t)n_seqs * n_tokens * c.n_kv_heads);
    if (x.chunks > 0 && n_best > 0) {
        const dim3 grid(units, (unsigned)x.chunks);
        if (head_dim == 128) hipLaunchKernelGGL((cache8_score_kernel<128>), grid, dim3(64), 0, stream, a);
        else hipLaunchKernelGGL((cache8_score_kernel<64>), grid, dim3(64), 0, stream, a);
        const int rc = check_launch();
        if (rc != PYR_OK) return rc;
    }
    if (head_dim == 128) launch<128>(x, a, units, stream);
    else launch<64>(x, a, units, stream);
    return check_launch();
}

}  // namespace pyr
