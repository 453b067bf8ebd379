// The blocks of a cache held in 8 bits that a token attends to, for every KV head: the first ones, the last ones, and those in between whose bounds
// promise the largest logits (Section 3.2's observation, that few tokens carry the attention, used at every step without the others being given up).
//
// The logit of a query with any K between a block's smallest lo and largest hi is at most sum_c max(q_c hi_c, q_c lo_c) = [max(q, 0); min(q, 0)] . [hi; lo],
// one product of twice the channels.  lo and hi are whole numbers times the block's power, and q is rounded to whole numbers from -127 to 127 times a power
// of its own, so that the product is one of 8-bit integers (v_mfma_i32_16x16x64_i8) and a score, a whole number below 2^22 times a power of two,
// is exact in fp32: which blocks are chosen does not depend on the order of a sum.  A block's score is the largest of the group's query heads.
// Bound: reading the bounds where there are many, the latency of a launch where there are few.
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

// Scores as numbers that compare like them.
__device__ __forceinline__ uint32_t key_of(float score) {
    const uint32_t bits = __float_as_uint(score);
    return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}

// A unit: a token of a sequence and a KV head.  What its tokens and blocks are.
struct Unit {
    int32_t slot, len, count, low, high, head, row;      // blocks it sees; candidates low .. high - 1; row of q's tokens
};
__device__ __forceinline__ Unit unit_of(const SelectArgs& a, int unit) {
    Unit u;
    const int hkv = a.c.n_kv_heads;
    u.row = unit / hkv;
    u.head = unit - u.row * hkv;
    const int b = u.row / a.n_tokens, token = u.row - b * a.n_tokens;
    u.slot = cache_slot(a.c, a.slots, b);
    u.len = u.slot < 0 ? 0 : cache_len(a.c, u.slot);
    u.count = (max(u.len - a.n_tokens + 1 + token, 0) + 31) >> 5;
    u.low = min(a.n_first, u.count);
    u.high = max(u.low, min(u.count - a.n_recent, a.max_blocks));
    return u;
}

// The keys of candidates begin .. end - 1, by the wavefronts of a workgroup; put(i, key)
template <int D, int kWaves, class Put>
__device__ __forceinline__ void score_blocks(const SelectArgs& a, const Unit& u, int begin, int end, Put put) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane >> 4, t = lane & 15;
    const int g = a.n_q_heads / a.c.n_kv_heads, tile_shift = a.c.shift - 5;
    const int32_t* row_pages = a.c.table + (int64_t)max(u.slot, 0) * a.c.max_pages;
    const uint16_t* q = a.q + ((int64_t)u.row * a.n_q_heads + u.head * g) * D;
    constexpr int kHalf = D / 64, kNone = -1000;
    // 16 query heads at a time (the first 16 stay in registers)
    i32x4 whole[2 * kHalf];
    int power[4];                                 // of rows 4 j + x; kNone: no query head
    auto take = [&](int first) {
        u32x4 words[kHalf][2];
        float top = 0.f;
        const bool mine = first + t < g;
#pragma unroll
        for (int s = 0; s < kHalf; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                words[s][h] = mine ? *(const u32x4*)(q + (int64_t)(first + t) * D + 64 * s + 16 * j + 8 * h) : u32x4{};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = fabsf(__uint_as_float(words[s][h][e] << 16)), y = fabsf(__uint_as_float(words[s][h][e] & 0xffff0000u));
                    top = fmaxf(top, fmaxf(x < INFINITY ? x : 0.f, y < INFINITY ? y : 0.f));
                }
            }
        auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        top = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
        p = __builtin_amdgcn_permlane16_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        top = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
        const uint32_t bits = __float_as_uint(top);
        const int e = min(max((int)(bits >> 23) - 127 - 6 + ((bits & 0x7fffff) > 0x7e0000 ? 1 : 0), -100), 122);
        const float by = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
        for (int s = 0; s < kHalf; ++s)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t up = 0, down = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t pair = words[s][w >> 1][2 * (w & 1) + (i >> 1)];
                    const float x = __uint_as_float(i & 1 ? pair & 0xffff0000u : pair << 16) * by;
                    const float y = fminf(fmaxf(__builtin_rintf(x), -127.f), 127.f);
                    const int n = x != x ? 0 : (int)y;
                    up |= (uint32_t)max(n, 0) << (8 * i);
                    down |= ((uint32_t)min(n, 0) & 255) << (8 * i);
                }
                whole[s][w] = (int)up;
                whole[kHalf + s][w] = (int)down;
            }
#pragma unroll
        for (int x = 0; x < 4; ++x) power[x] = __shfl(mine ? e : kNone, 4 * j + x);
    };
    if (g <= 16) take(0);
    // 64 blocks at a time: lane l holds page and power of the l-th
    for (int base = begin + 64 * wave; base < end; base += 64 * kWaves) {
        const int block = min(base + lane, end - 1);
        int page = row_pages[block >> tile_shift];
        if (page < 0 || page >= a.c.n_pages) page = 0;      // (the attention makes NaN of it)
        const int block_power = (int)(*Page8<D>(a.c, page).powers(u.head, block) & 255) - 127;
        i32x4 bounds[4][2 * kHalf];
#pragma unroll
        for (int s = 0; s < 4; ++s) {                       // (all loads of 64 blocks in flight)
            const int n = __shfl(block, 16 * s + t), p = __shfl(page, 16 * s + t);
            const i32x4* from = (const i32x4*)Page8<D>(a.c, p).bounds(u.head, n) + j;
#pragma unroll
            for (int i = 0; i < 2 * kHalf; ++i) bounds[s][i] = from[4 * i];
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int of_block = __shfl(block_power, 16 * s + t);
            float best = -INFINITY;
            for (int first = 0; first < g; first += 16) {
                if (g > 16) take(first);
                i32x4 d = {0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < 2 * kHalf; ++i) d = __builtin_amdgcn_mfma_i32_16x16x64_i8(whole[i], bounds[s][i], d, 0, 0, 0);
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int e = min(max(power[x] + of_block + 2, -120), 100);
                    const float score = (float)d[x] * __uint_as_float((uint32_t)(127 + e) << 23);
                    best = fmaxf(best, power[x] == kNone ? -INFINITY : score);
                }
            }
            auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(best), __float_as_uint(best), false, false);
            best = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
            p = __builtin_amdgcn_permlane16_swap(__float_as_uint(best), __float_as_uint(best), false, false);
            best = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
            const int n = base + 16 * s + t;
            if (j == 0 && n < end) put(n, key_of(best));
        }
    }
}

// grid: (units, chunks of candidates)
template <int D>
__global__ __launch_bounds__(256) void cache8_score_kernel(SelectArgs a) {
    const Unit u = unit_of(a, blockIdx.x);
    if (u.high - u.low <= a.n_best) return;
    const int begin = u.low + (int)blockIdx.y * a.chunk, end = min(u.high, begin + a.chunk);
    if (begin >= end) return;
    uint32_t* keys = a.keys + (int64_t)blockIdx.x * a.max_blocks;
    score_blocks<D, 4>(a, u, begin, end, [&](int n, uint32_t key) { keys[n] = key; });
}

// One workgroup a unit.  kKeys: keys in LDS, worked out here; 0: they are in memory.
// The n-th largest key is found byte by byte, from counts of the bytes among the keys that share the higher ones; of those equal to it the
// first are taken.
template <int D, int kKeys>
__global__ __launch_bounds__(256) void cache8_select_kernel(SelectArgs a) {
    constexpr int kWaves = 4, kThreads = 64 * kWaves;
    __shared__ uint32_t held[kKeys == 0 ? 1 : kKeys];
    __shared__ int counts[256], sums[kWaves], found[2];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Unit u = unit_of(a, blockIdx.x);
    const int width = a.n_first + a.n_recent + a.n_best, candidates = u.high - u.low;
    int32_t* out = a.blocks + (int64_t)blockIdx.x * width;
    const int chosen = min(candidates, a.n_best), tail = max(u.low, u.count - a.n_recent), all = u.low + chosen + (u.count - tail);
    for (int i = threadIdx.x; i < u.low; i += kThreads) out[i] = i;
    for (int i = threadIdx.x; i < u.count - tail; i += kThreads) out[u.low + chosen + i] = tail + i;
    for (int i = all + threadIdx.x; i < width; i += kThreads) out[i] = -1;
    if (candidates <= a.n_best) {
        for (int i = threadIdx.x; i < candidates; i += kThreads) out[u.low + i] = u.low + i;
        return;
    }
    if (a.n_best == 0) return;
    const uint32_t* keys = kKeys == 0 ? a.keys + (int64_t)blockIdx.x * a.max_blocks : held;
    if constexpr (kKeys != 0) {
        score_blocks<D, kWaves>(a, u, u.low, u.high, [&](int n, uint32_t key) { held[n - u.low] = key; });
        __syncthreads();
        keys -= u.low;
    }
    uint32_t prefix = 0;
    int wanted = a.n_best;                                    // so many of the keys that share the prefix, and all above
#pragma unroll 1
    for (int shift = 24; shift >= 0; shift -= 8) {
        counts[threadIdx.x] = 0;
        __syncthreads();
        for (int i = u.low + threadIdx.x; i < u.high; i += kThreads) {
            const uint32_t key = keys[i];
            if (shift == 24 || key >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&counts[key >> shift & 255], 1);
        }
        __syncthreads();
        // thread i: keys whose byte is at least 255 - i
        int sum = counts[255 - threadIdx.x];
        const int own = sum;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int other = __shfl_up(sum, d);
            if (lane >= d) sum += other;
        }
        if (lane == 63) sums[wave] = sum;
        __syncthreads();
        for (int w = 0; w < wave; ++w) sum += sums[w];
        if (sum >= wanted && sum - own < wanted) {
            found[0] = 255 - threadIdx.x;
            found[1] = wanted - (sum - own);
        }
        __syncthreads();
        prefix |= (uint32_t)found[0] << shift;
        wanted = found[1];
    }
    // in order: above the n-th largest, and the first `wanted` that are equal to it
    int before = 0, equal_before = 0;
    for (int base = u.low; base < u.high; base += kThreads) {
        const int i = base + threadIdx.x;
        const uint32_t key = i < u.high ? keys[i] : 0;
        const bool above = i < u.high && key > prefix, equal = i < u.high && key == prefix;
        const uint64_t equals = __builtin_amdgcn_ballot_w64(equal);
        __syncthreads();
        if (lane == 0) sums[wave] = __builtin_popcountll(equals);
        __syncthreads();
        int rank = equal_before + __builtin_popcountll(equals & ((1ull << lane) - 1));
        for (int w = 0; w < wave; ++w) rank += sums[w];
        for (int w = 0; w < kWaves; ++w) equal_before += sums[w];
        const bool taken = above || (equal && rank < wanted);
        const uint64_t takens = __builtin_amdgcn_ballot_w64(taken);
        __syncthreads();
        if (lane == 0) sums[wave] = __builtin_popcountll(takens);
        __syncthreads();
        int at = before + __builtin_popcountll(takens & ((1ull << lane) - 1));
        for (int w = 0; w < wave; ++w) at += sums[w];
        for (int w = 0; w < kWaves; ++w) before += sums[w];
        if (taken) out[u.low + at] = i;
    }
}

constexpr int kInLds = 4096;

}  // namespace

CacheSelect plan_cache8_select(int32_t n_seqs, int32_t n_tokens, int32_t n_kv_heads, int64_t max_len) {
    CacheSelect x{};
    const int64_t units = (int64_t)n_seqs * n_tokens * n_kv_heads, blocks = (max_len + 31) / 32;
    x.max_blocks = (int32_t)blocks;
    x.chunks = 0;
    if (blocks > kInLds || (units < 128 && blocks > 512)) {
        x.chunk = (int32_t)((blocks / 4096 + 256) / 256 * 256);
        x.chunks = (int32_t)((blocks + x.chunk - 1) / x.chunk);
        x.key_bytes = (size_t)units * blocks * sizeof(uint32_t);
    }
    return x;
}

int launch_cache8_select(const CacheSelect& x, const CacheView& c, int32_t head_dim, const void* q, const int32_t* slots, int32_t n_seqs, int32_t n_tokens,
                         int32_t n_q_heads, int32_t n_first, int32_t n_recent, int32_t n_best, int32_t* blocks, void* keys, hipStream_t stream) {
    const SelectArgs a{c, (const uint16_t*)q, slots, blocks, (uint32_t*)keys, n_tokens, n_q_heads, x.max_blocks, n_first, n_recent, n_best, x.chunk};
    const unsigned units = (unsigned)((int64_t)n_seqs * n_tokens * c.n_kv_heads);
    if (x.chunks > 0 && n_best > 0) {
        const dim3 grid(units, (unsigned)x.chunks);
        if (head_dim == 128) hipLaunchKernelGGL((cache8_score_kernel<128>), grid, dim3(256), 0, stream, a);
        else hipLaunchKernelGGL((cache8_score_kernel<64>), grid, dim3(256), 0, stream, a);
        const int rc = check_launch();
        if (rc != PYR_OK) return rc;
    }
    if (x.chunks > 0) {
        if (head_dim == 128) hipLaunchKernelGGL((cache8_select_kernel<128, 0>), dim3(units), dim3(256), 0, stream, a);
        else hipLaunchKernelGGL((cache8_select_kernel<64, 0>), dim3(units), dim3(256), 0, stream, a);
    } else {
        if (head_dim == 128) hipLaunchKernelGGL((cache8_select_kernel<128, kInLds>), dim3(units), dim3(256), 0, stream, a);
        else hipLaunchKernelGGL((cache8_select_kernel<64, kInLds>), dim3(units), dim3(256), 0, stream, a);
    }
    return check_launch();
}

}  // namespace pyr
