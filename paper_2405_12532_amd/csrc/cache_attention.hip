// Attention of a sequence's newest tokens over its cache held in 4 bits (Section 4.1, generation phase: the step that every generated token
// takes between two updates of the cache):
//   out[b,i,h,:] = sum_t softmax_t(scale * q[b,i,h,:] . k[t,h/g,:]) v[t,h/g,:],   t < len_b - n + 1 + i,  n tokens a sequence.
//
// One pass over the cache with the running reference and sum of a softmax.  A wavefront takes tiles of 32 tokens of one KV head and up to 16 * NT
// query rows (tokens x query heads of the group) as the columns of the products
//   S^T = K Q^T      16 tokens x 16 rows, contracted over 32 channels a step, K converted to bf16 (exactly) with its scale
//   O^T = V^T P^T    16 channels x 16 rows, contracted over the 32 tokens.  V's codes are converted without their scale, which depends on the
//                    token and the block of 32 channels: it is a factor of P instead, P' = P * 2^e per block, rounded to bf16 (as P is in pyr_attention)
// and the layout of the tile makes every operand what a lane loads or has computed: nothing passes through LDS but the wavefronts' results at
// the end.  One more product, of ones and the rounded P, sums what O is divided by: rounding P by itself (up to 2^-8) would show in rows that one token
// dominates; lse comes from the sum before rounding.  P, both sums and O are fp32.
// A row's reference is its largest logit when it was last moved, and it is moved when the weights of a tile add up to more than 2^12 in a lane; so most
// tiles neither look for a maximum nor rescale.  A tile adds at most 2^14 max|V| to an element of O, a wavefront's
// first one at most max|V| a token: less than 2^10 max|V| a token in all.  Two tiles are in flight per wavefront.
//
// Bound: reading the cache.  64 x 2048 tokens on 32 heads, d = 128: 87 us for 571 MB, 6.6 TB/s (counters: read = the cache's bytes; vector instructions
// 51 % of the time, 169 a tile, matrix pipe 20 %).  On the way there: through the caches, with P' made for every block 102, past them 94, P' made once for
// four blocks 87; four wavefronts a SIMD with two registers spilled 95, one copy of the loop with moves of registers instead of two 90.
#include <float.h>
#include <math.h>

#include "cache_device.h"

namespace pyr {
namespace {

constexpr float kGrowth = 4096.f;                 // how far a lane's weights of a tile may outgrow the reference

struct AttendArgs {
    CacheView c;
    const uint16_t* q;
    const int32_t* slots;
    void* out;                                    // splits == 1: bf16 [n, tokens, Hq, D]; else fp32 [splits, rows, D], not normalised
    float* lse;                                   // splits == 1: [rows] or NULL; else [splits, rows, 4]: reference, sum, sum of the rounded
    int32_t n_seqs, n_tokens, n_q_heads;
    int32_t chunk;                                // tiles of a split (the last one takes what is left)
    int32_t splits;
    float scale;                                  // softmax scale * log2(e)
};
static_assert(sizeof(AttendArgs) <= 112, "short arguments");

// What a wavefront holds of a tile.  R: how many times its 16 columns repeat the rows (see Rows).
template <int D, int R>
struct Tile {
    u32x4 k[D / 64], v[D / 64];
    u32x2 vs[D / 32 / R];
    uint32_t ks;
};

// kOnce: nobody else reads the tile.
template <int D, int R, bool kOnce>
__device__ __forceinline__ void load_tile(Tile<D, R>& t, const uint8_t* tile, int lane) {
    auto load = [](const uint8_t* p) { return kOnce ? __builtin_nontemporal_load((const u32x4*)p) : *(const u32x4*)p; };
#pragma unroll
    for (int h = 0; h < D / 64; ++h) t.k[h] = load(tile + (uint32_t)(h * 1024 + lane * 16));
    if (D == 128) t.ks = *(const uint16_t*)(tile + (uint32_t)(32 * D + lane * 2));
    else t.ks = tile[(uint32_t)(32 * D + (lane & 31) * 2 + (lane >> 5))];
#pragma unroll
    for (int h = 0; h < D / 64; ++h) t.v[h] = load(tile + (uint32_t)(16 * D + h * 1024 + lane * 16));
#pragma unroll
    for (int v = 0; v < D / 32 / R; ++v)
        t.vs[v] = *(const u32x2*)(tile + (uint32_t)(33 * D + (lane >> 4) * (D / 4) + 8 * ((lane & 15) / (16 / R)) + 8 * R * v));
}

__device__ __forceinline__ float times(float x, float y) {      // 0 where one of them is 0
    float z;
    asm("v_mul_legacy_f32 %0, %1, %2" : "=v"(z) : "v"(x), "v"(y));
    return z;
}
__device__ __forceinline__ float max_of_groups(float x) {      // over the lanes with the same lane & 15
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_of_groups(float x) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// An element of the output.  O is finite as long as V is, so that an infinite one comes from a block of V that is no number (its scale is +inf in P', and a
// code that is not 0 leaves it at that) or has left fp32's range: NaN either way.
__device__ __forceinline__ __bf16 quotient(float o, float f) { return (__bf16)(__builtin_isinf(o) ? NAN : o * f); }

// Up to 16 / R rows fill the columns of a product R times over: column c is row c % (16 / R), and of V's blocks v R .. v R + R - 1 it has the scales of
// block v R + c / (16 / R).  So P' is made once per R blocks, and of a block's products those of its columns count.
template <int D, int NT, int R>
struct Rows {
    bf16x8 q[NT][D / 32];                         // operand of step s: lane 16 j + col
    f32x4 o[NT][D / 16];
    f32x4 weight[NT];                             // sum of the rounded P, in every element
    float m[NT], l[NT];                           // reference; sum of P over the tokens that this lane sees
    int32_t seen[NT];                             // tokens that the row of this lane's column sees
};

// One tile's products.  masked: some row does not see all of its tokens.
template <int D, int NT, int R>
__device__ __forceinline__ void attend_tile(Rows<D, NT, R>& w, const Tile<D, R>& t, int first_token, bool masked, float scale, int lane) {
    constexpr int kSteps = D / 32;
    float p[NT][8];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        uint32_t codes[kSteps];
        float ks;
        if constexpr (D == 128) {
#pragma unroll
            for (int i = 0; i < 4; ++i) codes[i] = t.k[half][i];
            ks = scale_of(half == 0 ? t.ks & 255 : t.ks >> 8);
        } else {
            // (a lane of the lower half holds 32 channels of token t, one of the upper half of token 16 + t: the upper lanes take over 16 channels
            //  of the lower ones' blocks, and the other way round)
#pragma unroll
            for (int i = 0; i < 2; ++i) codes[i] = __builtin_amdgcn_permlane32_swap(t.k[0][i], t.k[0][i + 2], false, false)[half];
            ks = scale_of(__builtin_amdgcn_permlane32_swap(t.ks, t.ks, false, false)[half]);
        }
        f32x4 s[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) s[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const bf16x8 k = values_of(codes[i], ks);
#pragma unroll
            for (int n = 0; n < NT; ++n) s[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, w.q[n][i], s[n], 0, 0, 0);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) p[n][4 * half + e] = s[n][e];
    }
    bf16x8 ones;
#pragma unroll
    for (int e = 0; e < 8; ++e) ones[e] = (__bf16)1.f;
    if (masked) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int see = w.seen[n] - first_token - 4 * (lane >> 4);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (16 * (e >> 2) + (e & 3) >= see) p[n][e] = -INFINITY;
        }
    }
    // weights against the references as they are; where their sums show that a row has outgrown its own (or has none yet), again against new ones
    float x[NT][8], sum[NT];
    auto weigh = [&] {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[n][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[n][e], scale, -w.m[n]));
            sum[n] = ((x[n][0] + x[n][1]) + (x[n][2] + x[n][3])) + ((x[n][4] + x[n][5]) + (x[n][6] + x[n][7]));
        }
    };
    weigh();
    bool outgrown = false;
#pragma unroll
    for (int n = 0; n < NT; ++n) outgrown |= !(sum[n] <= kGrowth);
    if (__builtin_amdgcn_ballot_w64(outgrown) != 0) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float top = p[n][0];
#pragma unroll
            for (int e = 1; e < 8; ++e) top = fmaxf(top, p[n][e]);
            const float m = fmaxf(w.m[n], max_of_groups(top * scale));
            const float f = __builtin_amdgcn_exp2f(w.m[n] - m);
            w.m[n] = m;
            w.l[n] *= f;
            w.weight[n] *= f;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) w.o[n][i] *= f;
        }
        weigh();
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        w.l[n] += sum[n];
        bf16x8 rounded;
#pragma unroll
        for (int e = 0; e < 8; ++e) rounded[e] = (__bf16)x[n][e];
        w.weight[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, rounded, w.weight[n], 0, 0, 0);
    }
#pragma unroll
    for (int v = 0; v < D / 32 / R; ++v) {
        float vs[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) vs[e] = scale_of((t.vs[v][e >> 2] >> (8 * (e & 3))) & 255);
        // (0 times any scale is 0 here: a token that a row does not see may have any scale byte, NaN among them)
        bf16x8 ps[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 8; ++e) ps[n][e] = (__bf16)times(x[n][e], vs[e]);
#pragma unroll
        for (int i = 2 * R * v; i < 2 * R * (v + 1); ++i) {
            const bf16x8 y = values_of(t.v[i >> 2][i & 3], 1.f);
#pragma unroll
            for (int n = 0; n < NT; ++n) w.o[n][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, ps[n], w.o[n][i], 0, 0, 0);
        }
    }
}

template <int D, int NT, int R, int kWaves>
__global__ __launch_bounds__(64 * kWaves, NT == 1 && (D == 64 || R == 4) ? 3 : 2) void cache_attention_kernel(AttendArgs a) {
    constexpr int kRow = D + 4, kCols = 16 * NT / R;       // floats of a row in LDS; rows of a workgroup
    __shared__ __align__(16) float results[kWaves][kCols][kRow];
    __shared__ __align__(16) float stats[kWaves][kCols][4];      // reference, sum, sum of the rounded
    __shared__ int32_t places[kCols];                      // rows of q and out; -1: none
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane >> 4, c = lane & 15;
    const int hkv = a.c.n_kv_heads, g = a.n_q_heads / hkv, cols = a.n_tokens * g;
    // workgroup -> (sequence, column group, head), split: neighbours read neighbouring heads of the same pages
    int b = blockIdx.x / hkv, first_col = 0;
    const int head = blockIdx.x - b * hkv, split = blockIdx.y, begin = split * a.chunk;
    if (cols > kCols) {
        const int col_groups = (cols + kCols - 1) / kCols, all = b;
        b = all / col_groups;
        first_col = (all - b * col_groups) * kCols;
    }

    // the wavefront's tiles: begin + wave, + kWaves, ...; lane l holds the page of the l-th of 64 (asked for together with the length)
    const int slot = cache_slot(a.c, a.slots, b);
    const int32_t* row_pages = a.c.table + (int64_t)max(slot, 0) * a.c.max_pages;
    const int tile_shift = a.c.shift - 5;
    auto page_of = [&](int i) { return row_pages[min((begin + wave + (i + lane) * kWaves) >> tile_shift, a.c.max_pages - 1)]; };
    int pages = page_of(0);
    const int len = slot < 0 ? 0 : cache_len(a.c, slot);
    const int tiles = (len + 31) >> 5;
    const int end = split == a.splits - 1 ? tiles : min(tiles, begin + a.chunk);
    if (split > 0 && begin >= end) return;                           // (the join does not look at it)

    Rows<D, NT, R> w;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int at = 16 * n + c % (16 / R), col = first_col + at, token = (int)((uint32_t)col / (uint32_t)g);
        const int row = col < cols ? (b * a.n_tokens + token) * a.n_q_heads + head * g + (col - token * g) : -1;
        if (wave == 0 && j == 0) places[at] = row;
        w.seen[n] = len - a.n_tokens + 1 + token;
        w.m[n] = -FLT_MAX;
        w.l[n] = 0.f;
        w.weight[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            const int channel = D == 128 ? 32 * j + 8 * i : 32 * (j & 1) + 8 * (i + 2 * (j >> 1));
            w.q[n][i] = row >= 0 ? *(const bf16x8*)(a.q + (int64_t)row * D + channel) : bf16x8{};
        }
#pragma unroll
        for (int i = 0; i < D / 16; ++i) w.o[n][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int all_see = len - a.n_tokens + 1;                        // tokens below it are seen by every row

    bool bad = false;
    const int count = max(0, (end - begin - wave + kWaves - 1) / kWaves);
    auto fetch = [&](Tile<D, R>& t, int i) {                         // (i goes up by one from call to call)
        if (i >= count) return;
        if ((i & 63) == 0) {
            if (i > 0) pages = page_of(i);
            const bool outside = i + lane < count && (pages < 0 || pages >= a.c.n_pages);
            bad |= __builtin_amdgcn_ballot_w64(outside) != 0;
            if (outside) pages = 0;
        }
        const int page = __builtin_amdgcn_readlane(pages, i & 63);
        const int tile = begin + wave + i * kWaves;
        load_tile<D, R, NT == 1>(t, cache_tile<D>(a.c, page, head, tile & ((1 << tile_shift) - 1)), lane);
    };
    Tile<D, R> t0, t1;
    fetch(t0, 0);
    fetch(t1, 1);
    auto attend = [&](const Tile<D, R>& t, int i) {
        const int token = (begin + wave + i * kWaves) * 32;
        attend_tile<D, NT, R>(w, t, token, token + 32 > all_see, a.scale, lane);
    };
    for (int i = 0; i < count; i += 2) {
        attend(t0, i);
        fetch(t0, i + 2);
        if (i + 1 < count) {
            attend(t1, i + 1);
            fetch(t1, i + 3);
        }
    }

    // the wavefronts' results meet in LDS, weighted by 2^(reference - largest)
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int at = 16 * n + c % (16 / R);
        w.l[n] = bad ? NAN : sum_of_groups(w.l[n]);
        if (j == 0) *(f32x4*)stats[wave][at] = f32x4{w.m[n], w.l[n], bad ? NAN : w.weight[n][0], 0.f};
#pragma unroll
        for (int p = 0; p < D / 32; ++p) {
            // rows 4 j + r of products 2 p and 2 p + 1 are channels 32 p + 2 (4 j + r) and the next
            float* to = &results[wave][at][32 * p + 8 * j];
            const f32x4 x = w.o[n][2 * p], y = w.o[n][2 * p + 1];
            if (c / (16 / R) == p % R) {
                *(f32x4*)to = f32x4{x[0], y[0], x[1], y[1]};
                *(f32x4*)(to + 4) = f32x4{x[2], y[2], x[3], y[3]};
            }
        }
    }
    __syncthreads();
    const int64_t part = split * ((int64_t)a.n_seqs * a.n_tokens * a.n_q_heads);
#pragma unroll 1
    for (int i = threadIdx.x; i < kCols * (D / 4); i += 64 * kWaves) {
        const int r = i / (D / 4), c4 = i % (D / 4), row = places[r];
        if (row < 0) continue;
        float top = stats[0][r][0], sum = 0.f, weight = 0.f;
#pragma unroll
        for (int v = 1; v < kWaves; ++v) top = fmaxf(top, stats[v][r][0]);
        f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < kWaves; ++v) {
            const f32x4 st = *(const f32x4*)stats[v][r];
            const float f = __builtin_amdgcn_exp2f(st[0] - top);
            sum += f * st[1];
            weight += f * st[2];
            o += f * *(const f32x4*)&results[v][r][4 * c4];
        }
        if (a.splits == 1) {
            const float f = weight == 0.f ? 0.f : 1.f / weight;
            bf16x4 y;
#pragma unroll
            for (int x = 0; x < 4; ++x) y[x] = quotient(o[x], f);
            *(bf16x4*)((uint16_t*)a.out + (int64_t)row * D + 4 * c4) = y;
            if (a.lse != nullptr && c4 == 0) a.lse[row] = sum == 0.f ? -INFINITY : top + __builtin_amdgcn_logf(sum);
        } else {
            *(f32x4*)((float*)a.out + (part + row) * D + 4 * c4) = o;
            if (c4 == 0) *(f32x4*)(a.lse + 4 * (part + row)) = f32x4{top, sum, weight, 0.f};
        }
    }
}

typedef __attribute__((ext_vector_type(3))) float f32x3;

// The splits of a row, weighted by 2^(reference - largest) and added up: D / 4 threads a split, kSets splits of a row at a time.
struct JoinArgs {
    CacheView c;
    const int32_t* slots;
    const float* parts;
    const f32x4* stats;
    uint16_t* out;
    float* lse;
    int32_t rows, rows_of_seq, chunk, splits;
};
static_assert(sizeof(JoinArgs) <= 112, "short arguments");

template <int D, int kSets>
__global__ __launch_bounds__(256) void cache_join_kernel(JoinArgs a) {
    constexpr int kQuads = D / 4, kThreads = kQuads * kSets, kRows = 256 / kThreads;
    __shared__ f32x4 sums[kRows][kSets][kQuads];
    __shared__ float weights[kRows][kSets][2], tops[kRows][kSets];
    const int r = threadIdx.x / kThreads, set = threadIdx.x % kThreads / kQuads, quad = threadIdx.x % kQuads;
    const int row = min((int)blockIdx.x * kRows + r, a.rows - 1);          // (the last workgroup's spare threads: the last row again)
    auto stats_of = [&](int s) { return *(const f32x3*)(a.stats + (int64_t)s * a.rows + row); };
    auto part_of = [&](int s) { return *(const f32x4*)(a.parts + ((int64_t)s * a.rows + row) * D + 4 * quad); };
    // the first kAhead of a set are asked for together with the slot, whose length says afterwards whether they are there (1 x 16384 on 64/8 heads 11.6 ->
    // 10.1 us with the attention, 8 x 1800 11.2 -> 10.2)
    constexpr int kAhead = kSets == 2 ? 2 : 4;
    f32x3 st[kAhead];                    // (three: a register of a fourth is taken for something else, and its load waited for first)
    f32x4 part[kAhead];
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
        const int s = min(set + x * kSets, a.splits - 1);
        st[x] = stats_of(s);
        part[x] = part_of(s);
    }
    const int slot = cache_slot(a.c, a.slots, row / a.rows_of_seq);
    const int tiles = slot < 0 ? 0 : (cache_len(a.c, slot) + 31) >> 5;
    const int live = min(a.splits, max(1, (tiles + a.chunk - 1) / a.chunk));
    float top = -FLT_MAX;
#pragma unroll
    for (int x = 0; x < kAhead; ++x)
        if (set + x * kSets < live) top = fmaxf(top, st[x][0]);
#pragma unroll 4
    for (int s = set + kAhead * kSets; s < live; s += kSets) top = fmaxf(top, stats_of(s)[0]);
    tops[r][set] = top;
    __syncthreads();
#pragma unroll
    for (int x = 0; x < kSets; ++x) top = fmaxf(top, tops[r][x]);
    float sum = 0.f, weight = 0.f;
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
    auto add = [&](const f32x3& y, const f32x4& z) {
        const float f = __builtin_amdgcn_exp2f(y[0] - top);
        sum += f * y[1];
        weight += f * y[2];
        o += f * z;
    };
#pragma unroll
    for (int x = 0; x < kAhead; ++x)
        if (set + x * kSets < live) add(st[x], part[x]);
#pragma unroll 4
    for (int s = set + kAhead * kSets; s < live; s += kSets) add(stats_of(s), part_of(s));
    sums[r][set][quad] = o;
    if (quad == 0) {
        weights[r][set][0] = sum;
        weights[r][set][1] = weight;
    }
    __syncthreads();
    if (set != 0) return;
#pragma unroll
    for (int x = 1; x < kSets; ++x) {
        o += sums[r][x][quad];
        sum += weights[r][x][0];
        weight += weights[r][x][1];
    }
    const float f = weight == 0.f ? 0.f : 1.f / weight;
    bf16x4 y;
#pragma unroll
    for (int x = 0; x < 4; ++x) y[x] = quotient(o[x], f);
    *(bf16x4*)(a.out + (int64_t)row * D + 4 * quad) = y;
    if (a.lse != nullptr && quad == 0) a.lse[row] = sum == 0.f ? -INFINITY : top + __builtin_amdgcn_logf(sum);
}

template <int D>
int launch(const CacheAttention& x, const CacheView& c, const AttendArgs& a, void* out, float* lse, hipStream_t stream) {
    const dim3 blocks((unsigned)((int64_t)a.n_seqs * x.col_groups * c.n_kv_heads), (unsigned)x.splits), threads(64 * x.waves);
    constexpr int kMost = D / 32;      // columns of a product hold at most so many times the rows
    if (x.col_tiles == 2) hipLaunchKernelGGL((cache_attention_kernel<D, 2, 1, 4>), blocks, threads, 0, stream, a);
    else if (x.waves == 4) {
        if (x.repeats == 1) hipLaunchKernelGGL((cache_attention_kernel<D, 1, 1, 4>), blocks, threads, 0, stream, a);
        else if (x.repeats == 2) hipLaunchKernelGGL((cache_attention_kernel<D, 1, 2, 4>), blocks, threads, 0, stream, a);
        else hipLaunchKernelGGL((cache_attention_kernel<D, 1, kMost, 4>), blocks, threads, 0, stream, a);
    } else {
        if (x.repeats == 1) hipLaunchKernelGGL((cache_attention_kernel<D, 1, 1, 8>), blocks, threads, 0, stream, a);
        else if (x.repeats == 2) hipLaunchKernelGGL((cache_attention_kernel<D, 1, 2, 8>), blocks, threads, 0, stream, a);
        else hipLaunchKernelGGL((cache_attention_kernel<D, 1, kMost, 8>), blocks, threads, 0, stream, a);
    }
    const int rc = check_launch();
    if (rc != PYR_OK || a.splits == 1) return rc;
    const int32_t rows_of_seq = a.n_tokens * a.n_q_heads, rows = a.n_seqs * rows_of_seq;
    const JoinArgs j{c, a.slots, (const float*)a.out, (const f32x4*)a.lse, (uint16_t*)out, lse, rows, rows_of_seq, a.chunk, a.splits};
    constexpr int kFew = 2, kMany = 1024 / D;
    if (a.splits <= 2 * kFew) {
        constexpr int kRows = 256 / (D / 4 * kFew);
        hipLaunchKernelGGL((cache_join_kernel<D, kFew>), dim3((unsigned)((rows + kRows - 1) / kRows)), dim3(256), 0, stream, j);
    } else {
        hipLaunchKernelGGL((cache_join_kernel<D, kMany>), dim3((unsigned)rows), dim3(256), 0, stream, j);
    }
    return check_launch();
}

}  // namespace

// What is waited for at the end is the wavefront with the most tiles (0.4 us each), so few heads are split along the cache, until there are 2 * kUnits
// workgroups of kShortest tiles and more - unless a launch that joins the parts (2 to 3 us, and 3 us of the host's) costs more than it saves.
// Workgroups of eight wavefronts do with half as many parts; one fits a compute unit, so they are taken where they fill nearly all of them
// in one go.  Measured, us (four wavefronts, eight): one token of 1 x 1000 on 32/8 heads 9.5 / 8.2 (unsplit), 1 x 1434 on 32 12.2 / 10.2, 32 x 4096 on
// 32/8 29.7 / 26.6, 1 x 32768 on 32/8 13.6 / 12.9; 20 of 100 ... 8000 on 64/8 (160 heads) 31 / 38, 40 x 1500 on 32/8 (320 heads) 17 / 21.
// Unsplit as long as that is faster than the parts and their join (us, unsplit and split): 8 x 1200 on 32/8 heads 9.1 / 9.5, 8 x 1434 10.2 / 9.6 (64 heads), but
// with the calls of a step before it 1 x 1434 on 32 heads 27 / 30; 12 x 1500 10.5 / 10.9, 12 x 1800 11.4 / 11.1 (96); 16 x 1800 11.6 / 11.6 (128);
// 20 x 1800 on 64/8 12.4 / 15.1, 20 x 2100 13.8 / 15.0, lengths of 100 ... 2000 12.8 / 12.9 (160).  Heads of 128 channels that all have a place at once
// (three workgroups of four wavefronts a compute unit) are not split into more than have: 60 x 1800 on 64/8 heads (480) 24 / 30, 60 x 8000
// 85 / 93, though lengths of 300 ... 5000 take 44 / 41; with four tokens 60 x 1800 37.5 / 48, lengths of 100 ... 2000 32 / 40, of 300 ... 5000 70 / 71.
// More than 16 rows a head: parts twice as long, as their results are twice as large (us for parts of 16, 32 and 64 tiles:
// 8 x 4096 on 64/8 heads, four tokens 21.4 / 19.7 / 26; 16 x 2048, nine 36 / 35 / 32.5).
CacheAttention plan_cache_attention(int32_t n_seqs, int32_t n_tokens, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t max_len) {
    constexpr int64_t kShortest = 16, kUnits = 256, kFilled = 200;
    CacheAttention x{};
    const int cols = n_tokens * (n_q_heads / n_kv_heads);
    const int tiles = (cols + 15) / 16;
    x.col_tiles = tiles == 1 ? 1 : 2;
    x.col_groups = (tiles + x.col_tiles - 1) / x.col_tiles;
    x.repeats = cols <= 4 && head_dim == 128 ? 4 : cols <= 8 ? 2 : 1;
    const int64_t units = (int64_t)n_seqs * n_kv_heads * x.col_groups, key_tiles = (max_len + 31) / 32;
    const int64_t unsplit = x.col_tiles == 1 && units > kUnits * 9 / 16 && units <= kUnits ? 64 : 48;
    int64_t splits = 1;
    x.waves = 4;
    if (units > 0 && key_tiles <= unsplit) x.waves = x.col_tiles == 1 && units <= kUnits ? 8 : 4;
    else if (units > 0 && x.col_tiles == 1 && units <= kUnits && kUnits / units * units >= kFilled) {
        x.waves = 8;
        splits = kUnits / units;
    } else if (units > 0) {
        const bool in_one_go = head_dim == 128 && units > kUnits;
        splits = !in_one_go ? (2 * kUnits + units - 1) / units : units < 3 * kUnits ? 3 * kUnits / units : 1;
    }
    int64_t chunk = (key_tiles + splits - 1) / splits;
    const int64_t shortest = x.col_tiles * kShortest;
    if (splits > 1 && chunk < shortest) chunk = shortest;
    chunk = (chunk + x.waves - 1) / x.waves * x.waves;
    if (chunk == 0) chunk = x.waves;
    splits = (key_tiles + chunk - 1) / chunk;
    x.chunk = (int32_t)chunk;
    x.splits = splits < 1 ? 1 : (int32_t)splits;
    const int64_t rows = (int64_t)n_seqs * n_tokens * n_q_heads;
    x.part_bytes = x.splits == 1 ? 0 : (size_t)x.splits * rows * head_dim * sizeof(float);
    x.stat_bytes = x.splits == 1 ? 0 : (size_t)x.splits * rows * 4 * sizeof(float);
    return x;
}

int launch_cache_attention(const CacheAttention& x, const CacheView& c, int32_t head_dim, const void* q, const int32_t* slots, int32_t n_seqs,
                           int32_t n_tokens, int32_t n_q_heads, float scale_log2, void* out, float* lse, void* parts, float* stats, hipStream_t stream) {
    if (n_seqs == 0) return PYR_OK;
    AttendArgs a{c, (const uint16_t*)q, slots, out, lse, n_seqs, n_tokens, n_q_heads, x.chunk, x.splits, scale_log2};
    if (x.splits > 1) {
        a.out = parts;
        a.lse = stats;
    }
    return head_dim == 128 ? launch<128>(x, c, a, out, lse, stream) : launch<64>(x, c, a, out, lse, stream);
}

}  // namespace pyr
