// Attention of a sequence's newest tokens over its cache held in 8 bits, all of it or the blocks that a list names for every token and KV head
// (Section 4.1, generation phase: the step that every generated token takes between two updates of the cache):
//   out[b,i,h,:] = sum_t softmax_t(scale * q[b,i,h,:] . k[t,h/g,:]) v[t,h/g,:],   t < len_b - n + 1 + i,  n tokens a sequence.
//
// One pass over the blocks with the running reference and sum of a softmax.  A wavefront takes blocks of 32 tokens of one KV head and up to 16 * NT query
// rows (tokens x query heads of the group; with lists those of one token) as the columns of the products
//   S^T = K Q^T      16 tokens x 16 rows, contracted over 32 channels a step
//   O^T = V^T P^T    16 channels x 16 rows, contracted over the 32 tokens
// K and V are converted to bf16 with their power (exactly), and the layout of the block makes every operand what a lane loads or has computed: nothing
// passes through LDS but the wavefronts' results at the end.  P goes into the product as two bf16 numbers, the nearest one and the nearest one to what that
// leaves: sixteen bits, off by 2^-16 at most.  (One alone, off by 2^-8, took outputs from 0.0017 off, rms over rms, which is their own rounding, to 0.0018 to 0.0023.  The second
// product costs 0 to 3 % where bytes bound, 64 x 2048 on 32 heads 162 us either way; 16 x 2048 on 64/8 heads with nine tokens, bound by instructions, 30 us for 26.5.)  P, its sum
// and O are fp32.
// A row's reference is its largest logit when it was last moved, and it is moved when the weights of a block add up to more than 2^12 in a lane.
// Bound: reading the cache, past the caches: 64 x 2048 tokens on 32 heads of 128 channels in 162 us, 1077 MB at 6.6 TB/s (through the caches 184), vector
// instructions 25 % of a SIMD's cycles and matrix instructions 14 %; 32 x 307 ... 4915 tokens on 40 heads, four tokens each, 129 us, 6.1 TB/s; lists of 16 blocks, 64 x
// 2048, 47.5 us for 271 MB, 5.7 TB/s.  One sequence: dependent loads and launches (1 x 16384 on 64/8 heads 11.8 us a pass; 10.3 and 3.9 for the join in a kernel trace).
// More than 16 rows a head: instructions too (16 x 2048 on 64/8 heads, nine tokens, vector instructions 47 % of a SIMD's cycles and matrix instructions 32 %).
#include <float.h>
#include <math.h>

#include "cache8_device.h"

namespace pyr {
namespace {

constexpr float kGrowth = 4096.f;                 // how far a lane's weights of a block may outgrow the reference

struct AttendArgs {
    CacheView c;
    const uint16_t* q;
    const int32_t* slots;
    const int32_t* blocks;                        // lists [n, tokens, Hkv, n_blocks]
    void* out;                                    // splits == 1: bf16 [n, tokens, Hq, D]; else fp32 [splits, rows, D], not normalised
    float* lse;                                   // splits == 1: [rows] or NULL; else [splits, rows, 4]: reference, sum, the sum again (what O is divided by)
    int32_t n_seqs, n_tokens, n_blocks;
    int32_t chunk;                                // blocks of a split (the last one takes what is left)
    uint16_t n_q_heads, splits;
    float scale;                                  // softmax scale * log2(e)
};
static_assert(sizeof(AttendArgs) <= 112, "short arguments");

// What a wavefront holds of a block; token: its first one, -1: no block.
template <int D>
struct Tile {
    u32x4 k[D / 32], v[D / 32];
    float ks, vs;
    int32_t token;
};

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

// An element of the output: one whose sum has left fp32's range is NaN, as one that has a V that is no number.
__device__ __forceinline__ __bf16 quotient(float o, float f) { return (__bf16)(__builtin_isinf(o) ? NAN : o * f); }

// bytes of a word that are no numbers: their highest bits
__device__ __forceinline__ uint32_t no_numbers(uint32_t codes) { return ((codes & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

template <int D, int NT>
struct Rows {
    bf16x8 q[NT][D / 32];                         // operand of step i: lane 16 j + col
    f32x4 o[NT][D / 16];
    float m[NT], l[NT];                           // reference; sum of P over the tokens that this lane sees
    int32_t seen[NT];                             // tokens that the row of this lane's column sees
};

// One block's products.  masked: some row does not see all of its tokens; len: tokens there are.
template <int D, int NT>
__device__ __forceinline__ void attend_tile(Rows<D, NT>& w, Tile<D>& t, bool masked, int len, float scale, int lane) {
    float p[NT][8];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        f32x4 s[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) s[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            const u32x4& codes = t.k[half * (D / 64) + (i >> 1)];
            const bf16x8 k = values8_of(codes[2 * (i & 1)], codes[2 * (i & 1) + 1], t.ks);
#pragma unroll
            for (int n = 0; n < NT; ++n) s[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, w.q[n][i], s[n], 0, 0, 0);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) p[n][4 * half + e] = s[n][e];
    }
    if (masked) {
        const int mine = t.token + 4 * (lane >> 4);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int see = w.seen[n] - mine;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (16 * (e >> 2) + (e & 3) >= see) p[n][e] = -INFINITY;
        }
        // V behind the last token may be anything, 0 times which may be NaN
        uint32_t held[2] = {0, 0}, bad = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (16 * (e >> 2) + (e & 3) < len - mine) held[e >> 2] |= 0xffu << (8 * (e & 3));
#pragma unroll
        for (int g = 0; g < D / 32; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                t.v[g][i] &= held[i & 1];
                bad |= no_numbers(t.v[g][i]);
            }
        if (__builtin_amdgcn_ballot_w64(bad != 0) != 0) {
            // a V that is no number: NaN for the rows that see it, counted by one more product, and 0 for those that do not
#pragma unroll
            for (int g = 0; g < D / 32; ++g)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    bf16x8 none;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t high = no_numbers(t.v[g][2 * i + h]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) none[4 * h + e] = (__bf16)(float)(high >> (8 * e + 7) & 1);
                        t.v[g][2 * i + h] &= ~((high >> 7) * 255u);
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        bf16x8 sees;
                        const int see = w.seen[n] - mine;
#pragma unroll
                        for (int e = 0; e < 8; ++e) sees[e] = (__bf16)(16 * (e >> 2) + (e & 3) < see ? 1.f : 0.f);
                        const f32x4 count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(none, sees, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (count[e] > 0.f) w.o[n][2 * g + i][e] = NAN;
                    }
                }
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
#pragma unroll
            for (int i = 0; i < D / 16; ++i) w.o[n][i] *= f;
        }
        weigh();
    }
    // What P's nearest bf16 numbers leave, exactly: a product of a pair with -1 and 0 takes one of them off, where a subtraction would need it by itself first.  (In registers:
    // written as an operand, the instruction takes a constant of -1 for one of fp32, whose upper half is a bf16's.)
    uint32_t less_first = 0xbf80u, less_second = 0xbf800000u;
    asm volatile("" : "+s"(less_first), "+s"(less_second));
    bf16x8 high[NT], low[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        w.l[n] += sum[n];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const bf16x2 y = {(__bf16)x[n][e], (__bf16)x[n][e + 1]};
            high[n][e] = y[0];
            high[n][e + 1] = y[1];
            low[n][e] = (__bf16)__builtin_amdgcn_fdot2_f32_bf16(y, __builtin_bit_cast(bf16x2, less_first), x[n][e], false);
            low[n][e + 1] = (__bf16)__builtin_amdgcn_fdot2_f32_bf16(y, __builtin_bit_cast(bf16x2, less_second), x[n][e + 1], false);
        }
    }
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
        const bf16x8 y = values8_of(t.v[i >> 1][2 * (i & 1)], t.v[i >> 1][2 * (i & 1) + 1], t.vs);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            w.o[n][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, high[n], w.o[n][i], 0, 0, 0);
            w.o[n][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, low[n], w.o[n][i], 0, 0, 0);
        }
    }
}

// kOnce: nobody else reads a block.
template <int D, int NT, int kWaves, bool kListed, bool kOnce>
__global__ __launch_bounds__(64 * kWaves, NT == 1 && D == 64 ? 3 : 2) void cache8_attention_kernel(AttendArgs a) {
    constexpr int kRow = D + 4, kCols = 16 * NT;           // floats of a row in LDS; rows of a workgroup
    __shared__ __align__(16) float results[kWaves][kCols][kRow];
    __shared__ __align__(8) float stats[kWaves][kCols][2];       // reference, sum
    __shared__ int32_t places[kCols];                      // rows of q and out; -1: none
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane >> 4, c = lane & 15;
    const int hkv = a.c.n_kv_heads, g = a.n_q_heads / hkv, cols = kListed ? g : a.n_tokens * g;
    // workgroup -> (sequence or token, column group, head), split: neighbours read neighbouring heads of the same pages
    int b = blockIdx.x / hkv, first_col = 0;
    const int head = blockIdx.x - b * hkv, split = blockIdx.y, begin = split * a.chunk;
    if (cols > kCols) {
        const int col_groups = (cols + kCols - 1) / kCols, all = b;
        b = all / col_groups;
        first_col = (all - b * col_groups) * kCols;
    }
    const int first_row = kListed ? b : b * a.n_tokens;    // of q's tokens
    const int my_token = kListed ? b % a.n_tokens : 0;
    if (kListed) b /= a.n_tokens;

    // the wavefront's blocks: begin + wave, + kWaves, ... (of the list); lane l holds number, page and powers of the l-th of 64 (the first pages are asked for
    // together with the length)
    const int slot = cache_slot(a.c, a.slots, b);
    const int32_t* row_pages = a.c.table + (int64_t)max(slot, 0) * a.c.max_pages;
    const int32_t* list = kListed ? a.blocks + ((int64_t)first_row * hkv + head) * a.n_blocks : nullptr;
    const int tile_shift = a.c.shift - 5, most = a.c.max_pages << tile_shift;
    auto block_of = [&](int i) {
        const int at = begin + wave + (i + lane) * kWaves;
        if (!kListed) return at;
        const int block = at < a.n_blocks ? list[at] : -1;
        return block < most ? block : -1;
    };
    auto page_of = [&](int block) { return row_pages[min(max(block, 0) >> tile_shift, a.c.max_pages - 1)]; };
    int numbers = block_of(0), pages = page_of(numbers);
    const int len = slot < 0 ? 0 : cache_len(a.c, slot);
    const int sight = kListed ? len - a.n_tokens + 1 + my_token : len;      // tokens that some row sees
    const int tiles = kListed ? a.n_blocks : (len + 31) >> 5;
    const int end = split == a.splits - 1 ? tiles : min(tiles, begin + a.chunk);
    if (!kListed && split > 0 && begin >= end) return;               // (the join does not look at it)

    Rows<D, NT> w;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int at = 16 * n + c, col = first_col + at, token = kListed ? my_token : (int)((uint32_t)col / (uint32_t)g);
        const int row = col < cols ? (kListed ? first_row * a.n_q_heads + head * g + col : (first_row + token) * a.n_q_heads + head * g + (col - token * g)) : -1;
        if (wave == 0 && j == 0) places[at] = row;
        w.seen[n] = min(len - a.n_tokens + 1 + token, len);
        w.m[n] = -FLT_MAX;
        w.l[n] = 0.f;
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
            w.q[n][i] = row >= 0 ? *(const bf16x8*)(a.q + (int64_t)row * D + 64 * (i >> 1) + 16 * j + 8 * (i & 1)) : bf16x8{};
#pragma unroll
        for (int i = 0; i < D / 16; ++i) w.o[n][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int all_see = kListed ? sight : len - a.n_tokens + 1;      // tokens below it are seen by every row

    bool bad = false;
    uint32_t powers = 0;
    const int count = max(0, (end - begin - wave + kWaves - 1) / kWaves);
    auto fetch = [&](Tile<D>& t, int i) {                            // (i goes up by one from call to call)
        t.token = -1;
        if (i >= count) return;
        if ((i & 63) == 0) {
            if (i > 0) {
                numbers = block_of(i);
                pages = page_of(numbers);
            }
            // blocks of a list that hold no token that the row sees are left out
            const bool there = i + lane < count && numbers >= 0 && (!kListed || 32 * numbers < sight);
            if (!there) numbers = -1;
            const bool outside = there && (pages < 0 || pages >= a.c.n_pages);
            bad |= __builtin_amdgcn_ballot_w64(outside) != 0;
            if (outside || !there) pages = 0;
            const Page8<D> at(a.c, pages);
            powers = *at.powers(head, max(numbers, 0));
        }
        const int number = __builtin_amdgcn_readlane(numbers, i & 63);
        if (kListed && number < 0) return;
        t.token = 32 * number;
        const Page8<D> at(a.c, __builtin_amdgcn_readlane(pages, i & 63));
        const u32x4* from = (const u32x4*)at.codes(head, number);
#pragma unroll
        for (int x = 0; x < D / 32; ++x) t.k[x] = kOnce ? __builtin_nontemporal_load(from + (uint32_t)(64 * x + lane)) : from[(uint32_t)(64 * x + lane)];
#pragma unroll
        for (int x = 0; x < D / 32; ++x)
            t.v[x] = kOnce ? __builtin_nontemporal_load(from + (uint32_t)(64 * (D / 32 + x) + lane)) : from[(uint32_t)(64 * (D / 32 + x) + lane)];
        const uint32_t both = (uint32_t)__builtin_amdgcn_readlane((int)powers, i & 63);
        t.ks = scale_of(both & 255);
        t.vs = scale_of(both >> 8);
    };
    auto attend = [&](Tile<D>& t) {
        if (kListed && t.token < 0) return;
        attend_tile<D, NT>(w, t, t.token + 32 > all_see, sight, a.scale, lane);
    };
    Tile<D> t0, t1;
    fetch(t0, 0);
    fetch(t1, 1);
    for (int i = 0; i < count; i += 2) {
        attend(t0);
        fetch(t0, i + 2);
        if (i + 1 < count) {
            attend(t1);
            fetch(t1, i + 3);
        }
    }

    // the wavefronts' results meet in LDS, weighted by 2^(reference - largest)
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int at = 16 * n + c;
        w.l[n] = bad ? NAN : sum_of_groups(w.l[n]);
        if (j == 0) *(f32x2*)stats[wave][at] = f32x2{w.m[n], w.l[n]};
        if (first_col + at < cols) {
#pragma unroll
            for (int i = 0; i < D / 16; ++i) *(f32x4*)&results[wave][at][16 * i + 4 * j] = w.o[n][i];
        }
    }
    __syncthreads();
    const int64_t part = split * ((int64_t)a.n_seqs * a.n_tokens * a.n_q_heads);
    const int here = min(cols - first_col, kCols);
#pragma unroll 1
    for (int i = threadIdx.x; i < here * (D / 4); i += 64 * kWaves) {
        const int r = i / (D / 4), c4 = i % (D / 4), row = places[r];
        float top = stats[0][r][0], sum = 0.f;
#pragma unroll
        for (int v = 1; v < kWaves; ++v) top = fmaxf(top, stats[v][r][0]);
        f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < kWaves; ++v) {
            const f32x2 st = *(const f32x2*)stats[v][r];
            const float f = __builtin_amdgcn_exp2f(st[0] - top);
            sum += f * st[1];
            o += f * *(const f32x4*)&results[v][r][4 * c4];
        }
        if (a.splits == 1) {
            const float f = sum == 0.f ? 0.f : 1.f / sum;
            bf16x4 y;
#pragma unroll
            for (int x = 0; x < 4; ++x) y[x] = quotient(o[x], f);
            *(bf16x4*)((uint16_t*)a.out + (int64_t)row * D + 4 * c4) = y;
            if (a.lse != nullptr && c4 == 0) a.lse[row] = sum == 0.f ? -INFINITY : top + __builtin_amdgcn_logf(sum);
        } else {
            *(f32x4*)((float*)a.out + (part + row) * D + 4 * c4) = o;
            if (c4 == 0) *(f32x4*)(a.lse + 4 * (part + row)) = f32x4{top, sum, sum, 0.f};
        }
    }
}

template <int D, bool kListed, bool kOnce>
void launch(const CacheAttention& x, const AttendArgs& a, dim3 blocks, hipStream_t stream) {
    const dim3 threads(64 * x.waves);
    if (x.col_tiles == 2) hipLaunchKernelGGL((cache8_attention_kernel<D, 2, 4, kListed, false>), blocks, threads, 0, stream, a);
    else if (x.waves == 4) hipLaunchKernelGGL((cache8_attention_kernel<D, 1, 4, kListed, kOnce>), blocks, threads, 0, stream, a);
    else hipLaunchKernelGGL((cache8_attention_kernel<D, 1, 8, kListed, kOnce>), blocks, threads, 0, stream, a);
}

// Past the caches or through them, us: 64 x 2048 tokens on 32 heads 163 and 184, on 32/8 44 and 49.5, 64 x 8192 on 64/8 165 and 186.  Where sequences share all their pages, as branches of
// one prompt do, the other way round, by less: 71 and 62.5, 18.9 and 18.3, 64 and 61 (of four prompts 80 and 65, 20.1 and 19.3, 73 and 67); the host does not know.
template <int D>
void launch(const CacheAttention& x, const AttendArgs& a, dim3 blocks, hipStream_t stream) {
    if (a.blocks == nullptr) launch<D, false, true>(x, a, blocks, stream);
    else if (a.n_tokens == 1) launch<D, true, true>(x, a, blocks, stream);
    else launch<D, true, false>(x, a, blocks, stream);            // (a sequence's tokens choose much the same blocks)
}

}  // namespace

// n_blocks > 0: lists of so many blocks.
// What is waited for at the end is the wavefront with the most blocks (8 KB at 128 channels), so few heads are split along the cache until a workgroup of eight wavefronts has
// every compute unit to itself, and are taken by eight wavefronts unsplit up to one head a unit (two at 64 channels); more heads by four, two workgroups a unit.
// Splitting takes a launch that joins the parts.  Measured, us (pass with the join; w: wavefronts, s: parts), 128 channels:
//   heads x tokens   8 x 1000: w8 s1 7.3, w8 s4 7.1, w4 s8 6.8;  32 x 1434: w8 s1 11.5, w8 s4 9.6, w4 s8 8.9;  64 x 1200: w8 s1 10.6, w8 s4 10.2;  64 x 2048: w8 s1 14.8, w8 s4 11.6, w4 s8
//   12.0;  96 x 1500: w8 s1 12.8, w8 s2 11.7;  128 x 1800: w8 s1 14.6, w8 s2 15.2;  128 x 4000: w8 s1 27.3, w8 s2 26.0;  160 x 1800: w8 s1 15.4, w4 s1 17.8, w4 s4 20.6;  160 x 100 ... 8000:
//   w8 s1 43.3, w4 s4 37.8;  256 x 2000: w4 s1 23.5, w8 s1 23.6;  480 x 1800: w4 s1 37.9, w8 s1 38.5, w4 s2 41.0;  480 x 300 ... 5000: w4 s1 65.2, w4 s2 68.1;  8 x 65536: w8 s32 26.7, w4 s64 27.8
//   64 channels: 256 x 2000: w8 s1 13.1, w4 s1 14.9;  480 x 1800: 19.9 either way;  8 x 16384: w4 s64 9.3, w8 s32 9.1
//   24 rows a head: 64 x 4096: s1 35.5, s4 19.5, s8 21.4;  128 x 2048: s1 21.4, s2 19.5 (by the rule s1)
//   lists of 64 blocks: 8 heads: w8 s8 7.6, w8 s1 10.9;  64: w8 s4 11.6, w8 s1 14.9;  256: w4 s1 24.0, w8 s1 24.6;  of 16: 2048 heads: w4 s1 45.9, w8 s1 57.5
CacheAttention plan_cache8_attention(int32_t n_seqs, int32_t n_tokens, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t max_len, int32_t n_blocks) {
    constexpr int64_t kUnits = 256;
    CacheAttention x{};
    const int64_t groups = n_blocks > 0 ? (int64_t)n_seqs * n_tokens : n_seqs;
    const int cols = (n_blocks > 0 ? 1 : n_tokens) * (n_q_heads / n_kv_heads);
    const int tiles = (cols + 15) / 16;
    x.col_tiles = tiles == 1 ? 1 : 2;
    x.col_groups = (tiles + x.col_tiles - 1) / x.col_tiles;
    x.repeats = 1;
    const int64_t units = groups * n_kv_heads * x.col_groups, key_tiles = n_blocks > 0 ? n_blocks : (max_len + 31) / 32;
    x.waves = x.col_tiles == 1 && units <= (head_dim == 64 ? 2 * kUnits : kUnits - 1) ? 8 : 4;
    int64_t splits = 1;
    if (units > 0 && units <= kUnits / 2 && key_tiles > (units <= kUnits * 3 / 8 ? 40 : 72)) splits = kUnits / units;
    if (units > kUnits / 2 && units < kUnits && key_tiles >= 128 && head_dim == 128) {      // (long enough that all units have to help)
        x.waves = 4;
        splits = 2 * kUnits / units;
    }
    int64_t chunk = (key_tiles + splits - 1) / splits;
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

int launch_cache8_attention(const CacheAttention& x, const CacheView& c, int32_t head_dim, const void* q, const int32_t* slots, int32_t n_seqs,
                            int32_t n_tokens, int32_t n_q_heads, const int32_t* blocks, int32_t n_blocks, float scale_log2, void* out, float* lse, void* parts,
                            float* stats, hipStream_t stream) {
    if (n_seqs == 0) return PYR_OK;
    const bool split = x.splits > 1, listed = blocks != nullptr;
    const AttendArgs a{c, (const uint16_t*)q, slots, blocks, split ? parts : out, split ? stats : lse, n_seqs, n_tokens, n_blocks, x.chunk,
                       (uint16_t)n_q_heads, (uint16_t)x.splits, scale_log2};
    const dim3 grid((unsigned)((int64_t)n_seqs * (listed ? n_tokens : 1) * x.col_groups * c.n_kv_heads), (unsigned)x.splits);
    if (head_dim == 128) launch<128>(x, a, grid, stream);
    else launch<64>(x, a, grid, stream);
    const int rc = check_launch();
    if (rc != PYR_OK || !split) return rc;
    return launch_cache_join(c, head_dim, slots, (const float*)parts, stats, n_seqs, n_tokens * n_q_heads, listed ? 0 : x.chunk, x.splits, out, lse, stream);
}

}  // namespace pyr
