// Rows of K and V into the cache held in 4 bits (Algorithm 1, the new rows of KV = cat(PvC_past, KV); what Gather(KV, index) keeps of a prompt
// goes the same way, through its index) and back to bf16, and tokens of the cache into other pages of it, without their values being touched.
//
// A wavefront owns one tile (32 tokens of one KV head) of the destination, whole or in part, so no two of them write a byte, and the halves of a byte are
// tokens of the same tile.
// Bound: reading and writing HBM.  70 % of 8 x 2048 rows on 32 heads, d = 128, K and V: stored 43 us, 239 MB, 5.6 TB/s, read back 36 us, 6.5 TB/s; cut
// from 8 x 2048 tokens 29 us (122 MB with the whole lines that single tokens of a tile take, 4.2 TB/s), 4 x 32768 tokens on 8 heads cut to one half 48 us
// (255 MB so, 5.3 TB/s).  V's eight tokens gathered word by word took as long with 178 registers, and twice as long with 128 and spills.
#include "cache_device.h"

namespace pyr {
namespace {

// bf16 rows are read and written past the caches (nontemporal), codes are not: stored and read back 103 -> 78 us, cut and read back 97 -> 86 us.
constexpr int kWaves = 4;

__device__ __forceinline__ uint32_t max_u16(uint32_t a, uint32_t b) {      // of both halves
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
template <int kCtrl>
__device__ __forceinline__ uint32_t max_dpp(uint32_t x) { return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kCtrl, 0xf, 0xf, false)); }
__device__ __forceinline__ bf16x2 pair_of(uint32_t x) { return __builtin_bit_cast(bf16x2, x); }

// The codes of eight channels, whose block four neighbouring lanes hold; *byte: the block's scale.
__device__ __forceinline__ uint32_t codes_of(u32x4 x, uint32_t* byte) {
    uint32_t top = max_u16(max_u16(x[0] & 0x7fff7fffu, x[1] & 0x7fff7fffu), max_u16(x[2] & 0x7fff7fffu, x[3] & 0x7fff7fffu));
    top = max(top & 0xffff, top >> 16);
    top = max_dpp<0xb1>(top);       // the neighbour's, the other pair's
    top = max_dpp<0x4e>(top);
    *byte = scale_byte(top);
    const float scale = scale_of(*byte);
    uint32_t y = 0;
    y = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(y, pair_of(x[0]), scale, 0);
    y = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(y, pair_of(x[1]), scale, 1);
    y = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(y, pair_of(x[2]), scale, 2);
    y = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(y, pair_of(x[3]), scale, 3);
    return *byte == 255 ? 0 : y;
}

typedef __attribute__((address_space(3))) char* lptr_t;
typedef __attribute__((ext_vector_type(2))) int i32x2;

// Transposing LDS read (ds_read_b64_tr_b8).  Inside every group of 16 lanes, lane j receives byte (j & 7) of the 8-byte words addressed by lanes
// (j >> 3), 2 + (j >> 3), 4 + (j >> 3) ... 14 + (j >> 3), in this order.
__device__ __forceinline__ i32x2 lds_read_tr8(uint32_t lds_addr) {
    return __builtin_amdgcn_ds_read_tr8_b64_v2i32((i32x2 __attribute__((address_space(3)))*)(uintptr_t)lds_addr);
}

// A wavefront's own part of LDS: what its lanes have written before is what they read behind this.
__device__ __forceinline__ void meet() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Workgroups count through the head groups first: the heads of a row lie side by side in memory.
struct StoreArgs {
    CacheView c;
    const uint16_t *k, *v;
    const int32_t *row_idx, *offsets, *slots, *start;
    int32_t n_rows, n_list, tiles_of_piece, head_groups;
};
static_assert(sizeof(StoreArgs) <= 112, "short arguments");

// Rows are read and quantised as they lie in memory, 16 bytes a lane; their codes and scales meet in LDS, from where the lanes take them in
// the tile's order, V's through transposing reads that turn bytes of two channels of a token into words of eight tokens of a channel.
template <int D>
__global__ __launch_bounds__(64 * kWaves) void cache_store_kernel(StoreArgs a) {
    constexpr int kBlocks = D / 32, kHalves = D / 64, kRow = D / 2 + 16;      // bytes of a token's codes in LDS
    struct Staged {
        uint8_t k[32][kRow], v[32][kRow], scales[2 * D];
    };
    __shared__ __align__(16) Staged all_staged[kWaves];
    const int lane = threadIdx.x & 63, t = lane & 15, j = lane >> 4;
    const int place = blockIdx.x / a.head_groups, b = place / a.tiles_of_piece;
    const int head = (blockIdx.x - place * a.head_groups) * kWaves + (threadIdx.x >> 6);
    const int slot = cache_slot(a.c, a.slots, b);
    const int place_of_piece = a.start[b], offset = a.offsets[b];
    const int first = max(offset, 0), last = min(a.offsets[b + 1], a.n_list);
    bool again = false;                                           // an earlier row has the slot: its tile may be written by two wavefronts at once
    for (int i = lane; i < b; i += 64) again |= a.slots[i] == slot;
    if (slot < 0 || place_of_piece < 0 || first >= last || head >= a.c.n_kv_heads) return;
    const int64_t start = place_of_piece + ((int64_t)first - offset);      // (rows below 0 are not there: their tokens stay)
    const int64_t end = min(start + (last - first), (int64_t)cache_len(a.c, slot));      // tokens start .. end - 1 (the table holds anything behind the length)
    const int64_t token0 = (start & ~31) + 32 * (int64_t)(place - b * a.tiles_of_piece);
    if (token0 >= end) return;
    const int tile = (int)(token0 >> 5);
    const int page = a.c.table[(int64_t)slot * a.c.max_pages + (token0 >> a.c.shift)];
    // lane l: the row that token l & 31 of the tile gets; -1: none
    int from = -1;
    {
        const int64_t at = token0 + (lane & 31);
        if (at >= start && at < end) {
            const int row = first + (int)(at - start);
            from = a.row_idx != nullptr ? a.row_idx[row] : row;
            if (from < 0 || from >= a.n_rows) from = -1;
        }
    }
    if (page < 0 || page >= a.c.n_pages) return;
    const uint32_t stored = (uint32_t)__builtin_amdgcn_ballot_w64(from >= 0);                            // bit t: token t
    if (stored == 0 || __builtin_amdgcn_ballot_w64(again) != 0) return;
    uint8_t* const out = cache_tile<D>(a.c, page, head, tile & ((1 << (a.c.shift - 5)) - 1));

    // what is read: rows (one that is not there: row 0, not stored) and, where the tile is not written as a whole, V's codes
    constexpr int kLanes = D / 8, kLoads = 32 * kLanes / 64;      // lanes of a row
    const int64_t row_words = (int64_t)a.c.n_kv_heads * D;
    u32x4 kx[kLoads], vx[kLoads];
    auto some = [&](int i) { return (stored >> (i * (64 / kLanes)) & ((1u << (64 / kLanes)) - 1)) != 0; };      // (of a load's rows: one token is one load)
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        if (!some(i)) continue;
        const int64_t at = max(__shfl(from, i * (64 / kLanes) + lane / kLanes), 0) * row_words + head * D + 8 * (lane % kLanes);
        kx[i] = __builtin_nontemporal_load((const u32x4*)(a.k + at));
        vx[i] = __builtin_nontemporal_load((const u32x4*)(a.v + at));
    }
    uint32_t keep = 0;                                            // the bits of a word of V's codes that stay as they are
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if ((stored >> (16 * (e >> 2) + 4 * j + (e & 3)) & 1) == 0) keep |= 0xfu << (4 * e);
    u32x4* const codes = (u32x4*)(out + 16 * D) + lane;
    u32x4 old[kHalves] = {};
    if (stored != 0xffffffffu) {
#pragma unroll
        for (int h = 0; h < kHalves; ++h) old[h] = codes[64 * h];
    }

    Staged& staged = all_staged[threadIdx.x >> 6];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        if (!some(i)) continue;
        const int token = i * (64 / kLanes) + lane / kLanes, piece = lane % kLanes, block = piece >> 2;
        uint32_t ks, vs;
        *(uint32_t*)&staged.k[token][4 * piece] = codes_of(kx[i], &ks);
        *(uint32_t*)&staged.v[token][4 * piece] = codes_of(vx[i], &vs);
        if ((lane & 3) == 0) {
            const int half = token >> 4, low = token & 15;
            staged.scales[(block * 16 + low) * 2 + half] = (uint8_t)ks;
            staged.scales[D + (((low >> 2) * kBlocks + block) * 2 + half) * 4 + (low & 3)] = (uint8_t)vs;
        }
    }
    meet();
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
        const int token = 16 * (D == 128 ? h : j >> 1) + t, block = D == 128 ? j : j & 1;
        const u32x4 x = *(const u32x4*)&staged.k[token][16 * block];
        if (stored >> token & 1) *(u32x4*)(out + h * 1024 + lane * 16) = x;
    }
    // rows of the transposing reads: tokens 0, 2, 4, 6, 1, 3, 5, 7 of the lanes' eight, 16 * (e / 4) + 4 * j + e % 4; columns: 16 bytes, a block's
    const int e = (t >> 1 & 3) * 2 + (t >> 3);
    const uint32_t rows = (uint32_t)(uintptr_t)(lptr_t)&staged.v[16 * (e >> 2) + 4 * j + (e & 3)][8 * (t & 1)];
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
        u32x4 word;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const i32x2 x = lds_read_tr8(rows + 16 * (2 * h + p));
            const uint32_t even = x[0], odd = x[1];
            word[2 * p] = (even & 0x0f0f0f0fu) | (odd & 0x0f0f0f0fu) << 4;
            word[2 * p + 1] = (even >> 4 & 0x0f0f0f0fu) | (odd & 0xf0f0f0f0u);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) word[i] = (word[i] & ~keep) | (old[h][i] & keep);
        if (keep != 0xffffffffu) codes[64 * h] = word;
    }
    if (lane < 2 * D / 4) {
        const uint32_t x = *(const uint32_t*)&staged.scales[4 * lane];
        uint8_t* to = out + 32 * D + 4 * lane;
        if (stored == 0xffffffffu) *(uint32_t*)to = x;
        else {
            const bool is_k = lane < D / 4;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // K: [block][token 16][half], V: [j][block][half][s]
                const int token = is_k ? 16 * (i & 1) + (2 * lane + (i >> 1) & 15) : 16 * (lane & 1) + 4 * ((lane - D / 4) / (2 * kBlocks)) + i;
                if (stored >> token & 1) to[i] = (uint8_t)(x >> (8 * i));
            }
        }
    }
}

struct LoadArgs {
    CacheView c;
    const int32_t *slots, *offsets;
    uint16_t *k, *v;
    int32_t n_rows, max_len, tiles_of_seq, head_groups;
};
static_assert(sizeof(LoadArgs) <= 112, "short arguments");

// The values of a tile meet in LDS, from where a wavefront writes whole rows of the head, 16 bytes a lane.
template <int D>
__global__ __launch_bounds__(64 * kWaves) void cache_load_kernel(LoadArgs a) {
    constexpr int kBlocks = D / 32, kHalves = D / 64, kRow = D + 8;      // bf16 of a row in LDS
    __shared__ __align__(16) uint16_t staged[kWaves][32][kRow];
    const int lane = threadIdx.x & 63, t = lane & 15, j = lane >> 4;
    const int place = blockIdx.x / a.head_groups, b = place / a.tiles_of_seq, tile = place - b * a.tiles_of_seq;
    const int head = (blockIdx.x - place * a.head_groups) * kWaves + (threadIdx.x >> 6);
    const int slot = cache_slot(a.c, a.slots, b);
    const int first = a.offsets[b], last = min(a.offsets[b + 1], a.n_rows);
    if (slot < 0 || first < 0 || last <= first || head >= a.c.n_kv_heads) return;
    const int page = a.c.table[(int64_t)slot * a.c.max_pages + (tile >> (a.c.shift - 5))];
    const int count = min(min(last - first, cache_len(a.c, slot)), a.max_len) - 32 * tile;      // tokens of this tile and behind it
    if (count <= 0 || page < 0 || page >= a.c.n_pages) return;
    const uint8_t* const in = cache_tile<D>(a.c, page, head, tile & ((1 << (a.c.shift - 5)) - 1));
    uint16_t(*const rows)[kRow] = staged[threadIdx.x >> 6];
    const int64_t row_words = (int64_t)a.c.n_kv_heads * D, to = ((int64_t)first + 32 * tile) * row_words + head * D;
    u32x4 kc[kHalves], vc[kHalves], vs[kHalves];
    uint32_t ks[kHalves];
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
        kc[h] = *(const u32x4*)(in + h * 1024 + lane * 16);
        ks[h] = in[32 * D + ((D == 128 ? j : j & 1) * 16 + t) * 2 + (D == 128 ? h : j >> 1)];
        vc[h] = *(const u32x4*)(in + 16 * D + h * 1024 + lane * 16);
        vs[h] = *(const u32x4*)(in + 33 * D + j * (8 * kBlocks) + 16 * h);
    }
    auto write_rows = [&](uint16_t* out) {
        constexpr int kLanes = D / 8;                         // of a row
        meet();
#pragma unroll
        for (int i = 0; i < 32 * kLanes / 64; ++i) {
            const int token = i * (64 / kLanes) + lane / kLanes, channel = 8 * (lane % kLanes);
            const u32x4 x = *(const u32x4*)&rows[token][channel];
            if (token < count) __builtin_nontemporal_store(x, (u32x4*)(out + to + token * row_words + channel));
        }
        meet();
    };
    if (a.k != nullptr) {
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
            bf16x8* row = (bf16x8*)&rows[16 * (D == 128 ? h : j >> 1) + t][32 * (D == 128 ? j : j & 1)];
#pragma unroll
            for (int i = 0; i < 4; ++i) row[i] = values_of(kc[h][i], scale_of(ks[h]));
        }
        write_rows(a.k);
    }
    if (a.v != nullptr) {
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
#pragma unroll
            for (int p2 = 0; p2 < 2; ++p2) {
                const uint32_t c0 = vc[h][2 * p2], c1 = vc[h][2 * p2 + 1];
                // bytes of the two channels of tokens 0, 2, 4, 6 and 1, 3, 5, 7 of the lane's eight
                const uint32_t even = (c0 & 0x0f0f0f0fu) | (c1 & 0x0f0f0f0fu) << 4, odd = (c0 >> 4 & 0x0f0f0f0fu) | (c1 & 0xf0f0f0f0u);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float scale = scale_of(vs[h][2 * p2 + (e >> 2)] >> (8 * (e & 3)) & 255);
                    const uint32_t from = (e & 1 ? odd : even) >> (8 * (e >> 1));
                    *(bf16x2*)&rows[16 * (e >> 2) + 4 * j + (e & 3)][32 * (2 * h + p2) + 2 * t] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(from, scale, 0);
                }
            }
        }
        write_rows(a.v);
    }
}

struct MoveArgs {
    CacheView c;
    const int32_t *slots, *kept_idx, *seq_offsets, *out_offsets, *old_rows, *status;
    int32_t n_list, tiles_of_seq, head_groups;
};
static_assert(sizeof(MoveArgs) <= 112, "short arguments");

// Token t of a slot becomes what was its token kept_idx[out_offsets[b] + t] - seq_offsets[b]: old_rows [n, 1 + max_pages] holds the length and
// the pages that the slot had (cache_pages.hip has changed its row of the table already; nothing else has written to the old pages since).
// A wavefront takes every head_step-th head of a tile: finding the tile's sources is four loads that wait for one another.
// K's codes are gathered by 16 bytes.  V's are taken a source tile at a time (kept tokens come in order, so that there are two or three; any order
// works): read as they lie, turned in LDS to a row of bytes per token, the kept rows copied, and turned back into words of eight tokens.
template <int D>
__global__ __launch_bounds__(64 * kWaves) void cache_move_kernel(MoveArgs a) {
    constexpr int kBlocks = D / 32, kHalves = D / 64, kRow = D / 2 + 16;
    struct Staged {
        uint8_t words[kBlocks][4][16][8], source[32][kRow], kept[32][kRow];
    };
    __shared__ __align__(16) Staged all_staged[kWaves];
    const int lane = threadIdx.x & 63, t = lane & 15, j = lane >> 4;
    const int place = blockIdx.x / a.head_groups, b = place / a.tiles_of_seq, tile = place - b * a.tiles_of_seq;
    const int first_head = (blockIdx.x - place * a.head_groups) * kWaves + (threadIdx.x >> 6), head_step = a.head_groups * kWaves;
    const int tile_shift = a.c.shift - 5, tile_mask = (1 << tile_shift) - 1;
    const int status = *a.status, slot = cache_slot(a.c, a.slots, b), first = a.out_offsets[b], base = a.seq_offsets[b];
    if (status != 0 || slot < 0) return;
    const int page = a.c.table[(int64_t)slot * a.c.max_pages + (tile >> tile_shift)];
    const int32_t* old_row = a.old_rows + (int64_t)b * (1 + a.c.max_pages);
    const int old_len = old_row[0], at = first + 32 * tile + (lane & 31);
    const int kept = at >= 0 && at < a.n_list ? a.kept_idx[at] - base : -1;
    const int count = cache_len(a.c, slot) - 32 * tile;
    if (count <= 0 || page < 0 || page >= a.c.n_pages) return;
    // lane l: where token l & 31 of the tile comes from, as a token of the pool; -1: nowhere
    int from = -1;
    if ((lane & 31) < count && kept >= 0 && kept < old_len) {
        const int p = old_row[1 + (kept >> a.c.shift)];
        if (p >= 0 && p < a.c.n_pages) from = (p << a.c.shift) + (kept & ((1 << a.c.shift) - 1));
    }
    const uint32_t all = (uint32_t)__builtin_amdgcn_ballot_w64(from >= 0);
    auto source_of = [&](int token, int head) -> const uint8_t* {      // (a token that comes from nowhere: any, and what is read is not used)
        token = max(token, 0);
        return cache_tile<D>(a.c, token >> a.c.shift, head, (token >> 5) & tile_mask);
    };
    Staged& staged = all_staged[threadIdx.x >> 6];
    // scale bytes of V: lane t of a group takes slot t / 2, every second block
    const int se = t >> 1, stoken = 16 * (se >> 2) + 4 * j + (se & 3), sfrom = __shfl(from, stoken);
    // rows of the transposing reads.  Words: 8 lanes' columns r of two groups of eight tokens; kept: tokens 0, 2, 4, 6, 1, 3, 5, 7 of the lanes' eight
    const int e = (t >> 1 & 3) * 2 + (t >> 3), column = 8 * (j & 1);
    const uint32_t words = (uint32_t)(uintptr_t)(lptr_t)&staged.words[0][2 * (j >> 1) + (t & 1)][column + (t >> 1)][0];
    const uint32_t rows = (uint32_t)(uintptr_t)(lptr_t)&staged.kept[16 * (e >> 2) + 4 * j + (e & 3)][8 * (t & 1)];
    // the token whose columns a transposing read of words gives to a lane: byte t & 7 of group 2 * (j / 2) + t / 8
    const int we = (t & 3) * 2 + (t >> 2 & 1), wtoken = 16 * (we >> 2) + 4 * (2 * (j >> 1) + (t >> 3)) + (we & 3);
    for (int head = first_head; head < a.c.n_kv_heads; head += head_step) {
        uint8_t* const out = cache_tile<D>(a.c, page, head, tile & tile_mask);
        u32x4 kc[kHalves], x[kHalves], y[kHalves];
        uint8_t ks[kHalves], vs[kBlocks / 2];
        uint32_t left = all;
        // the tokens of the first source tile that is left; its words
        auto next = [&](u32x4 (&v)[kHalves]) -> uint32_t {
            if (left == 0) return 0;
            const int token = __builtin_amdgcn_readlane(from, __builtin_ctz(left));
            const uint32_t mine = left & (uint32_t)__builtin_amdgcn_ballot_w64(from >> 5 == token >> 5);
            left &= ~mine;
            const uint8_t* in = source_of(token, head) + 16 * D + lane * 16;
#pragma unroll
            for (int h = 0; h < kHalves; ++h) v[h] = *(const u32x4*)(in + h * 1024);
            return mine;
        };
        uint32_t mine = next(x);
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
            const int token = __shfl(from, 16 * (D == 128 ? h : j >> 1) + t), half = token >> 4 & 1, old = token & 15, block = D == 128 ? j : j & 1;
            const uint8_t* in = source_of(token, head);
            kc[h] = *(const u32x4*)(in + ((half * kBlocks + block) * 16 + old) * 16);
            ks[h] = in[32 * D + (block * 16 + old) * 2 + half];
        }
#pragma unroll
        for (int i = 0; i < kBlocks / 2; ++i)
            vs[i] = source_of(sfrom, head)[33 * D + (((sfrom >> 2 & 3) * kBlocks + 2 * i + (t & 1)) * 2 + (sfrom >> 4 & 1)) * 4 + (sfrom & 3)];
        // kept tokens that come from nowhere are zero (their scales are not: NaN)
#pragma unroll
        for (int i = 0; i < 32 * (D / 2) / 1024; ++i) *(u32x4*)&staged.kept[(i * 64 + lane) / (D / 32)][16 * (lane % (D / 32))] = u32x4{0, 0, 0, 0};
        while (mine != 0) {
            const uint32_t after = next(y);
#pragma unroll
            for (int p = 0; p < kBlocks; ++p) {
                const uint32_t c0 = x[p >> 1][2 * (p & 1)], c1 = x[p >> 1][2 * (p & 1) + 1];
                *(u32x2*)staged.words[p][j][t] = u32x2{(c0 & 0x0f0f0f0fu) | (c1 & 0x0f0f0f0fu) << 4, (c0 >> 4 & 0x0f0f0f0fu) | (c1 & 0xf0f0f0f0u)};
            }
            meet();
#pragma unroll
            for (int p = 0; p < kBlocks; ++p) {
                const i32x2 w = lds_read_tr8(words + p * (4 * 16 * 8));
                *(i32x2*)&staged.source[wtoken][16 * p + column] = w;
            }
            meet();
#pragma unroll
            for (int i = 0; i < 32 * (D / 2) / 1024; ++i) {
                const int token = (i * 64 + lane) / (D / 32), piece = 16 * (lane % (D / 32));
                const u32x4 row = *(const u32x4*)&staged.source[__shfl(from, token) & 31][piece];
                if (mine >> token & 1) *(u32x4*)&staged.kept[token][piece] = row;
            }
            meet();
            mine = after;
#pragma unroll
            for (int h = 0; h < kHalves; ++h) x[h] = y[h];
        }
        meet();
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
            const int token = 16 * (D == 128 ? h : j >> 1) + t, block = D == 128 ? j : j & 1;
            const bool there = all >> token & 1;
            *(u32x4*)(out + h * 1024 + lane * 16) = there ? kc[h] : u32x4{0, 0, 0, 0};
            out[32 * D + (block * 16 + t) * 2 + (token >> 4)] = there ? ks[h] : token < count ? 255 : 0;
            u32x4 word;
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const i32x2 w = lds_read_tr8(rows + 16 * (2 * h + p));
                const uint32_t even = w[0], odd = w[1];
                word[2 * p] = (even & 0x0f0f0f0fu) | (odd & 0x0f0f0f0fu) << 4;
                word[2 * p + 1] = (even >> 4 & 0x0f0f0f0fu) | (odd & 0xf0f0f0f0u);
            }
            *(u32x4*)(out + 16 * D + h * 1024 + lane * 16) = word;
        }
#pragma unroll
        for (int i = 0; i < kBlocks / 2; ++i)
            out[33 * D + (j * kBlocks + 2 * i + (t & 1)) * 8 + se] = sfrom >= 0 ? vs[i] : stoken < count ? 255 : 0;
        meet();
    }
}

}  // namespace

int launch_cache_store(const CacheView& c, int32_t head_dim, const void* k, const void* v, int32_t n_rows, const int32_t* row_idx, int32_t n_list,
                       const int32_t* offsets, const int32_t* slots, const int32_t* start, int32_t n_seqs, int32_t max_new, hipStream_t stream) {
    if (n_seqs == 0 || max_new == 0) return PYR_OK;
    const int32_t tiles = (int32_t)(((int64_t)max_new + 30) / 32) + 1;
    const StoreArgs a{c, (const uint16_t*)k, (const uint16_t*)v, row_idx, offsets, slots, start, n_rows, n_list, tiles, (c.n_kv_heads + kWaves - 1) / kWaves};
    const dim3 grid((unsigned)((int64_t)n_seqs * tiles * a.head_groups));
    if (head_dim == 128) hipLaunchKernelGGL(cache_store_kernel<128>, grid, dim3(64 * kWaves), 0, stream, a);
    else hipLaunchKernelGGL(cache_store_kernel<64>, grid, dim3(64 * kWaves), 0, stream, a);
    return check_launch();
}

int launch_cache_load(const CacheView& c, int32_t head_dim, const int32_t* slots, const int32_t* offsets, int32_t n_seqs, int32_t max_len,
                      void* k, void* v, int32_t n_rows, hipStream_t stream) {
    if (n_seqs == 0 || max_len == 0) return PYR_OK;
    const LoadArgs a{c, slots, offsets, (uint16_t*)k, (uint16_t*)v, n_rows, max_len, (int32_t)(((int64_t)max_len + 31) / 32), (c.n_kv_heads + kWaves - 1) / kWaves};
    const dim3 grid((unsigned)((int64_t)n_seqs * a.tiles_of_seq * a.head_groups));
    if (head_dim == 128) hipLaunchKernelGGL(cache_load_kernel<128>, grid, dim3(64 * kWaves), 0, stream, a);
    else hipLaunchKernelGGL(cache_load_kernel<64>, grid, dim3(64 * kWaves), 0, stream, a);
    return check_launch();
}

int launch_cache_move(const CacheView& c, int32_t head_dim, const int32_t* slots, const int32_t* kept_idx, int32_t n_list, const int32_t* seq_offsets,
                      const int32_t* out_offsets, const int32_t* old_rows, const int32_t* status, int32_t n_seqs, int32_t max_keep, hipStream_t stream) {
    if (n_seqs == 0 || max_keep == 0) return PYR_OK;
    MoveArgs a{c, slots, kept_idx, seq_offsets, out_offsets, old_rows, status, n_list, (int32_t)(((int64_t)max_keep + 31) / 32), (c.n_kv_heads + kWaves - 1) / kWaves};
    const int64_t places = (int64_t)n_seqs * a.tiles_of_seq;
    while (a.head_groups > 1 && places * ((a.head_groups + 1) / 2) >= 1024) a.head_groups = (a.head_groups + 1) / 2;
    const dim3 grid((unsigned)(places * a.head_groups));
    if (head_dim == 128) hipLaunchKernelGGL(cache_move_kernel<128>, grid, dim3(64 * kWaves), 0, stream, a);
    else hipLaunchKernelGGL(cache_move_kernel<64>, grid, dim3(64 * kWaves), 0, stream, a);
    return check_launch();
}

}  // namespace pyr
