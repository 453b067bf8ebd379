// Rows of K and V into the cache held in 4 bits (Algorithm 1, the new rows of KV = cat(PvC_past, KV); what Gather(KV, index) keeps of a prompt
// goes the same way, through its index) and back to bf16, and tokens of the cache into other pages of it, without their values being touched.
//
// A wavefront owns one tile (32 tokens of one KV head) of the destination, whole or in part, so no two of them write a byte, and the halves of a byte are
// tokens of the same tile.  K: lane 16 * block + token has the 32 channels of a scale to itself.  V: lane 16 * j + r has channels
// 2 r, 2 r + 1 of every block for eight tokens, so a block's largest magnitude is a maximum over 16 lanes.
// Bound: reading and writing HBM.
#include "cache_device.h"

namespace pyr {
namespace {

constexpr int kWaves = 4;

__device__ __forceinline__ uint32_t max_u16(uint32_t a, uint32_t b) {      // of both halves
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
template <int kCtrl>
__device__ __forceinline__ uint32_t max_dpp(uint32_t x) {
    return max_u16(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kCtrl, 0xf, 0xf, false));
}
__device__ __forceinline__ uint32_t max_of_16(uint32_t x) {                // of both halves, over 16 lanes
    x = max_dpp<0x140>(x);      // mirror of 16
    x = max_dpp<0x141>(x);      // of 8
    x = max_dpp<0x1b>(x);       // of 4
    return max_dpp<0xb1>(x);    // of 2
}
__device__ __forceinline__ bf16x2 pair_of(uint32_t x) { return __builtin_bit_cast(bf16x2, x); }
__device__ __forceinline__ uint32_t code4(uint32_t old, float a, float b, int sel) {
    return sel == 0   ? __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(old, a, b, 1.f, 0)
           : sel == 1 ? __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(old, a, b, 1.f, 1)
           : sel == 2 ? __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(old, a, b, 1.f, 2)
                      : __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(old, a, b, 1.f, 3);
}

// Workgroups count through the head groups first: the heads of a row lie side by side in memory.
struct StoreArgs {
    CacheView c;
    const uint16_t *k, *v;
    const int32_t *row_idx, *offsets, *slots, *start;
    int32_t n_rows, n_list;
};
static_assert(sizeof(StoreArgs) <= 112, "short arguments");

template <int D>
__global__ __launch_bounds__(64 * kWaves) void cache_store_kernel(StoreArgs a, int32_t tiles_of_piece, int32_t head_groups) {
    constexpr int kBlocks = D / 32, kHalves = D / 64;
    const int lane = threadIdx.x & 63, t = lane & 15, j = lane >> 4;
    const int place = blockIdx.x / head_groups, b = place / tiles_of_piece;
    const int head = (blockIdx.x - place * head_groups) * kWaves + (threadIdx.x >> 6);
    const int slot = cache_slot(a.c, a.slots, b);
    const int start = a.start[b];
    const int first = max(a.offsets[b], 0), last = min(a.offsets[b + 1], a.n_list);
    if (slot < 0 || start < 0 || first >= last || head >= a.c.n_kv_heads) return;
    const int64_t end = min((int64_t)start + (last - first), (int64_t)a.c.max_pages << a.c.shift);       // tokens start .. end - 1
    const int tile = (start >> 5) + (place - b * tiles_of_piece);
    const int64_t token0 = (int64_t)tile * 32;
    if (token0 >= end) return;
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
    uint8_t* const out = cache_tile<D>(a.c, page, head, tile & ((1 << (a.c.shift - 5)) - 1));

    // everything that is read: K (lane 16 * block + token), V (eight tokens, 16 * (e / 4) + 4 * j + e % 4, of channels 2 t, 2 t + 1 of every block), and, where
    // the tile is not written as a whole, V's codes (rows outside are read as row 0 and not used)
    const int64_t row_words = (int64_t)a.c.n_kv_heads * D;
    int krow[kHalves], row[8];
    uint32_t keep = 0;      // the bits of a word of V's codes that stay as they are
    u32x4 x[kHalves][4];
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
        krow[h] = __shfl(from, 16 * (D == 128 ? h : j >> 1) + t);
        const u32x4* k = (const u32x4*)(a.k + max(krow[h], 0) * row_words + head * D + 32 * (D == 128 ? j : j & 1));
#pragma unroll
        for (int i = 0; i < 4; ++i) x[h][i] = k[i];
    }
    uint32_t y[kBlocks][8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        row[e] = __shfl(from, 16 * (e >> 2) + 4 * j + (e & 3));
        if (row[e] < 0) keep |= 0xfu << (4 * e);
        const uint32_t* v = (const uint32_t*)(a.v + max(row[e], 0) * row_words + head * D) + t;
#pragma unroll
        for (int p = 0; p < kBlocks; ++p) y[p][e] = v[16 * p];
    }
    u32x4* const codes = (u32x4*)(out + 16 * D) + lane;
    uint8_t* const scales = out + 33 * D + j * (8 * kBlocks);
    u32x4 old[kHalves] = {};
    if (keep != 0 && keep != 0xffffffffu) {
#pragma unroll
        for (int h = 0; h < kHalves; ++h) old[h] = codes[64 * h];
    }

    // K
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
        const int half = D == 128 ? h : j >> 1, block = D == 128 ? j : j & 1;
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) top = max_u16(top, x[h][i >> 2][i & 3] & 0x7fff7fffu);
        const uint32_t byte = scale_byte(max(top & 0xffff, top >> 16));
        const float scale = scale_of(byte);
        u32x4 word;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t w = 0;
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, pair_of(x[h][i][0]), scale, 0);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, pair_of(x[h][i][1]), scale, 1);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, pair_of(x[h][i][2]), scale, 2);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, pair_of(x[h][i][3]), scale, 3);
            word[i] = byte == 255 ? 0 : w;
        }
        if (krow[h] >= 0) {
            *(u32x4*)(out + h * 1024 + lane * 16) = word;
            out[32 * D + (block * 16 + t) * 2 + half] = (uint8_t)byte;
        }
    }

    // V
    if (keep == 0xffffffffu) return;
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
        u32x4 word{0, 0, 0, 0};
#pragma unroll
        for (int p2 = 0; p2 < 2; ++p2) {
            const int p = 2 * h + p2;
            float f[8];
            u32x2 bytes{0, 0};
            uint32_t bad = 0;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const uint32_t a0 = y[p][e] & 0x7fff7fffu, a1 = y[p][e + 1] & 0x7fff7fffu;
                const uint32_t top = max_of_16(max(a0 & 0xffff, a0 >> 16) | max(a1 & 0xffff, a1 >> 16) << 16);
                const uint32_t s0 = scale_byte(top & 0xffff), s1 = scale_byte(top >> 16);
                if (s0 == 255) bad |= 0xfu << (4 * e);
                if (s1 == 255) bad |= 0xf0u << (4 * e);
                bytes[e >> 2] |= (s0 | s1 << 8) << (8 * (e & 3));
                f[e] = scale_of(254 - min(s0, 253u));
                f[e + 1] = scale_of(254 - min(s1, 253u));
            }
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                uint32_t w = 0;
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float v0 = __uint_as_float(q == 0 ? y[p][e] << 16 : y[p][e] & 0xffff0000u);
                    const float v1 = __uint_as_float(q == 0 ? y[p][e + 1] << 16 : y[p][e + 1] & 0xffff0000u);
                    w = code4(w, v0 * f[e], v1 * f[e + 1], e >> 1);
                }
                word[2 * p2 + q] = w & ~bad;
            }
            if (keep == 0) {
                if (t == 0) *(u32x2*)(scales + 8 * p) = bytes;
            } else if (t < 8) {
                const uint32_t byte = (t < 4 ? bytes[0] : bytes[1]) >> (8 * (t & 3));
                if ((keep >> (4 * t) & 1) == 0) scales[8 * p + t] = (uint8_t)byte;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) word[i] = (word[i] & ~keep) | (old[h][i] & keep);
        codes[64 * h] = word;
    }
}

struct LoadArgs {
    CacheView c;
    const int32_t *slots, *offsets;
    uint16_t *k, *v;
    int32_t n_rows, tiles_of_seq, head_groups;
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
    if (slot < 0 || first < 0 || head >= a.c.n_kv_heads) return;
    const int page = a.c.table[(int64_t)slot * a.c.max_pages + (tile >> (a.c.shift - 5))];
    const int count = min(last - first, cache_len(a.c, slot)) - 32 * tile;      // tokens of this tile and behind it
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
    auto meet = [] {                                          // (the wavefront's own part of LDS: its accesses keep their order)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    auto write_rows = [&](uint16_t* out) {
        constexpr int kLanes = D / 8;                         // of a row
        meet();
#pragma unroll
        for (int i = 0; i < 32 * kLanes / 64; ++i) {
            const int token = i * (64 / kLanes) + lane / kLanes, channel = 8 * (lane % kLanes);
            const u32x4 x = *(const u32x4*)&rows[token][channel];
            if (token < count) *(u32x4*)(out + to + token * row_words + channel) = x;
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
    int32_t n_list, tiles_of_seq;
};
static_assert(sizeof(MoveArgs) <= 112, "short arguments");

// Token t of a slot becomes what was its token kept_idx[out_offsets[b] + t] - seq_offsets[b]: old_rows [n, 1 + max_pages] holds the length and
// the pages that the slot had (cache_pages.hip has changed its row of the table already; nothing else has written to the old pages since).
// A wavefront takes every head_step-th head of a tile: finding the tile's sources is four loads that wait for one another.
template <int D>
__global__ __launch_bounds__(64 * kWaves) void cache_move_kernel(MoveArgs a, int32_t head_groups) {
    constexpr int kBlocks = D / 32, kHalves = D / 64;
    const int lane = threadIdx.x & 63, t = lane & 15, j = lane >> 4;
    const int place = blockIdx.x / head_groups, b = place / a.tiles_of_seq, tile = place - b * a.tiles_of_seq;
    const int first_head = (blockIdx.x - place * head_groups) * kWaves + (threadIdx.x >> 6), head_step = head_groups * kWaves;
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
    int kfrom[kHalves], vfrom[8];
#pragma unroll
    for (int h = 0; h < kHalves; ++h) kfrom[h] = __shfl(from, 16 * (D == 128 ? h : j >> 1) + t);
#pragma unroll
    for (int e = 0; e < 8; ++e) vfrom[e] = __shfl(from, 16 * (e >> 2) + 4 * j + (e & 3));
    // scale bytes of V: lane t of a group takes slot t / 2, every second block
    const int se = t >> 1, stoken = 16 * (se >> 2) + 4 * j + (se & 3), sfrom = __shfl(from, stoken);
    auto source = [&](int token, int head) -> const uint8_t* {      // (a token that comes from nowhere: any, and what is read is not used)
        token = max(token, 0);
        return cache_tile<D>(a.c, token >> a.c.shift, head, (token >> 5) & tile_mask);
    };
    for (int head = first_head; head < a.c.n_kv_heads; head += head_step) {
        uint8_t* const out = cache_tile<D>(a.c, page, head, tile & tile_mask);
        u32x4 kc[kHalves], vx[8][kHalves];
        uint8_t ks[kHalves], vs[kBlocks / 2];
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
            const uint8_t* in = source(kfrom[h], head);
            const int half = kfrom[h] >> 4 & 1, old = kfrom[h] & 15, block = D == 128 ? j : j & 1;
            kc[h] = *(const u32x4*)(in + ((half * kBlocks + block) * 16 + old) * 16);
            ks[h] = in[32 * D + (block * 16 + old) * 2 + half];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint8_t* in = source(vfrom[e], head);
#pragma unroll
            for (int h = 0; h < kHalves; ++h) vx[e][h] = *(const u32x4*)(in + 16 * D + h * 1024 + (16 * (vfrom[e] >> 2 & 3) + t) * 16);
        }
#pragma unroll
        for (int i = 0; i < kBlocks / 2; ++i)
            vs[i] = source(sfrom, head)[33 * D + (((sfrom >> 2 & 3) * kBlocks + 2 * i + (t & 1)) * 2 + (sfrom >> 4 & 1)) * 4 + (sfrom & 3)];
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
            const int half = D == 128 ? h : j >> 1, block = D == 128 ? j : j & 1;
            *(u32x4*)(out + h * 1024 + lane * 16) = kfrom[h] >= 0 ? kc[h] : u32x4{0, 0, 0, 0};
            out[32 * D + (block * 16 + t) * 2 + half] = kfrom[h] >= 0 ? ks[h] : 16 * half + t < count ? 255 : 0;
        }
        u32x4 y[kHalves] = {};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int shift = 4 * ((vfrom[e] >> 4 & 1) * 4 + (vfrom[e] & 3));
            const uint32_t mask = vfrom[e] >= 0 ? 15 : 0;
#pragma unroll
            for (int h = 0; h < kHalves; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) y[h][i] |= (vx[e][h][i] >> shift & mask) << (4 * e);
        }
#pragma unroll
        for (int h = 0; h < kHalves; ++h) *(u32x4*)(out + 16 * D + h * 1024 + lane * 16) = y[h];
#pragma unroll
        for (int i = 0; i < kBlocks / 2; ++i)
            out[33 * D + (j * kBlocks + 2 * i + (t & 1)) * 8 + se] = sfrom >= 0 ? vs[i] : stoken < count ? 255 : 0;
    }
}

}  // namespace

int launch_cache_store(const CacheView& c, int32_t head_dim, const void* k, const void* v, int32_t n_rows, const int32_t* row_idx, int32_t n_list,
                       const int32_t* offsets, const int32_t* slots, const int32_t* start, int32_t n_seqs, int32_t max_new, hipStream_t stream) {
    if (n_seqs == 0 || max_new == 0) return PYR_OK;
    const int32_t tiles = (max_new + 30) / 32 + 1;
    const StoreArgs a{c, (const uint16_t*)k, (const uint16_t*)v, row_idx, offsets, slots, start, n_rows, n_list};
    const int32_t head_groups = (c.n_kv_heads + kWaves - 1) / kWaves;
    const dim3 grid((unsigned)((int64_t)n_seqs * tiles * head_groups));
    if (head_dim == 128) hipLaunchKernelGGL(cache_store_kernel<128>, grid, dim3(64 * kWaves), 0, stream, a, tiles, head_groups);
    else hipLaunchKernelGGL(cache_store_kernel<64>, grid, dim3(64 * kWaves), 0, stream, a, tiles, head_groups);
    return check_launch();
}

int launch_cache_load(const CacheView& c, int32_t head_dim, const int32_t* slots, const int32_t* offsets, int32_t n_seqs, int32_t max_len,
                      void* k, void* v, int32_t n_rows, hipStream_t stream) {
    if (n_seqs == 0 || max_len == 0) return PYR_OK;
    const LoadArgs a{c, slots, offsets, (uint16_t*)k, (uint16_t*)v, n_rows, (max_len + 31) / 32, (c.n_kv_heads + kWaves - 1) / kWaves};
    const dim3 grid((unsigned)((int64_t)n_seqs * a.tiles_of_seq * a.head_groups));
    if (head_dim == 128) hipLaunchKernelGGL(cache_load_kernel<128>, grid, dim3(64 * kWaves), 0, stream, a);
    else hipLaunchKernelGGL(cache_load_kernel<64>, grid, dim3(64 * kWaves), 0, stream, a);
    return check_launch();
}

int launch_cache_move(const CacheView& c, int32_t head_dim, const int32_t* slots, const int32_t* kept_idx, int32_t n_list, const int32_t* seq_offsets,
                      const int32_t* out_offsets, const int32_t* old_rows, const int32_t* status, int32_t n_seqs, int32_t max_keep, hipStream_t stream) {
    if (n_seqs == 0 || max_keep == 0) return PYR_OK;
    const MoveArgs a{c, slots, kept_idx, seq_offsets, out_offsets, old_rows, status, n_list, (max_keep + 31) / 32};
    const int64_t places = (int64_t)n_seqs * a.tiles_of_seq;
    int32_t head_groups = (c.n_kv_heads + kWaves - 1) / kWaves;
    while (head_groups > 1 && places * ((head_groups + 1) / 2) >= 1024) head_groups = (head_groups + 1) / 2;
    const dim3 grid((unsigned)(places * head_groups));
    if (head_dim == 128) hipLaunchKernelGGL(cache_move_kernel<128>, grid, dim3(64 * kWaves), 0, stream, a, head_groups);
    else hipLaunchKernelGGL(cache_move_kernel<64>, grid, dim3(64 * kWaves), 0, stream, a, head_groups);
    return check_launch();
}

}  // namespace pyr
