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

struct StoreArgs {
    CacheView c;
    const uint16_t *k, *v;
    const int32_t *row_idx, *offsets, *slots, *start;
    int32_t n_rows, n_list;
};
static_assert(sizeof(StoreArgs) <= 112, "short arguments");

// grid: (n * tiles, head groups); tiles: of the longest piece
template <int D>
__global__ __launch_bounds__(64 * kWaves) void cache_store_kernel(StoreArgs a, int32_t tiles_of_piece) {
    constexpr int kBlocks = D / 32;
    const int lane = threadIdx.x & 63, t = lane & 15, j = lane >> 4;
    const int b = blockIdx.x / tiles_of_piece;
    const int slot = cache_slot(a.c, a.slots, b);
    const int start = a.start[b];
    const int first = max(a.offsets[b], 0), last = min(a.offsets[b + 1], a.n_list);
    if (slot < 0 || start < 0 || first >= last) return;
    const int64_t end = min((int64_t)start + (last - first), (int64_t)a.c.max_pages << a.c.shift);       // tokens start .. end - 1
    const int tile = (start >> 5) + (int)(blockIdx.x % tiles_of_piece);
    const int64_t token0 = (int64_t)tile * 32;
    if (token0 >= end) return;
    const int page = a.c.table[(int64_t)slot * a.c.max_pages + (token0 >> a.c.shift)];
    if (page < 0 || page >= a.c.n_pages) return;
    const int head = blockIdx.y * kWaves + (threadIdx.x >> 6);
    if (head >= a.c.n_kv_heads) return;
    uint8_t* const out = cache_tile<D>(a.c, page, head, tile & ((1 << (a.c.shift - 5)) - 1));

    // source row of a token of the tile; -1: the token is not stored
    auto row_of = [&](int token) -> int {
        const int64_t at = token0 + token;
        if (at < start || at >= end) return -1;
        const int row = first + (int)(at - start);
        const int r = a.row_idx != nullptr ? a.row_idx[row] : row;
        return r >= 0 && r < a.n_rows ? r : -1;
    };

    // K
#pragma unroll
    for (int h = 0; h < D / 64; ++h) {
        const int half = D == 128 ? h : j >> 1, block = D == 128 ? j : j & 1;
        const int row = row_of(16 * half + t);
        if (row >= 0) {
            const u32x4* from = (const u32x4*)(a.k + ((int64_t)row * a.c.n_kv_heads + head) * D + 32 * block);
            u32x4 x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = from[i];
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) top = max_u16(top, x[i >> 2][i & 3] & 0x7fff7fffu);
            const uint32_t byte = scale_byte(max(top & 0xffff, top >> 16));
            const float scale = scale_of(byte);
            u32x4 codes;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t y = 0;
                y = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(y, pair_of(x[i][0]), scale, 0);
                y = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(y, pair_of(x[i][1]), scale, 1);
                y = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(y, pair_of(x[i][2]), scale, 2);
                y = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(y, pair_of(x[i][3]), scale, 3);
                codes[i] = byte == 255 ? 0 : y;
            }
            *(u32x4*)(out + h * 1024 + lane * 16) = codes;
            out[32 * D + (block * 16 + t) * 2 + half] = (uint8_t)byte;
        }
    }

    // V: slot e of a lane is token 16 * (e / 4) + 4 * j + e % 4
    int row[8];
    uint32_t keep = 0;      // the bits of a word of codes that stay as they are
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        row[e] = row_of(16 * (e >> 2) + 4 * j + (e & 3));
        if (row[e] < 0) keep |= 0xfu << (4 * e);
    }
    if (keep == 0xffffffffu) return;
    uint32_t x[kBlocks][8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t* from = (const uint32_t*)(a.v + ((int64_t)max(row[e], 0) * a.c.n_kv_heads + head) * D) + t;
#pragma unroll
        for (int p = 0; p < kBlocks; ++p) x[p][e] = row[e] >= 0 ? from[16 * p] : 0;
    }
    u32x4* const codes = (u32x4*)(out + 16 * D) + lane;
    uint8_t* const scales = out + 33 * D + j * (8 * kBlocks);
#pragma unroll
    for (int h = 0; h < D / 64; ++h) {
        u32x4 y{0, 0, 0, 0};
#pragma unroll
        for (int p2 = 0; p2 < 2; ++p2) {
            const int p = 2 * h + p2;
            float f[8];
            u32x2 bytes{0, 0};
            uint32_t bad = 0;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const uint32_t a0 = x[p][e] & 0x7fff7fffu, a1 = x[p][e + 1] & 0x7fff7fffu;
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
                uint32_t word = 0;
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float v0 = __uint_as_float(q == 0 ? x[p][e] << 16 : x[p][e] & 0xffff0000u);
                    const float v1 = __uint_as_float(q == 0 ? x[p][e + 1] << 16 : x[p][e + 1] & 0xffff0000u);
                    word = code4(word, v0 * f[e], v1 * f[e + 1], e >> 1);
                }
                y[2 * p2 + q] = word & ~bad;
            }
            if (keep == 0) {
                if (t == 0) *(u32x2*)(scales + 8 * p) = bytes;
            } else if (t < 8) {
                const uint32_t byte = (t < 4 ? bytes[0] : bytes[1]) >> (8 * (t & 3));
                if ((keep >> (4 * t) & 1) == 0) scales[8 * p + t] = (uint8_t)byte;
            }
        }
        if (keep != 0) {
            const u32x4 old = codes[64 * h];
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = (y[i] & ~keep) | (old[i] & keep);
        }
        codes[64 * h] = y;
    }
}

struct LoadArgs {
    CacheView c;
    const int32_t *slots, *offsets;
    uint16_t *k, *v;
    int32_t n_rows, tiles_of_seq;
};
static_assert(sizeof(LoadArgs) <= 112, "short arguments");

// grid: (n * tiles, head groups)
template <int D>
__global__ __launch_bounds__(64 * kWaves) void cache_load_kernel(LoadArgs a) {
    constexpr int kBlocks = D / 32;
    const int lane = threadIdx.x & 63, t = lane & 15, j = lane >> 4;
    const int b = blockIdx.x / a.tiles_of_seq, tile = blockIdx.x % a.tiles_of_seq;
    const int slot = cache_slot(a.c, a.slots, b);
    const int first = a.offsets[b];
    if (slot < 0 || first < 0) return;
    const int count = min(min(a.offsets[b + 1], a.n_rows) - first, cache_len(a.c, slot)) - 32 * tile;      // tokens of this tile and behind it
    if (count <= 0) return;
    const int page = a.c.table[(int64_t)slot * a.c.max_pages + (tile >> (a.c.shift - 5))];
    if (page < 0 || page >= a.c.n_pages) return;
    const int head = blockIdx.y * kWaves + (threadIdx.x >> 6);
    if (head >= a.c.n_kv_heads) return;
    const uint8_t* const in = cache_tile<D>(a.c, page, head, tile & ((1 << (a.c.shift - 5)) - 1));
    const int64_t row0 = (int64_t)first + 32 * tile;
    const int hkv = a.c.n_kv_heads;
    if (a.k != nullptr) {
#pragma unroll
        for (int h = 0; h < D / 64; ++h) {
            const int half = D == 128 ? h : j >> 1, block = D == 128 ? j : j & 1;
            const u32x4 codes = *(const u32x4*)(in + h * 1024 + lane * 16);
            const float scale = scale_of(in[32 * D + (block * 16 + t) * 2 + half]);
            if (16 * half + t < count) {
                bf16x8* to = (bf16x8*)(a.k + ((row0 + 16 * half + t) * hkv + head) * D + 32 * block);
#pragma unroll
                for (int i = 0; i < 4; ++i) to[i] = values_of(codes[i], scale);
            }
        }
    }
    if (a.v != nullptr) {
#pragma unroll
        for (int h = 0; h < D / 64; ++h) {
            const u32x4 codes = *(const u32x4*)(in + 16 * D + h * 1024 + lane * 16);
            const u32x4 scales = *(const u32x4*)(in + 33 * D + j * (8 * kBlocks) + 16 * h);
#pragma unroll
            for (int p2 = 0; p2 < 2; ++p2) {
                const uint32_t c0 = codes[2 * p2], c1 = codes[2 * p2 + 1];
                // bytes of the two channels of tokens 0, 2, 4, 6 and 1, 3, 5, 7 of the lane's eight
                const uint32_t even = (c0 & 0x0f0f0f0fu) | (c1 & 0x0f0f0f0fu) << 4, odd = (c0 >> 4 & 0x0f0f0f0fu) | (c1 & 0xf0f0f0f0u);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int token = 16 * (e >> 2) + 4 * j + (e & 3);
                    const float scale = scale_of(scales[2 * p2 + (e >> 2)] >> (8 * (e & 3)) & 255);
                    const uint32_t from = (e & 1 ? odd : even) >> (8 * (e >> 1));
                    if (token < count) {
                        uint16_t* to = a.v + ((row0 + token) * hkv + head) * D + 32 * (2 * h + p2) + 2 * t;
                        *(bf16x2*)to = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(from, scale, 0);
                    }
                }
            }
        }
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
// grid: (n * tiles, head groups)
template <int D>
__global__ __launch_bounds__(64 * kWaves) void cache_move_kernel(MoveArgs a) {
    constexpr int kBlocks = D / 32;
    const int lane = threadIdx.x & 63, t = lane & 15, j = lane >> 4;
    if (*a.status != 0) return;
    const int b = blockIdx.x / a.tiles_of_seq, tile = blockIdx.x % a.tiles_of_seq;
    const int slot = cache_slot(a.c, a.slots, b);
    if (slot < 0) return;
    const int count = cache_len(a.c, slot) - 32 * tile;
    if (count <= 0) return;
    const int tile_shift = a.c.shift - 5, tile_mask = (1 << tile_shift) - 1;
    const int page = a.c.table[(int64_t)slot * a.c.max_pages + (tile >> tile_shift)];
    if (page < 0 || page >= a.c.n_pages) return;
    // lane l: where token l & 31 of the tile comes from, as a token of the pool; -1: nowhere
    int from = -1;
    if ((lane & 31) < count) {
        const int at = a.out_offsets[b] + 32 * tile + (lane & 31);
        const int old = at >= 0 && at < a.n_list ? a.kept_idx[at] - a.seq_offsets[b] : -1;
        const int32_t* old_row = a.old_rows + (int64_t)b * (1 + a.c.max_pages);
        if (old >= 0 && old < old_row[0]) {
            const int p = old_row[1 + (old >> a.c.shift)];
            if (p >= 0 && p < a.c.n_pages) from = (p << a.c.shift) + (old & ((1 << a.c.shift) - 1));
        }
    }
    int kfrom[2], vfrom[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) kfrom[h] = __shfl(from, D == 128 ? 16 * h + t : 16 * (j >> 1) + t);
#pragma unroll
    for (int e = 0; e < 8; ++e) vfrom[e] = __shfl(from, 16 * (e >> 2) + 4 * j + (e & 3));
    auto source = [&](int token, int head) -> const uint8_t* {
        const int old_page = token >> a.c.shift;
        return cache_tile<D>(a.c, old_page, head, (token >> 5) & tile_mask);
    };
    for (int head = blockIdx.y * kWaves + (threadIdx.x >> 6); head < a.c.n_kv_heads; head += gridDim.y * kWaves) {
        uint8_t* const out = cache_tile<D>(a.c, page, head, tile & tile_mask);
#pragma unroll
        for (int h = 0; h < D / 64; ++h) {
            const int half = D == 128 ? h : j >> 1, block = D == 128 ? j : j & 1;
            u32x4 codes{0, 0, 0, 0};
            uint8_t scale = 16 * half + t < count ? 255 : 0;
            if (kfrom[h] >= 0) {
                const uint8_t* in = source(kfrom[h], head);
                const int old_half = kfrom[h] >> 4 & 1, old = kfrom[h] & 15;
                codes = *(const u32x4*)(in + ((old_half * kBlocks + block) * 16 + old) * 16);
                scale = in[32 * D + (block * 16 + old) * 2 + old_half];
            }
            *(u32x4*)(out + h * 1024 + lane * 16) = codes;
            out[32 * D + (block * 16 + t) * 2 + half] = scale;
        }
        u32x4 y[D / 64] = {};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (vfrom[e] >= 0) {
                const uint8_t* in = source(vfrom[e], head);
                const int old = vfrom[e] & 31, old_j = old >> 2 & 3, shift = 4 * ((old >> 4) * 4 + (old & 3));
#pragma unroll
                for (int h = 0; h < D / 64; ++h) {
                    const u32x4 x = *(const u32x4*)(in + 16 * D + h * 1024 + (16 * old_j + t) * 16);
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[h][i] |= (x[i] >> shift & 15) << (4 * e);
                }
            }
        }
#pragma unroll
        for (int h = 0; h < D / 64; ++h) *(u32x4*)(out + 16 * D + h * 1024 + lane * 16) = y[h];
        // scale bytes: lane t of a group takes slot t / 2, every second block
        const int e = t >> 1;
        const int token = 16 * (e >> 2) + 4 * j + (e & 3);
        const int vf = __shfl(from, token);
#pragma unroll
        for (int i = 0; i < kBlocks / 2; ++i) {
            const int block = 2 * i + (t & 1);
            uint8_t scale = token < count ? 255 : 0;
            if (vf >= 0) {
                const int old = vf & 31;
                scale = source(vf, head)[33 * D + (((old >> 2 & 3) * kBlocks + block) * 2 + (old >> 4)) * 4 + (old & 3)];
            }
            out[33 * D + (j * kBlocks + block) * 8 + e] = scale;
        }
    }
}

}  // namespace

int launch_cache_store(const CacheView& c, int32_t head_dim, const void* k, const void* v, int32_t n_rows, const int32_t* row_idx, int32_t n_list,
                       const int32_t* offsets, const int32_t* slots, const int32_t* start, int32_t n_seqs, int32_t max_new, hipStream_t stream) {
    if (n_seqs == 0 || max_new == 0) return PYR_OK;
    const int32_t tiles = (max_new + 30) / 32 + 1;
    const StoreArgs a{c, (const uint16_t*)k, (const uint16_t*)v, row_idx, offsets, slots, start, n_rows, n_list};
    const dim3 grid((unsigned)((int64_t)n_seqs * tiles), (unsigned)((c.n_kv_heads + kWaves - 1) / kWaves));
    if (head_dim == 128) hipLaunchKernelGGL(cache_store_kernel<128>, grid, dim3(64 * kWaves), 0, stream, a, tiles);
    else hipLaunchKernelGGL(cache_store_kernel<64>, grid, dim3(64 * kWaves), 0, stream, a, tiles);
    return check_launch();
}

int launch_cache_load(const CacheView& c, int32_t head_dim, const int32_t* slots, const int32_t* offsets, int32_t n_seqs, int32_t max_len,
                      void* k, void* v, int32_t n_rows, hipStream_t stream) {
    if (n_seqs == 0 || max_len == 0) return PYR_OK;
    const LoadArgs a{c, slots, offsets, (uint16_t*)k, (uint16_t*)v, n_rows, (max_len + 31) / 32};
    const dim3 grid((unsigned)((int64_t)n_seqs * a.tiles_of_seq), (unsigned)((c.n_kv_heads + kWaves - 1) / kWaves));
    if (head_dim == 128) hipLaunchKernelGGL(cache_load_kernel<128>, grid, dim3(64 * kWaves), 0, stream, a);
    else hipLaunchKernelGGL(cache_load_kernel<64>, grid, dim3(64 * kWaves), 0, stream, a);
    return check_launch();
}

int launch_cache_move(const CacheView& c, int32_t head_dim, const int32_t* slots, const int32_t* kept_idx, int32_t n_list, const int32_t* seq_offsets,
                      const int32_t* out_offsets, const int32_t* old_rows, const int32_t* status, int32_t n_seqs, int32_t max_keep, hipStream_t stream) {
    if (n_seqs == 0 || max_keep == 0) return PYR_OK;
    const MoveArgs a{c, slots, kept_idx, seq_offsets, out_offsets, old_rows, status, n_list, (max_keep + 31) / 32};
    const dim3 grid((unsigned)((int64_t)n_seqs * a.tiles_of_seq), (unsigned)((c.n_kv_heads + kWaves - 1) / kWaves));
    if (head_dim == 128) hipLaunchKernelGGL(cache_move_kernel<128>, grid, dim3(64 * kWaves), 0, stream, a);
    else hipLaunchKernelGGL(cache_move_kernel<64>, grid, dim3(64 * kWaves), 0, stream, a);
    return check_launch();
}

}  // namespace pyr
