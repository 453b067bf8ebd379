// The cache held in 4 bits, as kernels see it: where a token's K and V lie, the conversions, exchanges inside a wavefront.
//
// A number is e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign) times a power of two shared by 32 channels of a head (e8m0: 2^(byte - 127),
// 255: not a number): the element and block of the OCP microscaling format MXFP4, which gfx950 converts from and to in one
// instruction for two numbers.  34 bytes a block of K and V together, 4.25 bits a number.
//
// A tile is 32 tokens of one KV head, 34 * d bytes, laid out so that a wavefront's loads of 16 bytes a lane are its operands of the
// 16x16x32 matrix instructions, without an exchange between lanes and without LDS (nb = d / 32 blocks, h = d / 64):
//   K codes   16 d bytes  [half 2][block nb][token 16][16 bytes]: lane 16 * block + token holds a block of one token, 32 channels of the
//                         contracted dimension of Q K^T
//   V codes   16 d bytes  [h][j 4][r 16][p 2][q 2][4 bytes]: lane 16 * j + r holds eight tokens, 4 j + s and 16 + 4 j + s (s < 4), of
//                         channels 64 h + 32 p + 2 r + q.  Those eight are the tokens whose logits the same lane receives from Q K^T.
//   K scales     d bytes  [block nb][token 16][half 2]
//   V scales     d bytes  [j 4][block nb][half 2][s 4]
// A page is [KV head][page_tokens / 32] tiles.
#pragma once

#include "pyr_internal.h"

namespace pyr {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;

// The parts of a pyr_cache that kernels use; token numbers in the pool (page * page_tokens + place) fit 31 bits.
struct CacheView {
    uint8_t* pages;
    int32_t* table;
    int32_t* lens;
    int32_t n_pages, n_slots, max_pages, shift /* log2(page_tokens) */, n_kv_heads;
};
struct PoolView : CacheView {
    int32_t* refs;
};

__device__ __forceinline__ int cache_slot(const CacheView& c, const int32_t* slots, int b) {      // -1: a row that is skipped
    const int slot = slots[b];
    return slot >= 0 && slot < c.n_slots ? slot : -1;
}
__device__ __forceinline__ int cache_len(const CacheView& c, int slot) {      // never more than a row of the table covers
    const int most = c.max_pages << c.shift;
    const int len = c.lens[slot];
    return len < 0 ? 0 : len < most ? len : most;
}

template <int D>
__device__ __forceinline__ uint8_t* cache_tile(const CacheView& c, int page, int head, int tile_of_page) {
    const int64_t tile = (((int64_t)page * c.n_kv_heads + head) << (c.shift - 5)) + tile_of_page;
    return c.pages + tile * (34 * D);
}

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }      // 255: +inf, which the conversions below take for NaN

// Eight codes of a word, lowest first, times scale.
__device__ __forceinline__ bf16x8 values_of(uint32_t codes, float scale) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The scale byte of a block whose largest magnitude has these bf16 bits (sign clear): the smallest power of two that brings it to 7 or
// less (which rounds to 6, the largest code); 255 if it is no finite number.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    if (top >= 0x7f80) return 255;
    const int e = (int)(top >> 7) - 2 + ((top & 0x7f) > 0x60 ? 1 : 0);
    return e < 1 ? 1 : e > 252 ? 252 : e;
}

}  // namespace pyr
