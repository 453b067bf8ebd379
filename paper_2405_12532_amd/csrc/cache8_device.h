// The cache held in 8 bits, as kernels see it: where a block's K, V, bounds and powers lie, the conversions.
//
// A number is e4m3 (OCP's FP8: four exponent bits, three mantissa bits, up to 448, no infinities, 0x7f and 0xff: not a number) times a power of two,
// 2^(byte - 127) with a byte from kLeastPower to kMostPower, one for the K and one for the V of a block: 32 tokens of a KV head.  A code keeps four
// significant bits of every number down to 2^-13.8 of the largest that its power was taken for, so that a channel far larger than the others does not cost them theirs, as one
// step for all of them would; gfx950 converts two codes to bf16 in one instruction, power included, exactly.
// A block keeps bounds of its K too, the largest and smallest code of every channel in whole units of 4, rounded outward (int8; +-127: not a number).
//
// A page holds, for hkv heads and T = page_tokens / 32 blocks of a head, up to a multiple of 256 bytes:
//   [hkv][T] 64 d bytes   K's codes [half 2][s d/64][j 4][t 16][byte 16]: token 16 half + t, channel 64 s + 16 j + byte
//                         V's codes [g d/32][j 4][r 16][p 2][e 8]: token 16 (e / 4) + 4 j + e % 4, channel 32 g + 16 p + r
//   [hkv][T]  2 d bytes   bounds of K: largest [d], smallest [d]
//   [hkv][T]  2 bytes     powers of K and of V
// so that a wavefront's loads of 16 bytes a lane are its operands of the 16x16x32 matrix instructions: lane 16 j + t holds 16 channels of a token of K,
// lane 16 j + r the eight tokens of a channel of V whose logits the same lane receives from Q K^T.
#pragma once

#include "cache_device.h"

namespace pyr {

constexpr int kLeastPower = 27, kMostPower = 246;      // 2^-100, 2^119

__host__ __device__ inline int64_t cache8_page_bytes(int32_t head_dim, int32_t n_kv_heads, int32_t blocks_of_head) {
    return ((int64_t)n_kv_heads * blocks_of_head * (66 * head_dim + 2) + 255) / 256 * 256;
}

// The parts of one page (below 2^31 bytes; the host checks).
template <int D>
struct Page8 {
    uint8_t* at;
    uint32_t blocks;              // of the page
    uint32_t head_shift;          // log2(blocks of a head)
    __device__ __forceinline__ Page8(const CacheView& c, int page) {
        head_shift = c.shift - 5;
        blocks = (uint32_t)c.n_kv_heads << head_shift;
        const uint32_t bytes = (blocks * (66 * D + 2) + 255) & ~255u;
        at = c.pages + (int64_t)page * bytes;
    }
    __device__ __forceinline__ uint32_t place(int head, int block) const { return ((uint32_t)head << head_shift) + (block & ((1 << head_shift) - 1)); }
    __device__ __forceinline__ uint8_t* codes(int head, int block) const { return at + place(head, block) * (64 * D); }
    __device__ __forceinline__ uint8_t* bounds(int head, int block) const { return at + blocks * (64 * D) + place(head, block) * (2 * D); }
    __device__ __forceinline__ uint16_t* powers(int head, int block) const { return (uint16_t*)(at + blocks * (66 * D)) + place(head, block); }
};

typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) short i16x2;

// Eight codes, lowest byte first, times scale (exact: four significant bits, and the powers keep to bf16's range).
__device__ __forceinline__ bf16x8 values8_of(uint32_t low, uint32_t high, float scale) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(low, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(low, scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(high, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(high, scale, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Four codes: the nearest to x / scale, ties to the even one.  What lies above 464 (and what is no number) becomes 0x7f or 0xff.
__device__ __forceinline__ uint32_t codes8_of(float x0, float x1, float x2, float x3, float scale) {
    i16x2 y = {0, 0};
    y = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(y, x0, x1, scale, false);
    y = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(y, x2, x3, scale, true);
    return __builtin_bit_cast(uint32_t, y);
}

__device__ __forceinline__ uint32_t max_u16(uint32_t a, uint32_t b) {      // of both halves
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

template <int kCtrl>
__device__ __forceinline__ uint32_t dpp(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kCtrl, 0xf, 0xf, false); }
// op over groups of kLanes lanes (8 or 16), in all of them; over the wavefront.
template <int kLanes, class Op>
__device__ __forceinline__ uint32_t within_lanes(uint32_t x, Op op) {
    x = op(x, dpp<0xb1>(x));              // the neighbour's, the other pair's
    x = op(x, dpp<0x4e>(x));
    x = op(x, dpp<0x141>(x));             // (eight lanes mirrored, then sixteen)
    return kLanes == 16 ? op(x, dpp<0x140>(x)) : x;
}
template <class Op>
__device__ __forceinline__ uint32_t within_wave(uint32_t x, Op op) {
    x = within_lanes<16>(x, op);
    const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = op(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return op(b[0], b[1]);
}

// The power byte of a block whose largest finite magnitude is top: the smallest with top <= 448 * 2^(byte - 127).
__device__ __forceinline__ int power8_of(float top) {
    const uint32_t bits = __float_as_uint(top);
    const int e = (int)(bits >> 23) - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0);
    return min(max(e, kLeastPower), kMostPower);
}

// Codes of a block whose power grows by 2^shift (scale: that power): rounded to the new step.
__device__ __forceinline__ uint32_t regrown(uint32_t codes, float scale) {
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, 1.f, true);
    return codes8_of(a[0], a[1], b[0], b[1], scale);
}

}  // namespace pyr
