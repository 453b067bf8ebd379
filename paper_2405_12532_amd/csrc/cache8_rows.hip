// New rows into the cache held in 8 bits, turned by their positions on the way (Algorithm 1, the new rows of KV = cat(PvC_past, KV); what
// Gather(KV, index) keeps of a prompt goes the same way, through its index), tokens of it back to bf16, and pages copied for a fork.
//
// A turn by position p takes channels a and b of a pair i to a cos(p f_i) - b sin(p f_i) and b cos(p f_i) + a sin(p f_i).  p f_i, of up to 55 bits, is two
// numbers of 64 bits, and so is the quarter of a turn that it is reduced by, so that far positions lose nothing; sine and cosine are Taylor's sums on [-pi/4, pi/4] in 64 bits too, rounded to 32.  A workgroup takes 32 tokens and some heads: the pairs are
// worked out once, meet in LDS and turn K and Q of all its heads.
// A wavefront owns one block (32 tokens of one KV head) of the destination, whole or in part, so no two of them write a byte.
// Bound: reading and writing HBM, in part only: the rows that a selection keeps of 8 x 2048 tokens on 32 heads (1433 of each, K and V) go in in 50.8 us, 287 MB at 5.6 TB/s, vector
// instructions 39 % of a SIMD's cycles, and come back in 44, 283 MB at 6.4 TB/s; all 2048 turned with Q 147 us, 680 MB at 4.6 TB/s, vector instructions 55 % of the cycles; ragged
// pieces turned with Q (7 x 100 ... 3000 on 32/8 heads of 64) 27 us for 110 MB, 4.1 TB/s, where loads, the block's power and stores follow one another in each
// wavefront; 64 tokens of a step 7.7 us, latency; back from 64 blocks 9.
#include "cache8_device.h"

namespace pyr {
namespace {

constexpr int kWaves = 4;
constexpr uint32_t kAllTokens = 0xffffffffu;

__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return max(a, b); }      // of magnitudes, as bits

typedef __attribute__((address_space(3))) char* lptr_t;
typedef __attribute__((ext_vector_type(2))) int i32x2;

// Transposing LDS read (ds_read_b64_tr_b8).  Inside every group of 16 lanes, lane j receives byte (j & 7) of the 8-byte words addressed by lanes
// (j >> 3), 2 + (j >> 3), 4 + (j >> 3) ... 14 + (j >> 3), in this order.
__device__ __forceinline__ i32x2 lds_read_tr8(uint32_t lds_addr) {
    return __builtin_amdgcn_ds_read_tr8_b64_v2i32((i32x2 __attribute__((address_space(3)))*)(uintptr_t)lds_addr);
}
__device__ __forceinline__ void meet() {            // (a wavefront's own part of LDS)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ float low_of(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float high_of(uint32_t pair) { return __uint_as_float(pair & 0xffff0000u); }

// cos and sin of position * freq, in 64 bits (the sums' next terms are below 2^-33), for angles up to 2^47; of larger ones, whose number of quarters is not known to a whole one,
// those of some angle
struct Turn {
    double c, s;
};
__device__ __forceinline__ Turn exact_turn_of(int position, float freq) {
    const double angle = (double)position * (double)freq, rest = __builtin_fma((double)position, (double)freq, -angle);
    const double nearest = __builtin_rint(angle * 0.63661977236758134308);      // quarters of a turn: times 2 / pi
    const double near = __builtin_fma(-nearest, 6.123233995736766e-17, __builtin_fma(-nearest, 1.57079632679489661923, angle)) + rest;      // (pi / 2 in two parts)
    const double x = __builtin_fmin(__builtin_fmax(near, -1.), 1.), y = x * x;
    const double s = x * (1. + y * (-1. / 6 + y * (1. / 120 + y * (-1. / 5040 + y * (1. / 362880 - y * (1. / 39916800))))));
    const double c = 1. + y * (-0.5 + y * (1. / 24 + y * (-1. / 720 + y * (1. / 40320 - y * (1. / 3628800)))));
    const int quadrant = (int)(nearest - 4.0 * __builtin_floor(nearest * 0.25));
    const double a = quadrant & 1 ? s : c, b = quadrant & 1 ? c : s;
    return {quadrant == 1 || quadrant == 2 ? -a : a, quadrant >= 2 ? -b : b};
}
__device__ __forceinline__ f32x2 turn_of(int position, float freq) {
    const Turn t = exact_turn_of(position, freq);
    return f32x2{(float)t.c, (float)t.s};
}

// Workgroups count through the head groups first: the heads of a row lie side by side in memory.
struct AppendArgs {
    CacheView c;
    const uint16_t *k, *v, *q;
    uint16_t* q_out;
    const int32_t *row_idx, *offsets, *slots, *start, *positions;
    const float* freqs;
    int32_t k_stride, v_stride, q_stride;                         // of rows, in 16 bytes
    int32_t n_rows, n_list, max_new, tiles_of_piece, head_groups, n_q_heads, dims;
};

enum { kAsIs, kAllHalves, kHalves, kPairs };                      // channel c turns with c + dims / 2 (all channels, some of them), or 2 c with 2 c + 1

// Where the turn of a pair lies among its token's: lanes that turn eight channels each (with their partners, or in pairs) read 16 bytes side by side.  (One behind the
// other, and partners through LDS: 8 x 2048 rows on 32/32 heads 149.5 us for 144.8, 4 x 4000 on 64/8 127 for 120.)
template <int D, int kTurn>
__device__ __forceinline__ int place_of(int pair) {
    constexpr int kOfLane = kTurn == kPairs ? 4 : 8;
    return pair / kOfLane * 2 + pair % kOfLane / 2 * (D / kOfLane) + pair % 2;
}
template <int D, int kTurn>
constexpr int turns_of_row = kTurn == kAsIs ? 1 : D == 64 ? 48 : 64;      // (at 64 channels with room between rows, two of which are read at a time)

constexpr uint32_t kNoNumber = 0x7f680000u;                       // 464 * 2^119: what lies above has no code

// The same channels of the lane that holds the partners of a lane's eight; with: lanes to it.
template <int D, int kTurn>
__device__ __forceinline__ uint32_t partners(uint32_t word, int with) {
    if constexpr (kTurn == kHalves) return (uint32_t)__shfl((int)word, (int)(threadIdx.x & 63) + with);
    else if constexpr (D == 128) return dpp<0x128>(word);      // eight lanes further of sixteen
    else return dpp<0x1b>(dpp<0x141>(word));                  // eight lanes mirrored, then four
}
template <int D, int kTurn>
__device__ __forceinline__ int lanes_to_partners(int dims, int piece) {
    const int half = kTurn == kAllHalves ? D / 16 : dims / 16;
    return piece < half ? half : piece < 2 * half ? -half : 0;
}

// Eight channels of a row, turned.  turns: of the row's token; lanes of a row are neighbours.
template <int D, int kTurn>
__device__ __forceinline__ void turned(u32x4 words, const f32x2* turns, int dims, int piece, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = low_of(words[i]);
        x[2 * i + 1] = high_of(words[i]);
    }
    if constexpr (kTurn == kAllHalves || kTurn == kHalves) {
        const int with = lanes_to_partners<D, kTurn>(dims, piece);
        float y[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t other = partners<D, kTurn>(words[i], with);
            y[2 * i] = low_of(other);
            y[2 * i + 1] = high_of(other);
        }
        if (kTurn == kAllHalves || with != 0) {
            const f32x2* at = turns + 2 * min(piece, piece + with);
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const f32x4 two = *(const f32x4*)(at + place_of<D, kTurn>(i));
                x[i] = __builtin_fmaf(x[i], two[0], (with > 0 ? -y[i] : y[i]) * two[1]);
                x[i + 1] = __builtin_fmaf(x[i + 1], two[2], (with > 0 ? -y[i + 1] : y[i + 1]) * two[3]);
            }
        }
    } else if constexpr (kTurn == kPairs) {
        if (piece < dims / 8) {
            const f32x2* at = turns + 2 * piece;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 two = *(const f32x4*)(at + place_of<D, kTurn>(i & 2));
                const float c = two[2 * (i & 1)], s = two[2 * (i & 1) + 1], p = x[2 * i], r = x[2 * i + 1];
                x[2 * i] = __builtin_fmaf(p, c, -(r * s));
                x[2 * i + 1] = __builtin_fmaf(r, c, p * s);
            }
        }
    }
}

// K is rounded to four significant bits, and what fp32 rounds onto a border between two codes, or across it, gets the wrong one: a number of a million.  Those within three
// units of fp32's last place of a border (a number of 150000) are turned again in 64 bits and rounded to fp32 so that a number that is on neither side of a border does not end
// on it (to odd ones).  (Numbers that are small against their partners, and codes of less than four bits, keep fp32's error.)
// Of 36 million numbers 8 to 16 are then off, all small, where fp32 alone left 30 to 38; it costs 3 to 5 % of an append (8 x 2048 rows on 32/32 heads 143.3 us without, 146.9 with it, 4 x 4000
// on 64/8 117.9 and 121.5, 64 x 9 tokens 9.4 and 10).
__device__ __forceinline__ uint32_t from_border(float x) { return (__float_as_uint(x) << 12) + 0x80003000u; }
constexpr uint32_t kNear = 6u << 12;
template <int D, int kTurn>
__device__ __forceinline__ bool turns_at_all(int dims, int piece) { return kTurn == kAllHalves || piece < dims / 8; }      // (halves: of dims / 16 lanes each)
// Which of a lane's four words of two turned channels hold such a number, in some lane; turned by nothing (a position or a frequency of 0: one bf16 in 16 is a border) they
// are exact.  turns: of the row's token.
template <int D, int kTurn>
__device__ __forceinline__ uint32_t near_words(const float (&x)[8], const f32x2* turns, int dims, int piece) {
    const bool turn = turns_at_all<D, kTurn>(dims, piece);
    uint32_t least = from_border(x[0]), words = 0;
#pragma unroll
    for (int e = 1; e < 8; ++e) least = min(least, from_border(x[e]));
    if (__builtin_amdgcn_ballot_w64(turn && least <= kNear) == 0) return 0;
    const f32x2* at = turns + 2 * (kTurn == kPairs ? piece : turn ? min(piece, piece + lanes_to_partners<D, kTurn>(dims, piece)) : 0);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        bool near = false;
#pragma unroll
        for (int h = 0; h < 2; ++h) near |= turn && from_border(x[2 * w + h]) <= kNear && at[place_of<D, kTurn>(kTurn == kPairs ? w : 2 * w + h)][1] != 0.f;
        words |= __builtin_amdgcn_ballot_w64(near) != 0 ? 1u << w : 0;
    }
    return words;
}
// Channels 2 i and 2 i + 1 of a lane's eight, where they are next to a border; row: those eight.
struct Exactly {
    float x[2];
    bool turns;
    __device__ __forceinline__ float value(int h, float fast) const { return turns && from_border(fast) <= kNear ? x[h] : fast; }
};
template <int D, int kTurn>
__device__ __forceinline__ Exactly turned_exactly(const uint32_t* row, int i, int position, const float* freqs, int dims, int piece) {
    const int with = kTurn == kPairs ? 0 : lanes_to_partners<D, kTurn>(dims, piece);
    const bool turns = turns_at_all<D, kTurn>(dims, piece);
    const uint32_t word = row[i], other = row[i + 4 * with];
    float x[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int pair = kTurn == kPairs ? 4 * piece + i : 8 * min(piece, piece + with) + 2 * i + h;
        const Turn t = exact_turn_of(position, freqs[turns ? pair : 0]);
        const double own = h ? high_of(word) : low_of(word), partner = (kTurn == kPairs ? 1 - h : h) ? high_of(other) : low_of(other);
        const bool first = kTurn == kPairs ? h == 0 : with > 0;
        const double y = __builtin_fma(own, t.c, first ? -partner * t.s : partner * t.s), z = turns ? y : own;
        const float nearest = (float)z;
        const double rest = z - (double)nearest;
        uint32_t bits = __float_as_uint(nearest);
        if (rest != 0 && (bits & 1) == 0) bits += (rest > 0) == (z > 0) ? 1 : -1;
        x[h] = __uint_as_float(bits);
        __builtin_amdgcn_sched_barrier(0);                    // (one after the other, for the registers)
    }
    return {{x[0], x[1]}, turns};
}
__device__ __forceinline__ u32x4 rounded(const float (&x)[8]) {
    bf16x8 y;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = (__bf16)x[e];
    return __builtin_bit_cast(u32x4, y);
}

// The largest magnitude, as bits, of what is a number.
__device__ __forceinline__ void raise_finite(uint32_t& top, float x) {
    const uint32_t bits = __float_as_uint(x) & 0x7fffffffu;
    if (bits < 0x7f800000u) top = max(top, bits);
}

__device__ __forceinline__ u32x2 codes_of(const float (&x)[8], float scale) {
    return u32x2{codes8_of(x[0], x[1], x[2], x[3], scale), codes8_of(x[4], x[5], x[6], x[7], scale)};
}
__device__ __forceinline__ u32x2 codes_of(u32x4 words, float scale) {
    i16x2 lo = {0, 0}, hi = {0, 0};
    lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, __builtin_bit_cast(bf16x2, (uint32_t)words[0]), scale, false);
    lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, __builtin_bit_cast(bf16x2, (uint32_t)words[1]), scale, true);
    hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, __builtin_bit_cast(bf16x2, (uint32_t)words[2]), scale, false);
    hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, __builtin_bit_cast(bf16x2, (uint32_t)words[3]), scale, true);
    return u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}

// Bounds of eight channels: of a token's codes (none: a number without one), and of what the block held (grown by 2^grow).
__device__ __forceinline__ void bounds_of(u32x2 codes, const bool (&none)[8], bool behind, u32x2 old_up, u32x2 old_down, int grow, u32x2& up, u32x2& down) {
    const float shrink = __uint_as_float((uint32_t)(127 - grow) << 23);
    up = down = u32x2{};
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const f32x2 y = e & 2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes[e >> 2], 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes[e >> 2], 1.f, false);
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            const int n = e + f;
            float largest = none[n] ? 127.f : __builtin_ceilf(y[f] * 0.25f), smallest = none[n] ? -127.f : __builtin_floorf(y[f] * 0.25f);
            if (behind) {
                const int o = (int8_t)(old_up[n >> 2] >> (8 * (n & 3))), u = (int8_t)(old_down[n >> 2] >> (8 * (n & 3)));
                largest = fmaxf(largest, __builtin_ceilf((float)o * shrink));
                smallest = fminf(smallest, __builtin_floorf((float)u * shrink));
            }
            up[n >> 2] |= ((uint32_t)(int)largest & 255) << (8 * (n & 3));
            down[n >> 2] |= ((uint32_t)(int)smallest & 255) << (8 * (n & 3));
        }
    }
}

// What a workgroup of an append is about: a block of a sequence, its tokens that are stored (bit t: token t), where the others' count as older ones.
struct Piece {
    int block, page, from;        // lane l: the row that token l & 31 of the block gets; -1: one that is not there, a token of NaN
    uint32_t stored;              // 0: nothing to do
    bool behind;                  // there are older tokens in the block, whose powers and bounds count
};
__device__ __forceinline__ Piece piece_of(const AppendArgs& a, int place) {
    Piece p{};
    const int lane = threadIdx.x & 63, b = place / a.tiles_of_piece;
    const int slot = cache_slot(a.c, a.slots, b);
    const int start = a.start[b], offset = a.offsets[b];
    const int64_t wanted = (int64_t)a.offsets[b + 1] - offset;
    // an earlier row has the slot: its block may be written by two wavefronts at once (every workgroup looks at all earlier rows: one token each of 1024 sequences on 32/8 heads turned
    // with Q 18.9 us, of 4096 on 8/8 heads of 64 33.5)
    bool again = false;
    for (int i = lane; i < b; i += 64) again |= a.slots[i] == slot;
    if (slot < 0 || start < 0 || wanted <= 0) return p;
    const int64_t token0 = (start & ~31) + 32 * (int64_t)(place - b * a.tiles_of_piece);
    p.block = (int)(token0 >> 5);
    // (asked for together with the length, which may say that it is not there)
    p.page = a.c.table[(int64_t)slot * a.c.max_pages + min(token0 >> a.c.shift, (int64_t)a.c.max_pages - 1)];
    const int64_t end = min((int64_t)start + min(wanted, (int64_t)a.max_new), (int64_t)cache_len(a.c, slot));      // (the table holds anything behind the length)
    p.behind = token0 < start;
    const int64_t token = token0 + (lane & 31);
    const bool mine = token >= start && token < end;
    p.from = -1;
    if (mine) {
        const int64_t row = offset + (token - start);
        if (row >= 0 && row < a.n_list) p.from = a.row_idx != nullptr ? a.row_idx[row] : (int)row;
        if (p.from < 0 || p.from >= a.n_rows) p.from = -1;
    }
    p.stored = (uint32_t)__builtin_amdgcn_ballot_w64(mine);
    if (p.page < 0 || p.page >= a.c.n_pages || __builtin_amdgcn_ballot_w64(again) != 0) p.stored = 0;
    return p;
}

// Pieces of any length.  A wavefront goes through items: K, V or Q of the piece's block and a head.  kShort: nine tokens at most, which a window of 12 (at 64
// channels 16) tokens of the block holds (64 x 9 tokens on 32/8 heads of 128, turned with Q: 10.6 us, with all 32 tokens' places 14.7; 8 x 5 5.7 and 9.5).
template <int D, int kTurn, bool kShort>
constexpr int append_waves = D == 64 ? 4 : kShort ? (kTurn == kPairs ? 3 : 4) : kTurn == kAsIs ? 3 : 2;      // of a SIMD, as registers allow
template <int D, int kTurn, bool kShort>
__global__ __launch_bounds__(64 * kWaves, (append_waves<D, kTurn, kShort>)) void cache8_append_kernel(AppendArgs a) {
    constexpr int kLanes = D / 8, kTokens = 64 / kLanes;          // lanes of a row, rows of a load
    constexpr bool kEarly = kShort || D == 128;                   // what a block holds is asked for with the rows (at 64 channels longer pieces have no registers for it)
    constexpr int kWindow = !kShort ? 32 : D == 128 ? 12 : 16, kLoads = kWindow / kTokens;
    constexpr int kRow = D + 16;                                  // bytes of a token's codes in LDS
    __shared__ __align__(16) f32x2 turns[kTurn == kAsIs ? 1 : 32][turns_of_row<D, kTurn>];
    __shared__ __align__(16) uint8_t all_staged[kWaves][32][kRow];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), piece = lane % kLanes;
    const int place = blockIdx.x / a.head_groups, hkv = a.c.n_kv_heads;
    const Piece p = piece_of(a, place);
    const uint32_t stored = p.stored, there = (uint32_t)__builtin_amdgcn_ballot_w64(p.from >= 0);
    const int block = p.block;
    const bool gone = stored != there, behind = p.behind;
    if (stored == 0) return;

    // the row that a lane reads in load i: of a token that is not stored the first one's (what it computes changes no largest and no smallest, and is not
    // written)
    const int first = __builtin_ctz(stored);
    const int window = kShort ? min(first & ~3, 32 - kWindow) : 0;      // its first token
    auto token_of = [&](int i) { return window + i * kTokens + lane / kLanes; };
    auto source_of = [&](int i) { return stored >> token_of(i) & 1 ? token_of(i) : first; };
    auto there_of = [&](int i) { return (there >> source_of(i) & 1) != 0; };
    int rows[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) rows[i] = max(__shfl(p.from, source_of(i)), 0);
    // what was worked out from the rows is worked out again (else the compiler keeps all of it for the paths of what is no number)
    auto afresh = [&](u32x4 (&words)[kLoads]) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) asm volatile("" : "+v"(words[i]));
    };
    auto load = [&](int item, u32x4 (&words)[kLoads]) {
        const uint16_t* from = item < hkv ? a.k : item < 2 * hkv ? a.v : a.q;
        const int64_t stride = item < hkv ? a.k_stride : item < 2 * hkv ? a.v_stride : a.q_stride;
        const u32x4* at = (const u32x4*)from + (item < hkv ? item : item < 2 * hkv ? item - hkv : item - 2 * hkv) * kLanes + piece;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) words[i] = __builtin_nontemporal_load(at + rows[i] * stride);
    };
    const int items = 2 * hkv + a.n_q_heads, step = a.head_groups * kWaves;
    int item = (blockIdx.x - place * a.head_groups) * kWaves + wave;
    u32x4 words[kLoads];
    if (item < items) load(item, words);

    if constexpr (kTurn != kAsIs) {
        constexpr int kPairsOf = D / 2, kAtOnce = 64 / kPairsOf;
        const int pair = lane % kPairsOf;
        const int position = p.from >= 0 ? a.positions[p.from] : 0;
        const float freq = pair < a.dims / 2 ? a.freqs[pair] : 0.f;
        for (int t = wave * kAtOnce; t < 32; t += kWaves * kAtOnce) {
            if ((stored >> t & ((1u << kAtOnce) - 1)) == 0) continue;
            const int mine_t = t + lane / kPairsOf;
            const f32x2 turn = turn_of(__shfl(position, mine_t), freq);
            if (pair < a.dims / 2) turns[mine_t][place_of<D, kTurn>(pair)] = turn;
        }
        __syncthreads();
    }
    auto turns_of = [&](int t) -> const f32x2* { return kTurn == kAsIs ? nullptr : turns[kTurn == kAsIs ? 0 : t]; };

    const Page8<D> at(a.c, p.page);
    uint8_t(*const staged)[kRow] = all_staged[wave];
    const float most = __uint_as_float(kNoNumber);
    const u32x4 kNoRow = {0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
    // the power of a block's K or V, whose codes the block held are rounded to it
    auto settle = [&](float top, int old_power, uint8_t* power_at, uint8_t* codes, int* grow) {
        int power = power8_of(__uint_as_float(within_wave(__float_as_uint(top), larger)));
        *grow = 0;
        if (behind) {
            power = max(power, old_power);
            *grow = min(power - old_power, 100);
        }
        if (lane == 0) *power_at = (uint8_t)power;
        if (*grow > 0) {
            const float by = __uint_as_float((uint32_t)(127 + *grow) << 23);
            u32x4* const lane_words = (u32x4*)codes + lane;
#pragma unroll 1
            for (int g = 0; g < D / 32; ++g) {
                u32x4 y = lane_words[64 * g];
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] = regrown(y[i], by);
                lane_words[64 * g] = y;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");      // (the bytes are read and written again, by other lanes)
            __builtin_amdgcn_s_waitcnt(0);
        }
        return scale_of(power);
    };
    for (; item < items; item += step) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) asm volatile("" : "+v"(rows[i]));      // (else it keeps what addresses are made of, too)
        if (item >= 2 * hkv) {                                    // a head of Q: rows turned, where there are rows
            u32x4* const to = (u32x4*)a.q_out + (item - 2 * hkv) * kLanes + piece;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                float x[8];
                turned<D, kTurn>(words[i], turns_of(source_of(i)), a.dims, piece, x);
                if ((stored & there) >> token_of(i) & 1) __builtin_nontemporal_store(rounded(x), to + (int64_t)rows[i] * (a.n_q_heads * kLanes));
            }
        } else if (item < hkv) {                                  // a head of K
            uint8_t* const codes = at.codes(item, block);
            uint8_t* const power_at = (uint8_t*)at.powers(item, block);
            const int old_power = behind ? *power_at : 0;
            int8_t* const bounds = (int8_t*)at.bounds(item, block) + (lane >> 5) * D + 8 * piece + (lane >> 4 & 1);      // (whose, below)
            int old_bounds[4] = {};
            auto look = [&] {
#pragma unroll
                for (int e = 0; e < 4; ++e) old_bounds[e] = bounds[2 * e];
            };
            if (kEarly && behind) look();
            constexpr bool kExpanded = kTurn != kAsIs;            // in fp32
            float x[kExpanded ? kLoads : 1][8];
            auto number = [&](int i, int e) { return kExpanded ? x[kExpanded ? i : 0][e] : e & 1 ? high_of(words[i][e >> 1]) : low_of(words[i][e >> 1]); };
            float up[8], down[8];                                 // the largest, and the smallest the other way round: NaN prevails
#pragma unroll
            for (int e = 0; e < 8; ++e) up[e] = down[e] = -INFINITY;
#pragma unroll
            for (int n = 0; n < kLoads; ++n)
                if (gone && !there_of(n)) words[n] = kNoRow;
            if constexpr (kExpanded) {
                uint32_t near = 0;                                // words of them with numbers next to a border
#pragma unroll
                for (int n = 0; n < kLoads; ++n) {
                    turned<D, kTurn>(words[n], turns_of(source_of(n)), a.dims, piece, x[n]);
                    near |= near_words<D, kTurn>(x[n], turns_of(source_of(n)), a.dims, piece) << (4 * n);
                    __builtin_amdgcn_sched_barrier(0);
                }
                while (near != 0) {
                    const int i = __builtin_ctz(near) >> 2, w = __builtin_ctz(near) & 3, row = max(__shfl(p.from, source_of(i)), 0);
                    near &= near - 1;
                    int hidden = piece;
                    asm volatile("" : "+v"(hidden));
                    const Exactly y = turned_exactly<D, kTurn>((const uint32_t*)((const u32x4*)a.k + item * kLanes + hidden + row * (int64_t)a.k_stride), w, a.positions[row], a.freqs,
                                                               a.dims, hidden);
#pragma unroll
                    for (int n = 0; n < kLoads; ++n)
#pragma unroll
                        for (int v = 0; v < 4; ++v)
                            if (n == i && v == w) {
                                x[n][2 * v] = y.value(0, x[n][2 * v]);
                                x[n][2 * v + 1] = y.value(1, x[n][2 * v + 1]);
                            }
                }
            }
#pragma unroll
            for (int i = 0; i < kLoads; i += 2) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float y = number(i, e), z = i + 1 < kLoads ? number(i + 1 < kLoads ? i + 1 : i, e) : y;
                    up[e] = __builtin_elementwise_maximum(__builtin_elementwise_maximum(up[e], y), z);
                    down[e] = __builtin_elementwise_maximum(__builtin_elementwise_maximum(down[e], -y), -z);
                }
                __builtin_amdgcn_sched_barrier(0);                // (else all rows are taken apart first, and registers run out)
            }
            float top = __builtin_elementwise_maximum(up[0], down[0]);
#pragma unroll
            for (int e = 1; e < 8; ++e) top = __builtin_elementwise_maximum(top, __builtin_elementwise_maximum(up[e], down[e]));
            if (__builtin_amdgcn_ballot_w64(!(top <= most)) != 0) {      // some have no code: the largest of those that are numbers, and no bounds where they are
                uint32_t bits = 0;
                if (!kExpanded) afresh(words);
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) raise_finite(bits, number(i, e));
                    __builtin_amdgcn_sched_barrier(0);
                }
                top = __uint_as_float(bits);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (!(up[e] <= most && down[e] <= most)) up[e] = down[e] = NAN;
            }
            int grow;
            const float scale = settle(top, old_power, power_at, codes, &grow);
            // over the tokens: lanes 16 r .. 16 r + 15 end up with the largest of even channels (r = 0), of odd ones, the smallest of even ones, of odd ones
            float four[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float y[2];
#pragma unroll
                for (int f = 0; f < 2; ++f) {
                    const auto z = __builtin_amdgcn_permlane32_swap(__float_as_uint(up[2 * e + f]), __float_as_uint(down[2 * e + f]), false, false);
                    y[f] = __builtin_elementwise_maximum(__uint_as_float(z[0]), __uint_as_float(z[1]));
                }
                const auto z = __builtin_amdgcn_permlane16_swap(__float_as_uint(y[0]), __float_as_uint(y[1]), false, false);
                four[e] = __builtin_elementwise_maximum(__uint_as_float(z[0]), __uint_as_float(z[1]));
                if (kLanes == 8) four[e] = __builtin_elementwise_maximum(four[e], __uint_as_float(dpp<0x128>(__float_as_uint(four[e]))));      // (eight lanes further)
            }
            const uint32_t c = codes8_of(four[0], four[1], four[2], four[3], scale);
            const f32x2 y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, 1.f, false), z = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, 1.f, true);
            if (!kEarly && behind) look();
            const float shrink = __uint_as_float((uint32_t)(127 - grow) << 23);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float code = e < 2 ? y[e & 1] : z[e & 1];
                float bound = code != code ? 127.f : __builtin_ceilf(code * 0.25f);
                if (behind) {
                    const float old = (float)old_bounds[e];
                    bound = fmaxf(bound, __builtin_ceilf((lane < 32 ? old : -old) * shrink));
                }
                if (kLanes == 16 || (lane & 8) == 0) bounds[2 * e] = (int8_t)(int)(lane < 32 ? bound : -bound);
            }
            // eight channels of a token a lane
            const uint32_t to = ((piece >> 3) * 4 + (piece >> 1 & 3)) * 256 + (piece & 1) * 8;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int t = token_of(i);
                const u32x2 y = kExpanded ? codes_of(x[kExpanded ? i : 0], scale) : codes_of(words[i], scale);
                if (stored >> t & 1) *(u32x2*)(codes + (t >> 4) * (16 * D) + to + (t & 15) * 16) = y;
            }
        } else {                                                  // a head of V
            uint8_t* const codes = at.codes(item - hkv, block) + 32 * D;
            uint8_t* const power_at = (uint8_t*)at.powers(item - hkv, block) + 1;
            const int old_power = behind ? *power_at : 0;
            u32x4* const lane_words = (u32x4*)codes + lane;
            u32x4 old[D / 32] = {};                               // of a block that is written in part
            if (kEarly && stored != kAllTokens) {
#pragma unroll
                for (int g = 0; g < D / 32; ++g) old[g] = lane_words[64 * g];
            }
            uint32_t pair = 0;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                if (gone && !there_of(i)) words[i] = kNoRow;
#pragma unroll
                for (int e = 0; e < 4; ++e) pair = max_u16(pair, words[i][e] & 0x7fff7fffu);
            }
            float top = __uint_as_float(max(pair & 0xffff0000u, pair << 16));
            if (__builtin_amdgcn_ballot_w64(!(top <= most)) != 0) {
                uint32_t bits = 0;
                afresh(words);
#pragma unroll
                for (int i = 0; i < kLoads; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        raise_finite(bits, low_of(words[i][e]));
                        raise_finite(bits, high_of(words[i][e]));
                    }
                top = __uint_as_float(bits);
            }
            int grow;
            const float scale = settle(top, old_power, power_at, codes, &grow);
            if (kEarly ? grow > 0 : stored != kAllTokens) {
#pragma unroll
                for (int g = 0; g < D / 32; ++g) old[g] = lane_words[64 * g];
            }
            // in LDS as rows, from where transposing reads give eight tokens of a channel
#pragma unroll
            for (int i = 0; i < kLoads; ++i) *(u32x2*)&staged[token_of(i)][8 * piece] = codes_of(words[i], scale);
            meet();
            const int r = lane & 15, j = lane >> 4, e = r >> 1;
            uint32_t keep[2] = {0, 0};                            // the bytes of a word that stay as they are: tokens 16 h + 4 j + i, i = 0 .. 3
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if ((stored >> (16 * (i >> 2) + 4 * j + (i & 3)) & 1) == 0) keep[i >> 2] |= 0xffu << (8 * (i & 3));
            const uint32_t from = (uint32_t)(uintptr_t)(lptr_t)&staged[16 * (e >> 2) + 4 * j + (e & 3)][8 * (r & 1)];
#pragma unroll
            for (int g = 0; g < D / 32; ++g) {
                const i32x2 y = lds_read_tr8(from + 32 * g), z = lds_read_tr8(from + 32 * g + 16);
                u32x4 word = {(uint32_t)y[0], (uint32_t)y[1], (uint32_t)z[0], (uint32_t)z[1]};
                if (stored != kAllTokens) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) word[i] = (word[i] & ~keep[i & 1]) | (old[g][i] & keep[i & 1]);
                }
                lane_words[64 * g] = word;
            }
            meet();                                               // (the next item's rows go to the same place)
        }
        if (item + step < items) load(item + step, words);
    }
}

// A step's new token: D / 8 lanes take a head, so that several heads share a wavefront and nothing has to cross lanes but a power.  A wavefront has one group of heads
// (64 sequences, 32/32 heads: 7.7 us, as pieces of any length 15.1; one on 8/8 heads of 64 3.5 and 5.3).
template <int D, int kTurn>
__global__ __launch_bounds__(64 * kWaves) void cache8_append_one_kernel(AppendArgs a) {
    constexpr int kLanes = D / 8, kHeads = 64 / kLanes;           // lanes of a head, heads of a wavefront
    __shared__ __align__(16) f32x2 turns[turns_of_row<D, kTurn>];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), piece = lane % kLanes;
    const int place = blockIdx.x / a.head_groups, group = (blockIdx.x - place * a.head_groups) * kWaves + wave;
    const int kv_groups = (a.c.n_kv_heads + kHeads - 1) / kHeads;
    const Piece p = piece_of(a, place);
    if (p.stored == 0) return;
    const int t = __builtin_ctz(p.stored), row = __builtin_amdgcn_readlane(p.from, t);
    const bool of_q = group >= kv_groups;
    const int heads = of_q ? a.n_q_heads : a.c.n_kv_heads, wanted_head = (of_q ? group - kv_groups : group) * kHeads + lane / kLanes;
    const bool real = wanted_head < heads;
    const int head = min(wanted_head, max(heads - 1, 0));
    const int64_t at_row = max(row, 0);
    u32x4 kx = {}, vx = {};
    if (!of_q) {
        kx = __builtin_nontemporal_load((const u32x4*)a.k + at_row * a.k_stride + head * kLanes + piece);
        vx = __builtin_nontemporal_load((const u32x4*)a.v + at_row * a.v_stride + head * kLanes + piece);
    } else if (heads > 0) {
        kx = __builtin_nontemporal_load((const u32x4*)a.q + at_row * a.q_stride + head * kLanes + piece);
    }
    const Page8<D> at(a.c, p.page);
    uint8_t* const codes = at.codes(head, p.block);
    uint16_t* const powers = at.powers(head, p.block);
    u32x2* const bounds = (u32x2*)at.bounds(head, p.block) + piece;      // largest; kLanes further the smallest
    uint32_t old_powers = 0;
    u32x2 old_up = {}, old_down = {};
    if (p.behind && !of_q) {
        old_powers = *powers;
        old_up = bounds[0];
        old_down = bounds[kLanes];
    }
    if constexpr (kTurn != kAsIs) {
        if (wave == 0) {
            const float freq = lane < a.dims / 2 ? a.freqs[lane] : 0.f;
            const f32x2 turn = turn_of(row >= 0 ? a.positions[row] : 0, freq);
            if (lane < a.dims / 2) turns[place_of<D, kTurn>(lane)] = turn;
        }
        __syncthreads();
    }
    float x[8];
    turned<D, kTurn>(kx, turns, a.dims, piece, x);
    if (kTurn != kAsIs && !of_q) {
        uint32_t near = near_words<D, kTurn>(x, turns, a.dims, piece);
        while (near != 0) {
            const int w = __builtin_ctz(near);
            near &= near - 1;
            const Exactly y = turned_exactly<D, kTurn>((const uint32_t*)((const u32x4*)a.k + at_row * a.k_stride + head * kLanes + piece), w, a.positions[at_row], a.freqs, a.dims, piece);
#pragma unroll
            for (int v = 0; v < 4; ++v)
                if (v == w) {
                    x[2 * v] = y.value(0, x[2 * v]);
                    x[2 * v + 1] = y.value(1, x[2 * v + 1]);
                }
        }
    }
    if (of_q) {
        if (real && row >= 0) __builtin_nontemporal_store(rounded(x), (u32x4*)a.q_out + (at_row * a.n_q_heads + head) * kLanes + piece);
        return;
    }
    if (row < 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = NAN;
        vx = u32x4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
    }
    uint32_t ktop = 0, vtop = 0;                                  // magnitudes, as bits: what is no number is above all others
#pragma unroll
    for (int e = 0; e < 8; ++e) ktop = max(ktop, __float_as_uint(x[e]) & 0x7fffffffu);
#pragma unroll
    for (int e = 0; e < 4; ++e) vtop = max_u16(vtop, vx[e] & 0x7fff7fffu);
    vtop = max(vtop & 0xffff0000u, vtop << 16);
    const bool special = __builtin_amdgcn_ballot_w64(ktop > kNoNumber || vtop > kNoNumber) != 0;
    bool none[8];                                                 // numbers without a code
#pragma unroll
    for (int e = 0; e < 8; ++e) none[e] = special && !(fabsf(x[e]) <= __uint_as_float(kNoNumber));
    if (special) {
        ktop = vtop = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            raise_finite(ktop, x[e]);
            raise_finite(vtop, e & 1 ? high_of(vx[e >> 1]) : low_of(vx[e >> 1]));
        }
    }
    int kp = power8_of(__uint_as_float(within_lanes<kLanes>(ktop, larger))), vp = power8_of(__uint_as_float(within_lanes<kLanes>(vtop, larger)));
    int kgrow = 0, vgrow = 0;
    if (p.behind) {
        const int old_kp = old_powers & 255, old_vp = old_powers >> 8;
        kp = max(kp, old_kp);
        vp = max(vp, old_vp);
        kgrow = min(kp - old_kp, 100);
        vgrow = min(vp - old_vp, 100);
    }
    const float kscale = scale_of(kp);
    const u32x2 k8 = codes_of(x, kscale), v8 = codes_of(vx, scale_of(vp));
    u32x2 up, down;
    bounds_of(k8, none, p.behind, old_up, old_down, kgrow, up, down);
    if (real) {
        bounds[0] = up;
        bounds[kLanes] = down;
        if (piece == 0) *powers = (uint16_t)(kp | vp << 8);
    }
    if (__builtin_amdgcn_ballot_w64(real && (kgrow > 0 || vgrow > 0)) != 0) {
        const float kby = __uint_as_float((uint32_t)(127 + kgrow) << 23), vby = __uint_as_float((uint32_t)(127 + vgrow) << 23);
#pragma unroll 1
        for (int g = 0; g < 16; ++g) {                            // (2 D words of 16 bytes each)
            u32x4* const kw = (u32x4*)codes + kLanes * g + piece;
            u32x4* const vw = (u32x4*)(codes + 32 * D) + kLanes * g + piece;
            u32x4 y = *kw, z = *vw;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                y[i] = regrown(y[i], kby);
                z[i] = regrown(z[i], vby);
            }
            if (real && kgrow > 0) *kw = y;
            if (real && vgrow > 0) *vw = z;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");    // (the bytes are written again below, by other lanes)
        __builtin_amdgcn_s_waitcnt(0);
    }
    if (!real) return;
    *(u32x2*)(codes + (t >> 4) * (16 * D) + ((piece >> 3) * 4 + (piece >> 1 & 3)) * 256 + (piece & 1) * 8 + (t & 15) * 16) = k8;
    uint8_t* const to = codes + 32 * D + (piece >> 2) * 1024 + (t >> 2 & 3) * 256 + (piece & 1) * 128 + (piece >> 1 & 1) * 8 + (t >> 4) * 4 + (t & 3);
#pragma unroll
    for (int e = 0; e < 8; ++e) to[16 * e] = (uint8_t)(v8[e >> 2] >> (8 * (e & 3)));
}

struct LoadArgs {
    CacheView c;
    const int32_t *slots, *first, *offsets;
    uint16_t *k, *v;
    int32_t n_rows, max_len, tiles_of_seq, head_groups;
};
static_assert(sizeof(LoadArgs) <= 112, "short arguments");

// A block's codes meet in LDS as rows, V's through transposing reads, from where a wavefront writes whole rows of the head, 16 bytes a lane.
template <int D>
__global__ __launch_bounds__(64 * kWaves) void cache8_load_kernel(LoadArgs a) {
    constexpr int kGroups = D / 32, kRow = D + 16;
    __shared__ __align__(16) uint8_t all_rows[kWaves][32][kRow];
    __shared__ __align__(16) uint8_t all_words[kWaves][kGroups][64][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, t = lane & 15, j = lane >> 4;
    const int place = blockIdx.x / a.head_groups, b = place / a.tiles_of_seq;
    const int head = (blockIdx.x - place * a.head_groups) * kWaves + wave;
    const int slot = cache_slot(a.c, a.slots, b);
    const int offset = a.offsets[b], end_row = min(a.offsets[b + 1], a.n_rows), begin = a.first != nullptr ? a.first[b] : 0;
    if (slot < 0 || offset < 0 || end_row <= offset || begin < 0 || head >= a.c.n_kv_heads) return;
    const int64_t token0 = (begin & ~31) + 32 * (int64_t)(place - b * a.tiles_of_seq);
    const int64_t end = min((int64_t)begin + min(end_row - offset, a.max_len), (int64_t)cache_len(a.c, slot));      // tokens begin .. end - 1
    if (token0 >= end) return;
    const int block = (int)(token0 >> 5);
    const int page = a.c.table[(int64_t)slot * a.c.max_pages + (token0 >> a.c.shift)];
    if (page < 0 || page >= a.c.n_pages) return;
    const Page8<D> at(a.c, page);
    const u32x4* in = (const u32x4*)at.codes(head, block) + lane;
    uint8_t(*const rows)[kRow] = all_rows[wave];
    uint8_t(*const words)[64][16] = all_words[wave];
    u32x4 kc[kGroups], vc[kGroups];
    const uint32_t powers = *at.powers(head, block);
#pragma unroll
    for (int g = 0; g < kGroups; ++g) kc[g] = in[64 * g];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) vc[g] = in[64 * (kGroups + g)];
    const int64_t row_words = (int64_t)a.c.n_kv_heads * D;
    auto write_rows = [&](uint16_t* out, float scale) {
        constexpr int kLanes = D / 8;
        meet();
#pragma unroll
        for (int i = 0; i < 32 * kLanes / 64; ++i) {
            const int token = i * (64 / kLanes) + lane / kLanes, channel = 8 * (lane % kLanes);
            const u32x2 x = *(const u32x2*)&rows[token][channel];
            const int64_t row = offset + (token0 + token - begin);
            if (token0 + token >= begin && token0 + token < end)
                __builtin_nontemporal_store(__builtin_bit_cast(u32x4, values8_of(x[0], x[1], scale)), (u32x4*)(out + row * row_words + head * D + channel));
        }
        meet();
    };
    if (a.k != nullptr) {
#pragma unroll
        for (int g = 0; g < kGroups; ++g) *(u32x4*)&rows[16 * (g / (D / 64)) + t][64 * (g % (D / 64)) + 16 * j] = kc[g];
        write_rows(a.k, scale_of(powers & 255));
    }
    if (a.v != nullptr) {
#pragma unroll
        for (int g = 0; g < kGroups; ++g) *(u32x4*)words[g][lane] = vc[g];
        meet();
        // a lane's word of a transposing read: channel r = t / 2 of eight, of both halves of 16 in turn; what it gets: those of token e of the group's eight
        const uint32_t from = (uint32_t)(uintptr_t)(lptr_t)&words[0][16 * j + (t >> 1) + 8 * (t & 1)][0];
        const int e = t & 7, token = 16 * (e >> 2) + 4 * j + (e & 3);
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
#pragma unroll
            for (int p = 0; p < 2; ++p)
                *(i32x2*)&rows[token][32 * g + 16 * p + 8 * (t >> 3)] = lds_read_tr8(from + 1024 * g + 8 * p);
        }
        write_rows(a.v, scale_of(powers >> 8));
    }
}

// The page of a parent that is filled in part, as it is.  grid: (n, pieces of a page)
__global__ __launch_bounds__(256) void cache8_fork_copy_kernel(CacheView c, const int32_t* __restrict__ parents, const int32_t* __restrict__ children,
                                                               const int32_t* __restrict__ status, uint32_t page_chunks, uint32_t piece_chunks) {
    const int state = *status, parent = parents[blockIdx.x], child = children[blockIdx.x];
    if (state != 0 || parent < 0) return;
    const int len = cache_len(c, parent), full = len >> c.shift;
    if ((len & ((1 << c.shift) - 1)) == 0) return;
    const int src = c.table[(int64_t)parent * c.max_pages + full], dst = c.table[(int64_t)child * c.max_pages + full];
    if (src < 0 || src >= c.n_pages || dst < 0 || dst >= c.n_pages) return;
    const u32x4* from = (const u32x4*)c.pages + (int64_t)src * page_chunks;
    u32x4* to = (u32x4*)c.pages + (int64_t)dst * page_chunks;
    constexpr int kMany = 4;
    const uint32_t end = min(page_chunks, (blockIdx.y + 1) * piece_chunks);
    for (uint32_t first = blockIdx.y * piece_chunks + threadIdx.x; first < end; first += 256 * kMany) {
        u32x4 x[kMany];
#pragma unroll
        for (int k = 0; k < kMany; ++k)
            if (first + 256 * k < end) x[k] = from[first + 256 * k];
#pragma unroll
        for (int k = 0; k < kMany; ++k)
            if (first + 256 * k < end) to[first + 256 * k] = x[k];
    }
}

template <int D, int kTurn, bool kShort>
void launch_append_items(AppendArgs a, int64_t pieces, hipStream_t stream) {
    const int64_t items = 2 * a.c.n_kv_heads + a.n_q_heads, most = (items + kWaves - 1) / kWaves;
    constexpr int64_t kHeld = 256 * append_waves<D, kTurn, kShort>;      // workgroups that the chip holds
    // Items of a wavefront: two share a reckoning of the turns, more of them leave too little in flight, and few pieces need all the workgroups they can get.  Measured,
    // us, one, two, four, turned with Q behind 77 tokens: 8 x 2048 tokens on 32/32 heads 193, 147, 149; 7 x 100 ... 3000 on 32/8 72, 52, 50; the same at 64 channels 35, 28.5, 26.5; 64 x 64 on 32/8 39, 32.6,
    // 33.5; 1 x 800 on 32/32 18.5, 16.4, 20; 16 x 200 on 8/8 18.4, 16.8, 17.1; 64 x 9 on 40/40 21.5, 19.2, 22, on 32/8 11.5, 10.5, 13.3; 2 x 500 on 12/12 heads of 64 7.9, 8.9, 10.2; 8 x 5 on 32/8
    // 5.5, 6.6, 8.8; 70 % of 8 x 2048 rows as they are on 32 heads 54.6, 52.7, 54.4
    const int64_t each = pieces * most > kHeld ? 2 : 1;
    a.head_groups = (int32_t)((most + each - 1) / each);
    hipLaunchKernelGGL((cache8_append_kernel<D, kTurn, kShort>), dim3((unsigned)(pieces * a.head_groups)), dim3(64 * kWaves), 0, stream, a);
}

template <int D, int kTurn>
void launch_append(AppendArgs a, int64_t pieces, hipStream_t stream) {
    if (a.max_new > 9) launch_append_items<D, kTurn, false>(a, pieces, stream);
    else if (a.max_new > 1) launch_append_items<D, kTurn, true>(a, pieces, stream);
    else {
        constexpr int kHeads = 512 / D;                           // (of a wavefront)
        const int groups = (a.c.n_kv_heads + kHeads - 1) / kHeads + (a.n_q_heads + kHeads - 1) / kHeads;
        a.head_groups = (groups + kWaves - 1) / kWaves;
        hipLaunchKernelGGL((cache8_append_one_kernel<D, kTurn>), dim3((unsigned)(pieces * a.head_groups)), dim3(64 * kWaves), 0, stream, a);
    }
}

}  // namespace

int launch_cache8_append(const CacheView& c, int32_t head_dim, const Cache8Rows& rows, const int32_t* offsets, const int32_t* slots, const int32_t* start,
                         int32_t n_seqs, int32_t max_new, hipStream_t stream) {
    const int64_t tiles = ((int64_t)max_new + 30) / 32 + 1;
    const AppendArgs a{c, (const uint16_t*)rows.k, (const uint16_t*)rows.v, (const uint16_t*)rows.q, (uint16_t*)rows.q_out, rows.row_idx, offsets, slots, start,
                       rows.positions, rows.freqs, rows.k_stride, rows.v_stride, rows.q_stride, rows.n_rows, rows.n_list, max_new, (int32_t)tiles, 0,
                       rows.n_q_heads, rows.dims};
    const int turn = rows.dims == 0 ? kAsIs : rows.interleaved ? kPairs : rows.dims == head_dim ? kAllHalves : kHalves;
    if (head_dim == 128) {
        if (turn == kAsIs) launch_append<128, kAsIs>(a, n_seqs * tiles, stream);
        else if (turn == kAllHalves) launch_append<128, kAllHalves>(a, n_seqs * tiles, stream);
        else if (turn == kHalves) launch_append<128, kHalves>(a, n_seqs * tiles, stream);
        else launch_append<128, kPairs>(a, n_seqs * tiles, stream);
    } else {
        if (turn == kAsIs) launch_append<64, kAsIs>(a, n_seqs * tiles, stream);
        else if (turn == kAllHalves) launch_append<64, kAllHalves>(a, n_seqs * tiles, stream);
        else if (turn == kHalves) launch_append<64, kHalves>(a, n_seqs * tiles, stream);
        else launch_append<64, kPairs>(a, n_seqs * tiles, stream);
    }
    return check_launch();
}

int launch_cache8_load(const CacheView& c, int32_t head_dim, const int32_t* slots, const int32_t* first, const int32_t* offsets, int32_t n_seqs,
                       int32_t max_len, void* k, void* v, int32_t n_rows, hipStream_t stream) {
    const int64_t tiles = ((int64_t)max_len + (first != nullptr ? 62 : 31)) / 32;
    const int groups = (c.n_kv_heads + kWaves - 1) / kWaves;
    const LoadArgs a{c, slots, first, offsets, (uint16_t*)k, (uint16_t*)v, n_rows, max_len, (int32_t)tiles, groups};
    const dim3 blocks((unsigned)(n_seqs * tiles * groups)), threads(64 * kWaves);
    if (head_dim == 128) hipLaunchKernelGGL((cache8_load_kernel<128>), blocks, threads, 0, stream, a);
    else hipLaunchKernelGGL((cache8_load_kernel<64>), blocks, threads, 0, stream, a);
    return check_launch();
}

int launch_cache8_fork_copy(const CacheView& c, int32_t head_dim, const int32_t* parents, const int32_t* children, int32_t n, const int32_t* status,
                            hipStream_t stream) {
    if (n == 0) return PYR_OK;
    const uint32_t chunks = (uint32_t)(cache8_page_bytes(head_dim, c.n_kv_heads, 1 << (c.shift - 5)) / 16);
    const uint32_t piece = chunks <= 1024 * 1024 ? 1024 : chunks / 1024;      // (a thousand pieces at most; 2^31 bytes are 2^27 chunks)
    hipLaunchKernelGGL(cache8_fork_copy_kernel, dim3((unsigned)n, (chunks + piece - 1) / piece), dim3(256), 0, stream, c, parents, children, status, chunks, piece);
    return check_launch();
}

}  // namespace pyr
