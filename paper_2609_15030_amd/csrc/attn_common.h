// Attention over packed or cached keys: what its kernels share.
//
// A row is one (token, query head).  The G = q_heads / kv_heads query heads of
// a key head stand beside one another, so the rows of a sequence under one key
// head are numbered token * G + head-in-group and a tile of rows reads each key
// once for the whole group.  Per row, with c = scale and log2(e) folded in,
//
//   t_j = c <q, k_j>,  p_j = 2^(t_j - m),  m = max t_j,  o = sum p_j v_j / sum p_j
//
// over the visible keys j < limit(row); a row that sees none is 0.  Keys are
// taken in tiles with the running m and l = sum p; a part of the keys leaves
// (m, l, sum p v), and parts join by 2^(m_part - m).  Scores, m, l and the sums
// are fp32; p is rounded to the type of v for the matrix product (bf16 p: half
// an ulp, unbiased, of the size of the rounding of the output itself).
//
// The kernels form S^T = K Q^T, whose accumulators (rows: keys, columns: rows of
// q) are the B operand of O^T = V^T P^T as they stand: a lane's accumulators
// belong to one q row, and the contraction index is permuted on the V side.
#pragma once
#include <type_traits>

#include "la_common.h"

namespace la {

typedef unsigned char fp8_t;               // e4m3 bits
// Codes of a cache whose blocks hold a scale for each key head: a code stands for
// itself times the scale.
struct e4m3_code { unsigned char bits; };  // scales: powers of two
struct int8_code { signed char bits; };
template <typename C> constexpr bool kBlockScaled = std::is_same<C, e4m3_code>::value || std::is_same<C, int8_code>::value;
// Where attention applies the scales.  A power of two goes into the conversion to bf16,
// exactly and for nothing.  Others would round there: those of keys multiply the scores
// and those of values the weights, in fp32 (before the weights' own rounding to bf16).
template <typename C> constexpr bool kScaleCodes = std::is_same<C, e4m3_code>::value;
template <typename C> constexpr bool kScaleScores = kBlockScaled<C> && !kScaleCodes<C>;
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr float kAttnLog2e = 1.4426950408889634f;

// Where keys and values come from: packed rows, or the blocks of a cache.
struct KvSource {
    const char *k, *v;             // packed: first row; cache: the layer's keys / values in block 0
    int64_t k_stride, v_stride;    // packed: bytes from one token to the next
    int64_t block_bytes;           // cache: bytes from one block to the next
    const int32_t *table;          // cache: [sequences, max_blocks]; NULL: packed
    int64_t max_blocks;
    int32_t n_blocks, bt_shift;    // blocks of 2^bt_shift tokens
    int32_t *err;
    const char *ks, *vs;           // block-scaled cache: the layer's scales in block 0, fp32 [kv_heads]
};

// Division of n < 2^31 by a divisor known to the host: a high product, an add and
// two shifts in place of the 30-odd instructions of a run-time division.
struct FastDiv {
    uint32_t m, s1, s2;
    __host__ static FastDiv by(uint32_t d) {
        uint32_t l = 0;
        while (((uint64_t)1 << l) < d) ++l;
        return {(uint32_t)((((((uint64_t)1 << l) - d) << 32) / d) + 1), l < 1 ? l : 1u, l < 1 ? 0u : l - 1};
    }
    __device__ inline int operator()(int n) const {
        const uint32_t t = __umulhi(m, (uint32_t)n);
        return (int)((t + (((uint32_t)n - t) >> s1)) >> s2);
    }
};

struct AttnArgs {
    const void *q;
    void *o;
    int64_t q_stride, o_stride;    // elements from one token to the next
    KvSource kv;
    const int32_t *cu;             // prompts: token offsets [n_seqs + 1]
    const int32_t *kv_len;         // keys of each sequence (NULL: as many as its tokens)
    const int32_t *cu_group;       // decode: sequences of each group [n_groups + 1], or NULL
    const int32_t *prefix_len;     // decode: shared keys of each group
    float c, v_scale;              // scale * k_scale * log2(e); value of a stored v of 1
    int32_t n_seqs, kv_heads, group, n_groups;
    FastDiv by_group, by_kv_heads; // row / group, item / kv_heads
    int32_t part_shift;            // prompts: keys of a part, as a power of two; 0: whole rows
    int32_t max_kv;                // longest kv_len that the tables and the workspace cover
    int32_t parts;                 // decode: parts the workspace holds for each row
    int32_t prefix_parts;          // decode: of these, the most of a prefix
    int32_t max_group;             // decode: sequences of a group that share, at most
    int32_t group_tiles;           // decode: row tiles of so many
    int32_t prefix_items;          // decode: workgroups of the prefixes, ahead of the others
    bool ordered;                  // prompts: sequences in `order` (up to 64), the longest first
    uint8_t order[64];
    bool direct;                   // decode: one part each, written straight to o
    float *part_o;                 // [slot][D]
    float2 *part_ml;               // [slot]
};

// Keys of one part of a shared prefix, and of a sequence's own keys (decode).
constexpr int kPrefixPart = 256;
constexpr int kOwnPart = 256;

// Prompts: rows of a tile in bf16.  Where a call's row tiles alone would leave much
// of the chip idle, every sequence's keys are cut into parts of 2^part_shift (0: not
// cut), the smallest power of two from 2^kPromptPartShift on that makes no more than
// prompt_grid workgroups.
constexpr int kPromptRows = 128;
constexpr int kPromptPartShift = 8;

__host__ __device__ inline int prompt_parts(int keys, int part_shift) {
    return part_shift && keys > (1 << part_shift) ? (int)(((uint32_t)keys + (1u << part_shift) - 1) >> part_shift) : 1;
}

// --- 16-byte pieces of rows, as the LDS tiles hold them ---------------------

template <typename T> struct Piece { static constexpr int N = 16 / sizeof(T); };   // elements

__device__ inline uint2 buf_load8(__amdgpu_buffer_rsrc_t r, uint32_t voff) {
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    const i32x2 v = __builtin_amdgcn_raw_buffer_load_b64(r, (int)voff, 0, 0);
    return make_uint2((uint32_t)v[0], (uint32_t)v[1]);
}

// Four codes as bf16 pairs, exactly; e4m3 times a power of two.
template <typename C> __device__ inline uint2 bf16_of4(uint32_t x, float scale = 1.0f) {
    bf16x2 a, b;
    if constexpr (std::is_same<C, int8_code>::value) {
        a = bf16x2{(__bf16)(float)(int8_t)x, (__bf16)(float)(int8_t)(x >> 8)};
        b = bf16x2{(__bf16)(float)(int8_t)(x >> 16), (__bf16)(float)(int8_t)(x >> 24)};
    } else {
        a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, false);
        b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, true);
    }
    return make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
}

// The registers of one piece in flight: 16 bytes, or 8 that become 16.
template <typename C> struct Raw { std::conditional_t<sizeof(C) == 1, uint2, uint4> x; };

template <typename C> __device__ inline Raw<C> load_piece(__amdgpu_buffer_rsrc_t r, uint32_t voff) {
    if constexpr (sizeof(C) == 1) return {buf_load8(r, voff)};
    else return {buf_load16(r, voff, 0)};
}

template <typename C> __device__ inline uint4 piece_of(const Raw<C> &p, float scale = 1.0f) {
    if constexpr (sizeof(C) == 1) {
        const uint2 a = bf16_of4<C>(p.x.x, scale), b = bf16_of4<C>(p.x.y, scale);
        return make_uint4(a.x, a.y, b.x, b.y);
    } else {
        return p.x;
    }
}

// Whether a piece holds an infinity or NaN (an exponent of all ones).  bf16: both
// exponents of a word at once, a one added to each carries into the sign's place.
template <typename T> __device__ inline bool has_nonfinite(const uint4 &x) {
    if constexpr (sizeof(T) == 2) {
        constexpr uint32_t E = 0x7F807F80u, ONE = 0x00800080u;
        return ((((x.x & E) + ONE) | ((x.y & E) + ONE) | ((x.z & E) + ONE) | ((x.w & E) + ONE)) & 0x80008000u) != 0;
    } else {
        constexpr uint32_t E = 0x7F800000u;
        return (x.x & E) == E || (x.y & E) == E || (x.z & E) == E || (x.w & E) == E;
    }
}

// Those made zero.
template <typename T> __device__ inline void drop_nonfinite(uint4 &x) {
    uint32_t *w = &x.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 2) {
            if ((w[i] & 0x7F80u) == 0x7F80u) w[i] &= 0xFFFF0000u;
            if ((w[i] & 0x7F800000u) == 0x7F800000u) w[i] &= 0x0000FFFFu;
        } else {
            if ((w[i] & 0x7F800000u) == 0x7F800000u) w[i] = 0;
        }
    }
}

// Byte offsets of runs of 16 cached tokens behind a layer's keys (and values), for
// one key head: lane j holds run j of the 1,024 tokens from `base` on.  A run lies
// in one block; its offset is read from its lane when it is needed, which takes two
// instructions where a table entry read then and there took a scalar load (whose
// wait is also one for every LDS read in flight) and some twenty instructions.  Runs
// past the last key are at block 0's offset; those in a block that the table does not
// name too, and are in `bad`.
constexpr int kRunTokens = 16;
struct Runs {
    int64_t at;
    uint64_t bad;
    float ks, vs;                  // block-scaled cache: the lane's run's scales
    // The lane's block id of the 1,024 tokens `ahead` of base.  Compared by distance: a
    // sequence may end so near 2^31 that the token itself passes it.
    __device__ static inline int fetch(const KvSource &s, const int32_t *table_row, int base, int ahead, int hi) {
        const int off = ahead + kRunTokens * (int)(threadIdx.x & 63);
        return off < hi - base ? table_row[(base + off) >> s.bt_shift] : 0;
    }
    __device__ inline void set(const KvSource &s, int id, int base, int kvh, int row_bytes) {
        const bool ok = (uint32_t)id < (uint32_t)s.n_blocks;
        bad = __ballot(!ok);
        if (!ok && s.err) atomicAdd(s.err, 1);
        const uint32_t t = (uint32_t)base + kRunTokens * (threadIdx.x & 63);
        at = (int64_t)(ok ? id : 0) * s.block_bytes +
             (int64_t)((kvh << s.bt_shift) + (int)(t & ((1u << s.bt_shift) - 1))) * row_bytes;    // may pass 2 GB within a block
    }
    // Scales of the lane's run, of block `id` (as fetched `ahead` of base); 1 past the last
    // key and in blocks that are none, whose bytes may be anything.
    __device__ static inline void fetch_scales(const KvSource &s, int id, int base, int ahead, int hi, int kvh, float *ks, float *vs) {
        *ks = *vs = 1.f;
        if (ahead + kRunTokens * (int)(threadIdx.x & 63) < hi - base && (uint32_t)id < (uint32_t)s.n_blocks) {
            const int64_t b = (int64_t)id * s.block_bytes + 4 * (int64_t)kvh;
            *ks = *(const float *)(s.ks + b);
            *vs = *(const float *)(s.vs + b);
        }
    }
    __device__ inline float k_scale(int r) const { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks), r)); }
    __device__ inline float v_scale(int r) const { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vs), r)); }
    __device__ inline int64_t run(int r) const {
        const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)at, r);
        const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(at >> 32), r);
        return (int64_t)((uint64_t)hi << 32 | lo);
    }
    __device__ inline bool named(int r) const { return !(bad >> r & 1); }
};

// What the scores of a run with key scale ks are multiplied by.  Not zero: masked scores
// are minus infinity when they are multiplied.  The least subnormal: a factor is off by at
// most 2^-149 then, and a score of fp32's size by 2^-21, where the least normal number would
// let large queries give keys of the least scale up to 16 times their weight.
__device__ inline float run_factor(float c, float ks) { return fmaxf(c * ks, 0x1p-149f); }

// Maximum and sum over the four lanes (l, l + 16, l + 32, l + 48) that share a
// q row of a 16-column accumulator.
__device__ inline float row_max16(float x) {
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ inline float row_sum16(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// Eight (bf16) values of two accumulators as a B operand.
__device__ inline bf16x8 pack8(f32x4 a, f32x4 b) {
    return bf16x8{(__bf16)a[0], (__bf16)a[1], (__bf16)a[2], (__bf16)a[3],
                  (__bf16)b[0], (__bf16)b[1], (__bf16)b[2], (__bf16)b[3]};
}

__device__ inline i16x4 lds_tr(const void *p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)p);
}

__device__ inline bf16x8 join_tr(i16x4 a, i16x4 b) {
    const i16x8 x = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    return __builtin_bit_cast(bf16x8, x);
}

// (m, l, x) joined by the weight of a part's (mp, lp, xp): the running sums
// shrink by *w, the part's by *wp.
__device__ inline void join_weights(float &m, float &l, float mp, float lp, float *w, float *wp) {
    const float m2 = fmaxf(m, mp), mu = m2 == -INFINITY ? 0.f : m2;
    *w = __builtin_amdgcn_exp2f(m - mu);
    *wp = __builtin_amdgcn_exp2f(mp - mu);
    m = m2;
    l = __builtin_fmaf(lp, *wp, l * *w);
}
__device__ inline f32x4 join4(f32x4 x, f32x4 xp, float w, float wp) {
    f32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_fmaf(xp[i], wp, x[i] * w);
    return r;
}

// What a row's sums are multiplied by for its output.
__device__ inline float row_scale(const AttnArgs &a, float l) { return l > 0.f || l != l ? a.v_scale / l : 0.f; }

// Four consecutive outputs.
__device__ inline void store4(float *p, f32x4 x) { *(f32x4 *)p = x; }
__device__ inline void store4(__bf16 *p, f32x4 x) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    *(bf16x4 *)p = bf16x4{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
}

// Inclusive sum over the wave's lanes.
__device__ inline int wave_scan(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true);       // rows of 16: shifts by 1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);      // row ends to the next row, then to the upper half
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);
    return x;
}

// The sequence of row `tok`, by offsets cu [n + 1], one sequence a lane; its rows are
// [*first, *end).  False for rows before the first sequence and behind the last.
__device__ inline bool sequence_of(const int32_t *cu, int n, int tok, int *seq, int *first, int *end) {
    const int lane = threadIdx.x & 63;
    for (int i0 = 0; i0 < n; i0 += 64) {
        const int i = min(i0 + lane, n - 1), c0 = cu[i], c1 = cu[i + 1];
        const uint64_t past = __ballot(c1 > tok);
        if (!past) continue;
        const int at = __builtin_ctzll(past);
        *seq = i0 + at;
        *first = __builtin_amdgcn_readlane(c0, at);
        *end = __builtin_amdgcn_readlane(c1, at);
        return *first <= tok;
    }
    return false;
}

// Where the first of n ascending truths `past(i)` may be: in [result, result + 64), or
// nowhere.  Each step asks 64 at once, evenly spaced: three of them for 262,144, where
// going through the sequences takes one for every 64.
template <typename F> __device__ inline int narrow_to_64(int n, F past) {
    const uint32_t lane = threadIdx.x & 63;
    uint32_t lo = 0, hi = (uint32_t)n;
    while (hi - lo > 64) {
        const uint32_t step = (hi - lo + 63) >> 6;
        const uint64_t yes = __ballot(past((int)(min(lo + (lane + 1) * step, hi) - 1)));
        if (!yes) return (int)hi - 1;
        lo += (uint32_t)__builtin_ctzll(yes) * step;
        hi = min(hi, lo + step);
    }
    return (int)lo;
}

// The sequence of row `tok` and the row's position, which is its place from the end of
// kv_len's keys; false outside every sequence.  The lengths are read beside the offsets,
// not after the sequence is known.
__device__ inline bool position_of(const int32_t *cu, const int32_t *kv_len, int n, int tok, int *seq, int *pos) {
    const int i0 = narrow_to_64(n, [&](int i) { return cu[i + 1] > tok; });
    const int i = min(i0 + (int)(threadIdx.x & 63), n - 1), c0 = cu[i], c1 = cu[i + 1], len = kv_len[i];
    const uint64_t past = __ballot(c1 > tok);
    if (!past) return false;
    const int at = __builtin_ctzll(past);
    *seq = i0 + at;
    *pos = __builtin_amdgcn_readlane(len, at) - (__builtin_amdgcn_readlane(c1, at) - tok);
    return __builtin_amdgcn_readlane(c0, at) <= tok;
}

}  // namespace la
