// New keys and values into a cache of 8-bit codes with a scale for each block and key
// head, and cached rows of any type back out.
//
// A unit is the keys, or the values, of one head in one block: bt x d codes, and a scale
// s of its own in the block.  The tokens that a call writes into it, of largest
// magnitude A, ask for
//
//   e4m3  the smallest 2^e with A <= 448 2^e: a float's relative precision is the same at
//         every power of two, so none is lost, and codes move to a larger scale exactly
//         (those that fall below the smallest normal apart)
//   int8  A / 127, rounded up to 8 significant bits
//
// and at least 2^-100.  Tokens that stay before them in the block keep its scale from
// shrinking, and follow it when it grows: code s_old / s, to nearest even.  With 8 bits
// in s and in a bf16 value (15 in code s_old), a quotient is a tie or at least 2^-17 of
// it away from one, so that one division, whoever does it, has one answer.
//
// Both kernels are bound by memory once they are large: 47,248 tokens x 8 heads x 128 as
// e4m3 59.7 us (290 MB, 4.9 TB/s), 32,768 x 4 x 128 into int8 blocks of 64 21.2 (4.7);
// 77,472 x 8 x 128 int8 back in bf16 94.9 (5.0).  Small calls are a chain of loads:
// lengths, table, scale (64 tokens 4.5 us).
#pragma once
#include "blocks.h"

namespace la {

constexpr float kLeastScale = 0x1p-100f;
constexpr uint32_t kLargestBf16 = 0x7F00;          // 2^127: what lies beyond is written as this, so that code s is finite

template <typename C> __device__ inline float scale_of(float most) {
    const uint32_t u = __float_as_uint(most);
    float s;
    if constexpr (kScaleCodes<C>) {
        // 448 = 1.75 2^8
        const int e = (int)(u >> 23) - 8 + ((u & 0x7FFFFF) > 0x600000);
        s = e > 0 ? __uint_as_float((uint32_t)e << 23) : 0.f;
    } else {
        s = __uint_as_float((__float_as_uint(most / 127.f) + 0xFFFFu) & 0xFFFF0000u);
    }
    return fmaxf(s, kLeastScale);
}

// A scale that a block holds; what no write can have left there counts as the least.  The
// largest that one can is that of 2^127: past it (a stray scale in a block that is used
// again) ordinary tokens would all become code 0.
template <typename C> __device__ inline float held_scale(float s) {
    const float t = __uint_as_float(__float_as_uint(s) & (kScaleCodes<C> ? 0xFF800000u : 0xFFFF0000u));
    return s == t && s >= kLeastScale && s <= scale_of<C>(__uint_as_float(kLargestBf16 << 16)) ? s : kLeastScale;
}

// x / s correctly rounded where the quotient has few bits (a tie), by r = 1 / s: the
// product's error, and one step against it.
__device__ inline float quotient(float x, float r, float s) {
    const float t = x * r;
    return __builtin_fmaf(__builtin_fmaf(-t, s, x), r, t);
}

// Four quotients of at most 448 (127) to codes.
template <typename C> __device__ inline uint32_t codes_of4(const float *y) {
    if constexpr (kScaleCodes<C>) {
        const int r = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], r, true);
    } else {
        uint32_t b[4];                              // 1.5 2^23 + y: the sum rounds, its low byte is the integer
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = __float_as_uint(y[i] + 0x1.8p23f) & 0xFFu;
        return b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24;
    }
}

// Eight bf16 values over s.  ODD: there may be infinities, values beyond 2^127 and NaN.
template <typename C, bool ODD> __device__ inline uint2 codes_of8(const uint4 &raw, float r, float s) {
    const uint32_t *w = &raw.x;
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float x = __uint_as_float((i & 1) ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
        if constexpr (ODD) {
            if (x == x) x = fminf(fmaxf(x, -0x1p127f), 0x1p127f);
            else if (!kScaleCodes<C>) x = 0.f;
        }
        y[i] = kScaleCodes<C> ? x * r : quotient(x, r, s);
    }
    return make_uint2(codes_of4<C>(y), codes_of4<C>(y + 4));
}

// Four codes of scale s_old over s.
template <typename C> __device__ inline uint32_t move4(uint32_t x, float s_old, float r, float s) {
    float y[4];
    if constexpr (kScaleCodes<C>) {
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(x, true);
        const float f = s_old * r;                  // powers of two
        y[0] = a[0] * f, y[1] = a[1] * f, y[2] = b[0] * f, y[3] = b[1] * f;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = quotient((float)(int8_t)(x >> 8 * i) * s_old, r, s);
    }
    return codes_of4<C>(y);
}

// The largest bf16 magnitude of four words, as bits in both halves.
__device__ inline uint32_t most_of(uint32_t m, const uint4 &x) {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    const uint32_t *w = &x.x;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, m), __builtin_bit_cast(u16x2, w[i] & 0x7FFF7FFFu)));
    return m;
}

// The same without NaN, cut at 2^127.
__device__ inline uint32_t most_finite_of(uint32_t m, const uint4 &x) {
    const uint32_t *w = &x.x;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t h = (i & 1 ? w[i / 2] >> 16 : w[i / 2]) & 0x7FFFu;
        if (h <= 0x7F80u) m = max(m, min(h, kLargestBf16));
    }
    return m;
}

// Maximum over the wave of both halves.
__device__ inline uint32_t wave_most(uint32_t m) {
    uint32_t x = max(m & 0xFFFFu, m >> 16);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) x = max(x, (uint32_t)__shfl_xor((int)x, d));
    return x;
}

// Workgroups of four waves take units of one block that the call writes into, one or four
// waves a unit, each with P pieces of 8 values a lane in registers, so that values are
// read once and a block's scale is known before any of its codes is formed.
//
// Sequence i's blocks have numbers from cu[i] / bt + 2 i on, so that a workgroup finds
// its own without a sum over the sequences before it: n tokens lie in at most n / bt + 2
// blocks.
__device__ inline bool spot_of(const KvWriteArgs &a, int64_t w, int *seq, int *c0, int *c1, int *len, int64_t *nth) {
    auto first_of = [&](int i) { return (int64_t)(max(a.cu[i], 0) >> a.bt_shift) + 2 * (int64_t)i; };
    const int i0 = narrow_to_64(a.n_seqs, [&](int i) { return first_of(i + 1) > w; });
    const int i = min(i0 + (int)(threadIdx.x & 63), a.n_seqs - 1);
    const int b0 = max(a.cu[i], 0), b1 = max(a.cu[i + 1], 0), n = a.kv_len[i];       // lengths beside the offsets
    const uint64_t past = __ballot((b1 >> a.bt_shift) + 2 * (int64_t)(i + 1) > w);
    if (!past) return false;
    const int l = __builtin_ctzll(past);
    *seq = i0 + l;
    *c0 = __builtin_amdgcn_readlane(b0, l);
    *c1 = __builtin_amdgcn_readlane(b1, l);
    *len = __builtin_amdgcn_readlane(n, l);
    *nth = w - (*c0 >> a.bt_shift) - 2 * (int64_t)*seq;
    return *nth >= 0 && *c1 > *c0;
}

struct KvCodesArgs {
    KvWriteArgs w;
    int64_t first_group;           // the launch's first workgroup
    int32_t team_shift;            // waves of a unit, as a power of two
    int32_t unit_groups;           // workgroups of one block
};

template <typename C, int D, int P>
__global__ __launch_bounds__(256) void kv_write_codes_kernel(KvCodesArgs args) {
    const KvWriteArgs &a = args.w;
    constexpr int V = D / 8;
    __shared__ uint32_t most_sm[4];
    __shared__ float old_sm[4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t group = args.first_group + blockIdx.x, w = group / args.unit_groups;
    const int ug = (int)(group - w * args.unit_groups);
    int seq, c0, c1, keys;
    int64_t nth;
    if (!spot_of(a, w, &seq, &c0, &c1, &keys, &nth)) return;
    const int64_t len = keys, p0 = len - (c1 - c0), j = (p0 >> a.bt_shift) + nth, base = j * (1 << a.bt_shift);
    if (base >= len) return;
    const int id = j >= 0 && j < a.max_blocks ? a.table[seq * a.max_blocks + j] : -1;
    if ((uint32_t)id >= (uint32_t)a.n_blocks) {
        if (threadIdx.x == 0 && ug == 0 && a.err) atomicAdd(a.err, 1);
        return;
    }
    // rows [a0, a1) of the block are written, those before a0 stay
    const int64_t tok0 = c0 + (base - p0);                     // token of row 0
    const int bt = 1 << a.bt_shift, a0 = (int)max(p0 - base, (int64_t)0);
    const int a1 = (int)min(min(len - base, (int64_t)bt), a.n_tokens - tok0);
    if (a1 <= a0) return;                                      // offsets past the call's rows
    const int team = 1 << args.team_shift, tw = wave & (team - 1), unit = (ug << (2 - args.team_shift)) + (wave >> args.team_shift);
    const bool live = unit < 2 * a.kv_heads;
    const int h = live ? unit >> 1 : 0;
    const bool is_v = unit & 1;
    const char *src = (const char *)(is_v ? a.v : a.k) + ((is_v ? a.v_stride : a.k_stride) * tok0 + (int64_t)h * D) * 2;
    const int64_t stride = 2 * (is_v ? a.v_stride : a.k_stride);
    const int64_t block = (int64_t)id * a.block_bytes;
    float *const scale_at = (float *)((is_v ? a.vs : a.ks) + block) + h;
    char *const codes = (is_v ? a.cv : a.ck) + block + ((int64_t)h << a.bt_shift) * D;

    const int piece = lane % V * 8;
    auto row_of = [&](int i) { return ((tw * P + i) * 64 + lane) / V; };
    uint4 raw[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int row = row_of(i);
        raw[i] = make_uint4(0, 0, 0, 0);
        if (live && row >= a0 && row < a1) raw[i] = *(const uint4 *)(src + row * stride + piece * 2);
    }
    float old = kLeastScale;
    if (live && a0 > 0 && tw == 0) old = held_scale<C>(*scale_at);
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < P; ++i) m = most_of(m, raw[i]);
    uint32_t most = wave_most(m);
    // The waves of a unit agree on its magnitude; its old scale is read by one, before
    // another may have written the new.
    auto agree = [&]() {
        if (team == 1) return;
        __syncthreads();
        if (lane == 0) {
            most_sm[wave] = most;
            if (tw == 0) old_sm[wave] = old;
        }
        __syncthreads();
        for (int i = 0; i < team; ++i) most = max(most, most_sm[wave - tw + i]);
        old = old_sm[wave - tw];
    };
    agree();
    const bool odd = __builtin_amdgcn_readfirstlane((int)(most > kLargestBf16));      // of a unit: not the same for the workgroup
    bool nan = false;
    if (odd) {
        nan = most > 0x7F80u;
        m = 0;
#pragma unroll
        for (int i = 0; i < P; ++i) m = most_finite_of(m, raw[i]);
        most = wave_most(m);
    }
    agree();                                                   // once more for all, since its barrier is the workgroup's
    float s = scale_of<C>(__uint_as_float(most << 16));
    if (a0 > 0) s = fmaxf(s, old);
    const float r = 1.f / s;
    if (!live) return;
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int row = row_of(i);
        if (row >= a0 && row < a1) {
            const uint2 x = odd ? codes_of8<C, true>(raw[i], r, s) : codes_of8<C, false>(raw[i], r, s);
            *(uint2 *)(codes + row * D + piece) = x;
        }
    }
    if (s > old && a0 > 0) {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int row = row_of(i);
            if (row < a0) {
                const uint2 x = *(const uint2 *)(codes + row * D + piece);
                *(uint2 *)(codes + row * D + piece) = make_uint2(move4<C>(x.x, old, r, s), move4<C>(x.y, old, r, s));
            }
        }
    }
    if (tw == 0 && lane == 0) {
        *scale_at = s;
        if (nan && !kScaleCodes<C> && a.err) atomicAdd(a.err, 1);
    }
}

// --- cached rows back out ----------------------------------------------------

struct KvReadArgs {
    KvWriteArgs w;
    int32_t lanes;                 // of a token, four pieces each (64: a wave takes one token, 256 pieces a turn)
    FastDiv by_lanes;
};

// Products f of eight e4m3 codes and a layer's scale, on their way to bf16.  The scale has 24
// bits, so that fp32 has rounded them and bf16 would again: where the first rounding made a
// tie between two bf16 values, a step of fp32 takes the product back to the side that it is
// on, and the second rounding alone counts (else 6 products of a million come out wrong).
// fp64 holds the product.  One branch for all eight: one for each took 4 % of the call.
__device__ inline void take_off_ties(float (&f)[8], const uint32_t *w, float s) {
    bool tie = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) tie |= (__float_as_uint(f[i]) & 0xFFFF) == 0x8000;
    if (!tie) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint2 b = bf16_of4<fp8_t>(w[i / 4]);
        const uint32_t h = i & 2 ? b.y : b.x;
        const double x = __uint_as_float(i & 1 ? h & 0xFFFF0000u : h << 16), rest = fabs(x * s) - fabs((double)f[i]);
        uint32_t u = __float_as_uint(f[i]);
        if ((u & 0xFFFF) == 0x8000) u += rest > 0.0 ? 1 : rest < 0.0 ? -1 : 0;
        f[i] = __uint_as_float(u);
    }
}

// A wave takes as many tokens as fill it, four 16-byte pieces of the result a lane: with
// one token a wave, few or short heads left most lanes without work (8 heads of 64: 1.3
// times the time that a copy takes).
template <typename T, typename C, int D>
__global__ __launch_bounds__(256) void kv_read_kernel(KvReadArgs args) {
    const KvWriteArgs &a = args.w;
    constexpr int N = 16 / sizeof(T), V = D / N, R = 4;        // values of a piece, pieces of a row, pieces of a lane
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int group = args.by_lanes(lane), per_wave = args.by_lanes(64);
    const int64_t first = a.first_token + ((int64_t)blockIdx.x * kWriteTokens + wave) * per_wave, tok = first + group;
    if (first >= a.n_tokens) return;
    // the wave's first token's sequence, then those of the others, in the same 64 or behind them
    const bool mine = group < per_wave && tok < a.n_tokens;
    int i0 = narrow_to_64(a.n_seqs, [&](int i) { return a.cu[i + 1] > first; });
    int i = min(i0 + lane, a.n_seqs - 1), c0 = a.cu[i], c1 = a.cu[i + 1], len = a.kv_len[i], seq = -1, pos = 0;
    bool in = false;
    for (uint64_t left = __ballot(mine); left;) {
        const int t = __builtin_amdgcn_readlane((int)tok, __builtin_ctzll(left));
        const uint64_t past = __ballot(c1 > t);
        if (!past) {
            if ((i0 += 64) >= a.n_seqs) break;
            i = min(i0 + lane, a.n_seqs - 1);
            c0 = a.cu[i];
            c1 = a.cu[i + 1];
            len = a.kv_len[i];
            continue;
        }
        const int at = __builtin_ctzll(past), end = __builtin_amdgcn_readlane(c1, at);
        if (mine && seq < 0 && (int)tok < end) {
            seq = i0 + at;
            pos = __builtin_amdgcn_readlane(len, at) - (end - (int)tok);
            in = (int)tok >= __builtin_amdgcn_readlane(c0, at);
        }
        left = __ballot(mine && seq < 0);
    }
    if (!in) return;
    const int64_t j = pos >> a.bt_shift;
    int id = pos >= 0 && j < a.max_blocks ? a.table[seq * a.max_blocks + j] : -1;
    const bool named = (uint32_t)id < (uint32_t)a.n_blocks;
    const int l = lane - group * args.lanes, pieces = 2 * a.kv_heads * V;
    if (!named) {
        if (l == 0 && a.err) atomicAdd(a.err, 1);
        id = 0;
    }
    const int slot = pos & ((1 << a.bt_shift) - 1);
    const int64_t block = (int64_t)id * a.block_bytes;
    typedef typename std::conditional<N * sizeof(C) == 16, uint4, typename std::conditional<N * sizeof(C) == 8, uint2, uint32_t>::type>::type Raw;
    for (int e0 = l; e0 < pieces; e0 += R * args.lanes) {
        Raw raw[R];
        float s[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int e = min(e0 + i * args.lanes, pieces - 1);
            const bool is_v = e >= a.kv_heads * V;
            const int x = is_v ? e - a.kv_heads * V : e, h = x / V, p = x % V;
            raw[i] = *(const Raw *)((is_v ? a.cv : a.ck) + block + (((int64_t)h << a.bt_shift) + slot) * (int64_t)(D * sizeof(C)) +
                                    p * (int)(N * sizeof(C)));
            s[i] = 1.f;
            if constexpr (kBlockScaled<C>) s[i] = *((const float *)((is_v ? a.vs : a.ks) + block) + h);
            else if constexpr (sizeof(C) == 1) s[i] = is_v ? a.v_scale : a.k_scale;
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int e = e0 + i * args.lanes;
            if (e >= pieces) break;
            const bool is_v = e >= a.kv_heads * V;
            T *dst = (is_v ? (T *)a.v : (T *)a.k) + tok * (is_v ? a.v_stride : a.k_stride) + (is_v ? e - a.kv_heads * V : e) * N;
            if constexpr (sizeof(C) == sizeof(T)) {                 // as it stands
                *(uint4 *)dst = named ? raw[i] : make_uint4(0, 0, 0, 0);
                continue;
            }
            const uint32_t *w = (const uint32_t *)&raw[i];
            float f[N];
#pragma unroll
            for (int v = 0; v < N; v += 4) {
                uint2 b{};                                          // four values in bf16, exact
                if constexpr (sizeof(C) == 1) b = bf16_of4<C>(w[v / 4]);
                else if constexpr (sizeof(C) == 2) b = make_uint2(w[v / 2], w[v / 2 + 1]);
                f[v] = __uint_as_float(b.x << 16) * s[i];
                f[v + 1] = __uint_as_float(b.x & 0xFFFF0000u) * s[i];
                f[v + 2] = __uint_as_float(b.y << 16) * s[i];
                f[v + 3] = __uint_as_float(b.y & 0xFFFF0000u) * s[i];
            }
            if constexpr (std::is_same<C, fp8_t>::value && sizeof(T) == 2) take_off_ties(f, w, s[i]);
#pragma unroll
            for (int v = 0; v < N; ++v)
                if (!named) f[v] = 0.f;
            if constexpr (sizeof(T) == 2) *(bf16x8 *)dst = pack8(f32x4{f[0], f[1], f[2], f[3]}, f32x4{f[4], f[5], f[6], f[7]});
            else store4(dst, f32x4{f[0], f[1], f[2], f[3]});
        }
    }
}

}  // namespace la
