// Rotary positions: the first r dims of a head as r / 2 pairs, pair i of a token at
// position p turned by p freq_i, times a magnitude a.
//
//   (y1, y2) = a (x1 cos - x2 sin, x1 sin + x2 cos);   transposed: sin -> -sin
//
// Angles: freq_i / 2 pi is a binary fraction of a turn, 64 bits, so that its product
// with p is exact but for whole turns, which the multiplication drops; 32 bits of it
// (2^-32 turns) go on.  The nearest quarter turn comes off as an integer, and Taylor's
// polynomials of degree 9 and 10 take the rest (pi / 4 at most: the terms left out are
// below 2e-9).  An angle formed in fp32 would be off by 0.004 at position 100,000.
//
// A wave takes up to 192 pieces of one token's heads, three a lane, whose loads are in
// flight while its lanes work out the token's angles, one a lane, and hand them over
// through LDS: all heads share them.  Pieces are 16 bytes (two of them with pairs
// (i, i + r / 2)), at any alignment.  Where they do not divide a run of values, its last
// piece reaches back over what is before it and stores only what is its own (in place it may
// so read what another lane has turned already, and drops what it makes of it).
//
// Bound by memory: 32,768 tokens x 20 heads x 128 in bf16 66.2 us (335 MB, 5.1 TB/s).
// Small calls are bound by what a position takes: lengths, angle, product (64 tokens 4.5
// us).  Four to six pieces a lane were as fast or up to 8 % slower.
#pragma once
#include "attn_common.h"

namespace la {

struct RopeRows {
    const void *x;
    void *y;
    int64_t x_stride, y_stride;    // elements from one token to the next
    int32_t heads;
};

struct RopeArgs {
    RopeRows q, k;
    const uint64_t *turns;         // [r / 2]
    const int32_t *positions;      // [n_tokens], or NULL and
    const int32_t *cu, *kv_len;    // those of la_kv_write
    int64_t n_tokens, first_token;
    int32_t n_seqs, dim, rotary;
    int32_t pieces, turned;        // of a head, and those of them that are turned
    FastDiv by_pieces;
    int32_t items, share, splits;  // pieces of a token; of a wave, a multiple of 64; waves of a token
    float magnitude;
    bool transpose;
    bool whole;                    // pieces divide what is turned: none begins inside another's angles
};

constexpr int kRopeItems = 3;      // pieces of a lane
constexpr int kRopeTokens = 4;     // tokens of a workgroup, one for each wave
constexpr int kRopeDims = 512;     // largest r

// Place of angle i in LDS.  Pieces of eight angles lie 64 bytes apart, four of them on the
// same banks: eight bytes of padding behind each eight angles spread them (8,192 tokens x
// 20 heads of 256: 37 us, 43 without).  Pieces of four do better without (36 against 40).
template <int ANGLES> __device__ inline int angle_at(int i) { return ANGLES == 8 ? i + (i >> 3) : i; }

// cos and sin of t 2^-32 turns.
__device__ inline float2 cos_sin(uint32_t t) {
    const uint32_t quarter = (t + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(t - (quarter << 30)) * 1.4629180792671596e-9f;      // 2 pi 2^-32
    const float z = x * x;
    float s = __builtin_fmaf(z, 2.7557319224e-6f, -1.9841269841e-4f);                     // 1 / 9!, -1 / 7!
    s = __builtin_fmaf(z, s, 8.3333333333e-3f);
    s = __builtin_fmaf(z, s, -1.6666666667e-1f);
    s = __builtin_fmaf(x * z, s, x);
    float c = __builtin_fmaf(z, -2.7557319224e-7f, 2.4801587302e-5f);                     // -1 / 10!, 1 / 8!
    c = __builtin_fmaf(z, c, -1.3888888889e-3f);
    c = __builtin_fmaf(z, c, 4.1666666667e-2f);
    c = __builtin_fmaf(z, c, -0.5f);
    c = __builtin_fmaf(z, c, 1.f);
    const bool odd = quarter & 1;
    const float a = odd ? s : c, b = odd ? c : s;
    return make_float2((quarter + 1) & 2 ? -a : a, quarter & 2 ? -b : b);
}

#define LA_GLOBAL __attribute__((address_space(1)))

// 16 bytes of values, at any alignment of T.
template <typename T> struct Span {
    static constexpr int N = 16 / sizeof(T);
    typedef T vec __attribute__((ext_vector_type(N)));
    typedef vec loose __attribute__((aligned(sizeof(T))));
    typedef uint32_t two __attribute__((ext_vector_type(2)));
    typedef two loose2 __attribute__((aligned(2)));
    typedef uint32_t loose1 __attribute__((aligned(2)));
    typedef LA_GLOBAL T *Out;              // a flat store would wait for LDS as well
    vec v;
    __device__ inline void load(const T *p) { v = *(const loose *)p; }
    // The first n.
    __device__ inline void load_first(const T *p, int n) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = i < n ? p[i] : (T)0.f;
    }
    __device__ inline void store_first(Out p, int n) const {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n) p[i] = v[i];
    }
    // The last n, as 8, 4 and 2 bytes (fp32: 8 and 4) by the bits of n.
    __device__ inline void store_last(Out p, int n) const {
        if (n == N) {
            *(LA_GLOBAL loose *)p = v;
            return;
        }
        const uint4 w = __builtin_bit_cast(uint4, v);
        if constexpr (sizeof(T) == 2) {
            if (n & 4) *(LA_GLOBAL loose2 *)(p + 4) = two{w.z, w.w};
            if (n & 2) *(LA_GLOBAL loose1 *)(p + (n & 4 ? 2 : 6)) = n & 4 ? w.y : w.w;
            if (n & 1) *(LA_GLOBAL unsigned short *)(p + N - n) = (unsigned short)((n < 4 ? n < 2 ? w.w : w.z : n < 6 ? w.y : w.x) >> 16);
        } else {
            if (n & 2) *(LA_GLOBAL loose2 *)(p + 2) = two{w.z, w.w};
            if (n & 1) *(LA_GLOBAL uint32_t *)(p + N - n) = n < 2 ? w.w : w.y;
        }
    }
};

// SHORT: the values to turn (their half) are fewer than a piece has.
template <typename T, bool PAIRS, bool SHORT>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
    constexpr int N = Span<T>::N, ANGLES = PAIRS ? N / 2 : N;      // of a piece
    __shared__ float2 turn_sm[kRopeTokens][kRopeDims / 2 * 9 / 8];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // eight workgroups of a share side by side: an XCD (workgroup id mod 8) has as many of each
    const int set = (int)((blockIdx.x >> 3) / (uint32_t)a.splits), of = 8 * set + (int)(blockIdx.x & 7);
    const int64_t tok = a.first_token + (int64_t)of * kRopeTokens + wave;
    if (tok >= a.n_tokens) return;
    const int e0 = ((int)(blockIdx.x >> 3) - set * a.splits) * a.share, stop = min(a.items, e0 + a.share), half = a.rotary >> 1;

    Span<T> x[kRopeItems], x2[kRopeItems];
    typedef typename Span<T>::Out Out;
    Out to[kRopeItems];
    int at[kRopeItems], n[kRopeItems];                             // first angle (-1: a piece that is copied), values
#pragma unroll
    for (int i = 0; i < kRopeItems; ++i) {
        const int e = e0 + 64 * i + lane;
        n[i] = 0;
        if (e >= stop) continue;
        int head = a.by_pieces(e);
        const int j = e - head * a.pieces;
        const bool is_k = head >= a.q.heads;
        if (is_k) head -= a.q.heads;
        const T *px = (const T *)(is_k ? a.k.x : a.q.x) + tok * (is_k ? a.k.x_stride : a.q.x_stride) + (int64_t)head * a.dim;
        T *py = (T *)(is_k ? a.k.y : a.q.y) + tok * (is_k ? a.k.y_stride : a.q.y_stride) + (int64_t)head * a.dim;
        const bool turned = j < a.turned;
        const int end = turned ? (PAIRS ? a.rotary : half) : a.dim;
        int d = turned ? N * j : a.rotary + N * (j - a.turned);
        n[i] = min(N, end - d);
        if (!SHORT || !turned) d += n[i] - N;                      // the last piece reaches back over what is before it
        at[i] = turned ? d / (N / ANGLES) : -1;
        if (!turned && px == py) n[i] = 0;                         // in place: there already
        to[i] = (Out)(py + d);
        if (SHORT && turned) {
            x[i].load_first(px + d, n[i]);
            if (!PAIRS && turned) x2[i].load_first(px + half + d, n[i]);
        } else if (n[i] > 0) {
            x[i].load(px + d);
            if (!PAIRS && turned) x2[i].load(px + half + d);
        }
    }
    auto store = [&](const Span<T> &y, Out p, int count) {
        if constexpr (SHORT) y.store_first(p, count);
        else y.store_last(p, count);
    };

    const uint64_t turns0 = a.turns[min(lane, half - 1)];          // in flight beside what the position takes
    int pos;
    if (a.positions) {
        pos = a.positions[tok];
    } else {
        int seq;
        if (!position_of(a.cu, a.kv_len, a.n_seqs, (int)tok, &seq, &pos)) return;
    }
    for (int i = lane; i < half; i += 64) {
        const uint64_t turns = i < 64 ? turns0 : a.turns[i];
        float2 t = cos_sin((uint32_t)((uint64_t)(int64_t)pos * turns >> 32));
        t.x *= a.magnitude;
        t.y *= a.transpose ? -a.magnitude : a.magnitude;
        turn_sm[wave][angle_at<ANGLES>(i)] = t;
    }
    __builtin_amdgcn_wave_barrier();                               // a wave's LDS operations are in order

#pragma unroll
    for (int i = 0; i < kRopeItems; ++i) {
        if (n[i] <= 0) continue;
        if (at[i] < 0) {
            x[i].store_last(to[i], n[i]);
            continue;
        }
        float2 t[ANGLES];
#pragma unroll
        for (int k = 0; k < ANGLES; ++k) t[k] = turn_sm[wave][a.whole ? angle_at<ANGLES>(at[i]) + k : angle_at<ANGLES>(at[i] + k)];
        Span<T> y, y2;
#pragma unroll
        for (int k = 0; k < ANGLES; ++k) {
            const float u = (float)(PAIRS ? x[i].v[2 * k] : x[i].v[k]), w = (float)(PAIRS ? x[i].v[2 * k + 1] : x2[i].v[k]);
            const float s = __builtin_fmaf(u, t[k].x, -(w * t[k].y)), r = __builtin_fmaf(u, t[k].y, w * t[k].x);
            if constexpr (PAIRS) {
                y.v[2 * k] = (T)s;
                y.v[2 * k + 1] = (T)r;
            } else {
                y.v[k] = (T)s;
                y2.v[k] = (T)r;
            }
        }
        store(y, to[i], n[i]);
        if constexpr (!PAIRS) store(y2, to[i] + half, n[i]);
    }
}

}  // namespace la
