// Attention of single tokens over a cache, and the joining of parts.
//
// attn_rows_kernel: a workgroup takes one part of the keys that a sequence has
// to itself, for up to 16 query heads of one key head.  Every key and value is
// used once by one wave, so nothing is shared: each of the eight waves takes
// key tiles of its own, K goes from memory straight into the registers that the
// product reads, V through LDS of the wave's own (its fragments are columns),
// and the waves' m, l and sums meet at the end.
#pragma once
#include "attn_tile.h"

namespace la {

constexpr int kRowsThreads = 512;
constexpr int kRowsWaves = kRowsThreads / 64;
constexpr int kRowsHeads = 16;

// Keys of a wave's tile, and one tile of V in LDS (vpos as the row tiles').
template <typename T, int D> struct RowsTile {
    static constexpr int KT = sizeof(T) == 2 ? 32 : 16;
    static constexpr int PPR = D / Piece<T>::N;
};

// Own keys of sequence s of a decode call: [*first, *end); and the parts its prefix has.
__device__ inline void own_keys(const AttnArgs &a, int s, bool count, int *first, int *end, int *prefix_parts) {
    const int n = a.kv_len[s];
    if (count && n > a.max_kv && a.kv.err) atomicAdd(a.kv.err, 1);
    *end = max(0, min(n, a.max_kv));
    *first = 0;
    *prefix_parts = 0;
    if (!a.cu_group) return;
    const int lane = threadIdx.x & 63;
    int g = 0;
    for (int i0 = 0; i0 < a.n_groups; i0 += 64) {      // groups that begin at or before s
        const int i = i0 + lane;
        g += __popcll(__ballot(i < a.n_groups && a.cu_group[i] <= s));
    }
    if (g == 0) return;
    g = __builtin_amdgcn_readfirstlane(g - 1);
    const int s1 = a.cu_group[g + 1];
    if (s >= s1) return;
    const int shared = min(group_prefix(a, g, s1 - a.cu_group[g]), *end);
    *first = shared;
    *prefix_parts = (shared + a.prefix_part_tokens - 1) / a.prefix_part_tokens;
}

// Parts of own keys [first, end): they begin at the 16-token line at or before first.
__device__ inline int own_parts(const AttnArgs &a, int first, int end) {
    return end <= first ? 0 : (end - (first & ~15) + a.part_tokens - 1) / a.part_tokens;
}

template <typename T, typename C, int D>
__global__ __launch_bounds__(kRowsThreads) void attn_rows_kernel(AttnArgs a, bool direct) {
    using L = AttnTile<T, D>;
    using M = MT<T>;
    constexpr int KT = RowsTile<T, D>::KT, PPR = RowsTile<T, D>::PPR, NT = KT / 16, DT = D / 16;
    constexpr int NQ = sizeof(T) == 2 ? D / 32 : D / 16;
    constexpr int RPL = 64 / PPR, VL = KT / RPL;               // V rows a load, loads of a tile
    constexpr int RB = D * sizeof(C), CB = Piece<T>::N * sizeof(C);
    constexpr int VBYTES = kRowsWaves * KT * PPR * 16, OBYTES = kRowsWaves * kRowsHeads * D * 4;
    __shared__ uint4 smem[(VBYTES > OBYTES ? VBYTES : OBYTES) / 16];
    __shared__ float2 wml[kRowsWaves][kRowsHeads];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    // key head fastest, then the row tiles of a wide group, the part, the sequence
    uint32_t r = blockIdx.x;
    const int kvh = (int)(r % (uint32_t)a.kv_heads);
    r /= (uint32_t)a.kv_heads;
    const int tiles = (a.group + kRowsHeads - 1) / kRowsHeads;
    const int h0 = (int)(r % (uint32_t)tiles) * kRowsHeads;
    r /= (uint32_t)tiles;
    const int own_max = a.parts - a.prefix_parts;
    const int part = (int)(r % (uint32_t)own_max), seq = (int)(r / (uint32_t)own_max);
    int first, end, pp;
    own_keys(a, seq, part == 0 && kvh == 0 && h0 == 0 && threadIdx.x == 0, &first, &end, &pp);
    const int lo = (first & ~15) + part * a.part_tokens;
    const int hi = min(end, lo + a.part_tokens);
    if (lo >= hi && !(direct && part == 0)) return;
    const bool live = h0 + col < a.group;
    const int head = kvh * a.group + h0 + (live ? col : 0);
    const int32_t *table_row = a.kv.table + (int64_t)seq * a.kv.max_blocks;

    uint4 qf[NQ];
    {
        const T *qp = (const T *)a.q + seq * a.q_stride + (int64_t)head * D;
#pragma unroll
        for (int s = 0; s < NQ; ++s) qf[s] = live ? *(const uint4 *)(qp + (4 * s + g) * Piece<T>::N) : make_uint4(0, 0, 0, 0);
    }
    f32x4 acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = zero4();
    float m = -INFINITY, l = 0.f;
    uint4 *vt = smem + wave * KT * PPR;
    for (int t0 = lo + wave * KT; t0 < hi; t0 += kRowsWaves * KT) {
        Raw<C> kr[NT][NQ], vr[VL];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const auto res = kv_rows<true>(a.kv, 0, table_row, 0, kvh, RB, t0 + 16 * n, 16, hi);
#pragma unroll
            for (int k = 0; k < NQ; ++k) kr[n][k] = load_piece<C>(res, (uint32_t)(col * RB + (4 * k + g) * CB));
        }
#pragma unroll
        for (int i = 0; i < VL; ++i) {
            const auto res = kv_rows<true>(a.kv, 1, table_row, 0, kvh, RB, t0 + RPL * i, RPL, hi);
            vr[i] = load_piece<C>(res, (uint32_t)((lane / PPR) * RB + (lane % PPR) * CB));
        }
        f32x4 s[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            s[n] = zero4();
#pragma unroll
            for (int k = 0; k < NQ; ++k) {
                const uint4 kf = piece_of<C>(kr[n][k]);
                if constexpr (sizeof(T) == 2) {
                    s[n] = M::mma(__builtin_bit_cast(bf16x8, kf), __builtin_bit_cast(bf16x8, qf[k]), s[n]);
                } else {
                    const float *x = (const float *)&kf, *y = (const float *)&qf[k];
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[n] = M::mma(x[e], y[e], s[n]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < VL; ++i) vt[L::vpos(RPL * i + lane / PPR, lane % PPR)] = piece_of<C>(vr[i]);
        const bool masked = t0 < first || t0 + KT > hi;
        float top = -INFINITY;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float x = s[n][i] * a.c;
                const int tok = t0 + 16 * n + 4 * g + i;
                if (masked && (tok < first || tok >= hi)) x = -INFINITY;
                s[n][i] = x;
                top = fmaxf(top, x);
            }
        const float m2 = fmaxf(m, row_max16(top));
        const float mu = m2 == -INFINITY ? 0.f : m2;
        const float shrink = __builtin_amdgcn_exp2f(m - mu);
        m = m2;
        l *= shrink;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[n][i] = __builtin_amdgcn_exp2f(s[n][i] - mu);
                l += s[n][i];
            }
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[d][i] *= shrink;
        const char *vb = (const char *)vt;
        if constexpr (sizeof(T) == 2) {
            const bf16x8 p = pack8(s[0], s[1]);
            const int vr0 = 4 * g + (col >> 2);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const int pc = 2 * d + ((col & 3) >> 1), half = 8 * (col & 1);
                acc[d] = M::mma(join_tr(lds_tr(vb + L::vpos(vr0, pc) * 16 + half), lds_tr(vb + L::vpos(vr0 + 16, pc) * 16 + half)),
                                p, acc[d]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int d = 0; d < DT; ++d)
                    acc[d] = M::mma(*(const float *)(vb + L::vpos(4 * g + i, 4 * d + (col >> 2)) * 16 + 4 * (col & 3)), s[0][i],
                                    acc[d]);
        }
    }
    // the waves' results: every wave scales its sums to the common maximum
    l = row_sum16(l);
    if (g == 0) wml[wave][col] = make_float2(m, l);
    __syncthreads();
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kRowsWaves; ++w) top = fmaxf(top, wml[w][col].x);
    const float mu = top == -INFINITY ? 0.f : top;
    const float scale = __builtin_amdgcn_exp2f(m - mu);
    float *so = (float *)smem;                                  // [wave][head][D], V no longer needed
#pragma unroll
    for (int d = 0; d < DT; ++d) *(f32x4 *)&so[(wave * kRowsHeads + col) * D + 16 * d + 4 * g] = acc[d] * scale;
    __syncthreads();
    for (int e = threadIdx.x; e < kRowsHeads * D / 4; e += kRowsThreads) {
        const int h = e / (D / 4), d = e % (D / 4) * 4;
        if (h0 + h >= a.group) continue;
        f32x4 x = zero4();
        float lt = 0.f, mt = -INFINITY;
#pragma unroll
        for (int w = 0; w < kRowsWaves; ++w) mt = fmaxf(mt, wml[w][h].x);
        const float mh = mt == -INFINITY ? 0.f : mt;
#pragma unroll
        for (int w = 0; w < kRowsWaves; ++w) {
            x += *(const f32x4 *)&so[(w * kRowsHeads + h) * D + d];
            lt += wml[w][h].y * __builtin_amdgcn_exp2f(wml[w][h].x - mh);
        }
        const int64_t row = (int64_t)seq * a.kv_heads * a.group + kvh * a.group + h0 + h;
        if (direct) {
            const float inv = lt > 0.f || lt != lt ? a.v_scale / lt : 0.f;
            store4((T *)a.o + seq * a.o_stride + (int64_t)(kvh * a.group + h0 + h) * D + d, x * inv);
        } else {
            const int64_t slot = row * a.parts + pp + part;
            store4(a.part_o + slot * D + d, x);
            if (d == 0) a.part_ml[slot] = make_float2(mt, lt);
        }
    }
}

// Joins the parts of every row that has them: a wave a row.  Lane p holds part
// p's weight (64 parts a step); D / 64 sums each.
template <typename T, int D>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a, int64_t n_rows) {
    constexpr int E = D / 64;
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (row >= n_rows) return;
    const int heads = a.kv_heads * a.group;
    const int64_t tok = row / heads;
    const int head = (int)(row - tok * heads);
    int n;
    if (a.cu) {
        int seq, local;
        if (!item_of(a.n_seqs, (int)tok, [&](int i) { return a.cu[i + 1] - a.cu[i]; }, &seq, &local)) return;
        const int new_tokens = a.cu[seq + 1] - a.cu[seq], rows = new_tokens * a.group, keys = prompt_keys(a, seq);
        if (prompt_parts(rows, keys) == 1) return;             // written by its tile
        const int limit = max(0, min(keys, keys - new_tokens + local + 1)), pt = prompt_part_tokens(rows, keys);
        n = (limit + pt - 1) / pt;
    } else {
        int first, end, pp;
        own_keys(a, (int)tok, false, &first, &end, &pp);
        n = pp + own_parts(a, first, end);
    }
    const float2 *ml = a.part_ml + row * a.parts;
    const float *po = a.part_o + row * a.parts * D;
    float m = -INFINITY, l = 0.f, x[E];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = 0.f;
    for (int p0 = 0; p0 < n; p0 += 64) {
        const float2 y = p0 + lane < n ? ml[p0 + lane] : make_float2(-INFINITY, 0.f);
        float top = y.x;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
        const float m2 = fmaxf(m, top), mu = m2 == -INFINITY ? 0.f : m2;
        const float shrink = __builtin_amdgcn_exp2f(m - mu);
        const float w = __builtin_amdgcn_exp2f(y.x - mu);
        m = m2;
        l *= shrink;
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] *= shrink;
        l += w * y.y;                                            // this lane's part
        const int most = min(64, n - p0);
        for (int p = 0; p < most; ++p) {
            const float wp = __shfl(w, p);
            const float *src = po + (int64_t)(p0 + p) * D + lane * E;
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] += wp * src[e];
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) l += __shfl_xor(l, d);
    const float inv = l > 0.f || l != l ? a.v_scale / l : 0.f;
    T *op = (T *)a.o + tok * a.o_stride + (int64_t)head * D + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) op[e] = from_f32<T>(x[e] * inv);
}

}  // namespace la
