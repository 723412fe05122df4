// Causal attention of bf16 prompts: workgroups of 128 rows, four waves of 32, over
// 64-key tiles in LDS; two workgroups share a CU.
//
// 32x32x16 products: a K or V fragment that a wave reads from LDS serves 32 rows
// (16 a wave, as in attn_tile.h, is bound by LDS: 579 against 956 TFLOP/s for
// 32,768 tokens; 64 rows a wave leave one wave a SIMD, whose own exponentials
// then wait for its products: 860).
//
// A row's chain is scores -> maximum -> weights -> product with V.  A wave runs it
// as a pipeline of half tiles (32 keys): while the weights of half h are formed,
// the matrix unit computes the scores of half h + 1 and the product of half
// h - 1, none of which wait for one another.
//
// The exponent's reference m is not the running maximum but a value that it may
// pass by kLag: sums are scaled only when a row's maximum rises above that, which
// after the first tiles is rare.  Weights stay below 2^kLag, far inside bf16 and
// fp32.  The choice is each row's own: it depends on no other row.
#pragma once
#include "attn_tile.h"

namespace la {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kWideThreads = 256;
constexpr float kLag = 8.f;

// LDS: rows of 16-byte pieces; keys padded by one piece (the 16 rows of a piece
// fall on different banks), values by four (the 8 rows x 64 bytes of a
// fragment's transposed reads fall on every bank twice).
template <int D> struct WideLds {
    static constexpr int KT = 64, PPR = D / 8, KS = PPR + 1, VS = PPR + 4;
    uint4 k[2][KT * KS], v[2][KT * VS];
    int least[4], dropped;
};

// Maximum over the two lanes (l, l + 32) of a 32-column accumulator's row.
__device__ inline float half_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

template <typename C, int D, bool PAGED>
__device__ __forceinline__ void wide_run(const AttnArgs &a, const RowTile &t, WideLds<D> &sm) {
    using L = WideLds<D>;
    constexpr int KT = L::KT, PPR = L::PPR, RPL = 64 / PPR, LOADS = KT / (4 * RPL), KD = D / 16, MT32 = D / 32;
    constexpr int CB = 8 * sizeof(C), RB = D * sizeof(C);

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, hf = lane >> 5;
    const int32_t *table_row = PAGED ? a.kv.table + (int64_t)t.seq * a.kv.max_blocks : nullptr;
    const int64_t seq_row0 = PAGED ? 0 : t.tok0;
    const int lrow = lane / PPR, lp = lane % PPR;
    const uint32_t kvoff = (uint32_t)(lrow * (PAGED ? RB : (int)a.kv.k_stride) + lp * CB);
    const uint32_t vvoff = (uint32_t)(lrow * (PAGED ? RB : (int)a.kv.v_stride) + lp * CB);

    int kid[LOADS], vid[LOADS];                  // block ids of the next tiles to load
    auto look = [&](int t0, int (&ids)[LOADS]) {
        if constexpr (PAGED) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) ids[i] = block_of(a.kv, table_row, t0 + (4 * i + wave) * RPL, t.hi);
        }
    };
    Raw<C> fk[LOADS], fv[LOADS];
    auto load_k = [&](int t0) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            fk[i] = load_piece<C>(kv_rows<PAGED>(a.kv, PAGED ? kid[i] : 0, seq_row0, t.kvh, RB, t0 + (4 * i + wave) * RPL, RPL, t.hi).k, kvoff);
    };
    auto load_v = [&](int t0) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            fv[i] = load_piece<C>(kv_rows<PAGED>(a.kv, PAGED ? vid[i] : 0, seq_row0, t.kvh, RB, t0 + (4 * i + wave) * RPL, RPL, t.hi).v, vvoff);
    };
    look(t.lo, kid);
    load_k(t.lo);
    look(t.lo, vid);
    load_v(t.lo);
    look(t.lo + KT, kid);

    const int row = t.row0 + 32 * wave + col;
    const bool live = row < t.n_rows;
    const int limit = row_limit(a, t, row), edge = min(limit, t.hi);
    const int64_t tok = t.tok0 + (live ? row / a.group : 0);
    const int head = t.kvh * a.group + (live ? row % a.group : 0);
    bf16x8 qf[KD];
    {
        const __bf16 *qp = (const __bf16 *)a.q + tok * a.q_stride + (int64_t)head * D + 8 * hf;
#pragma unroll
        for (int k = 0; k < KD; ++k) qf[k] = __builtin_bit_cast(bf16x8, live ? *(const uint4 *)(qp + 16 * k) : make_uint4(0, 0, 0, 0));
    }
    int least = live ? limit : 0x7fffffff;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) least = min(least, __shfl_xor(least, d));
    if (lane == 0) sm.least[wave] = least;
    if (threadIdx.x == 0) sm.dropped = 0;
    __syncthreads();
    // the keys that every row of the workgroup sees
    const int all_see = __builtin_amdgcn_readfirstlane(min(min(sm.least[0], sm.least[1]), min(sm.least[2], sm.least[3])));

    auto store_k = [&](int b) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) sm.k[b][((4 * i + wave) * RPL + lrow) * L::KS + lp] = piece_of<C>(fk[i]);
    };
    auto store_v = [&](int b, bool mixed) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            uint4 v = piece_of<C>(fv[i]);
            if (mixed && drop_nonfinite<__bf16>(v)) sm.dropped = 1;
            sm.v[b][((4 * i + wave) * RPL + lrow) * L::VS + lp] = v;
        }
    };

    f32x16 acc[MT32];
    float m = -INFINITY, mu = 0.f, l = 0.f;
#pragma unroll
    for (int d = 0; d < MT32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;
    // scores of 32 keys: rows 32 half .. of the key tile in buffer b
    auto scores = [&](int b, int half, f32x16 &s) {
        const uint4 *kp = &sm.k[b][(32 * half + col) * L::KS + hf];
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int k = 0; k < KD; ++k) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kp[2 * k]), qf[k], s, 0, 0, 0);
    };
    // weights of the 32 keys from t0 on; returns what the row's sums so far shrink by
    auto weights = [&](int t0, bool masked, f32x16 &s, bf16x8 (&p)[2]) {
        if (masked) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (t0 + 8 * (i >> 2) + 4 * hf + (i & 3) >= edge) s[i] = -INFINITY;
        }
        float top = fmaxf(s[0], s[1]);
#pragma unroll
        for (int i = 2; i < 16; i += 2) top = fmaxf(fmaxf(top, s[i]), s[i + 1]);
        top = half_max(top) * a.c;
        float shrink = 1.f;
        if (top > m + kLag) {
            shrink = __builtin_amdgcn_exp2f(m - top);
            m = mu = top;
        }
        l *= shrink;
        float e[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], a.c, -mu));
            l += e[i];
        }
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) p[k][i] = (__bf16)e[8 * k + i];
        return shrink;
    };
    // sums += V^T P of 32 keys: rows 32 half .. of the value tile in buffer b
    auto product = [&](int b, int half, const bf16x8 (&p)[2]) {
        const char *vp = (const char *)&sm.v[b][(32 * half + 4 * hf + ((lane & 15) >> 2)) * L::VS] + 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int d = 0; d < MT32; ++d) {
                const char *x = vp + 16 * k * L::VS * 16 + 64 * d;
                acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(join_tr(lds_tr(x), lds_tr(x + 8 * L::VS * 16)), p[k], acc[d], 0, 0, 0);
            }
    };
    // The weights are complete before the sums shrink: without the empty statement
    // the compiler moves their exponentials behind the branch, away from the products.
    auto settle = [&](bf16x8 (&p)[2], float shrink) {
        __asm__ volatile("" : "+v"(p[0]), "+v"(p[1]), "+v"(l));
        if (__any(shrink != 1.f)) {
#pragma unroll
            for (int d = 0; d < MT32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[d][i] *= shrink;
        }
    };

    // Turn j takes key tile j + 1 and value tile j, both in LDS since the last
    // barrier, and brings in key tile j + 2 and value tile j + 1.  It begins with
    // the weights of half 2 j and the scores of half 2 j + 1.
    f32x16 s0, s1;
    bf16x8 p0[2], p1[2];
    store_k(0);
    store_v(0, t.lo + KT > all_see);
    load_k(t.lo + KT);
    look(t.lo + KT, vid);
    look(t.lo + 2 * KT, kid);
    __syncthreads();
    scores(0, 0, s0);
    scores(0, 1, s1);
    (void)weights(t.lo, true, s0, p0);           // sums are still zero
    store_k(1);
    __syncthreads();
    int b = 0;
    auto turn = [&](int t0, bool masked) {
        load_k(t0 + 2 * KT);
        load_v(t0 + KT);
        look(t0 + 3 * KT, kid);
        look(t0 + 2 * KT, vid);
        scores(b ^ 1, 0, s0);
        float shrink = weights(t0 + 32, masked, s1, p1);
        product(b, 0, p0);
        settle(p1, shrink);
        scores(b ^ 1, 1, s1);
        shrink = weights(t0 + KT, masked, s0, p0);
        product(b, 1, p1);
        settle(p0, shrink);
        store_k(b);
        store_v(b ^ 1, t0 + 2 * KT > all_see);
        __syncthreads();
        b ^= 1;
    };
    int t0 = t.lo;
    for (; t0 + 2 * KT <= min(all_see, t.hi); t0 += KT) turn(t0, false);
    for (; t0 < t.hi; t0 += KT) turn(t0, true);

    if (!live) return;
    l += __shfl_xor(l, 32);
    if (sm.dropped) {
        const int first = all_see <= t.lo ? t.lo : t.lo + (all_see - t.lo) / KT * KT;
#pragma unroll
        for (int d = 0; d < MT32; ++d)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                f32x4 y = {acc[d][4 * q], acc[d][4 * q + 1], acc[d][4 * q + 2], acc[d][4 * q + 3]};
                add_nonfinite<C, D, PAGED>(a, table_row, seq_row0, t.kvh, first, t.hi, limit, 32 * d + 8 * q + 4 * hf, y);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[d][4 * q + i] = y[i];
            }
    }
    const bool whole = t.n_parts == 1;
    if (!whole && limit <= t.lo) return;
    const float x = row_scale(a, l);
    const int64_t slot = t.slot0 + ((tok - t.tok0) * (a.kv_heads * a.group) + head) * t.slot_parts + t.part;
    __bf16 *op = (__bf16 *)a.o + tok * a.o_stride + (int64_t)head * D + 4 * hf;
    float *pp = a.part_o + slot * D + 4 * hf;
#pragma unroll
    for (int d = 0; d < MT32; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const f32x4 y = {acc[d][4 * q], acc[d][4 * q + 1], acc[d][4 * q + 2], acc[d][4 * q + 3]};
            if (whole) store4(op + 32 * d + 8 * q, y * x);
            else store4(pp + 32 * d + 8 * q, y);
        }
    if (!whole && hf == 0) a.part_ml[slot] = make_float2(m, l);
}

template <typename C, int D, bool PAGED>
__global__ __launch_bounds__(kWideThreads, 2) void attn_wide_kernel(AttnArgs a) {
    __shared__ WideLds<D> sm;
    RowTile t;
    if (prompt_tile_of<kPromptRows>(a, blockIdx.x, &t)) wide_run<C, D, PAGED>(a, t, sm);
}

}  // namespace la
