// Attention of 128-row tiles in bf16, four waves of 32 rows, over 64-key tiles in
// LDS; two workgroups share a CU.  Prompts, and the shared prefix of decode groups.
//
// 32x32x16 products: a K or V fragment that a wave reads from LDS serves 32 rows
// (16 a wave, as in attn_tile.h, is bound by LDS: 579 against 956 TFLOP/s for
// 32,768 tokens; 64 rows a wave leave one wave a SIMD, whose own exponentials
// then wait for its products: 860).  As it stands the kernel takes that prompt at
// 1,025 to 1,048 TFLOP/s, from card to card (a product of 8,192 x 8,192 x 8,192:
// 1,177 to 1,200), the suffixes of 16 prompts over an 8-bit cache at 893 to 923 and
// over a bf16 one at 882 to 896.
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
    union {
        struct {
            uint4 k[2][KT * KS], v[2][KT * VS];
        };
        float out[4][32][D + 4];                 // results on their way out; the padding puts 8 rows on different banks
    };
    int64_t where[4][32];                        // and where their rows go, in elements (-1: nowhere)
    int dropped;
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
    using Loads = KvLoads<C, PAGED, 4, RPL, LOADS, RB>;
    Loads ld{table_row, seq_row0, t.kvh, t.hi, wave, {}, 0, 0};
    const uint32_t kvoff = ld.voff(lrow, a.kv.k_stride, lp * CB), vvoff = ld.voff(lrow, a.kv.v_stride, lp * CB);
    typename Loads::Place kplace, vplace;
    Raw<C> fk[LOADS], fv[LOADS];
    // A turn's loads: keys of the tile at t0, values of the tile before it.
    auto loads = [&](int t0) {
        vplace = kplace;
        ld.load(fv, a.kv.v, vplace, a.kv.v_stride, vvoff, t0 - KT, KT);
        ld.place(a.kv, t0, &kplace);
        ld.load(fk, a.kv.k, kplace, a.kv.k_stride, kvoff, t0, KT);
    };
    ld.begin(a.kv, t.lo);
    ld.place(a.kv, t.lo, &kplace);
    ld.load(fk, a.kv.k, kplace, a.kv.k_stride, kvoff, t.lo, KT);

    const int row = t.row0 + 32 * wave + col;
    const bool live = row < t.n_rows;
    const int limit = row_limit(a, t, row), edge = min(limit, t.hi);
    const int row_tok = live ? a.by_group(row) : 0;
    const int64_t tok = t.tok0 + row_tok;
    const int head = t.kvh * a.group + (live ? row - row_tok * a.group : 0);
    bf16x8 qf[KD];
    {
        const __bf16 *qp = (const __bf16 *)a.q + tok * a.q_stride + (int64_t)head * D + 8 * hf;
#pragma unroll
        for (int k = 0; k < KD; ++k) qf[k] = __builtin_bit_cast(bf16x8, live ? *(const uint4 *)(qp + 16 * k) : make_uint4(0, 0, 0, 0));
    }
    if (threadIdx.x == 0) sm.dropped = 0;
    const int all_see = t.all_see;

    auto store_k = [&](int b) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) sm.k[b][((4 * i + wave) * RPL + lrow) * L::KS + lp] = Loads::piece(fk[i], kplace, i);
    };
    auto store_v = [&](int b, bool mixed) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            uint4 v = Loads::piece(fv[i], vplace, i);
            if (mixed && has_nonfinite<__bf16>(v)) {
                drop_nonfinite<__bf16>(v);
                sm.dropped = 1;
            }
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
            const int seen = edge - t0 - 4 * hf;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = seen > 8 * (i >> 2) + (i & 3) ? s[i] : -INFINITY;
        }
        float top = fmaxf(s[0], s[1]);
#pragma unroll
        for (int i = 2; i < 16; i += 2) top = fmaxf(fmaxf(top, s[i]), s[i + 1]);
        top = half_max(top) * a.c;
        float shrink = 1.f;
        if (top > m + kLag) {
            shrink = __builtin_amdgcn_exp2f(m - top);
            m = top;
            mu = top + (top - top);              // a score past fp32's range: NaN, where infinity would weigh every key 0
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
    loads(t.lo + KT);
    __syncthreads();
    scores(0, 0, s0);
    scores(0, 1, s1);
    (void)weights(t.lo, true, s0, p0);           // sums are still zero
    store_k(1);
    store_v(0, t.lo + KT > all_see);
    __syncthreads();
    int b = 0;
    auto turn = [&](int t0, bool masked) {
        loads(t0 + 2 * KT);
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

    l += __shfl_xor(l, 32);
    if (sm.dropped && live) {
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
    // Results go out as whole rows, through LDS: a lane holds four dims here and
    // there of one row, and storing those as they are took as long as two turns.
    const bool whole = t.n_parts == 1;
    const float x = whole ? row_scale(a, l) : 1.f;
    if (hf == 0) {
        int64_t at = -1;
        if (live && whole) {
            at = tok * a.o_stride + (int64_t)head * D;
        } else if (live && limit > t.lo) {
            const int64_t slot = t.slot0 + ((tok - t.tok0) * (a.kv_heads * a.group) + head) * t.slot_parts + t.part;
            a.part_ml[slot] = make_float2(m, l);
            at = slot * D;
        }
        sm.where[wave][col] = at;
    }
#pragma unroll
    for (int d = 0; d < MT32; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *(f32x4 *)&sm.out[wave][col][32 * d + 8 * q + 4 * hf] =
                f32x4{acc[d][4 * q], acc[d][4 * q + 1], acc[d][4 * q + 2], acc[d][4 * q + 3]} * x;
    // rows of this wave only: its LDS operations are in order
    if (whole) {
        constexpr int RL = D / 8, RS = 64 / RL;  // lanes a row, rows a step
#pragma unroll
        for (int r0 = 0; r0 < 32; r0 += RS) {
            const int r = r0 + lane / RL, e = lane % RL * 8;
            const f32x4 y0 = *(const f32x4 *)&sm.out[wave][r][e], y1 = *(const f32x4 *)&sm.out[wave][r][e + 4];
            const int64_t at = sm.where[wave][r];
            if (at >= 0) *(bf16x8 *)((__bf16 *)a.o + at + e) = pack8(y0, y1);
        }
    } else {
        constexpr int RL = D / 4, RS = 64 / RL;
#pragma unroll 4
        for (int r0 = 0; r0 < 32; r0 += RS) {
            const int r = r0 + lane / RL, e = lane % RL * 4;
            const f32x4 y = *(const f32x4 *)&sm.out[wave][r][e];
            const int64_t at = sm.where[wave][r];
            if (at >= 0) store4(a.part_o + at + e, y);
        }
    }
}

template <typename C, int D, bool PAGED>
__global__ __launch_bounds__(kWideThreads, 2) void attn_wide_kernel(AttnArgs a) {
    __shared__ WideLds<D> sm;
    RowTile t;
    if (prompt_tile_of<kPromptRows>(a, blockIdx.x, &t)) wide_run<C, D, PAGED>(a, t, sm);
}

}  // namespace la
