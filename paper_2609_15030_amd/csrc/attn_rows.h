// Attention of single tokens over a cache, and the joining of parts.
//
// One launch holds two kinds of workgroups.  The first ones take the shared
// prefixes, as tiles of rows (attn_wide.h; fp32: attn_tile.h).  The others take
// the keys that each sequence has to itself, a part at a time, for up to 16 query
// heads of one key head: every key and value is used once by one wave, so nothing
// is shared; each of the four waves takes key tiles of its own, K goes from
// memory straight into the registers that the product reads, V through LDS of the
// wave's own (its fragments are columns), and the waves' m, l and sums meet at the
// end.
//
// Many long sequences are bound by memory: 96 of 1 to 32,768 keys, 4 key heads of
// 128 in 8 bits, 66 us at 4.8 TB/s (a large copy reaches 5.1), their join 5.6; whole
// calls of 64 of 8,000 in bf16 207 us at 5.1, in 8 bits 131 at 4.0, of 64 of 4,000 with
// 8 key heads in fp32 378 at 5.5.  A single one is a chain (lengths -> table -> keys -> join): 3,584 keys, 2 heads,
// 7.5 us, its join 2.6.  64 sequences behind 6,144 shared keys: 22.9 us, of which
// memory alone would take 9.5; a prefix part is a chain of four key tiles.
#pragma once
#include "attn_tile.h"
#include "attn_wide.h"

namespace la {

constexpr int kDecodeWaves = 4;
constexpr int kRowsThreads = 64 * kDecodeWaves;
constexpr int kRowsHeads = 16;

template <typename T, int D> struct RowsLds {
    static constexpr int KT = sizeof(T) == 2 ? 32 : 16;       // keys of a wave's tile
    static constexpr int PS = D * (int)sizeof(T) / 16 + 1;    // 16-byte pieces of a row in LDS, one of them padding
    union {
        uint4 v[kDecodeWaves][KT * PS];
        float sum[kDecodeWaves][kRowsHeads][D];
    };
    float m[kDecodeWaves][kRowsHeads], l[kDecodeWaves][kRowsHeads];
};

// What a sequence of a decode call has to itself: keys [first, end), and the parts
// of the prefix before them.
struct OwnKeys {
    int first, end, prefix_parts;
    // Parts of the own keys: they begin at the 16-token line at or before the first.
    __device__ inline int lo() const { return first & ~15; }
    __device__ inline int parts() const { return end <= first ? 0 : (end - lo() + kOwnPart - 1) / kOwnPart; }
};

// Sequence s's own keys, for every lane its s.  Sequences outside every group share
// nothing.  Up to 64 groups are read at once, one a lane, beside kv_len: a search
// would be a chain of loads, each as long as memory takes to answer.
__device__ inline OwnKeys own_keys(const AttnArgs &a, int s) {
    OwnKeys k{0, 0, 0};
    const int len = a.kv_len[s];
    if (!a.cu_group) {
        k.end = max(0, min(len, a.max_kv));
        return k;
    }
    int shared = 0;
    for (int g0 = 0; g0 < a.n_groups; g0 += 64) {
        const int n = min(64, a.n_groups - g0), g = g0 + min((int)(threadIdx.x & 63), n - 1);
        const int c0 = max(0, a.cu_group[g]), c1 = group_end(a, c0, a.cu_group[g + 1]), p = a.prefix_len[g];
        for (int i = 0; i < n; ++i) {
            const int b0 = __builtin_amdgcn_readlane(c0, i), b1 = __builtin_amdgcn_readlane(c1, i);
            if (s >= b0 && s < b1 && b1 - b0 > 1) shared = __builtin_amdgcn_readlane(p, i);
        }
    }
    k.end = max(0, min(len, a.max_kv));
    k.first = max(0, min(min(shared, a.prefix_parts * kPrefixPart), k.end));
    k.prefix_parts = (k.first + kPrefixPart - 1) / kPrefixPart;
    return k;
}
// Lane `at`'s, for all.
__device__ inline OwnKeys own_keys_of_lane(const OwnKeys &k, int at) {
    return {__builtin_amdgcn_readlane(k.first, at), __builtin_amdgcn_readlane(k.end, at), __builtin_amdgcn_readlane(k.prefix_parts, at)};
}

// Workgroup b of n that take the own keys.
template <typename T, typename C, int D>
__device__ __forceinline__ void rows_run(const AttnArgs &a, int b, int n_blocks, RowsLds<T, D> &sm) {
    using M = MT<T>;
    using L = RowsLds<T, D>;
    constexpr bool F8 = sizeof(C) == 1;
    constexpr int KT = L::KT, PS = L::PS, NT = KT / 16, DT = D / 16;
    constexpr int NQ = sizeof(T) == 2 ? D / 32 : D / 16;       // 16-byte pieces of a q row for each lane
    constexpr int RB = D * sizeof(C);                          // bytes of a stored row
    constexpr int NK = RB / 64, VPR = RB / 16, VR = 64 / VPR, VL = 16 / VR;    // loads of 16 keys, of 16 values

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int tiles = (a.group + kRowsHeads - 1) / kRowsHeads, heads = tiles * a.kv_heads;
    // the call's items (part of a sequence, key head, row tile; the last fastest), and this workgroup's share
    auto parts_of = [&](const OwnKeys &k) { return a.direct ? 1 : k.parts(); };
    int total = 0, sum = 0;                      // sum: of the last step of 64 sequences, up to each lane
    OwnKeys lane_keys{0, 0, 0};
    for (int i0 = 0; i0 < a.n_seqs; i0 += 64) {
        lane_keys = own_keys(a, min(i0 + lane, a.n_seqs - 1));
        sum = wave_scan(i0 + lane < a.n_seqs ? parts_of(lane_keys) : 0);
        total += __builtin_amdgcn_readlane(sum, 63);
    }
    const int per = total * heads / n_blocks, extra = total * heads - per * n_blocks;
    int item = b * per + min(b, extra);
    const int stop = item + per + (b < extra);
    if (b == 0 && a.kv.err)
        for (int i = threadIdx.x; i < a.n_seqs; i += kRowsThreads)
            if (a.kv_len[i] > a.max_kv) atomicAdd(a.kv.err, 1);
    if (item >= stop) return;
    int seq = 0, part = item / heads, at = item - part * heads, i0 = 0;
    if (a.n_seqs > 64) {
        for (; i0 < a.n_seqs; i0 += 64) {        // the step that holds the first item's sequence
            lane_keys = own_keys(a, min(i0 + lane, a.n_seqs - 1));
            sum = wave_scan(i0 + lane < a.n_seqs ? parts_of(lane_keys) : 0);
            const int n = __builtin_amdgcn_readlane(sum, 63);
            if (part < n) break;
            part -= n;
        }
    }
    {
        const int l0 = __builtin_ctzll(__ballot(sum > part));
        part -= l0 ? __builtin_amdgcn_readlane(sum, l0 - 1) : 0;
        seq = i0 + l0;
    }
    OwnKeys own = own_keys_of_lane(lane_keys, seq - i0);

    for (; item < stop; ++item) {
        const int kvh = at / tiles, h0 = (at - kvh * tiles) * kRowsHeads;
        const int lo = own.lo() + part * kOwnPart, first = own.first;
        const int hi = min(own.end, lo + kOwnPart);
        const int live_heads = min(kRowsHeads, a.group - h0);
        const bool live = col < live_heads;
        const int head = kvh * a.group + h0 + (live ? col : 0);
        // the part's runs of 16 keys, one a lane
        static_assert(kOwnPart <= 64 * kRunTokens, "a lane for each run");
        Runs runs;
        runs.set(a.kv, Runs::fetch(a.kv, a.kv.table + (int64_t)seq * a.kv.max_blocks, lo, 0, hi), lo, kvh, RB);
        uint4 qf[NQ];
        {
            const T *qp = (const T *)a.q + seq * a.q_stride + (int64_t)head * D;
#pragma unroll
            for (int s = 0; s < NQ; ++s) {
                // an 8-bit key load holds 16 dims of a lane: the pieces of two products
                const int p = F8 ? 8 * (s >> 1) + 2 * g + (s & 1) : 4 * s + g;
                qf[s] = live ? *(const uint4 *)(qp + p * Piece<T>::N) : make_uint4(0, 0, 0, 0);
            }
        }
        f32x4 acc[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d) acc[d] = zero4();
        float m = -INFINITY, l = 0.f;
        char *const vt = (char *)sm.v[wave];
        // the wave's tiles: two of them in flight; those past the last key load nothing
        constexpr int STEP = kDecodeWaves * KT, TILES = kOwnPart / STEP;
        static_assert(TILES % 2 == 0, "two tiles a turn");
        struct Flight { uint4 k[NT][NK], v[NT][VL]; } f0, f1;
        auto load = [&](int t0, Flight &f) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int r = ((t0 - lo) / kRunTokens + n) & 63, rows = min(hi - t0 - 16 * n, 16);
                const int64_t at = runs.run(r);
                const uint32_t bytes = rows > 0 && runs.named(r) ? (uint32_t)(rows * RB) : 0u;    // the others read as zero
                const auto kres = make_rsrc(a.kv.k + at, bytes), vres = make_rsrc(a.kv.v + at, bytes);
#pragma unroll
                for (int k = 0; k < NK; ++k) f.k[n][k] = buf_load16(kres, (uint32_t)(col * RB + 16 * g), 64 * k);
#pragma unroll
                for (int i = 0; i < VL; ++i) f.v[n][i] = buf_load16(vres, (uint32_t)(16 * lane), 1024 * i);
            }
        };
        auto compute = [&](int t0, const Flight &f) {
            if (t0 >= hi) return;
            f32x4 s[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                s[n] = zero4();
#pragma unroll
                for (int k = 0; k < NK; ++k) {
                    const uint4 x = f.k[n][k];
                    if constexpr (F8) {
                        const uint2 e0 = bf16_of_fp8(x.x), e1 = bf16_of_fp8(x.y), e2 = bf16_of_fp8(x.z), e3 = bf16_of_fp8(x.w);
                        s[n] = M::mma(__builtin_bit_cast(bf16x8, make_uint4(e0.x, e0.y, e1.x, e1.y)),
                                      __builtin_bit_cast(bf16x8, qf[2 * k]), s[n]);
                        s[n] = M::mma(__builtin_bit_cast(bf16x8, make_uint4(e2.x, e2.y, e3.x, e3.y)),
                                      __builtin_bit_cast(bf16x8, qf[2 * k + 1]), s[n]);
                    } else if constexpr (sizeof(T) == 2) {
                        s[n] = M::mma(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, qf[k]), s[n]);
                    } else {
                        const float *e = (const float *)&x, *y = (const float *)&qf[k];
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[n] = M::mma(e[j], y[j], s[n]);
                    }
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < VL; ++i) {
                    const int row = 16 * n + VR * i + lane / VPR;
                    uint4 *const to = (uint4 *)vt + row * PS;
                    uint4 x = f.v[n][i];
                    // keys that the prefix's part has: a weight of zero would not undo an infinity
                    if (t0 < first && t0 + row < first) x = make_uint4(0, 0, 0, 0);
                    if constexpr (F8) {
                        const uint2 e0 = bf16_of_fp8(x.x), e1 = bf16_of_fp8(x.y), e2 = bf16_of_fp8(x.z), e3 = bf16_of_fp8(x.w);
                        to[2 * (lane % VPR)] = make_uint4(e0.x, e0.y, e1.x, e1.y);
                        to[2 * (lane % VPR) + 1] = make_uint4(e2.x, e2.y, e3.x, e3.y);
                    } else {
                        to[lane % VPR] = x;
                    }
                }
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
            if constexpr (sizeof(T) == 2) {
                const bf16x8 p = pack8(s[0], s[1]);
                const char *x = vt + (4 * g + (col >> 2)) * PS * 16 + 8 * (col & 3);
#pragma unroll
                for (int d = 0; d < DT; ++d) acc[d] = M::mma(join_tr(lds_tr(x + 32 * d), lds_tr(x + 16 * PS * 16 + 32 * d)), p, acc[d]);
            } else {
                const char *x = vt + 4 * g * PS * 16 + 4 * col;
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int d = 0; d < DT; ++d) acc[d] = M::mma(*(const float *)(x + i * PS * 16 + 64 * d), s[0][i], acc[d]);
            }
        };
        const int w0 = lo + wave * KT;
        load(w0, f0);
        load(w0 + STEP, f1);
#pragma unroll
        for (int i = 0; i < TILES; i += 2) {
            compute(w0 + i * STEP, f0);
            if (i + 2 < TILES) load(w0 + (i + 2) * STEP, f0);
            compute(w0 + (i + 1) * STEP, f1);
            if (i + 3 < TILES) load(w0 + (i + 3) * STEP, f1);
        }
        // the waves' results: every wave scales its sums to the common maximum
        if (g == 0) sm.m[wave][col] = m;
        l = row_sum16(l);
        __syncthreads();
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < kDecodeWaves; ++w) top = fmaxf(top, sm.m[w][col]);
        const float scale = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.f : top));
        if (live) {
#pragma unroll
            for (int d = 0; d < DT; ++d) *(f32x4 *)&sm.sum[wave][col][16 * d + 4 * g] = acc[d] * scale;
            if (g == 0) sm.l[wave][col] = l * scale;
        }
        __syncthreads();
        const int64_t head_row0 = (int64_t)kvh * a.group + h0;
        for (int e = threadIdx.x; e < live_heads * (D / 4); e += kRowsThreads) {
            const int h = e / (D / 4), d = e % (D / 4) * 4;
            f32x4 x = zero4();
            float lt = 0.f;
#pragma unroll
            for (int w = 0; w < kDecodeWaves; ++w) {
                x += *(const f32x4 *)&sm.sum[w][h][d];
                lt += sm.l[w][h];
            }
            if (a.direct) {
                store4((T *)a.o + seq * a.o_stride + (head_row0 + h) * D + d, x * row_scale(a, lt));
            } else {
                const int64_t slot = ((int64_t)seq * a.kv_heads * a.group + head_row0 + h) * a.parts + own.prefix_parts + part;
                store4(a.part_o + slot * D + d, x);
                if (d == 0) {
                    float mt = sm.m[0][h];
#pragma unroll
                    for (int w = 1; w < kDecodeWaves; ++w) mt = fmaxf(mt, sm.m[w][h]);
                    a.part_ml[slot] = make_float2(mt, lt);
                }
            }
        }
        // the next item: the next head, part or sequence that has one
        if (++at == heads && item + 1 < stop) {
            at = 0;
            if (++part >= parts_of(own)) {
                part = 0;
                do {
                    if (++seq >= a.n_seqs) return;
                    if (seq - i0 == 64) {
                        i0 += 64;
                        lane_keys = own_keys(a, min(i0 + lane, a.n_seqs - 1));
                    }
                    own = own_keys_of_lane(lane_keys, seq - i0);
                } while (parts_of(own) == 0);
            }
        }
        __syncthreads();                                        // sums read before the next item's V lands there
    }
}

template <typename T, typename C, int D>
__global__ __launch_bounds__(kRowsThreads, 2) void attn_decode_kernel(AttnArgs a) {
    constexpr bool WIDE = sizeof(T) == 2;
    constexpr int ROWS = WIDE ? kPromptRows : kTileRows;
    static_assert(kRowsThreads == kWideThreads && kRowsThreads == kTileThreads, "one launch for both");
    __shared__ union Lds {
        std::conditional_t<WIDE, WideLds<D>, TileLds<D>> tile;
        RowsLds<T, D> rows;
    } sm;
    if ((int)blockIdx.x < a.prefix_items) {
        RowTile t;
        if (!prefix_tile_of<ROWS>(a, blockIdx.x, &t)) return;
        if constexpr (WIDE) wide_run<C, D, true>(a, t, sm.tile);
        else tile_run<D, true>(a, t, sm.tile);
    } else {
        rows_run<T, C, D>(a, (int)blockIdx.x - a.prefix_items, (int)gridDim.x - a.prefix_items, sm.rows);
    }
}

// Joins the parts of prompt rows, those of the sequences that have several: D / 4
// lanes a row, 1,024 / D rows a workgroup.
template <typename T, int D>
__global__ __launch_bounds__(256) void attn_join_prompt_kernel(AttnArgs a) {
    constexpr int LANES = D / 4, ROWS = 256 / LANES, AHEAD = 8;
    const int heads = a.kv_heads * a.group, wl = threadIdx.x & 63;
    int before = 0, slots = 0, seq = -1, local = 0, c0 = 0, new_tokens = 0, keys = 0;
    int stride = 1;
    for (int i0 = 0; i0 < a.n_seqs; i0 += 64) {
        const int i = min(i0 + wl, a.n_seqs - 1);
        const int b0 = a.cu[i], n = a.cu[i + 1] - b0, k = prompt_keys(a, i);
        const int parts = prompt_parts(k, a.part_shift);
        const bool in = i0 + wl < a.n_seqs && parts > 1;
        const int x = wave_scan(in ? (n * heads + ROWS - 1) / ROWS : 0), y = wave_scan(in ? n * heads * parts : 0);
        const uint64_t past = __ballot(before + x > (int)blockIdx.x);
        if (!past) {
            before += __builtin_amdgcn_readlane(x, 63);
            slots += __builtin_amdgcn_readlane(y, 63);
            continue;
        }
        const int at = __builtin_ctzll(past);
        seq = i0 + at;
        local = (int)blockIdx.x - before - (at ? __builtin_amdgcn_readlane(x, at - 1) : 0);
        slots += at ? __builtin_amdgcn_readlane(y, at - 1) : 0;
        c0 = __builtin_amdgcn_readlane(b0, at);
        new_tokens = __builtin_amdgcn_readlane(n, at);
        keys = __builtin_amdgcn_readlane(k, at);
        stride = __builtin_amdgcn_readlane(parts, at);
        break;
    }
    if (seq < 0) return;
    const int lane = threadIdx.x % LANES, row = local * ROWS + threadIdx.x / LANES;
    if (row >= new_tokens * heads) return;
    const int tok = a.by_group(a.by_kv_heads(row)), head = row - tok * heads;
    const int limit = max(0, keys - new_tokens + tok + 1), parts = (int)(((uint32_t)limit + (1u << a.part_shift) - 1) >> a.part_shift);
    const int64_t slot = slots + (int64_t)row * stride;
    const float2 *ml = a.part_ml + slot;
    const float *po = a.part_o + slot * D + 4 * lane;
    float m = -INFINITY, l = 0.f;
    f32x4 x = zero4();
    for (int p0 = 0; p0 < parts; p0 += AHEAD) {
        f32x4 xp[AHEAD];
        float2 y[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int p = min(p0 + i, parts - 1);
            xp[i] = *(const f32x4 *)(po + (int64_t)p * D);
            y[i] = ml[p];
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (p0 + i >= parts) break;
            float w, wp;
            join_weights(m, l, y[i].x, y[i].y, &w, &wp);
            x = join4(x, xp[i], w, wp);
        }
    }
    store4((T *)a.o + (int64_t)(c0 + tok) * a.o_stride + (int64_t)head * D + 4 * lane, x * row_scale(a, l));
}

// Joins the parts of a single token's row: a workgroup a row, D / 4 lanes a part.
template <typename T, int D>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a) {
    constexpr int LANES = D / 4, SETS = 256 / LANES;
    __shared__ f32x4 xs[SETS][LANES];
    __shared__ float2 mls[SETS];
    const int set = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    const int heads = a.kv_heads * a.group;
    const uint32_t row = blockIdx.x, seq = row / (uint32_t)heads, head = row - seq * (uint32_t)heads;
    const OwnKeys own = own_keys(a, (int)seq);
    const int parts = own.prefix_parts + own.parts();
    const float2 *ml = a.part_ml + (int64_t)row * a.parts;
    const float *po = a.part_o + (int64_t)row * a.parts * D + 4 * lane;
    float m = -INFINITY, l = 0.f;
    f32x4 x = zero4();
#pragma unroll 4
    for (int p = set; p < parts; p += SETS) {
        const float2 y = ml[p];
        const f32x4 xp = *(const f32x4 *)(po + (int64_t)p * D);
        float w, wp;
        join_weights(m, l, y.x, y.y, &w, &wp);
        x = join4(x, xp, w, wp);
    }
    xs[set][lane] = x;
    if (lane == 0) mls[set] = make_float2(m, l);
    __syncthreads();
    if (set > 0) return;
#pragma unroll
    for (int i = 1; i < SETS; ++i) {
        float w, wp;
        join_weights(m, l, mls[i].x, mls[i].y, &w, &wp);
        x = join4(x, xs[i][lane], w, wp);
    }
    store4((T *)a.o + (int64_t)seq * a.o_stride + (int64_t)head * D + 4 * lane, x * row_scale(a, l));
}

}  // namespace la
