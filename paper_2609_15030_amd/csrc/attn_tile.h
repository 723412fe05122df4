// Attention of tiles of 64 rows, 16 for each of four waves, over key tiles in
// LDS: prompts of few rows, fp32 prompts, and the shared prefix of a decode
// group (rows: the group's sequences; every row reads the same keys).
#pragma once
#include "attn_common.h"

namespace la {

constexpr int kTileThreads = 256;
constexpr int kTileRows = 64;

// Key tile of the kernel and the layout of one tile in LDS: rows of 16-byte
// pieces.  kpos: 16 rows of one piece (a K fragment) fall on 16 different pieces
// of the 64 banks; vpos: so do the 16 rows x 32 bytes (bf16) or 4 rows x 64
// bytes (fp32) that a V fragment reads at once.
template <typename T, int D> struct AttnTile {
    static constexpr int N = Piece<T>::N, PPR = D / N;
    static constexpr int KT = sizeof(T) == 2 || D == 64 ? 64 : 32;
    static constexpr int RPL = 64 / PPR;                  // rows that a wave loads at once
    static constexpr int LOADS = KT / (4 * RPL);
    __device__ static inline int kpos(int row, int p) {
        if constexpr (PPR == 8) return row * PPR + (p ^ ((row >> 1) & 7));
        else return row * PPR + (p ^ (row & 15));
    }
    __device__ static inline int vpos(int row, int p) {
        if constexpr (sizeof(T) == 4) return row * PPR + (p ^ (((row >> 2) & 3) << 2));
        else if constexpr (PPR == 8) return row * PPR + (p ^ (((row >> 1) & 3) << 1));
        else return row * PPR + (p ^ ((row & 7) << 1));
    }
};

// The tile of rows that a workgroup works on (all values uniform).
struct RowTile {
    int kvh, seq;             // key head; row of the block table
    int64_t tok0;             // q token of row 0
    int row0, n_rows;         // first row of the tile, rows of the sequence or group
    int pos0;                 // prompts: position of token 0
    int keys;                 // keys of the sequence, or of the prefix
    int lo, hi;               // keys of this part
    int part, n_parts;        // n_parts == 1: results go straight to o
    bool prefix;
};

// Keys that a row sees.
__device__ inline int row_limit(const AttnArgs &a, const RowTile &t, int row) {
    if (row >= t.n_rows) return 0;
    const int tok = row / a.group;
    if (t.prefix) return min(t.keys, min(a.kv_len[t.tok0 + tok], a.max_kv));
    return max(0, min(t.keys, t.pos0 + tok + 1));
}

// Shared keys of a group: none if it has only one member (its keys are then all its own).
__device__ inline int group_prefix(const AttnArgs &a, int g, int members) {
    if (members < 2) return 0;
    return max(0, min(a.prefix_len[g], a.prefix_parts * a.prefix_part_tokens));
}

// Keys of sequence i of a prompt call.
__device__ inline int prompt_keys(const AttnArgs &a, int i) {
    return a.kv_len ? max(0, min(a.kv_len[i], a.max_kv)) : a.cu[i + 1] - a.cu[i];
}

// The work of block `b`; false: none.  The key head is the fastest index, so that
// the heads of one row tile run side by side and, with 8 heads or a divisor of 8,
// an XCD (workgroup id mod 8) keeps to one head's keys.  A prompt's longest
// (last) tiles come first.
template <int ROWS>
__device__ inline bool row_tile_of(const AttnArgs &a, RowTile *t) {
    const uint32_t b = blockIdx.x;
    const int r = (int)(b / (uint32_t)a.kv_heads);
    t->kvh = (int)(b - (uint32_t)r * (uint32_t)a.kv_heads);
    t->prefix = a.cu_group != nullptr;
    if (t->prefix) {
        const int tile = r % a.group_tiles, q = r / a.group_tiles;
        t->part = q % a.prefix_parts;
        const int g = q / a.prefix_parts;
        if (g >= a.n_groups) return false;
        const int s0 = a.cu_group[g], members = a.cu_group[g + 1] - s0;
        t->seq = s0;
        t->tok0 = s0;
        t->n_rows = members * a.group;
        t->row0 = tile * ROWS;
        t->pos0 = 0;
        t->keys = group_prefix(a, g, members);
        t->n_parts = 2;
        t->lo = t->part * a.prefix_part_tokens;
        t->hi = min(t->keys, t->lo + a.prefix_part_tokens);
        return t->row0 < t->n_rows && t->lo < t->hi;
    }
    auto items = [&](int i) {
        const int rows = (a.cu[i + 1] - a.cu[i]) * a.group;
        return (rows + ROWS - 1) / ROWS * prompt_parts(rows, prompt_keys(a, i));
    };
    int seq, local;
    if (!item_of(a.n_seqs, r, items, &seq, &local)) return false;
    t->seq = seq;
    t->tok0 = a.cu[seq];
    const int rows = (a.cu[seq + 1] - a.cu[seq]) * a.group;
    t->keys = prompt_keys(a, seq);
    const int tiles = (rows + ROWS - 1) / ROWS;
    t->n_rows = rows;
    t->n_parts = prompt_parts(rows, t->keys);
    t->part = local / tiles;
    t->row0 = (tiles - 1 - local % tiles) * ROWS;
    t->pos0 = t->keys - rows / a.group;
    t->prefix = false;
    t->hi = row_limit(a, *t, min(t->row0 + ROWS, t->n_rows) - 1);
    t->lo = 0;
    if (t->n_parts > 1) {
        const int pt = prompt_part_tokens(rows, t->keys);
        t->lo = t->part * pt;
        t->hi = min(t->hi, t->lo + pt);
        return t->lo < t->hi || (t->part == 0);
    }
    return true;
}

// Stored values of v at token `tok`, dims d .. d + 3, of one key head (zero in a
// block that the table does not name).
template <typename C, int D, bool PAGED>
__device__ inline f32x4 v_at(const AttnArgs &a, const int32_t *table_row, int64_t seq_row0, int kvh, int tok, int d) {
    const char *p;
    if constexpr (PAGED) {
        const int id = table_row[tok >> a.kv.bt_shift];
        if ((uint32_t)id >= (uint32_t)a.kv.n_blocks) return zero4();
        p = a.kv.v + (int64_t)id * a.kv.block_bytes +
            (int64_t)D * sizeof(C) * (((int64_t)kvh << a.kv.bt_shift) + (tok & ((1 << a.kv.bt_shift) - 1)));
    } else {
        p = a.kv.v + (seq_row0 + tok) * a.kv.v_stride + (int64_t)kvh * D * sizeof(C);
    }
    const C *e = (const C *)p + d;
    if constexpr (sizeof(C) == 1) {
        const uint2 x = bf16_of_fp8(*(const uint32_t *)e);
        return f32x4{__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xFFFF0000u), __uint_as_float(x.y << 16),
                     __uint_as_float(x.y & 0xFFFF0000u)};
    } else {
        return f32x4{to_f32(e[0]), to_f32(e[1]), to_f32(e[2]), to_f32(e[3])};
    }
}

// Adds the infinities and NaN of v that tiles with a mask left out of their
// products to the rows that see their tokens (tokens t0 .. t1 - 1).  The row's
// lane holds dims 4 g + i of each of the tiles of TS dims in acc.
template <typename C, int D, bool PAGED>
__device__ inline void add_nonfinite(const AttnArgs &a, const int32_t *table_row, int64_t seq_row0, int kvh, int t0,
                                     int t1, int limit, int d, f32x4 &acc) {
    for (int t = t0; t < min(t1, limit); ++t) {
        const f32x4 x = v_at<C, D, PAGED>(a, table_row, seq_row0, kvh, t, d);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if ((__float_as_uint(x[i]) & 0x7F800000u) == 0x7F800000u) acc[i] += x[i];
    }
}

template <typename T, typename C, int D, bool PAGED>
__global__ __launch_bounds__(kTileThreads) void attn_tile_kernel(AttnArgs a) {
    using L = AttnTile<T, D>;
    using M = MT<T>;
    constexpr int KT = L::KT, NT = KT / 16, DT = D / 16;
    constexpr int NQ = sizeof(T) == 2 ? D / 32 : D / 16;       // 16-byte pieces of a q row for each lane
    constexpr int CB = Piece<T>::N * sizeof(C);                // stored bytes of one piece
    __shared__ uint4 kbuf[2][KT * L::PPR];
    __shared__ uint4 vbuf[2][KT * L::PPR];
    __shared__ int least[4], dropped;

    RowTile t;
    if (!row_tile_of<kTileRows>(a, &t)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int row = t.row0 + 16 * wave + col;
    const int limit = row_limit(a, t, row);
    const bool live = row < t.n_rows;
    const int64_t tok = t.tok0 + (live ? row / a.group : 0);
    const int head = t.kvh * a.group + (live ? row % a.group : 0);
    const int32_t *table_row = PAGED ? a.kv.table + (int64_t)t.seq * a.kv.max_blocks : nullptr;
    const int64_t seq_row0 = PAGED ? 0 : t.tok0;

    uint4 qf[NQ];
    {
        const T *qp = (const T *)a.q + tok * a.q_stride + (int64_t)head * D;
#pragma unroll
        for (int s = 0; s < NQ; ++s) {
            const int p = 4 * s + g;                            // bf16: dims 32 s + 8 g ..; fp32: 16 s + 4 g ..
            qf[s] = live ? *(const uint4 *)(qp + p * Piece<T>::N) : make_uint4(0, 0, 0, 0);
        }
    }
    // the keys that every row of the workgroup sees, and the most that a row of the wave sees
    {
        int lo = live ? limit : 0x7fffffff;
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) lo = min(lo, __shfl_xor(lo, d));
        if (lane == 0) least[wave] = lo;
        if (threadIdx.x == 0) dropped = 0;
    }
    int wave_hi = limit;
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) wave_hi = max(wave_hi, __shfl_xor(wave_hi, d));
    wave_hi = __builtin_amdgcn_readfirstlane(min(wave_hi, t.hi));
    __syncthreads();
    const int all_see = __builtin_amdgcn_readfirstlane(min(min(least[0], least[1]), min(least[2], least[3])));

    Raw<C> kr[L::LOADS], vr[L::LOADS];
    const int lrow = lane / L::PPR, lp = lane % L::PPR;
    auto load = [&](int t0) {
#pragma unroll
        for (int i = 0; i < L::LOADS; ++i) {
            const int r = (4 * i + wave) * L::RPL;
            const auto kres = kv_rows<PAGED>(a.kv, 0, table_row, seq_row0, t.kvh, D * (int)sizeof(C), t0 + r, L::RPL, t.hi);
            const auto vres = kv_rows<PAGED>(a.kv, 1, table_row, seq_row0, t.kvh, D * (int)sizeof(C), t0 + r, L::RPL, t.hi);
            const int ks = PAGED ? D * (int)sizeof(C) : (int)a.kv.k_stride, vs = PAGED ? D * (int)sizeof(C) : (int)a.kv.v_stride;
            kr[i] = load_piece<C>(kres, (uint32_t)(lrow * ks + lp * CB));
            vr[i] = load_piece<C>(vres, (uint32_t)(lrow * vs + lp * CB));
        }
    };
    auto store = [&](int b, int t0) {
        const bool mixed = t0 + KT > all_see;
#pragma unroll
        for (int i = 0; i < L::LOADS; ++i) {
            const int r = (4 * i + wave) * L::RPL + lrow;
            kbuf[b][L::kpos(r, lp)] = piece_of<C>(kr[i]);
            uint4 v = piece_of<C>(vr[i]);
            if (mixed && drop_nonfinite<T>(v)) dropped = 1;
            vbuf[b][L::vpos(r, lp)] = v;
        }
    };

    f32x4 acc[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) acc[i] = zero4();
    float m = -INFINITY, l = 0.f;
    if (t.lo < t.hi) {
        load(t.lo);
        store(0, t.lo);
    }
    __syncthreads();
    int b = 0;
    for (int t0 = t.lo; t0 < t.hi; t0 += KT, b ^= 1) {
        const bool more = t0 + KT < t.hi;
        if (more) load(t0 + KT);
        if (t0 < wave_hi) {
            f32x4 s[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                s[n] = zero4();
#pragma unroll
                for (int k = 0; k < NQ; ++k) {
                    const uint4 kf = kbuf[b][L::kpos(16 * n + col, 4 * k + g)];
                    if constexpr (sizeof(T) == 2) {
                        s[n] = M::mma(__builtin_bit_cast(bf16x8, kf), __builtin_bit_cast(bf16x8, qf[k]), s[n]);
                    } else {
                        const float *x = (const float *)&kf, *y = (const float *)&qf[k];
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[n] = M::mma(x[e], y[e], s[n]);
                    }
                }
            }
            const bool masked = t0 + KT > all_see;
            float top = -INFINITY;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float x = s[n][i] * a.c;
                    if (masked && t0 + 16 * n + 4 * g + i >= limit) x = -INFINITY;
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
            const char *vt = (const char *)vbuf[b];
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int k = 0; k < NT / 2; ++k) {
                    const bf16x8 p = pack8(s[2 * k], s[2 * k + 1]);
                    const int r = 32 * k + 4 * g + (col >> 2);
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        const int pc = 2 * d + ((col & 3) >> 1), half = 8 * (col & 1);
                        const bf16x8 v = join_tr(lds_tr(vt + L::vpos(r, pc) * 16 + half),
                                                 lds_tr(vt + L::vpos(r + 16, pc) * 16 + half));
                        acc[d] = M::mma(v, p, acc[d]);
                    }
                }
            } else {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int d = 0; d < DT; ++d) {
                            const int r = 16 * n + 4 * g + i;
                            const float v = *(const float *)(vt + L::vpos(r, 4 * d + (col >> 2)) * 16 + 4 * (col & 3));
                            acc[d] = M::mma(v, s[n][i], acc[d]);
                        }
            }
        }
        if (more) store(b ^ 1, t0 + KT);
        __syncthreads();
    }
    l = row_sum16(l);
    if (dropped && live) {
        const int first = max(t.lo, (all_see - t.lo) / KT * KT + t.lo);
#pragma unroll
        for (int d = 0; d < DT; ++d)
            add_nonfinite<C, D, PAGED>(a, table_row, seq_row0, t.kvh, first, t.hi, limit, 16 * d + 4 * g, acc[d]);
    }
    if (!live) return;
    if (t.n_parts == 1) {
        const float inv = l > 0.f || l != l ? a.v_scale / l : 0.f;
        T *op = (T *)a.o + tok * a.o_stride + (int64_t)head * D;
#pragma unroll
        for (int d = 0; d < DT; ++d) store4(op + 16 * d + 4 * g, acc[d] * inv);
    } else if (limit > t.lo) {
        const int64_t slot = (tok * (a.kv_heads * a.group) + head) * a.parts + t.part;
#pragma unroll
        for (int d = 0; d < DT; ++d) store4(a.part_o + slot * D + 16 * d + 4 * g, acc[d]);
        if (g == 0) a.part_ml[slot] = make_float2(m, l);
    }
}

}  // namespace la
