// What the kernels over tiles of rows share (their work, their loads), and fp32
// attention of such tiles: four waves of 16 rows over key tiles in LDS.  Prompts,
// and the shared prefix of a decode group (rows: the group's sequences; every row
// reads the same keys).
#pragma once
#include "attn_common.h"

namespace la {

// A workgroup's loads of key tiles: wave w of NW takes runs of
// RPL rows, run i at rows (NW i + w) RPL of the tile.
//
// Packed rows: one resource from the tile's first row to the last key; rows past
// it read as zero.  Cached rows: at the tile's offsets (place), which serve its
// keys and its values.  Rows past the last key are whatever the block holds there:
// a masked tile's weights are zero and its values' infinities and NaN dropped.  Rows
// of a block that the table does not name are made zero on their way to LDS
// (missing).  Everything but `voff` is uniform.
template <typename C, bool PAGED, int NW, int RPL, int LOADS, int RB> struct KvLoads {
    static constexpr int STEP = NW * RPL;        // rows from one run of a wave to the next
    static_assert(STEP % kRunTokens == 0 || kRunTokens % STEP == 0, "a wave's rows lie in one run of 16");
    struct Place {
        int64_t at[LOADS];
        uint32_t missing;
    };
    const int32_t *table_row;
    int64_t seq_row0;
    int kvh, hi, wave;
    Runs runs;
    int base, next;                              // first token of `runs`; the lane's block id of the 1,024 tokens behind

    __device__ inline void begin(const KvSource &s, int lo) {
        if constexpr (PAGED) {
            base = lo & ~(64 * kRunTokens - 1);
            const int id = Runs::fetch(s, table_row, base, 0, hi);
            next = Runs::fetch(s, table_row, base, 64 * kRunTokens, hi);
            runs.set(s, id, base, kvh, RB);
        }
    }
    // The place of tile t0; tiles come in order.
    __device__ inline void place(const KvSource &s, int t0, Place *p) {
        if constexpr (PAGED) {
            if (t0 - base >= 64 * kRunTokens) {
                base += 64 * kRunTokens;
                runs.set(s, next, base, kvh, RB);
                next = Runs::fetch(s, table_row, base, 64 * kRunTokens, hi);
            }
            const int r0 = ((t0 - base) + wave * RPL) / kRunTokens;
            p->missing = 0;
            if (runs.bad) {
#pragma unroll
                for (int i = 0; i < LOADS; ++i) p->missing |= (uint32_t)!runs.named(r0 + i * STEP / kRunTokens) << i;
            }
#pragma unroll
            for (int i = 0; i < LOADS; ++i) p->at[i] = runs.run(r0 + i * STEP / kRunTokens) + i * STEP % kRunTokens * RB;
        }
    }
    // A lane's byte offset within its run, from its row of the RPL and piece.
    __device__ inline uint32_t voff(int row, int64_t stride, int piece_at) const {
        return (uint32_t)(PAGED ? (wave * RPL % kRunTokens + row) * RB : row * (int)stride) + (uint32_t)piece_at;
    }
    __device__ inline void load(Raw<C> (&f)[LOADS], const char *from, const Place &p, int64_t stride, uint32_t voff, int t0, int tile) const {
        if constexpr (PAGED) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) f[i] = *(const Raw<C> *)(from + p.at[i] + voff);
        } else {
            const int n = hi - t0;
            const auto res = make_rsrc(from + (n > 0 ? (seq_row0 + t0) * stride : 0) + (int64_t)kvh * RB,
                                       n > 0 ? (uint32_t)(min(n, tile) - 1) * (uint32_t)stride + RB : 0u);
#pragma unroll
            for (int i = 0; i < LOADS; ++i) f[i] = load_piece<C>(res, voff + (uint32_t)((NW * i + wave) * RPL) * (uint32_t)stride);
        }
    }
    // Run i's piece as it goes to LDS.
    __device__ static inline uint4 piece(const Raw<C> &f, const Place &p, int i) {
        if (PAGED && p.missing && (p.missing >> i & 1)) return make_uint4(0, 0, 0, 0);
        return piece_of<C>(f);
    }
};

// The tile of rows that a workgroup works on (all values uniform).
struct RowTile {
    int kvh, seq;             // key head; row of the block table
    int64_t tok0;             // q token of row 0
    int row0, n_rows;         // first row of the tile, rows of the sequence or group
    int pos0;                 // prompts: position of token 0
    int all_see;              // keys that every row of the tile sees
    int keys;                 // keys of the sequence, or of the prefix
    int lo, hi;               // keys of this part
    int part, n_parts;        // n_parts == 1: results go straight to o
    int64_t slot0;            // else to slot0 + (token * q heads + head) * slot_parts + part
    int slot_parts;
    bool prefix;
};

// Keys that a row sees.
__device__ inline int row_limit(const AttnArgs &a, const RowTile &t, int row) {
    if (row >= t.n_rows) return 0;
    const int tok = a.by_group(row);
    if (t.prefix) return max(0, min(t.keys, min(a.kv_len[t.tok0 + tok], a.max_kv)));
    return max(0, min(t.keys, t.pos0 + tok + 1));
}

// The end of the group of sequences [c0, c1), cut to the call's and to max_group: those
// behind it have all their keys to themselves (attn_rows.h decides the same way).
__device__ inline int group_end(const AttnArgs &a, int c0, int c1) { return min(min(c1, c0 + a.max_group), a.n_seqs); }

// Shared keys of a group: none if it has only one member (its keys are then all its own).
__device__ inline int group_prefix(const AttnArgs &a, int g, int members) {
    if (members < 2) return 0;
    return max(0, min(a.prefix_len[g], min(a.prefix_parts * kPrefixPart, a.max_kv)));
}

// Keys of sequence i of a prompt call.
__device__ inline int prompt_keys(const AttnArgs &a, int i) {
    return a.kv_len ? max(0, min(a.kv_len[i], a.max_kv)) : a.cu[i + 1] - a.cu[i];
}

// The work of item `b` of a call; false: none.  The key head is the fastest
// index, so that the heads of one row tile run side by side and, with 8 heads or
// a divisor of 8, an XCD (workgroup id mod 8) keeps to one head's keys.  A
// prompt's longest (last) tiles come first.
template <int ROWS>
__device__ inline bool prefix_tile_of(const AttnArgs &a, uint32_t b, RowTile *t) {
    int r = a.by_kv_heads((int)b);
    t->kvh = (int)b - r * a.kv_heads;
    t->prefix = true;
    const int tile = r % a.group_tiles;
    r /= a.group_tiles;
    t->part = r % a.prefix_parts;
    const int g = r / a.prefix_parts;
    const int s0 = max(0, a.cu_group[g]), members = group_end(a, s0, a.cu_group[g + 1]) - s0;
    t->seq = s0;
    t->tok0 = s0;
    t->n_rows = members * a.group;
    t->row0 = tile * ROWS;
    t->pos0 = 0;
    t->keys = group_prefix(a, g, members);
    t->n_parts = 2;
    t->slot0 = (int64_t)s0 * a.kv_heads * a.group * a.parts;
    t->slot_parts = a.parts;
    t->lo = t->part * kPrefixPart;
    t->hi = min(t->keys, t->lo + kPrefixPart);
    if (t->row0 >= t->n_rows || t->lo >= t->hi) return false;
    const int first = a.by_group(t->row0), last = a.by_group(min(t->row0 + ROWS, t->n_rows) - 1);
    int least = t->keys, most = 0;
    for (int s = first + (int)(threadIdx.x & 63); s <= last; s += 64) {
        const int len = a.kv_len[s0 + s];
        least = min(least, len);
        most = max(most, len);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        least = min(least, __shfl_xor(least, d));
        most = max(most, __shfl_xor(most, d));
    }
    t->all_see = max(0, __builtin_amdgcn_readfirstlane(least));
    t->hi = min(t->hi, __builtin_amdgcn_readfirstlane(most));      // keys that no row sees are not read: their blocks may be gone
    return t->lo < t->hi;
}

// The work of a prompt call's item.  One load of the lengths serves a step of 64
// sequences; the item's sequence is then read from its lane.
template <int ROWS>
__device__ inline bool prompt_tile_of(const AttnArgs &a, uint32_t b, RowTile *t) {
    const int lane = threadIdx.x & 63;
    const int r = a.by_kv_heads((int)b);
    t->kvh = (int)b - r * a.kv_heads;
    t->prefix = false;
    int before = 0, slots = 0;
    for (int i0 = 0; i0 < a.n_seqs; i0 += 64) {
        const int i = a.ordered ? a.order[min(lane, a.n_seqs - 1)] : min(i0 + lane, a.n_seqs - 1);
        const int c0 = a.cu[i], c1 = a.cu[i + 1];
        const int keys = prompt_keys(a, i), rows = (c1 - c0) * a.group;
        const int parts = prompt_parts(keys, a.part_shift);
        const bool in = i0 + lane < a.n_seqs;
        const int x = wave_scan(in ? (rows + ROWS - 1) / ROWS * parts : 0);
        const int y = wave_scan(in && parts > 1 ? rows * a.kv_heads * parts : 0);
        const uint64_t past = __ballot(before + x > r);
        if (!past) {
            before += __builtin_amdgcn_readlane(x, 63);
            slots += __builtin_amdgcn_readlane(y, 63);
            continue;
        }
        const int at = __builtin_ctzll(past);
        const int local = r - before - (at ? __builtin_amdgcn_readlane(x, at - 1) : 0);
        t->slot0 = slots + (at ? __builtin_amdgcn_readlane(y, at - 1) : 0);
        t->seq = __builtin_amdgcn_readlane(i, at);
        t->tok0 = __builtin_amdgcn_readlane(c0, at);
        t->n_rows = __builtin_amdgcn_readlane(rows, at);
        t->keys = __builtin_amdgcn_readlane(keys, at);
        t->n_parts = t->slot_parts = __builtin_amdgcn_readlane(parts, at);
        const int tiles = (t->n_rows + ROWS - 1) / ROWS;
        t->part = 0;
        int tile = local;
        while (tile >= tiles) {                  // few parts: cheaper than a division
            tile -= tiles;
            ++t->part;
        }
        t->row0 = (tiles - 1 - tile) * ROWS;
        t->pos0 = t->keys - (__builtin_amdgcn_readlane(c1, at) - (int)t->tok0);
        t->all_see = row_limit(a, *t, t->row0);
        t->hi = row_limit(a, *t, min(t->row0 + ROWS, t->n_rows) - 1);
        t->lo = 0;
        if (t->n_parts > 1) {
            t->lo = t->part << a.part_shift;
            t->hi = t->lo + min(t->hi - t->lo, 1 << a.part_shift);      // lo + 2^part_shift may be 2^31
            return t->lo < t->hi;
        }
        return true;
    }
    return false;
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

// fp32: key tiles of 32 keys, double buffered, and two more in flight in registers,
// so that a tile's loads have two tiles' time to arrive.  Bound by the matrix unit
// where a call fills the chip (8,192 tokens x 8 heads x 64: 101 TFLOP/s of the 154
// that a large product reaches; suffixes of 16 prompts over a cache, 8 heads x 128: 111), by the uneven tiles of its parts where it does
// not (1,791 + 640 + 257 tokens: 61 us, 62 TFLOP/s).  At 32 keys and 64 dims four
// workgroups share a CU; at 64 keys two did (66 us).
//
// LDS: 16-byte pieces, one piece of padding behind each row.  With it the 16 rows
// of one piece (a K fragment) fall on different banks, and so do the 4 rows x 64
// bytes of a V fragment; and a lane's addresses differ by constants, which an
// exclusive-or of row and piece would not give (it took 40 more registers).
constexpr int kTileWaves = 4, kTileRows = 16 * kTileWaves, kTileThreads = 64 * kTileWaves;

template <int D> struct TileLds {
    static constexpr int KT = 32, PPR = D / 4, PS = PPR + 1;
    union {
        struct {
            uint4 k[2][KT * PS], v[2][KT * PS];
        };
        float out[kTileWaves][16][D + 4];        // results on their way out; the padding puts 16 rows on different banks
    };
    int64_t where[kTileWaves][16];               // and where their rows go, in elements (-1: nowhere)
    int dropped;
};

template <int D, bool PAGED>
__device__ __forceinline__ void tile_run(const AttnArgs &a, const RowTile &t, TileLds<D> &sm) {
    using L = TileLds<D>;
    constexpr int KT = L::KT, NT = KT / 16, DT = D / 16, NQ = D / 16;          // NQ: 16-byte pieces of a q row for each lane
    constexpr int RPL = 64 / L::PPR, LOADS = KT / (kTileWaves * RPL), RB = D * sizeof(float);
    static_assert(LOADS >= 1 && LOADS * kTileWaves * RPL == KT, "key tile");

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int row = t.row0 + 16 * wave + col;
    const int limit = row_limit(a, t, row);
    const bool live = row < t.n_rows;
    const int row_tok = live ? a.by_group(row) : 0;
    const int64_t tok = t.tok0 + row_tok;
    const int head = t.kvh * a.group + (live ? row - row_tok * a.group : 0);
    const int32_t *table_row = PAGED ? a.kv.table + (int64_t)t.seq * a.kv.max_blocks : nullptr;
    const int64_t seq_row0 = PAGED ? 0 : t.tok0;
    const int lrow = lane / L::PPR, lp = lane % L::PPR;
    using Loads = KvLoads<float, PAGED, kTileWaves, RPL, LOADS, RB>;
    Loads ld{table_row, seq_row0, t.kvh, t.hi, wave, {}, 0, 0};
    const uint32_t kvoff = ld.voff(lrow, a.kv.k_stride, 16 * lp), vvoff = ld.voff(lrow, a.kv.v_stride, 16 * lp);
    struct Flight {
        Raw<float> k[LOADS], v[LOADS];
        typename Loads::Place p;
    } f0, f1;
    auto load = [&](int t0, Flight &f) {
        ld.place(a.kv, t0, &f.p);
        ld.load(f.k, a.kv.k, f.p, a.kv.k_stride, kvoff, t0, KT);
        ld.load(f.v, a.kv.v, f.p, a.kv.v_stride, vvoff, t0, KT);
    };
    ld.begin(a.kv, t.lo);
    load(t.lo, f0);
    load(t.lo + KT, f1);

    uint4 qf[NQ];
    {
        const float *qp = (const float *)a.q + tok * a.q_stride + (int64_t)head * D + 4 * g;
#pragma unroll
        for (int s = 0; s < NQ; ++s) qf[s] = live ? *(const uint4 *)(qp + 16 * s) : make_uint4(0, 0, 0, 0);
    }
    const int all_see = t.all_see;
    int wave_hi = limit;                         // the most keys that a row of the wave sees
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) wave_hi = max(wave_hi, __shfl_xor(wave_hi, d));
    wave_hi = __builtin_amdgcn_readfirstlane(min(wave_hi, t.hi));
    if (threadIdx.x == 0) sm.dropped = 0;
    __syncthreads();

    auto store = [&](int b, int t0, const Flight &f) {
        const bool mixed = t0 + KT > all_see;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = ((kTileWaves * i + wave) * RPL + lrow) * L::PS + lp;
            sm.k[b][at] = Loads::piece(f.k[i], f.p, i);
            uint4 v = Loads::piece(f.v[i], f.p, i);
            if (mixed && has_nonfinite<float>(v)) {
                drop_nonfinite<float>(v);
                sm.dropped = 1;
            }
            sm.v[b][at] = v;
        }
    };

    f32x4 acc[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) acc[i] = zero4();
    float m = -INFINITY, l = 0.f;
    auto compute = [&](int b, int t0) {
        if (t0 >= wave_hi) return;
        f32x4 s[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            s[n] = zero4();
#pragma unroll
            for (int k = 0; k < NQ; ++k) {
                const uint4 kf = sm.k[b][(16 * n + col) * L::PS + 4 * k + g];
                const float *x = (const float *)&kf, *y = (const float *)&qf[k];
#pragma unroll
                for (int e = 0; e < 4; ++e) s[n] = MT<float>::mma(x[e], y[e], s[n]);
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
        const char *at = (const char *)sm.v[b] + 4 * g * L::PS * 16 + 4 * col;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int d = 0; d < DT; ++d)
                    acc[d] = MT<float>::mma(*(const float *)(at + (16 * n + i) * L::PS * 16 + 64 * d), s[n][i], acc[d]);
    };
    // Two tiles a turn, so that the register sets and buffers are constants; the
    // loads run past the last tile (as zeros) rather than being skipped, since a
    // loop that can leave between two register sets makes every wait a wait for all.
    store(0, t.lo, f0);
    load(t.lo + 2 * KT, f0);
    __syncthreads();
    for (int t0 = t.lo; t0 < t.hi; t0 += 2 * KT) {
        compute(0, t0);
        store(1, t0 + KT, f1);
        load(t0 + 3 * KT, f1);
        __syncthreads();
        compute(1, t0 + KT);
        store(0, t0 + 2 * KT, f0);
        load(t0 + 4 * KT, f0);
        __syncthreads();
    }
    l = row_sum16(l);
    if (sm.dropped && live) {
        const int first = all_see <= t.lo ? t.lo : t.lo + (all_see - t.lo) / KT * KT;
#pragma unroll
        for (int d = 0; d < DT; ++d)
            add_nonfinite<float, D, PAGED>(a, table_row, seq_row0, t.kvh, first, t.hi, limit, 16 * d + 4 * g, acc[d]);
    }
    // Results go out as whole rows, through LDS (the last barrier is behind every read of its tiles).
    const bool whole = t.n_parts == 1;
    const float x = whole ? row_scale(a, l) : 1.f;
    if (g == 0) {
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
    for (int d = 0; d < DT; ++d) *(f32x4 *)&sm.out[wave][col][16 * d + 4 * g] = acc[d] * x;
    constexpr int RL = D / 4, RS = 64 / RL;      // lanes a row, rows a step
#pragma unroll
    for (int r0 = 0; r0 < 16; r0 += RS) {
        const int r = r0 + lane / RL, e = lane % RL * 4;
        const f32x4 y = *(const f32x4 *)&sm.out[wave][r][e];
        const int64_t at = sm.where[wave][r];
        if (at < 0) continue;
        store4((whole ? (float *)a.o : a.part_o) + at + e, y);
    }
}

template <int D, bool PAGED>
__global__ __launch_bounds__(kTileThreads) void attn_tile_kernel(AttnArgs a) {
    __shared__ TileLds<D> sm;
    RowTile t;
    if (prompt_tile_of<kTileRows>(a, blockIdx.x, &t)) tile_run<D, PAGED>(a, t, sm);
}

}  // namespace la
