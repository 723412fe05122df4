// The blocks of an attention cache: new keys and values written into them, and
// their bookkeeping (copy, fork, extend, free, compact) on the device.
//
// Bytes: a copied or moved block is read and written once (a fork copies only a
// last block that its tokens end inside); beside that 4 bytes for each table entry
// and block id.  Copies run at the rate of a large copy (5.0 TB/s) once they are
// many; small calls are bound by their launches and by chains of loads (row ->
// table entry -> id), which is why a call is few kernels and a thread's loads
// within one pass are independent.  Measured, in us: 64 forks of 517 to 3,584 tokens
// with their 64 children freed 16.3 (fork_take 3, fork 7, free_rows 4, free_push 2.7);
// 16 rows of 17 to 3,328 tokens with four freed, compacted and grown
// again 49.9 (rank 5, move 28 at 4.9 TB/s, extend 6.5, free_rows 4, free_push 4.7).
// Freeing in one workgroup instead of two kernels took 9 to 25: one CU's atomics are too slow.
//
// Handing out and taking back in a fixed order is one workgroup's work, pass after
// pass: extend visits every entry of its rows (4 rows of 210 entries 4.4 us, 64 of
// 2,048 73, 256 of 2,048 286), free every id of the pool (one row freed from 3,000
// ids 6 us, 33,000 13, 1,048,576 171, 2,097,152 350).
//
// Block ids live in a table [rows, max_blocks] (-1: none); ref[b] counts the
// entries that name b; the free ids are a stack, the next one at its top.
// Everything that hands out or takes back several blocks does so in a fixed
// order (calls, entries or ids ascending), so no result depends on timing.
#pragma once
#include "attn_common.h"

namespace la {

struct BlockPoolArgs {
    char *cache;
    int64_t block_vec;             // 16-byte vectors of a block
    int64_t n_blocks, n_rows, max_blocks;
    int32_t bt_shift;
    int32_t *table, *ref, *free_list, *free_count, *err;
};

constexpr int kBlockThreads = 1024;
constexpr int kPartVec = 2 * kBlockThreads;        // 32 KB of a block for each workgroup
constexpr int32_t kFreed = -(1 << 30);             // mark of a block whose last entry just went

__device__ inline void count_error(const BlockPoolArgs &p) {
    if (p.err) atomicAdd(p.err, 1);
}

// Free blocks on the stack; a count outside it is cut, so that no call leaves the list.
__device__ inline int free_blocks(const BlockPoolArgs &p) { return (int)max((int64_t)0, min((int64_t)*p.free_count, p.n_blocks)); }

// Vectors [part * kPartVec, ...) of one block to another, loads first.
__device__ inline void copy_block_part(const BlockPoolArgs &p, int64_t src, int64_t dst, int64_t part) {
    const f32x4 *s = (const f32x4 *)p.cache + src * p.block_vec;
    f32x4 *d = (f32x4 *)p.cache + dst * p.block_vec;
    const int64_t v0 = part * kPartVec + threadIdx.x, v1 = v0 + kBlockThreads;
    f32x4 x0 = zero4(), x1 = zero4();
    if (v0 < p.block_vec) x0 = __builtin_nontemporal_load(s + v0);
    if (v1 < p.block_vec) x1 = __builtin_nontemporal_load(s + v1);
    if (v0 < p.block_vec) d[v0] = x0;
    if (v1 < p.block_vec) d[v1] = x1;
}

// Exclusive sum of x over the workgroup's 1,024 threads, and the total.
__device__ inline int block_sum_before(int x, int *total) {
    __shared__ int sums[kBlockThreads / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int y = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int z = __shfl_up(y, d);
        if (lane >= d) y += z;
    }
    __syncthreads();                               // sums of the last call are no longer read
    if (lane == 63) sums[wave] = y;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kBlockThreads / 64; ++w) {
        before += w < wave ? sums[w] : 0;
        all += sums[w];
    }
    *total = all;
    return before + y - x;
}

__global__ __launch_bounds__(kBlockThreads) void blocks_copy_kernel(BlockPoolArgs p, const int32_t *src, const int32_t *dst) {
    const int64_t i = blockIdx.x;
    const int32_t s = src[i], d = dst[i];
    if (s == -1 || d == -1) return;
    if (s < 0 || s >= p.n_blocks || d < 0 || d >= p.n_blocks) {
        if (threadIdx.x == 0 && blockIdx.y == 0) count_error(p);
        return;
    }
    copy_block_part(p, s, d, blockIdx.y);
}

// --- fork --------------------------------------------------------------------

struct ForkArgs {
    BlockPoolArgs p;
    const int32_t *parent, *child, *len;
    int32_t n;
};

// What fork i does: false if its rows are no rows.  *full: whole blocks shared;
// *tail: the parent's last block, inside which its tokens end (-1: they end with a
// whole block; -2: the parent has no block there).
__device__ inline bool fork_of(const ForkArgs &a, int i, int *full, int *tail) {
    const int pr = a.parent[i], ch = a.child[i];
    if (pr < 0 || pr >= a.p.n_rows || ch < 0 || ch >= a.p.n_rows || pr == ch) return false;
    const int64_t most = a.p.max_blocks << a.p.bt_shift;
    const int len = (int)max((int64_t)0, min((int64_t)a.len[i], most));
    *full = len >> a.p.bt_shift;
    *tail = -1;
    if (len & ((1 << a.p.bt_shift) - 1)) {
        const int id = a.p.table[(int64_t)pr * a.p.max_blocks + *full];
        *tail = (uint32_t)id < (uint64_t)a.p.n_blocks ? id : -2;
    }
    return true;
}

// One workgroup: a fresh block for every fork whose parent ends inside one, in
// the order of the forks.
__global__ __launch_bounds__(kBlockThreads) void fork_take_kernel(ForkArgs a) {
    const int have = free_blocks(a.p);
    int taken = 0;
    for (int i0 = 0; i0 < a.n; i0 += kBlockThreads) {
        const int i = i0 + threadIdx.x;
        int full = 0, tail = -1, total;
        const bool ok = i < a.n && fork_of(a, i, &full, &tail);
        if (i < a.n && (!ok || tail == -2 || a.len[i] < 0 || a.len[i] > (a.p.max_blocks << a.p.bt_shift))) count_error(a.p);
        const bool want = ok && tail >= 0;
        const int k = taken + block_sum_before(want, &total);
        if (want) {
            int id = k < have ? a.p.free_list[have - 1 - k] : -1;
            if ((uint32_t)id < (uint64_t)a.p.n_blocks) {
                a.p.ref[id] = 1;
            } else {
                id = -1;
                count_error(a.p);
            }
            a.p.table[(int64_t)a.child[i] * a.p.max_blocks + full] = id;
        }
        taken += total;
    }
    if (threadIdx.x == 0) *a.p.free_count = have - min(have, taken);
}

// Workgroup (x, i): x = 0 shares fork i's whole blocks and clears the entries
// behind them; x > 0 copies a part of its last block.
__global__ __launch_bounds__(kBlockThreads) void fork_kernel(ForkArgs a) {
    const int i = blockIdx.y;
    int full, tail;
    if (!fork_of(a, i, &full, &tail)) return;
    const BlockPoolArgs &p = a.p;
    const int32_t *src = p.table + (int64_t)a.parent[i] * p.max_blocks;
    int32_t *dst = p.table + (int64_t)a.child[i] * p.max_blocks;
    if (blockIdx.x == 0) {
        for (int64_t j = threadIdx.x; j < p.max_blocks; j += kBlockThreads) {      // 64 bits: a row may have 2^31 - 1 entries
            if (j == full && tail >= 0) continue;
            int id = j < full ? src[j] : -1;
            if (id != -1 && (uint32_t)id >= (uint64_t)p.n_blocks) {
                count_error(p);
                id = -1;
            }
            if (id >= 0) atomicAdd(&p.ref[id], 1);
            dst[j] = id;
        }
        return;
    }
    if (tail < 0) return;
    const int id = dst[full];
    if (id >= 0) copy_block_part(p, tail, id, blockIdx.x - 1);
}

// --- extend ------------------------------------------------------------------

// One workgroup: a fresh block for every missing entry below ceil(len / block
// tokens), in the order of the rows and entries.
__global__ __launch_bounds__(kBlockThreads) void extend_kernel(BlockPoolArgs p, const int32_t *rows, const int32_t *len, int32_t n) {
    constexpr int E = 8;                           // entries of a thread
    const int have = free_blocks(p);
    const int64_t all = n * p.max_blocks;
    int taken = 0;
    for (int64_t e0 = 0; e0 < all; e0 += kBlockThreads * E) {
        const int64_t first = e0 + threadIdx.x * E;
        int32_t *at[E];
        int want = 0, total;
        int i = first >= all ? n : first >> 32 ? (int)(first / p.max_blocks) : (int)((uint32_t)first / (uint32_t)p.max_blocks);
        int64_t j = first - i * p.max_blocks;
        int row = i < n ? rows[i] : -1, tokens = i < n ? len[i] : 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            at[e] = nullptr;
            if (j == p.max_blocks) {
                j = 0;
                ++i;
                row = i < n ? rows[i] : -1;
                tokens = i < n ? len[i] : 0;
            }
            if (i < n) {
                const bool none = row < 0 || row >= p.n_rows;
                if (j == 0 && (none || tokens < 0 || tokens > (p.max_blocks << p.bt_shift))) count_error(p);
                if (!none && (j << p.bt_shift) < tokens) {
                    int32_t *entry = p.table + row * p.max_blocks + j;
                    if (*entry == -1) {
                        at[e] = entry;
                        ++want;
                    }
                }
            }
            ++j;
        }
        int k = taken + block_sum_before(want, &total);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (!at[e]) continue;
            const int id = k < have ? p.free_list[have - 1 - k] : -1;
            if ((uint32_t)id < (uint64_t)p.n_blocks) {
                p.ref[id] = 1;
                *at[e] = id;
            } else {
                count_error(p);
            }
            ++k;
        }
        taken += total;
    }
    if (threadIdx.x == 0) *p.free_count = have - min(have, taken);
}

// --- free --------------------------------------------------------------------

// Takes the entries of the rows back; a block whose last one goes is marked.
__global__ __launch_bounds__(256) void free_rows_kernel(BlockPoolArgs p, const int32_t *rows) {
    const int row = rows[blockIdx.y];
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (row < 0 || row >= p.n_rows) {
        if (j == 0) count_error(p);
        return;
    }
    if (j >= p.max_blocks) return;
    const int id = atomicExch(&p.table[row * p.max_blocks + j], -1);
    if (id == -1) return;
    if ((uint32_t)id >= (uint64_t)p.n_blocks) {
        count_error(p);
        return;
    }
    const int old = atomicSub(&p.ref[id], 1);
    if (old == 1) {
        atomicAdd(&p.ref[id], kFreed);
    } else if (old <= 0) {
        atomicAdd(&p.ref[id], 1);
        count_error(p);
    }
}

// One workgroup: the marked blocks go on the stack, ids ascending.  A wave takes
// 64 E ids at a time, 64 side by side.  E = 16 for large pools, whose passes are a
// chain; E = 4 up to kPushSmall ids, which are one pass (2.6 us where 16 take 4.4, with
// the counts in cache; 4.7 behind a large copy).
constexpr int kPushSmall = 4 * kBlockThreads;
template <int E>
__global__ __launch_bounds__(kBlockThreads) void free_push_kernel(BlockPoolArgs p) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int at = free_blocks(p);
    for (int64_t b0 = 0; b0 < p.n_blocks; b0 += kBlockThreads * E) {
        const int64_t first = b0 + wave * (64 * E) + lane;
        uint32_t marked = 0;
        int total;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int64_t id = first + 64 * e;
            if (p.ref[min(id, p.n_blocks - 1)] == kFreed && id < p.n_blocks) marked |= 1u << e;
        }
        int mine = 0;                              // of the wave: all, and those before this lane's e-th
        int before[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const uint64_t here = __ballot(marked >> e & 1);
            before[e] = mine + __popcll(here & ((1ull << lane) - 1));
            mine += __popcll(here);
        }
        const int k = at + __builtin_amdgcn_readfirstlane(block_sum_before(lane == 0 ? mine : 0, &total));
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (!(marked >> e & 1)) continue;
            const int64_t id = first + 64 * e;
            p.ref[id] = 0;
            if (k + before[e] < p.n_blocks) p.free_list[k + before[e]] = (int32_t)id;
        }
        at += total;
    }
    __syncthreads();
    if (threadIdx.x == 0) *p.free_count = (int)min((int64_t)at, p.n_blocks);
}

// --- compact -----------------------------------------------------------------

// Workspace of a compaction: live blocks of each 1,024 ids, then the sources and
// the destinations of the moves, in the same order, and each id's rank among the
// moves (ids that stay: 0; free ones: -1).
struct CompactArgs {
    BlockPoolArgs p;
    int32_t *counts, *src, *dst, *rank, *remap;
    int32_t n_chunks;
};

__global__ __launch_bounds__(kBlockThreads) void compact_count_kernel(CompactArgs a) {
    const int64_t id = (int64_t)blockIdx.x * kBlockThreads + threadIdx.x;
    int total;
    block_sum_before(id < a.p.n_blocks && a.p.ref[id] > 0, &total);
    if (threadIdx.x == 0) a.counts[blockIdx.x] = total;
}

// Live blocks (all, and below id `to` of a chunk's start), summed by one workgroup.
__device__ inline int counts_before(const CompactArgs &a, int to) {
    int x = 0, total;
    for (int i = threadIdx.x; i < to; i += kBlockThreads) x += a.counts[i];
    block_sum_before(x, &total);
    return total;
}

// With n live blocks: the k-th live id at or past n goes to the k-th free id
// below n.  Each workgroup ranks 1,024 ids.  SMALL (up to kCompactSmall chunks):
// each counts the whole pool itself, so that no launch has to do it before (5 us in
// one kernel, 2.2 + 4.4 and the gap between them in two, for 3,000 ids).
constexpr int kCompactSmall = 32;
template <bool SMALL>
__global__ __launch_bounds__(kBlockThreads) void compact_rank_kernel(CompactArgs a) {
    const BlockPoolArgs &p = a.p;
    int n, below, stay;
    if constexpr (SMALL) {
        uint32_t live = 0;                         // bit c: id 1,024 c + thread
#pragma unroll 8
        for (int c = 0; c < a.n_chunks; ++c) {
            const int id = c * kBlockThreads + threadIdx.x;
            if (p.ref[min((int64_t)id, p.n_blocks - 1)] > 0 && id < p.n_blocks) live |= 1u << c;
        }
        block_sum_before(__popc(live), &n);
        block_sum_before(__popc(live & ((1u << blockIdx.x) - 1)), &below);
        const int whole = n / kBlockThreads + ((int)threadIdx.x < n % kBlockThreads);      // of this thread's ids, those below n
        block_sum_before(__popc(whole < 32 ? live & ((1u << whole) - 1) : live), &stay);
    } else {
        n = counts_before(a, a.n_chunks);
        below = counts_before(a, blockIdx.x);
        // live ids below n: whole chunks, then the chunk that n falls into
        const int cn = n / kBlockThreads;
        int in_chunk;
        const int64_t id = (int64_t)cn * kBlockThreads + threadIdx.x;
        block_sum_before(id < n && id < p.n_blocks && p.ref[id] > 0, &in_chunk);
        stay = counts_before(a, cn) + in_chunk;
    }
    const int64_t id = (int64_t)blockIdx.x * kBlockThreads + threadIdx.x;
    const bool live = id < p.n_blocks && p.ref[id] > 0;
    int total;
    const int rank = below + block_sum_before(live, &total);
    if (id >= p.n_blocks) return;
    if (id < n) {
        if (!live) a.dst[id - rank] = (int32_t)id;
        a.rank[id] = live ? 0 : -1;
    } else {
        if (live) a.src[rank - stay] = (int32_t)id;
        a.rank[id] = live ? rank - stay : -1;
    }
    if (id == p.n_blocks - 1) {
        a.counts[a.n_chunks] = n;
        a.counts[a.n_chunks + 1] = n - stay;       // moves
    }
}

// Moves: workgroups [0, copy_blocks) stride over (move, part); then the table's
// entries, 1,024 a workgroup; then the stack and the new ids, 1,024 ids each.
__global__ __launch_bounds__(kBlockThreads) void compact_move_kernel(CompactArgs a, int32_t copy_blocks, int32_t parts,
                                                                     int32_t table_blocks) {
    const BlockPoolArgs &p = a.p;
    const int n = a.counts[a.n_chunks], moves = a.counts[a.n_chunks + 1];
    int b = blockIdx.x;
    if (b < copy_blocks) {
        for (int64_t x = b; x < (int64_t)moves * parts; x += copy_blocks) {
            const int k = (int)(x / parts), part = (int)(x - (int64_t)k * parts);
            copy_block_part(p, a.src[k], a.dst[k], part);
        }
        return;
    }
    b -= copy_blocks;
    if (b < table_blocks) {
        const int64_t e = (int64_t)b * kBlockThreads + threadIdx.x;
        if (e >= p.n_rows * p.max_blocks) return;
        const int id = p.table[e];
        if (id == -1) return;
        if ((uint32_t)id >= (uint64_t)p.n_blocks) {
            count_error(p);
            return;
        }
        const int k = a.rank[id];
        if (k < 0) {                               // a free block: left there, the entry would name what moves in
            p.table[e] = -1;
            count_error(p);
        } else if (id >= n) {
            p.table[e] = a.dst[k];
        }
        return;
    }
    b -= table_blocks;
    const int64_t id = (int64_t)b * kBlockThreads + threadIdx.x;
    if (id >= p.n_blocks) return;
    const int k = a.rank[id];
    if (id >= n) {
        if (k >= 0) p.ref[a.dst[k]] = p.ref[id];
        p.ref[id] = 0;
        p.free_list[p.n_blocks - 1 - id] = (int32_t)id;
    }
    if (a.remap) a.remap[id] = k < 0 ? -1 : id >= n ? a.dst[k] : (int32_t)id;
    if (id == 0) *p.free_count = (int)(p.n_blocks - n);
}

// --- new keys and values -----------------------------------------------------

struct KvWriteArgs {
    const void *k, *v;
    int64_t k_stride, v_stride;    // elements from one token to the next
    char *ck, *cv;                 // the layer's keys and values in block 0
    int64_t block_bytes, max_blocks, n_tokens, first_token;    // first_token: the launch's
    const int32_t *table, *cu, *kv_len;
    int32_t *err;
    float k_scale, v_scale;        // what a stored 8-bit 1 stands for
    int32_t n_seqs, kv_heads, n_blocks, bt_shift;
};

constexpr int kWriteTokens = 4;    // tokens a workgroup writes, one for each wave

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

// Four values to e4m3: beyond the largest finite value they become it, NaN stays.
__device__ inline uint32_t fp8_of4(const float *x) {
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = x[i] != x[i] ? x[i] : fminf(fmaxf(x[i], -448.f), 448.f);
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], r, true);
}

// A wave writes one token: 8 values of a key and a value row at a time, 16-byte
// loads; what it needs to find the place (the sequence, its length, the block) is a
// chain of four loads, which bounds small calls (64 tokens: 3.6 us); large ones are
// bound by memory (47,248 tokens x 8 heads x 128 into an 8-bit cache: 58 us, 5.0
// TB/s of reads and writes, what a large copy reaches).
template <typename T, typename C, int D>
__global__ __launch_bounds__(256) void kv_write_kernel(KvWriteArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t tok = a.first_token + (int64_t)blockIdx.x * kWriteTokens + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (tok >= a.n_tokens) return;
    int seq, first, end;
    if (!sequence_of(a.cu, a.n_seqs, (int)tok, &seq, &first, &end)) return;
    const int pos = a.kv_len[seq] - (end - (int)tok);
    const int64_t j = pos >> a.bt_shift;
    const int id = pos >= 0 && j < a.max_blocks ? a.table[seq * a.max_blocks + j] : -1;
    if ((uint32_t)id >= (uint32_t)a.n_blocks) {
        if (lane == 0 && a.err) atomicAdd(a.err, 1);
        return;
    }
    const int slot = pos & ((1 << a.bt_shift) - 1);
    constexpr int V = D / 8;                        // 8-value pieces of a row
    const int pieces = a.kv_heads * V;
    for (int e = lane; e < 2 * pieces; e += 64) {
        const bool is_v = e >= pieces;
        const int x = is_v ? e - pieces : e, h = x / V, p = x % V;
        const T *src = is_v ? (const T *)a.v + tok * a.v_stride : (const T *)a.k + tok * a.k_stride;
        src += h * D + p * 8;
        char *dst = (is_v ? a.cv : a.ck) + id * a.block_bytes +
                    (((int64_t)h << a.bt_shift) + slot) * (int64_t)(D * sizeof(C)) + p * (int)(8 * sizeof(C));
        if constexpr (sizeof(C) == 1) {
            const uint4 raw = *(const uint4 *)src;
            const uint32_t *w = &raw.x;
            const float scale = is_v ? a.v_scale : a.k_scale;
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = __uint_as_float((i & 1) ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16) / scale;
            *(uint2 *)dst = make_uint2(fp8_of4(f), fp8_of4(f + 4));
        } else if constexpr (sizeof(C) == 2) {
            *(uint4 *)dst = *(const uint4 *)src;
        } else {
            const uint4 x0 = *(const uint4 *)src, x1 = *((const uint4 *)src + 1);
            *(uint4 *)dst = x0;
            *((uint4 *)dst + 1) = x1;
        }
    }
}

}  // namespace la
