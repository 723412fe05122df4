// C ABI of the attention side of the library (gfx950): attention of prompts and
// of single tokens over packed or cached keys, writes into the cache, and the
// bookkeeping of its blocks.  Host side: argument checks, workspace sizes and
// launches.  Kernels live in the headers included below.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "linattn.h"
#include "la_host.h"
#include "attn_tile.h"
#include "attn_rows.h"
#include "attn_wide.h"
#include "blocks.h"
#include "kv_codes.h"

namespace {

using la::host::aligned16;
using la::host::fail;
using la::host::hip_check;

constexpr int64_t kMaxInt = 0x7fffffff;
// A launch has fewer than 2^32 threads along an axis: workgroups of `threads`, at most.
constexpr int64_t max_grid(int threads) { return 0xffffffffll / threads; }

int64_t dtype_size(int32_t d) { return d == LA_F32 ? 4 : d == LA_BF16 ? 2 : 1; }
bool block_scaled(int32_t d) { return d == LA_FP8_E4M3_BLOCK || d == LA_INT8_BLOCK; }
int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }
int shift_of(int32_t pow2) { return __builtin_ctz((unsigned)pow2); }

la_status check_attn_shape(const la_attn_shape *s) {
    if (!s) return fail(LA_ERR_INVALID_ARG, "shape is NULL");
    if (s->n_seqs < 1 || s->q_heads < 1 || s->kv_heads < 1)
        return fail(LA_ERR_INVALID_ARG, "n_seqs=%d, q_heads=%d, kv_heads=%d must be positive", s->n_seqs, s->q_heads, s->kv_heads);
    if (s->q_heads % s->kv_heads != 0)
        return fail(LA_ERR_INVALID_ARG, "q_heads=%d is no multiple of kv_heads=%d", s->q_heads, s->kv_heads);
    if (s->io_dtype != LA_F32 && s->io_dtype != LA_BF16)
        return fail(LA_ERR_INVALID_ARG, "io_dtype=%d must be LA_F32 or LA_BF16", s->io_dtype);
    if (s->head_dim != 64 && s->head_dim != 128)
        return fail(LA_ERR_UNSUPPORTED, "head_dim=%d: 64 and 128 are built", s->head_dim);
    if (!(s->scale > 0.f) || !std::isfinite(s->scale))
        return fail(LA_ERR_INVALID_ARG, "scale=%g must be positive and finite", (double)s->scale);
    return LA_OK;
}

// What a score is multiplied by to become a base-2 exponent.  Masked scores are
// minus infinity when they are multiplied, so it may not have become zero.
la_status exponent_scale(const la_attn_shape *s, float k_scale, float *out) {
    *out = s->scale * k_scale * la::kAttnLog2e;
    if (!std::isnormal(*out))
        return fail(LA_ERR_INVALID_ARG, "scale=%g times k_scale=%g is out of fp32's range", (double)s->scale, (double)k_scale);
    return LA_OK;
}

// A token stride in elements: 0 stands for packed rows.
la_status token_stride(int64_t given, int64_t heads, const la_attn_shape *s, const char *what, int64_t *out) {
    const int64_t packed = heads * s->head_dim;
    *out = given ? given : packed;
    if (*out < packed || *out > ((int64_t)1 << 24) || *out * dtype_size(s->io_dtype) % 16 != 0)
        return fail(LA_ERR_INVALID_ARG, "%s=%lld must be at least %lld, at most 2^24 and a multiple of 16 bytes", what,
                    (long long)*out, (long long)packed);
    return LA_OK;
}

la_status check_layer(const la_kv_layer *y, int32_t io_dtype) {
    if (!y) return fail(LA_ERR_INVALID_ARG, "layer is NULL");
    if (y->dtype != LA_F32 && y->dtype != LA_BF16 && y->dtype != LA_FP8_E4M3 && !block_scaled(y->dtype))
        return fail(LA_ERR_INVALID_ARG, "cache dtype=%d", y->dtype);
    if ((y->dtype == LA_F32) != (io_dtype == LA_F32))
        return fail(LA_ERR_UNSUPPORTED, "an fp32 cache goes with fp32 queries, a bf16 or 8-bit one with bf16");
    if (y->kv_heads < 1) return fail(LA_ERR_INVALID_ARG, "kv_heads=%d", y->kv_heads);
    if (y->head_dim != 64 && y->head_dim != 128)
        return fail(LA_ERR_UNSUPPORTED, "head_dim=%d: 64 and 128 are built", y->head_dim);
    const int32_t bt = y->block_tokens;
    if (bt < 16 || bt > 256 || (bt & (bt - 1)))
        return fail(LA_ERR_UNSUPPORTED, "block_tokens=%d: powers of two from 16 to 256 are built", bt);
    if (y->n_blocks < 1 || y->n_blocks > 0x7fffffff) return fail(LA_ERR_INVALID_ARG, "n_blocks=%lld", (long long)y->n_blocks);
    const int64_t part = (int64_t)y->kv_heads * bt * y->head_dim * dtype_size(y->dtype);
    if (y->block_bytes < 0 || y->block_bytes % 16 || y->k_offset < 0 || y->v_offset < 0 || y->k_offset % 16 || y->v_offset % 16 ||
        y->k_offset > y->block_bytes - part || y->v_offset > y->block_bytes - part)
        return fail(LA_ERR_INVALID_ARG, "keys at %lld and values at %lld (%lld bytes each) must lie in a block of %lld bytes, on 16-byte lines",
                    (long long)y->k_offset, (long long)y->v_offset, (long long)part, (long long)y->block_bytes);
    if (y->k_offset < y->v_offset + part && y->v_offset < y->k_offset + part)
        return fail(LA_ERR_INVALID_ARG, "keys and values overlap in the block");
    if (!(y->k_scale > 0.f) || !(y->v_scale > 0.f) || !std::isfinite(y->k_scale) || !std::isfinite(y->v_scale))
        return fail(LA_ERR_INVALID_ARG, "k_scale=%g and v_scale=%g must be positive and finite", (double)y->k_scale, (double)y->v_scale);
    if (y->dtype != LA_FP8_E4M3 && (y->k_scale != 1.f || y->v_scale != 1.f))
        return fail(LA_ERR_INVALID_ARG, "k_scale and v_scale other than 1 go with an 8-bit cache of one scale");
    if (block_scaled(y->dtype)) {
        const int64_t size = 4 * (int64_t)y->kv_heads, ks = y->k_scales, vs = y->v_scales;
        if (ks < 0 || vs < 0 || ks % 4 || vs % 4 || ks > y->block_bytes - size || vs > y->block_bytes - size)
            return fail(LA_ERR_INVALID_ARG, "scales at %lld and %lld (%lld bytes each) must lie in a block of %lld bytes, on 4-byte lines",
                        (long long)ks, (long long)vs, (long long)size, (long long)y->block_bytes);
        auto meet = [](int64_t a, int64_t n, int64_t b, int64_t m) { return a < b + m && b < a + n; };
        if (meet(ks, size, vs, size) || meet(ks, size, y->k_offset, part) || meet(ks, size, y->v_offset, part) ||
            meet(vs, size, y->k_offset, part) || meet(vs, size, y->v_offset, part))
            return fail(LA_ERR_INVALID_ARG, "scales overlap keys, values or one another in the block");
    }
    if (y->max_blocks < 1 || y->max_blocks > 0x7fffff00 / bt)
        return fail(LA_ERR_INVALID_ARG, "max_blocks=%lld must be positive and cover fewer than 2^31 tokens", (long long)y->max_blocks);
    if (!y->block_table) return fail(LA_ERR_INVALID_ARG, "block_table is required");
    if (!y->cache || !aligned16(y->cache))
        return fail(LA_ERR_INVALID_ARG, "cache is required, 16-byte aligned");
    return LA_OK;
}

la_status check_layer_of(const la_kv_layer *y, const la_attn_shape *s) {
    if (la_status e = check_layer(y, s->io_dtype)) return e;
    if (y->kv_heads != s->kv_heads || y->head_dim != s->head_dim)
        return fail(LA_ERR_INVALID_ARG, "the layer has %d heads of %d, the shape %d of %d", y->kv_heads, y->head_dim, s->kv_heads,
                    s->head_dim);
    return LA_OK;
}

la::KvSource cached(const la_kv_layer *y) {
    la::KvSource k{};
    k.k = (const char *)y->cache + y->k_offset;
    k.v = (const char *)y->cache + y->v_offset;
    k.block_bytes = y->block_bytes;
    k.table = y->block_table;
    k.max_blocks = y->max_blocks;
    k.n_blocks = (int32_t)y->n_blocks;
    k.bt_shift = shift_of(y->block_tokens);
    k.err = y->err_count;
    if (block_scaled(y->dtype)) {
        k.ks = (const char *)y->cache + y->k_scales;
        k.vs = (const char *)y->cache + y->v_scales;
    }
    return k;
}

// --- prompts -----------------------------------------------------------------

// Workgroups of a split call, at most: two on every CU; fp32, whose products take
// eight times as long and whose partial sums so weigh less, eight.  (256 tokens at
// 3,328 x 8 heads: 77 us whole, 23 split; three fp32 prompts of 1,791, 640 and 257:
// 101 whole, 61 split.)
constexpr int64_t prompt_grid(bool f32) { return f32 ? 2048 : 512; }

struct PromptPlan {
    int64_t tokens = 0, items = 0;      // items: row tiles times parts, of one key head
    int64_t slots = 0, joins = 0;       // (row, part) results in the workspace; workgroups that join them
    int32_t max_kv = 0;
    int part_shift = 0;                 // keys of a part, as a power of two; 0: rows are not split
    bool ordered = false;
    uint8_t order[64];                  // sequences, the longest first
};

la_status plan_prompt(const la_attn_shape *s, const int32_t *cu, const int32_t *kv_len, PromptPlan *p) {
    if (!cu) return fail(LA_ERR_INVALID_ARG, "cu_seqlens_host is required");
    if (cu[0] != 0) return fail(LA_ERR_INVALID_ARG, "cu_seqlens[0]=%d", cu[0]);
    const int64_t group = s->q_heads / s->kv_heads;
    const bool f32 = s->io_dtype == LA_F32;
    auto keys_of = [&](int i) { return kv_len ? kv_len[i] : cu[i + 1] - cu[i]; };
    auto tiles = [&](int rows, int shift) {
        int64_t n = 0;
        for (int i = 0; i < s->n_seqs; ++i) n += up((cu[i + 1] - cu[i]) * group, rows) * la::prompt_parts(keys_of(i), shift);
        return n;
    };
    for (int i = 0; i < s->n_seqs; ++i) {
        const int64_t n = (int64_t)cu[i + 1] - cu[i];
        if (n < 0) return fail(LA_ERR_INVALID_ARG, "cu_seqlens decreases at sequence %d", i);
        if (n * group > 0x7fffff00) return fail(LA_ERR_INVALID_ARG, "sequence %d is too long for one launch", i);
        if (keys_of(i) < 0) return fail(LA_ERR_INVALID_ARG, "kv_len[%d]=%d", i, keys_of(i));
        p->max_kv = std::max(p->max_kv, keys_of(i));
    }
    p->tokens = cu[s->n_seqs];
    const int tile = f32 ? la::kTileRows : la::kPromptRows;
    p->items = tiles(tile, 0);
    // two parts save no more than joining them costs (512 tokens x 8 heads: 15.5 us whole, 15.7 in two)
    if (p->items * s->kv_heads <= prompt_grid(f32) / 2 && p->max_kv > 2 << la::kPromptPartShift)
        for (int shift = la::kPromptPartShift; (1 << shift) < p->max_kv; ++shift) {
            const int64_t n = tiles(tile, shift);
            if (n * s->kv_heads > prompt_grid(f32)) continue;
            p->part_shift = shift;
            p->items = n;
            break;
        }
    // A long sequence's tiles that begin late are what a large call ends on (16 prompts
    // with suffixes of 80 to 8,064 tokens: 615 us, 700 in the caller's order).
    if (!p->part_shift && s->n_seqs > 1 && s->n_seqs <= 64 && p->items * s->kv_heads > prompt_grid(f32)) {
        p->ordered = true;
        for (int i = 0; i < s->n_seqs; ++i) p->order[i] = (uint8_t)i;
        std::stable_sort(p->order, p->order + s->n_seqs, [&](int x, int y) { return keys_of(x) > keys_of(y); });
    }
    if (p->part_shift)
        for (int i = 0; i < s->n_seqs; ++i) {
            const int64_t rows = (int64_t)(cu[i + 1] - cu[i]) * s->q_heads, parts = la::prompt_parts(keys_of(i), p->part_shift);
            if (parts == 1) continue;
            p->slots += rows * parts;
            p->joins += up(rows, 1024 / s->head_dim);
        }
    static_assert(la::kWideThreads == 256 && la::kTileThreads == 256, "workgroups of a prompt");
    if (p->items * s->kv_heads > max_grid(256) || p->joins > max_grid(256) || p->slots > kMaxInt)
        return fail(LA_ERR_INVALID_ARG, "too many row tiles for one launch");
    return LA_OK;
}

size_t parts_bytes(int64_t slots, int d) { return (size_t)slots * (d * sizeof(float) + sizeof(float2)); }

void carve_parts(la::AttnArgs *a, void *ws, int64_t slots, int d) {
    a->part_o = (float *)ws;
    a->part_ml = (float2 *)((char *)ws + (size_t)slots * d * sizeof(float));
}

template <typename T, typename C, int D, bool PAGED>
la_status launch_prompt(const la::AttnArgs &a, const PromptPlan &p, hipStream_t st) {
    const dim3 grid((unsigned)(p.items * a.kv_heads));
    if constexpr (sizeof(T) == 2)
        hipLaunchKernelGGL((la::attn_wide_kernel<C, D, PAGED>), grid, dim3(la::kWideThreads), 0, st, a);
    else hipLaunchKernelGGL((la::attn_tile_kernel<D, PAGED>), grid, dim3(la::kTileThreads), 0, st, a);
    if (la_status e = hip_check("attention prompt launch")) return e;
    if (p.joins == 0) return LA_OK;
    hipLaunchKernelGGL((la::attn_join_prompt_kernel<T, D>), dim3((unsigned)p.joins), dim3(256), 0, st, a);
    return hip_check("attention join launch");
}

template <typename T, typename C, bool PAGED>
la_status prompt_of_dim(int d, const la::AttnArgs &a, const PromptPlan &p, hipStream_t st) {
    return d == 64 ? launch_prompt<T, C, 64, PAGED>(a, p, st) : launch_prompt<T, C, 128, PAGED>(a, p, st);
}

la_status run_prompt(const la_attn_shape *s, la::AttnArgs &a, const la_kv_layer *layer, const PromptPlan &p, void *ws,
                     size_t ws_bytes, hipStream_t st) {
    const size_t need = parts_bytes(p.slots, s->head_dim);
    if (need && (!ws || ws_bytes < need))
        return fail(LA_ERR_WORKSPACE, "workspace of %zu bytes, %zu required", ws ? ws_bytes : 0, need);
    if (need && !aligned16(ws)) return fail(LA_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    a.kv_heads = s->kv_heads;
    a.group = s->q_heads / s->kv_heads;
    a.by_group = la::FastDiv::by((uint32_t)a.group);
    a.by_kv_heads = la::FastDiv::by((uint32_t)a.kv_heads);
    a.n_seqs = s->n_seqs;
    a.max_kv = p.max_kv;
    a.part_shift = p.part_shift;
    a.ordered = p.ordered;
    if (p.ordered) std::copy(p.order, p.order + 64, a.order);
    carve_parts(&a, ws, p.slots, s->head_dim);
    (void)hipGetLastError();
    const int d = s->head_dim;
    if (!layer)
        return s->io_dtype == LA_F32 ? prompt_of_dim<float, float, false>(d, a, p, st) : prompt_of_dim<__bf16, __bf16, false>(d, a, p, st);
    if (layer->dtype == LA_F32) return prompt_of_dim<float, float, true>(d, a, p, st);
    if (layer->dtype == LA_BF16) return prompt_of_dim<__bf16, __bf16, true>(d, a, p, st);
    if (layer->dtype == LA_FP8_E4M3_BLOCK) return prompt_of_dim<__bf16, la::e4m3_code, true>(d, a, p, st);
    if (layer->dtype == LA_INT8_BLOCK) return prompt_of_dim<__bf16, la::int8_code, true>(d, a, p, st);
    return prompt_of_dim<__bf16, la::fp8_t, true>(d, a, p, st);
}

la_status check_qo(const la_attn_shape *s, const void *q, const void *o, la::AttnArgs *a) {
    if (!q || !o) return fail(LA_ERR_INVALID_ARG, "q and o are required");
    if (!aligned16(q) || !aligned16(o)) return fail(LA_ERR_INVALID_ARG, "q and o must be 16-byte aligned");
    if (la_status e = token_stride(s->q_stride, s->q_heads, s, "q_stride", &a->q_stride)) return e;
    if (la_status e = token_stride(s->o_stride, s->q_heads, s, "o_stride", &a->o_stride)) return e;
    a->q = q;
    a->o = const_cast<void *>(o);
    return LA_OK;
}

// --- decode ------------------------------------------------------------------

// Workgroups for own keys: two on every CU.  Those of shared prefixes come on top and
// start first; the own keys' follow as they end.  Three on every CU where a cache in one
// byte a value is read and nothing is shared.
constexpr int kRowsGrid = 512, kOwnRowsGrid = 768;

struct DecodePlan {
    int own_parts, prefix_parts;
    bool direct;                       // one part each: no join
};

DecodePlan plan_decode(int64_t max_kv_len, int64_t max_prefix) {
    DecodePlan p{};
    p.own_parts = (int)std::max<int64_t>(1, up(max_kv_len, la::kOwnPart));
    p.prefix_parts = (int)up(max_prefix, la::kPrefixPart);
    p.direct = p.own_parts == 1 && p.prefix_parts == 0;
    return p;
}

la_status check_decode_sizes(const la_attn_shape *s, int64_t max_kv_len, int64_t max_prefix_len) {
    if (la_status e = check_attn_shape(s)) return e;
    if (max_kv_len < 0 || max_kv_len > 0x7fffff00 || max_prefix_len < 0 || max_prefix_len > max_kv_len)
        return fail(LA_ERR_INVALID_ARG, "max_kv_len=%lld, max_prefix_len=%lld", (long long)max_kv_len, (long long)max_prefix_len);
    return LA_OK;
}

template <typename T, typename C, int D>
la_status launch_decode(const la::AttnArgs &a, int64_t rows_blocks, hipStream_t st) {
    bool own = false;
    if constexpr (sizeof(C) == 1) {
        own = a.prefix_items == 0;
        if (own) hipLaunchKernelGGL((la::attn_decode_own_kernel<T, C, D>), dim3((unsigned)rows_blocks), dim3(la::kRowsThreads), 0, st, a);
    }
    if (!own)
        hipLaunchKernelGGL((la::attn_decode_kernel<T, C, D>), dim3((unsigned)(a.prefix_items + rows_blocks)), dim3(la::kRowsThreads), 0,
                           st, a);
    if (la_status e = hip_check("attention decode launch")) return e;
    if (a.direct) return LA_OK;
    hipLaunchKernelGGL((la::attn_join_kernel<T, D>), dim3((unsigned)(a.n_seqs * a.kv_heads * a.group)), dim3(256), 0, st, a);
    return hip_check("attention join launch");
}

template <typename T, typename C>
la_status decode_of_dim(int d, const la::AttnArgs &a, int64_t rows_blocks, hipStream_t st) {
    return d == 64 ? launch_decode<T, C, 64>(a, rows_blocks, st) : launch_decode<T, C, 128>(a, rows_blocks, st);
}

// --- blocks ------------------------------------------------------------------

la_status check_pool(const la_block_pool *p, bool tables, bool bytes, la::BlockPoolArgs *a) {
    if (!p) return fail(LA_ERR_INVALID_ARG, "pool is NULL");
    if (p->n_blocks < 0 || p->n_blocks > 0x3fffffff) return fail(LA_ERR_INVALID_ARG, "n_blocks=%lld", (long long)p->n_blocks);
    if (bytes) {
        if (p->block_bytes < 16 || p->block_bytes % 16 || up(p->block_bytes / 16, la::kPartVec) > 65534)
            return fail(LA_ERR_INVALID_ARG, "block_bytes=%lld must be a positive multiple of 16 below 2 GB", (long long)p->block_bytes);
        if (p->n_blocks > 0 && (!p->cache || !aligned16(p->cache)))
            return fail(LA_ERR_INVALID_ARG, "cache is required, 16-byte aligned");
    }
    if (tables) {
        if (p->block_tokens < 1 || (p->block_tokens & (p->block_tokens - 1)))
            return fail(LA_ERR_INVALID_ARG, "block_tokens=%d must be a power of two", p->block_tokens);
        if (p->n_rows < 0 || p->n_rows > 0x7fffffff || p->max_blocks < 1 || p->max_blocks > 0x7fffffff / p->block_tokens)
            return fail(LA_ERR_INVALID_ARG, "a table of %lld rows of %lld blocks", (long long)p->n_rows, (long long)p->max_blocks);
        if (!p->table || !p->ref_count || !p->free_list || !p->free_count)
            return fail(LA_ERR_INVALID_ARG, "table, ref_count, free_list and free_count are required");
    }
    a->cache = (char *)p->cache;
    a->block_vec = p->block_bytes / 16;
    a->n_blocks = p->n_blocks;
    a->n_rows = p->n_rows;
    a->max_blocks = p->max_blocks;
    a->bt_shift = tables ? shift_of(p->block_tokens) : 0;
    a->table = p->table;
    a->ref = p->ref_count;
    a->free_list = p->free_list;
    a->free_count = p->free_count;
    a->err = p->err_count;
    return LA_OK;
}

la_status check_rows(const void *rows, int64_t n, const char *what) {
    if (n < 0 || n > 65535) return fail(LA_ERR_INVALID_ARG, "%s: %lld rows, at most 65535 in one call", what, (long long)n);
    if (n > 0 && !rows) return fail(LA_ERR_INVALID_ARG, "%s: row lists are required", what);
    return LA_OK;
}

template <typename T, typename C>
la_status launch_kv_write(int d, la::KvWriteArgs &a, hipStream_t st) {
    constexpr int64_t STEP = max_grid(256) * la::kWriteTokens;
    for (a.first_token = 0; a.first_token < a.n_tokens; a.first_token += STEP) {
        const dim3 grid((unsigned)up(std::min(a.n_tokens - a.first_token, STEP), la::kWriteTokens));
        if (d == 64) hipLaunchKernelGGL((la::kv_write_kernel<T, C, 64>), grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((la::kv_write_kernel<T, C, 128>), grid, dim3(256), 0, st, a);
        if (la_status e = hip_check("cache write launch")) return e;
    }
    return LA_OK;
}

// P: pieces of 8 values a lane holds of a unit.
template <typename C, int D, int P>
la_status launch_kv_codes_of(la::KvCodesArgs &a, int waves, hipStream_t st) {
    a.team_shift = shift_of(waves);
    a.unit_groups = (int32_t)up(2 * (int64_t)a.w.kv_heads * waves, 4);
    const int64_t groups = ((a.w.n_tokens >> a.w.bt_shift) + 2 * (int64_t)a.w.n_seqs) * a.unit_groups, step = max_grid(256);
    for (a.first_group = 0; a.first_group < groups; a.first_group += step) {
        const dim3 grid((unsigned)std::min(groups - a.first_group, step));
        hipLaunchKernelGGL((la::kv_write_codes_kernel<C, D, P>), grid, dim3(256), 0, st, a);
        if (la_status e = hip_check("cache write launch")) return e;
    }
    return LA_OK;
}

// One wave a unit while its registers hold it, four beyond (39,934 tokens x 8 heads: blocks
// of 128 x 128 values in four waves of 8 pieces 53 us, in two of 16 56; blocks of 64 x 128
// in one wave of 16 pieces 53, in two of 8 54).
template <typename C, int D>
la_status launch_kv_codes(la::KvCodesArgs &a, hipStream_t st) {
    const int pieces = (D / 8 << a.w.bt_shift) / 64;           // of a unit for each lane of a wave
    if constexpr (D == 64) {
        if (pieces == 2) return launch_kv_codes_of<C, D, 2>(a, 1, st);
    }
    switch (pieces) {
    case 4: return launch_kv_codes_of<C, D, 4>(a, 1, st);
    case 8: return launch_kv_codes_of<C, D, 8>(a, 1, st);
    case 16: return launch_kv_codes_of<C, D, 16>(a, 1, st);
    case 32: return launch_kv_codes_of<C, D, 8>(a, 4, st);
    default: return launch_kv_codes_of<C, D, 16>(a, 4, st);
    }
}

template <typename T, typename C>
la_status launch_kv_read(int d, const la::KvWriteArgs &w, hipStream_t st) {
    la::KvReadArgs a{};
    a.w = w;
    a.lanes = (int32_t)std::min<int64_t>(64, up(2 * (int64_t)w.kv_heads * d * (int64_t)sizeof(T) / 16, 4));
    a.by_lanes = la::FastDiv::by((uint32_t)a.lanes);
    const int64_t tokens = 64 / a.lanes * la::kWriteTokens, step = max_grid(256) * tokens;    // of a workgroup, of a launch
    for (a.w.first_token = 0; a.w.first_token < w.n_tokens; a.w.first_token += step) {
        const dim3 grid((unsigned)up(std::min(w.n_tokens - a.w.first_token, step), tokens));
        if (d == 64) hipLaunchKernelGGL((la::kv_read_kernel<T, C, 64>), grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((la::kv_read_kernel<T, C, 128>), grid, dim3(256), 0, st, a);
        if (la_status e = hip_check("cache read launch")) return e;
    }
    return LA_OK;
}

// Arguments of a call that writes or reads the rows of a layer; *n_tokens 0: nothing to do.
la_status kv_rows_args(const la_kv_layer *layer, int32_t io_dtype, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                       const int32_t *cu_seqlens_dev, int32_t n_seqs, int64_t n_tokens, const int32_t *kv_len_dev, la::KvWriteArgs *a) {
    if (n_seqs < 0 || n_tokens < 0 || n_tokens > 0x7fffff00)
        return fail(LA_ERR_INVALID_ARG, "n_seqs=%d, n_tokens=%lld", n_seqs, (long long)n_tokens);
    a->n_tokens = n_seqs == 0 ? 0 : n_tokens;
    if (a->n_tokens == 0) return LA_OK;
    if (!k || !v || !cu_seqlens_dev || !kv_len_dev) return fail(LA_ERR_INVALID_ARG, "k, v, cu_seqlens_dev and kv_len_dev are required");
    if (!aligned16(k) || !aligned16(v)) return fail(LA_ERR_INVALID_ARG, "k and v must be 16-byte aligned");
    la_attn_shape s{};
    s.head_dim = layer->head_dim;
    s.io_dtype = io_dtype;
    if (la_status e = token_stride(k_stride, layer->kv_heads, &s, "k_stride", &a->k_stride)) return e;
    if (la_status e = token_stride(v_stride, layer->kv_heads, &s, "v_stride", &a->v_stride)) return e;
    a->k = k;
    a->v = v;
    a->ck = (char *)layer->cache + layer->k_offset;
    a->cv = (char *)layer->cache + layer->v_offset;
    if (block_scaled(layer->dtype)) {
        a->ks = (char *)layer->cache + layer->k_scales;
        a->vs = (char *)layer->cache + layer->v_scales;
    }
    a->block_bytes = layer->block_bytes;
    a->max_blocks = layer->max_blocks;
    a->table = layer->block_table;
    a->cu = cu_seqlens_dev;
    a->kv_len = kv_len_dev;
    a->err = layer->err_count;
    a->k_scale = layer->k_scale;
    a->v_scale = layer->v_scale;
    a->n_seqs = n_seqs;
    a->kv_heads = layer->kv_heads;
    a->n_blocks = (int32_t)layer->n_blocks;
    a->bt_shift = shift_of(layer->block_tokens);
    return LA_OK;
}

}  // namespace

extern "C" {

size_t la_attn_prefill_workspace_bytes(const la_attn_shape *shape, const int32_t *cu_seqlens_host, const int32_t *kv_len_host) {
    PromptPlan p;
    if (check_attn_shape(shape) || plan_prompt(shape, cu_seqlens_host, kv_len_host, &p)) return 0;
    return std::max<size_t>(16, parts_bytes(p.slots, shape->head_dim));
}

la_status la_attn_prefill(const la_attn_shape *shape, const void *q, const void *k, const void *v, const int32_t *cu_seqlens_dev,
                          const int32_t *cu_seqlens_host, void *o, void *workspace, size_t ws_bytes, void *stream) {
    if (la_status e = check_attn_shape(shape)) return e;
    PromptPlan p;
    if (la_status e = plan_prompt(shape, cu_seqlens_host, nullptr, &p)) return e;
    if (p.tokens == 0) return LA_OK;
    la::AttnArgs a{};
    if (la_status e = check_qo(shape, q, o, &a)) return e;
    if (!k || !v || !cu_seqlens_dev) return fail(LA_ERR_INVALID_ARG, "k, v and cu_seqlens_dev are required");
    if (!aligned16(k) || !aligned16(v)) return fail(LA_ERR_INVALID_ARG, "k and v must be 16-byte aligned");
    int64_t ks, vs;
    if (la_status e = token_stride(shape->k_stride, shape->kv_heads, shape, "k_stride", &ks)) return e;
    if (la_status e = token_stride(shape->v_stride, shape->kv_heads, shape, "v_stride", &vs)) return e;
    a.kv.k = (const char *)k;
    a.kv.v = (const char *)v;
    a.kv.k_stride = ks * dtype_size(shape->io_dtype);
    a.kv.v_stride = vs * dtype_size(shape->io_dtype);
    a.cu = cu_seqlens_dev;
    if (la_status e = exponent_scale(shape, 1.f, &a.c)) return e;
    a.v_scale = 1.f;
    return run_prompt(shape, a, nullptr, p, workspace, ws_bytes, (hipStream_t)stream);
}

la_status la_attn_prefill_paged(const la_attn_shape *shape, const la_kv_layer *layer, const void *q, const int32_t *cu_seqlens_dev,
                                const int32_t *cu_seqlens_host, const int32_t *kv_len_dev, const int32_t *kv_len_host, void *o,
                                void *workspace, size_t ws_bytes, void *stream) {
    if (la_status e = check_attn_shape(shape)) return e;
    if (la_status e = check_layer_of(layer, shape)) return e;
    if (!kv_len_host) return fail(LA_ERR_INVALID_ARG, "kv_len_host is required");
    PromptPlan p;
    if (la_status e = plan_prompt(shape, cu_seqlens_host, kv_len_host, &p)) return e;
    if (p.tokens == 0) return LA_OK;
    if (p.max_kv > layer->max_blocks * layer->block_tokens)
        return fail(LA_ERR_INVALID_ARG, "kv_len reaches %d, the block table %lld tokens", p.max_kv,
                    (long long)(layer->max_blocks * layer->block_tokens));
    la::AttnArgs a{};
    if (la_status e = check_qo(shape, q, o, &a)) return e;
    if (!cu_seqlens_dev || !kv_len_dev) return fail(LA_ERR_INVALID_ARG, "cu_seqlens_dev and kv_len_dev are required");
    a.kv = cached(layer);
    a.cu = cu_seqlens_dev;
    a.kv_len = kv_len_dev;
    if (la_status e = exponent_scale(shape, layer->k_scale, &a.c)) return e;
    a.v_scale = layer->v_scale;
    return run_prompt(shape, a, layer, p, workspace, ws_bytes, (hipStream_t)stream);
}

size_t la_attn_decode_workspace_bytes(const la_attn_shape *shape, int64_t max_kv_len, int64_t max_prefix_len) {
    if (check_decode_sizes(shape, max_kv_len, max_prefix_len)) return 0;
    const DecodePlan p = plan_decode(max_kv_len, max_prefix_len);
    return p.direct ? 16 : parts_bytes((int64_t)shape->n_seqs * shape->q_heads * (p.own_parts + p.prefix_parts), shape->head_dim);
}

la_status la_attn_decode(const la_attn_shape *shape, const la_kv_layer *layer, const void *q, const int32_t *kv_len_dev,
                         int64_t max_kv_len, const la_prefix_groups *groups, void *o, void *workspace, size_t ws_bytes,
                         void *stream) {
    const int64_t max_prefix = groups && groups->n_groups > 0 ? groups->max_prefix_len : 0;
    if (la_status e = check_decode_sizes(shape, max_kv_len, max_prefix)) return e;
    if (la_status e = check_layer_of(layer, shape)) return e;
    if (max_kv_len > layer->max_blocks * layer->block_tokens)
        return fail(LA_ERR_INVALID_ARG, "max_kv_len=%lld, the block table covers %lld tokens", (long long)max_kv_len,
                    (long long)(layer->max_blocks * layer->block_tokens));
    la::AttnArgs a{};
    if (la_status e = check_qo(shape, q, o, &a)) return e;
    if (!kv_len_dev) return fail(LA_ERR_INVALID_ARG, "kv_len_dev is required");
    const bool shared = max_prefix > 0;
    if (groups && groups->n_groups < 0) return fail(LA_ERR_INVALID_ARG, "n_groups=%d", groups->n_groups);
    if (shared && (!groups->cu_group_dev || !groups->prefix_len_dev))
        return fail(LA_ERR_INVALID_ARG, "cu_group_dev and prefix_len_dev are required with a shared prefix");
    if (shared && (groups->max_group < 0 || groups->max_group > shape->n_seqs))
        return fail(LA_ERR_INVALID_ARG, "max_group=%d of %d sequences", groups->max_group, shape->n_seqs);
    const DecodePlan p = plan_decode(max_kv_len, max_prefix);
    a.parts = p.own_parts + p.prefix_parts;
    a.direct = p.direct;
    const int64_t rows = (int64_t)shape->n_seqs * shape->q_heads;
    const size_t need = p.direct ? 0 : parts_bytes(rows * a.parts, shape->head_dim);
    if (need && (!workspace || ws_bytes < need))
        return fail(LA_ERR_WORKSPACE, "workspace of %zu bytes, %zu required", workspace ? ws_bytes : 0, need);
    if (need && !aligned16(workspace)) return fail(LA_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    a.kv = cached(layer);
    a.kv_len = kv_len_dev;
    if (la_status e = exponent_scale(shape, layer->k_scale, &a.c)) return e;
    a.v_scale = layer->v_scale;
    a.n_seqs = shape->n_seqs;
    a.kv_heads = shape->kv_heads;
    a.group = shape->q_heads / shape->kv_heads;
    a.by_group = la::FastDiv::by((uint32_t)a.group);
    a.by_kv_heads = la::FastDiv::by((uint32_t)a.kv_heads);
    a.max_kv = (int32_t)max_kv_len;
    carve_parts(&a, workspace, rows * a.parts, shape->head_dim);
    const int64_t items = rows / a.group * up(a.group, la::kRowsHeads) * p.own_parts;
    int64_t prefix_items = 0;
    if (shared) {
        a.cu_group = groups->cu_group_dev;
        a.prefix_len = groups->prefix_len_dev;
        a.n_groups = groups->n_groups;
        a.prefix_parts = p.prefix_parts;
        a.max_group = groups->max_group;
        a.group_tiles = (int32_t)up((int64_t)groups->max_group * a.group, shape->io_dtype == LA_F32 ? la::kTileRows : la::kPromptRows);
        prefix_items = (int64_t)a.group_tiles * p.prefix_parts * groups->n_groups * a.kv_heads;
    }
    if (items > kMaxInt || rows > max_grid(256) || prefix_items + kRowsGrid > max_grid(la::kRowsThreads))
        return fail(LA_ERR_INVALID_ARG, "too many parts for one launch");
    a.prefix_items = (int32_t)prefix_items;
    const bool wide_cache = layer->dtype == LA_F32 || layer->dtype == LA_BF16;
    const int64_t blocks = std::min<int64_t>(items, wide_cache || prefix_items ? kRowsGrid : kOwnRowsGrid);
    hipStream_t st = (hipStream_t)stream;
    (void)hipGetLastError();
    if (layer->dtype == LA_F32) return decode_of_dim<float, float>(shape->head_dim, a, blocks, st);
    if (layer->dtype == LA_BF16) return decode_of_dim<__bf16, __bf16>(shape->head_dim, a, blocks, st);
    if (layer->dtype == LA_FP8_E4M3_BLOCK) return decode_of_dim<__bf16, la::e4m3_code>(shape->head_dim, a, blocks, st);
    if (layer->dtype == LA_INT8_BLOCK) return decode_of_dim<__bf16, la::int8_code>(shape->head_dim, a, blocks, st);
    return decode_of_dim<__bf16, la::fp8_t>(shape->head_dim, a, blocks, st);
}

la_status la_kv_write(const la_kv_layer *layer, int32_t io_dtype, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                      const int32_t *cu_seqlens_dev, int32_t n_seqs, int64_t n_tokens, const int32_t *kv_len_dev, void *stream) {
    if (io_dtype != LA_F32 && io_dtype != LA_BF16)
        return fail(LA_ERR_INVALID_ARG, "io_dtype=%d must be LA_F32 or LA_BF16", io_dtype);
    if (la_status e = check_layer(layer, io_dtype)) return e;
    la::KvWriteArgs a{};
    if (la_status e = kv_rows_args(layer, io_dtype, k, k_stride, v, v_stride, cu_seqlens_dev, n_seqs, n_tokens, kv_len_dev, &a)) return e;
    if (a.n_tokens == 0) return LA_OK;
    hipStream_t st = (hipStream_t)stream;
    (void)hipGetLastError();
    if (block_scaled(layer->dtype)) {
        la::KvCodesArgs c{};
        c.w = a;
        const bool d64 = layer->head_dim == 64;
        if (layer->dtype == LA_INT8_BLOCK) return d64 ? launch_kv_codes<la::int8_code, 64>(c, st) : launch_kv_codes<la::int8_code, 128>(c, st);
        return d64 ? launch_kv_codes<la::e4m3_code, 64>(c, st) : launch_kv_codes<la::e4m3_code, 128>(c, st);
    }
    if (layer->dtype == LA_F32) return launch_kv_write<float, float>(layer->head_dim, a, st);
    if (layer->dtype == LA_BF16) return launch_kv_write<__bf16, __bf16>(layer->head_dim, a, st);
    return launch_kv_write<__bf16, la::fp8_t>(layer->head_dim, a, st);
}

la_status la_kv_read(const la_kv_layer *layer, int32_t io_dtype, void *k, int64_t k_stride, void *v, int64_t v_stride,
                     const int32_t *cu_seqlens_dev, int32_t n_seqs, int64_t n_tokens, const int32_t *kv_len_dev, void *stream) {
    if (io_dtype != LA_F32 && io_dtype != LA_BF16)
        return fail(LA_ERR_INVALID_ARG, "io_dtype=%d must be LA_F32 or LA_BF16", io_dtype);
    // an fp32 cache goes with fp32 rows; the others are read as either
    if (la_status e = check_layer(layer, layer && layer->dtype != LA_F32 ? LA_BF16 : io_dtype)) return e;
    la::KvWriteArgs a{};
    if (la_status e = kv_rows_args(layer, io_dtype, k, k_stride, v, v_stride, cu_seqlens_dev, n_seqs, n_tokens, kv_len_dev, &a)) return e;
    if (a.n_tokens == 0) return LA_OK;
    hipStream_t st = (hipStream_t)stream;
    (void)hipGetLastError();
    const int d = layer->head_dim;
    const bool f32 = io_dtype == LA_F32;
    switch (layer->dtype) {
    case LA_F32: return launch_kv_read<float, float>(d, a, st);
    case LA_BF16: return f32 ? launch_kv_read<float, __bf16>(d, a, st) : launch_kv_read<__bf16, __bf16>(d, a, st);
    case LA_FP8_E4M3: return f32 ? launch_kv_read<float, la::fp8_t>(d, a, st) : launch_kv_read<__bf16, la::fp8_t>(d, a, st);
    case LA_FP8_E4M3_BLOCK: return f32 ? launch_kv_read<float, la::e4m3_code>(d, a, st) : launch_kv_read<__bf16, la::e4m3_code>(d, a, st);
    default: return f32 ? launch_kv_read<float, la::int8_code>(d, a, st) : launch_kv_read<__bf16, la::int8_code>(d, a, st);
    }
}

la_status la_blocks_copy(const la_block_pool *pool, const int32_t *src_ids_dev, const int32_t *dst_ids_dev, int64_t n, void *stream) {
    la::BlockPoolArgs p{};
    if (la_status e = check_pool(pool, false, true, &p)) return e;
    if (n < 0 || n > kMaxInt) return fail(LA_ERR_INVALID_ARG, "n=%lld", (long long)n);
    if (n == 0) return LA_OK;
    if (!src_ids_dev || !dst_ids_dev) return fail(LA_ERR_INVALID_ARG, "src_ids and dst_ids are required");
    (void)hipGetLastError();
    constexpr int64_t STEP = max_grid(la::kBlockThreads);
    for (int64_t i = 0; i < n; i += STEP) {
        const dim3 grid((unsigned)std::min(n - i, STEP), (unsigned)up(p.block_vec, la::kPartVec));
        hipLaunchKernelGGL(la::blocks_copy_kernel, grid, dim3(la::kBlockThreads), 0, (hipStream_t)stream, p, src_ids_dev + i,
                           dst_ids_dev + i);
        if (la_status e = hip_check("block copy launch")) return e;
    }
    return LA_OK;
}

la_status la_blocks_fork(const la_block_pool *pool, const int32_t *parent_rows_dev, const int32_t *child_rows_dev,
                         const int32_t *len_dev, int64_t n, void *stream) {
    la::ForkArgs a{};
    if (la_status e = check_pool(pool, true, true, &a.p)) return e;
    if (la_status e = check_rows(parent_rows_dev, n, "fork")) return e;
    if (n == 0) return LA_OK;
    if (!child_rows_dev || !len_dev) return fail(LA_ERR_INVALID_ARG, "child rows and lengths are required");
    a.parent = parent_rows_dev;
    a.child = child_rows_dev;
    a.len = len_dev;
    a.n = (int32_t)n;
    hipStream_t st = (hipStream_t)stream;
    (void)hipGetLastError();
    hipLaunchKernelGGL(la::fork_take_kernel, dim3(1), dim3(la::kBlockThreads), 0, st, a);
    if (la_status e = hip_check("fork launch")) return e;
    hipLaunchKernelGGL(la::fork_kernel, dim3((unsigned)(1 + up(a.p.block_vec, la::kPartVec)), (unsigned)n), dim3(la::kBlockThreads), 0, st, a);
    return hip_check("fork launch");
}

la_status la_blocks_extend(const la_block_pool *pool, const int32_t *rows_dev, const int32_t *len_dev, int64_t n, void *stream) {
    la::BlockPoolArgs p{};
    if (la_status e = check_pool(pool, true, false, &p)) return e;
    if (la_status e = check_rows(rows_dev, n, "extend")) return e;
    if (n == 0) return LA_OK;
    if (!len_dev) return fail(LA_ERR_INVALID_ARG, "lengths are required");
    (void)hipGetLastError();
    hipLaunchKernelGGL(la::extend_kernel, dim3(1), dim3(la::kBlockThreads), 0, (hipStream_t)stream, p, rows_dev, len_dev, (int32_t)n);
    return hip_check("extend launch");
}

la_status la_blocks_free(const la_block_pool *pool, const int32_t *rows_dev, int64_t n, void *stream) {
    la::BlockPoolArgs p{};
    if (la_status e = check_pool(pool, true, false, &p)) return e;
    if (la_status e = check_rows(rows_dev, n, "free")) return e;
    if (n == 0) return LA_OK;
    hipStream_t st = (hipStream_t)stream;
    (void)hipGetLastError();
    hipLaunchKernelGGL(la::free_rows_kernel, dim3((unsigned)up(p.max_blocks, 256), (unsigned)n), dim3(256), 0, st, p, rows_dev);
    if (la_status e = hip_check("free launch")) return e;
    hipLaunchKernelGGL(p.n_blocks <= la::kPushSmall ? la::free_push_kernel<4> : la::free_push_kernel<16>, dim3(1),
                       dim3(la::kBlockThreads), 0, st, p);
    return hip_check("free launch");
}

size_t la_blocks_compact_workspace_bytes(int64_t n_blocks) {
    if (n_blocks < 0 || n_blocks > 0x3fffffff) return 0;
    return (size_t)(up(n_blocks, la::kBlockThreads) + 2 + 3 * n_blocks) * sizeof(int32_t);
}

la_status la_blocks_compact(const la_block_pool *pool, int32_t *new_ids_dev, void *workspace, size_t ws_bytes, void *stream) {
    la::CompactArgs a{};
    if (la_status e = check_pool(pool, true, true, &a.p)) return e;
    if (a.p.n_blocks == 0) return LA_OK;
    const size_t need = la_blocks_compact_workspace_bytes(a.p.n_blocks);
    if (!workspace || ws_bytes < need)
        return fail(LA_ERR_WORKSPACE, "workspace of %zu bytes, %zu required", workspace ? ws_bytes : 0, need);
    if ((uintptr_t)workspace % sizeof(int32_t)) return fail(LA_ERR_INVALID_ARG, "workspace must be 4-byte aligned");
    a.n_chunks = (int32_t)up(a.p.n_blocks, la::kBlockThreads);
    a.counts = (int32_t *)workspace;
    a.src = a.counts + a.n_chunks + 2;
    a.dst = a.src + a.p.n_blocks;
    a.rank = a.dst + a.p.n_blocks;
    a.remap = new_ids_dev;
    const int64_t parts = up(a.p.block_vec, la::kPartVec), table_blocks = up(a.p.n_rows * a.p.max_blocks, la::kBlockThreads);
    const int64_t copy_blocks = std::min<int64_t>(a.p.n_blocks * parts, 2048);
    if (copy_blocks + table_blocks + a.n_chunks > max_grid(la::kBlockThreads)) return fail(LA_ERR_INVALID_ARG, "the table is too large for one launch");
    hipStream_t st = (hipStream_t)stream;
    (void)hipGetLastError();
    if (a.n_chunks <= la::kCompactSmall) {
        hipLaunchKernelGGL(la::compact_rank_kernel<true>, dim3((unsigned)a.n_chunks), dim3(la::kBlockThreads), 0, st, a);
    } else {
        hipLaunchKernelGGL(la::compact_count_kernel, dim3((unsigned)a.n_chunks), dim3(la::kBlockThreads), 0, st, a);
        if (la_status e = hip_check("compaction launch")) return e;
        hipLaunchKernelGGL(la::compact_rank_kernel<false>, dim3((unsigned)a.n_chunks), dim3(la::kBlockThreads), 0, st, a);
    }
    if (la_status e = hip_check("compaction launch")) return e;
    hipLaunchKernelGGL(la::compact_move_kernel, dim3((unsigned)(copy_blocks + table_blocks + a.n_chunks)), dim3(la::kBlockThreads), 0, st, a,
                       (int32_t)copy_blocks, (int32_t)parts, (int32_t)table_blocks);
    return hip_check("compaction launch");
}

}  // extern "C"
