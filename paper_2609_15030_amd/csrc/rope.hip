// C ABI of rotary positions: frequencies on the host, the rotation on the device.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "linattn.h"
#include "la_host.h"
#include "rope.h"

namespace {

using la::host::aligned16;
using la::host::fail;
using la::host::hip_check;

la_status check_rows(const la_rope_plan *p, const la_rope_rows *r, const char *what, la::RopeRows *out) {
    if (r->heads < 1) return fail(LA_ERR_INVALID_ARG, "%s: heads=%d", what, r->heads);
    if (!r->x || !r->y || !aligned16(r->x) || !aligned16(r->y))
        return fail(LA_ERR_INVALID_ARG, "%s: x and y are required, 16-byte aligned", what);
    const int64_t size = p->io_dtype == LA_F32 ? 4 : 2, packed = (int64_t)r->heads * p->head_dim;
    const int64_t xs = r->x_stride ? r->x_stride : packed, ys = r->y_stride ? r->y_stride : packed;
    for (int64_t s : {xs, ys})
        if (s < packed || s > ((int64_t)1 << 24) || s * size % 16 != 0)
            return fail(LA_ERR_INVALID_ARG, "%s: a stride of %lld must be at least %lld, at most 2^24 and a multiple of 16 bytes", what,
                        (long long)s, (long long)packed);
    if (r->x == r->y && xs != ys) return fail(LA_ERR_INVALID_ARG, "%s: in place with strides of %lld and %lld", what, (long long)xs, (long long)ys);
    *out = {r->x, r->y, xs, ys, r->heads};
    return LA_OK;
}

template <typename T, bool PAIRS, bool SHORT>
la_status launch_of(la::RopeArgs &a, hipStream_t st) {
    constexpr int64_t SET = 8 * la::kRopeTokens;                   // tokens of eight workgroups
    const int64_t step = 0x7fffffffll / (256 * 8) / a.splits * SET;            // of a launch
    for (a.first_token = 0; a.first_token < a.n_tokens; a.first_token += step) {
        const int64_t sets = (std::min(a.n_tokens - a.first_token, step) + SET - 1) / SET;
        hipLaunchKernelGGL((la::rope_kernel<T, PAIRS, SHORT>), dim3((unsigned)(8 * sets * a.splits)), dim3(256), 0, st, a);
        if (la_status e = hip_check("rotary positions launch")) return e;
    }
    return LA_OK;
}

template <typename T>
la_status launch(la::RopeArgs &a, bool pairs, hipStream_t st) {
    if ((pairs ? a.rotary : a.rotary / 2) < la::Span<T>::N) return pairs ? launch_of<T, true, true>(a, st) : launch_of<T, false, true>(a, st);
    return pairs ? launch_of<T, true, false>(a, st) : launch_of<T, false, false>(a, st);
}

}  // namespace

extern "C" {

la_status la_rope_frequencies(int32_t rotary_dim, double base, const la_rope_scaling *scaling, double *freq_out) {
    if (rotary_dim < 2 || rotary_dim % 2 || rotary_dim > la::kRopeDims)
        return fail(LA_ERR_INVALID_ARG, "rotary_dim=%d must be even, from 2 to %d", rotary_dim, la::kRopeDims);
    if (!(base > 0) || !std::isfinite(base)) return fail(LA_ERR_INVALID_ARG, "base=%g must be positive and finite", base);
    if (!freq_out) return fail(LA_ERR_INVALID_ARG, "freq_out is NULL");
    const int32_t kind = scaling ? scaling->kind : LA_ROPE_UNSCALED;
    const double factor = kind == LA_ROPE_UNSCALED ? 1.0 : scaling->factor;
    if (kind < LA_ROPE_UNSCALED || kind > LA_ROPE_PARTS) return fail(LA_ERR_INVALID_ARG, "scaling kind=%d", kind);
    if (!(factor > 0) || !std::isfinite(factor)) return fail(LA_ERR_INVALID_ARG, "scaling factor=%g must be positive and finite", factor);
    if (kind == LA_ROPE_PARTS && (!(scaling->original_len > 0) || !(scaling->high > scaling->low) || !std::isfinite(scaling->original_len) ||
                                  !std::isfinite(scaling->low) || !std::isfinite(scaling->high)))
        return fail(LA_ERR_INVALID_ARG, "scaling by parts: original_len=%g must be positive, low=%g below high=%g", scaling->original_len,
                    scaling->low, scaling->high);
    if (kind == LA_ROPE_BASE && rotary_dim > 2) base *= std::pow(factor, rotary_dim / (rotary_dim - 2.0));
    for (int i = 0; i < rotary_dim / 2; ++i) {
        double f = std::pow(base, -2.0 * i / rotary_dim);
        if (kind == LA_ROPE_LINEAR) f /= factor;
        if (kind == LA_ROPE_PARTS) {
            const double turns = scaling->original_len * f / 6.283185307179586476925;
            const double keep = std::min(1.0, std::max(0.0, (turns - scaling->low) / (scaling->high - scaling->low)));
            f *= keep + (1.0 - keep) / factor;
        }
        freq_out[i] = f;
    }
    return LA_OK;
}

la_status la_rope_turns(const double *freq, int32_t n, uint64_t *turns_out) {
    if (n < 1 || n > la::kRopeDims / 2) return fail(LA_ERR_INVALID_ARG, "n=%d frequencies, 1 to %d", n, la::kRopeDims / 2);
    if (!freq || !turns_out) return fail(LA_ERR_INVALID_ARG, "freq and turns_out are required");
    for (int i = 0; i < n; ++i)
        if (!std::isfinite(freq[i])) return fail(LA_ERR_INVALID_ARG, "freq[%d]=%g", i, freq[i]);
    for (int i = 0; i < n; ++i) {
        // beyond half a turn the quotient would have fewer than 64 bits behind its whole turns: the
        // angle in (-pi, pi] by its sine and cosine, which the C library reduces exactly
        long double f = freq[i];
        if (std::fabs(f) > 3.14L) f = std::atan2(std::sin(f), std::cos(f));
        const long double t = f / 6.283185307179586476925286766559L, x = std::ldexp(t - std::floor(t), 64);
        turns_out[i] = x < 18446744073709551615.0L ? (uint64_t)x : 0;
    }
    return LA_OK;
}

la_status la_rope_apply(const la_rope_plan *plan, const la_rope_rows *q, const la_rope_rows *k, int64_t n_tokens,
                        const la_rope_positions *at, int32_t transpose, void *stream) {
    if (!plan) return fail(LA_ERR_INVALID_ARG, "plan is NULL");
    if (plan->io_dtype != LA_F32 && plan->io_dtype != LA_BF16)
        return fail(LA_ERR_INVALID_ARG, "io_dtype=%d must be LA_F32 or LA_BF16", plan->io_dtype);
    const int32_t r = plan->rotary_dim, d = plan->head_dim, n = plan->io_dtype == LA_F32 ? 4 : 8;
    if (d < 8 || d % 8) return fail(LA_ERR_UNSUPPORTED, "head_dim=%d: multiples of 8 are built", d);
    if (r < 2 || r % 2 || r > d) return fail(LA_ERR_INVALID_ARG, "rotary_dim=%d must be even, from 2 to head_dim=%d", r, d);
    if (r > la::kRopeDims) return fail(LA_ERR_UNSUPPORTED, "rotary_dim=%d: up to %d are built", r, la::kRopeDims);
    if (plan->layout != LA_ROPE_HALVES && plan->layout != LA_ROPE_PAIRS) return fail(LA_ERR_INVALID_ARG, "layout=%d", plan->layout);
    if (!std::isfinite(plan->magnitude)) return fail(LA_ERR_INVALID_ARG, "magnitude=%g must be finite", (double)plan->magnitude);
    if (n_tokens < 0 || n_tokens > 0x7fffff00) return fail(LA_ERR_INVALID_ARG, "n_tokens=%lld", (long long)n_tokens);
    if (!at) return fail(LA_ERR_INVALID_ARG, "positions are required");
    if (at->n_seqs < 0) return fail(LA_ERR_INVALID_ARG, "n_seqs=%d", at->n_seqs);
    if (n_tokens == 0 || (!q && !k) || (!at->positions_dev && at->n_seqs == 0)) return LA_OK;
    if (!at->positions_dev && (!at->cu_seqlens_dev || !at->kv_len_dev))
        return fail(LA_ERR_INVALID_ARG, "positions_dev, or cu_seqlens_dev and kv_len_dev, are required");
    if (!plan->turns_dev) return fail(LA_ERR_INVALID_ARG, "turns_dev is required");
    la::RopeArgs a{};
    if (q)
        if (la_status e = check_rows(plan, q, "q", &a.q)) return e;
    if (k)
        if (la_status e = check_rows(plan, k, "k", &a.k)) return e;
    a.turns = plan->turns_dev;
    a.positions = at->positions_dev;
    a.cu = at->cu_seqlens_dev;
    a.kv_len = at->kv_len_dev;
    a.n_tokens = n_tokens;
    a.n_seqs = at->n_seqs;
    a.dim = d;
    a.rotary = r;
    const bool pairs = plan->layout == LA_ROPE_PAIRS, copies = (q && q->x != q->y) || (k && k->x != k->y);
    a.turned = ((pairs ? r : r / 2) + n - 1) / n;
    a.pieces = a.turned + (copies ? (d - r + n - 1) / n : 0);
    a.by_pieces = la::FastDiv::by((uint32_t)a.pieces);
    const int64_t items = ((int64_t)a.q.heads + a.k.heads) * a.pieces;
    a.items = (int32_t)items;                                  // rows of at most 2^24 values
    a.splits = (int32_t)((items + 64 * la::kRopeItems - 1) / (64 * la::kRopeItems));
    a.share = (int32_t)((items + a.splits - 1) / a.splits + 63) & ~63;
    a.magnitude = plan->magnitude;
    a.transpose = transpose != 0;
    a.whole = (pairs ? r : r / 2) % n == 0;
    (void)hipGetLastError();
    return plan->io_dtype == LA_F32 ? launch<float>(a, pairs, (hipStream_t)stream) : launch<__bf16>(a, pairs, (hipStream_t)stream);
}

}  // extern "C"
