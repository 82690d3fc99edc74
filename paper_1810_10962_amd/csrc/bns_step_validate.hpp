// Argument checks of the calls around a step on a model's own answers that need neither a device nor the HIP headers (plain C++, as bns_lm_validate.hpp).
#pragma once
#include <algorithm>
#include <memory>
#include <new>

#include "bns_lm_validate.hpp"

namespace bns {

// A tensor of heads: elements from token to token and from head to head, both filled in.
struct HeadStrides {
    int64_t token, head;
};

inline bool aligned_to(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// Pointers to elements of a size.
template <typename... P>
inline bool aligned_all(size_t bytes, const P*... p) {
    return (aligned_to(p, bytes) && ...);
}

constexpr int64_t kMostReach = int64_t(1) << 48;

// What a dimension of `count` entries, `stride` elements apart, reaches over when each entry takes `entry` elements.
inline __int128 reach_of(int64_t count, int64_t stride, __int128 entry) { return static_cast<__int128>(count - 1) * stride + entry; }

// Strides in elements, 0 filled in; that of a dimension of one entry is made to suit the other.  BNS_EINVAL unless the heads of a token end before the
// next token begins, or the tokens of a head before the next head.
inline bns_status head_strides(const bns_head_strides& given, int64_t tokens, int64_t heads, int64_t width, HeadStrides* got) {
    if (given.token < 0 || given.head < 0) return BNS_EINVAL;
    if (given.token >= kMostReach || given.head >= kMostReach) return BNS_EUNSUPPORTED;
    *got = {given.token ? given.token : heads * width, given.head ? given.head : width};
    if (tokens == 0 || heads == 0) return BNS_OK;
    if (heads == 1) got->head = width;
    if (tokens == 1) {
        if (got->head < width) return BNS_EINVAL;
        if (reach_of(heads, got->head, width) >= kMostReach) return BNS_EUNSUPPORTED;
        got->token = int64_t(reach_of(heads, got->head, width));
    }
    const bool by_token = got->head >= width && got->token >= reach_of(heads, got->head, width);
    const bool by_head = got->token >= width && got->head >= reach_of(tokens, got->token, width);
    if (!by_token && !by_head) return BNS_EINVAL;
    return reach_of(tokens, got->token, reach_of(heads, got->head, width)) < kMostReach ? BNS_OK : BNS_EUNSUPPORTED;
}

struct QkDims {
    int64_t tokens;
    HeadStrides x[2], out[2], dx[2];    // queries, keys
    int32_t heads[2];
    int32_t width, rotated;
};

inline bns_status check_qk(const bns_qk* s, QkDims* d) {
    if (!s) return BNS_EINVAL;
    if (s->tokens < 0 || s->q_heads < 0 || s->k_heads < 0 || s->width <= 0 || s->rotated < 0 || s->rotated > s->width || s->rotated % 2) return BNS_EINVAL;
    if (s->interleaved != 0 && s->interleaved != 1) return BNS_EINVAL;
    if (!known_dtype(s->dtype) || !known_dtype(s->weight_dtype) || !(s->eps >= 0.f) || !(s->eps < __builtin_inff())) return BNS_EINVAL;
    if (s->tokens >= int64_t(1) << 31 || s->q_heads >= 1 << 20 || s->k_heads >= 1 << 20 || s->width > 512) return BNS_EUNSUPPORTED;
    d->tokens = s->tokens;
    d->heads[0] = s->q_heads;
    d->heads[1] = s->k_heads;
    d->width = s->width;
    d->rotated = s->rotated;
    const bns_head_strides given[6] = {s->q, s->k, s->q_out, s->k_out, s->dq, s->dk};
    HeadStrides* const got[6] = {&d->x[0], &d->x[1], &d->out[0], &d->out[1], &d->dx[0], &d->dx[1]};
    for (int i = 0; i < 6; ++i) {
        const bns_status st = head_strides(given[i], s->tokens, d->heads[i % 2], s->width, got[i]);
        if (st != BNS_OK) return st;
    }
    return BNS_OK;
}

// A tensor of heads as the overlap checks see it: rows of the outer dimension, each from its first element to its last.
struct HeadMatrix {
    Matrix m;
    size_t row;
    HeadStrides strides;
};
inline HeadMatrix head_matrix(const void* p, int64_t tokens, int64_t heads, int64_t width, const HeadStrides& s, size_t element) {
    if (tokens == 0 || heads == 0) return {{nullptr, 0, 0}, 0, s};
    const bool by_token = s.head >= width && s.token >= reach_of(heads, s.head, width);
    const int64_t inner = by_token ? (heads - 1) * s.head + width : (tokens - 1) * s.token + width;
    return {matrix(p, by_token ? tokens : heads, inner, by_token ? s.token : s.head, element), size_t(inner) * element, s};
}
// As for matrices; `in_place`: the very same tensor is fine.
inline bool collide(const HeadMatrix& out, const HeadMatrix& in, bool in_place) {
    if (!out.m.p || !in.m.p) return false;
    if (out.m.p == in.m.p) return !(in_place && out.strides.token == in.strides.token && out.strides.head == in.strides.head);
    return collide(out.m, in.m, false, out.row, in.row);
}

struct LogprobDims {
    int64_t tokens, logits_stride, dlogits_stride;
    int32_t vocab, top;
};

inline bns_status check_logprob(const bns_logprob* s, LogprobDims* d) {
    if (!s) return BNS_EINVAL;
    if (s->tokens < 0 || s->vocab <= 0 || s->top < 0 || s->top > s->vocab || !known_dtype(s->dtype)) return BNS_EINVAL;
    if (!(s->temperature > 0.f) || !(s->temperature < __builtin_inff())) return BNS_EINVAL;
    const int64_t lim = int64_t(1) << 31;
    if (s->tokens >= lim || s->vocab >= 1 << 30 || s->top > 128) return BNS_EUNSUPPORTED;
    if (s->temperature < 1e-6f || s->temperature > 1e6f) return BNS_EUNSUPPORTED;      // (log2(e) / tau and differences times it stay finite)
    d->tokens = s->tokens;
    d->vocab = s->vocab;
    d->top = s->top;
    if ((d->logits_stride = stride_of(s->logits_stride, s->vocab)) < 0) return BNS_EINVAL;
    if ((d->dlogits_stride = stride_of(s->dlogits_stride, s->vocab)) < 0) return BNS_EINVAL;
    if (d->logits_stride >= lim || d->dlogits_stride >= lim) return BNS_EUNSUPPORTED;
    return BNS_OK;
}

constexpr int32_t kMostGradients = 65536;

// Whether a tensor ends below 2^48 (the kernels keep more than the address in a word).
inline bool low_address(const void* p, int64_t elements, int32_t dtype) {
    const uint64_t most = uint64_t(1) << 48, at = reinterpret_cast<uintptr_t>(p);
    return at < most && uint64_t(elements) * dtype_bytes(dtype) <= most - at;
}

// The entries of a list of gradients; `scaled`: with where they go.
inline bns_status check_gradients(const bns_gradient* g, int32_t count, bool scaled) {
    if (count < 0 || (count > 0 && !g)) return BNS_EINVAL;
    if (count > kMostGradients) return BNS_EUNSUPPORTED;
    int64_t all = 0;
    for (int32_t i = 0; i < count; ++i) {
        if (g[i].elements < 0 || !known_dtype(g[i].dtype) || g[i].reserved != 0) return BNS_EINVAL;
        if (g[i].elements >= int64_t(1) << 40) return BNS_EUNSUPPORTED;
        all += g[i].elements;       // (below 2^56)
        if (g[i].elements == 0) continue;
        if (!g[i].grad || !aligned_to(g[i].grad, dtype_bytes(g[i].dtype))) return BNS_EINVAL;
        if (scaled && (!g[i].out || !aligned_to(g[i].out, dtype_bytes(g[i].dtype)))) return BNS_EINVAL;
        if (!low_address(g[i].grad, g[i].elements, g[i].dtype) || (scaled && !low_address(g[i].out, g[i].elements, g[i].dtype))) return BNS_EUNSUPPORTED;
    }
    return all < int64_t(1) << 43 ? BNS_OK : BNS_EUNSUPPORTED;
}

// Whether a result shares bytes with another result or with a gradient that is not its own, in one pass over all of them by address.
struct Span {
    uintptr_t from, to;
    bool out;
};
inline bns_status gradients_apart(const bns_gradient* g, int32_t count) {
    constexpr int kFew = 256;       // (spans that need no memory from the heap)
    Span few[kFew];
    std::unique_ptr<Span[]> many;
    if (count > kFew / 2 && !(many = std::unique_ptr<Span[]>(new (std::nothrow) Span[size_t(count) * 2]))) return BNS_EDEVICE;
    Span* const s = many ? many.get() : few;
    size_t n = 0;
    for (int32_t i = 0; i < count; ++i) {
        if (g[i].elements == 0) continue;
        const size_t bytes = size_t(g[i].elements) * dtype_bytes(g[i].dtype);
        const uintptr_t in = reinterpret_cast<uintptr_t>(g[i].grad), out = reinterpret_cast<uintptr_t>(g[i].out);
        s[n++] = {out, out + bytes, true};
        if (in != out) s[n++] = {in, in + bytes, false};
    }
    const auto before = [](const Span& a, const Span& b) { return a.from < b.from; };
    if (!std::is_sorted(s, s + n, before)) std::sort(s, s + n, before);
    uintptr_t out_to = 0, any_to = 0;
    for (size_t i = 0; i < n; ++i) {
        if (s[i].from < (s[i].out ? any_to : out_to)) return BNS_EINVAL;
        any_to = std::max(any_to, s[i].to);
        if (s[i].out) out_to = std::max(out_to, s[i].to);
    }
    return BNS_OK;
}

}  // namespace bns
