// Argument checks of the language-model operators that need neither a device nor the HIP headers (plain C++, as bns_validate.hpp).
#pragma once
#include "bns_validate.hpp"

namespace bns {

inline int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
inline size_t dtype_bytes(int32_t dtype) { return dtype == BNS_F32 ? 4 : 2; }
inline bool known_dtype(int32_t dtype) { return dtype == BNS_F32 || dtype == BNS_BF16; }

// A call that moves more than this between memory and the compute units finds nothing of it in the memory-side cache (256 MB) a second time.
constexpr size_t kStreamBytes = size_t(224) << 20;

// A row-major matrix as the overlap checks see it: the bytes from its first element to its last.
struct Matrix {
    const void* p;
    int64_t stride;     // in bytes
    size_t bytes;
};

inline Matrix matrix(const void* p, int64_t rows, int64_t width, int64_t stride, size_t element) {
    return {p, int64_t(size_t(stride) * element), rows > 0 ? (size_t(rows - 1) * size_t(stride) + size_t(width)) * element : 0};
}

// Whether an output and an input collide; `in_place`: the very same tensor is fine.  Rows of two matrices that interleave
// (two halves of one wider matrix) do not collide: equal strides, and every row of one ends before the next of the other begins.
inline bool collide(const Matrix& out, const Matrix& in, bool in_place, size_t out_row, size_t in_row) {
    if (!out.p || !in.p || out.bytes == 0 || in.bytes == 0) return false;
    if (!overlap(out.p, out.bytes, in.p, in.bytes)) return false;
    if (out.p == in.p && out.stride == in.stride) return !in_place;
    if (out.stride != in.stride || out.stride <= 0) return true;
    const int64_t apart = int64_t(reinterpret_cast<uintptr_t>(in.p) - reinterpret_cast<uintptr_t>(out.p));
    const int64_t shift = ((apart % out.stride) + out.stride) % out.stride;
    return !(shift >= int64_t(out_row) && shift + int64_t(in_row) <= out.stride);
}

// 0 stands for dense rows; -1: not allowed
inline int64_t stride_of(int64_t given, int64_t width) {
    if (given == 0) return width;
    return given >= width ? given : -1;
}

struct RmsDims {
    int64_t rows, x_stride, residual_stride, sum_stride, y_stride;
    int32_t width, groups;      // groups: scales per row
};

inline bns_status check_rms(const bns_rms* r, RmsDims* d) {
    if (!r) return BNS_EINVAL;
    if (r->rows < 0 || r->width <= 0 || !known_dtype(r->dtype) || !known_dtype(r->weight_dtype)) return BNS_EINVAL;
    if (r->out != BNS_OUT_SAME && r->out != BNS_OUT_E4M3) return BNS_EINVAL;
    if (!(r->eps >= 0.f) || !(r->eps < __builtin_inff())) return BNS_EINVAL;
    if (r->group != 0 && r->group != 32 && r->group != 64 && r->group != 128) return BNS_EINVAL;
    if (r->pow2_scales != 0 && r->pow2_scales != 1) return BNS_EINVAL;
    if (r->out == BNS_OUT_SAME && (r->group != 0 || r->pow2_scales != 0)) return BNS_EINVAL;
    const int64_t lim = int64_t(1) << 31;
    if (r->rows >= lim || r->width > 16384) return BNS_EUNSUPPORTED;
    d->rows = r->rows;
    d->width = r->width;
    d->groups = r->group ? int32_t((r->width + r->group - 1) / r->group) : 1;
    const int64_t given[4] = {r->x_stride, r->residual_stride, r->sum_stride, r->y_stride};
    int64_t* const got[4] = {&d->x_stride, &d->residual_stride, &d->sum_stride, &d->y_stride};
    for (int i = 0; i < 4; ++i) {
        if ((*got[i] = stride_of(given[i], r->width)) < 0) return BNS_EINVAL;
        if (*got[i] >= lim) return BNS_EUNSUPPORTED;
    }
    return BNS_OK;
}

struct HeadDims {
    int64_t tokens, hidden_stride, weight_stride;
    int32_t width, vocab, dtype, piece;
};

inline bns_status check_head(const bns_head* h, HeadDims* d) {
    if (!h) return BNS_EINVAL;
    if (h->tokens < 0 || h->width <= 0 || h->vocab <= 0 || h->piece < 0 || !known_dtype(h->dtype)) return BNS_EINVAL;
    const int64_t lim = int64_t(1) << 31;
    if (h->tokens > (1 << 20) || h->width > 65536 || h->vocab >= (1 << 24)) return BNS_EUNSUPPORTED;
    d->tokens = h->tokens;
    d->width = h->width;
    d->vocab = h->vocab;
    d->dtype = h->dtype;
    d->piece = h->piece;
    if ((d->hidden_stride = stride_of(h->hidden_stride, h->width)) < 0) return BNS_EINVAL;
    if ((d->weight_stride = stride_of(h->weight_stride, h->width)) < 0) return BNS_EINVAL;
    if (d->hidden_stride >= lim || d->weight_stride >= lim) return BNS_EUNSUPPORTED;
    return BNS_OK;
}

struct DistillDims {
    int64_t tokens, logits_stride, dlogits_stride;
    int32_t vocab, k;
};

inline bns_status check_distill(const bns_distill* s, DistillDims* d) {
    if (!s) return BNS_EINVAL;
    if (s->tokens < 0 || s->vocab <= 0 || s->k <= 0 || !known_dtype(s->dtype)) return BNS_EINVAL;
    if (!(s->temperature > 0.f) || !(s->temperature < __builtin_inff())) return BNS_EINVAL;
    const int64_t lim = int64_t(1) << 31;
    if (s->tokens >= lim || s->vocab >= (1 << 30) || s->k > 1024) return BNS_EUNSUPPORTED;
    d->tokens = s->tokens;
    d->vocab = s->vocab;
    d->k = s->k;
    if ((d->logits_stride = stride_of(s->logits_stride, s->vocab)) < 0) return BNS_EINVAL;
    if ((d->dlogits_stride = stride_of(s->dlogits_stride, s->vocab)) < 0) return BNS_EINVAL;
    if (d->logits_stride >= lim || d->dlogits_stride >= lim) return BNS_EUNSUPPORTED;
    return BNS_OK;
}

}  // namespace bns
