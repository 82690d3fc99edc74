// The norm of many gradients together, and their scaling down to a largest norm.  See include/bns.h for the equations.
//
// Two passes: the norm reads every element, the scaling reads and writes it; both are bound by HBM, or by their launches where elements are few.  All gradients
// are cut into pieces of kPiece bytes, numbered through, and a launch deals the pieces to its blocks in turn.  Squares are formed and added in fp64 (a
// conversion and a fused multiply-add an element), in the same order in every call: by thread, wave, block, and at the end over the blocks'
// sums.  Every block of the scaling adds the blocks' sums up itself, so that a clip is two launches.  The scaling takes the pieces from the last to the
// first: what the norm has read last is still in the memory-side cache.
//
// The list comes with the kernel's arguments where it is short, else through the workspace, written there by launches that carry it.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "bns_internal.hpp"
#include "bns_lm_words.hpp"
#include "bns_step_validate.hpp"

using namespace bns;

namespace {

constexpr int kThreads = 256;
constexpr int kPiece = 32768;           // bytes of a gradient that a block takes at a time
constexpr int kMostBlocks = 1024;
constexpr int kShort = 96;              // entries that travel with a launch

struct Entry {
    const void* grad;
    void* out;
    int64_t elements;
    uint32_t first;                     // number of its first piece
    uint32_t f32;
};

struct List {
    Entry entry[kShort];
};
struct ListInWorkspace {};

struct GradsArgs {
    double* partial;                    // [blocks] sums of squares
    const Entry* list;                  // a long one, in the workspace
    double* squares;                    // norm: written (may be NULL); scaling: read where `partial` is NULL
    float* norm;
    float max_norm;
    int32_t entries, blocks;            // blocks: of the norm's launch
    uint32_t pieces;
};

__global__ void __launch_bounds__(kShort) grads_list_kernel(List list, Entry* out, int entries) {
    if (int(threadIdx.x) < entries) out[threadIdx.x] = list.entry[threadIdx.x];
}

__device__ __forceinline__ const Entry& entry_at(const GradsArgs&, const List& list, int i) { return list.entry[i]; }
__device__ __forceinline__ const Entry& entry_at(const GradsArgs& a, const ListInWorkspace&, int i) { return a.list[i]; }

// The entry that piece p belongs to: the last one whose first piece is p or less (entries have a piece at least).
template <typename L>
__device__ __forceinline__ Entry entry_of(const GradsArgs& a, const L& list, uint32_t p) {
    int lo = 0, hi = a.entries;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (entry_at(a, list, mid).first <= p) lo = mid;
        else hi = mid;
    }
    return entry_at(a, list, lo);
}

__device__ __forceinline__ double block_sum(double v, double* lds) {
    v = wave_sum(v);
    __syncthreads();
    if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < kThreads / kWave; ++i) s += lds[i];
    return s;
}

template <typename T, bool NT>
__device__ __forceinline__ void add_squares(const T* p, int n, double (&s)[4]) {
    constexpr int E = Words<T>::kElems, kAtOnce = 4;
    for (int v = int(threadIdx.x) * E; v < n; v += kThreads * E * kAtOnce) {
        u4 w[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int at = v + j * kThreads * E;
            if (at + E <= n) w[j] = get16<NT>(p + at);
            else w[j] = u4{0, 0, 0, 0};
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            float f[E];
            Words<T>::unpack(w[j], f);
#pragma unroll
            for (int i = 0; i < E; ++i) s[i % 4] = fma(double(f[i]), double(f[i]), s[i % 4]);
        }
    }
    const int rest = n % E;
    if (int(threadIdx.x) < rest) {
        const double f = load_scalar<T>(p + n - rest + threadIdx.x);
        s[0] = fma(f, f, s[0]);
    }
}

template <typename T, bool NT>
__device__ __forceinline__ void scale_piece(const T* p, T* out, int n, float c, float c2) {
    constexpr int E = Words<T>::kElems, kAtOnce = 4;
    for (int v = int(threadIdx.x) * E; v < n; v += kThreads * E * kAtOnce) {
        u4 w[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int at = v + j * kThreads * E;
            if (at + E <= n) w[j] = get16<NT>(p + at);
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int at = v + j * kThreads * E;
            if (at + E > n) continue;
            float f[E];
            Words<T>::unpack(w[j], f);
#pragma unroll
            for (int i = 0; i < E; ++i) f[i] = f[i] * c * c2;
            Words<T>::template store<NT>(out + at, E, f);
        }
    }
    const int rest = n % E;
    if (int(threadIdx.x) < rest) Words<T>::put_one(out + n - rest + threadIdx.x, load_scalar<T>(p + n - rest + threadIdx.x) * c * c2);
}

// What piece p is: calls work(gradient, result, elements) with pointers of its type.
template <typename Work>
__device__ __forceinline__ void with_piece(const Entry& e, uint32_t p, Work&& work) {
    const int64_t per = e.f32 ? kPiece / 4 : kPiece / 2, at = int64_t(p - e.first) * per;
    const int n = int(min(per, e.elements - at));
    if (e.f32) work(static_cast<const float*>(e.grad) + at, static_cast<float*>(e.out) + at, n);
    else work(static_cast<const bf16_t*>(e.grad) + at, static_cast<bf16_t*>(e.out) + at, n);
}

template <typename L, bool NT>
__global__ void __launch_bounds__(kThreads) grads_norm_kernel(GradsArgs a, L list) {
    __shared__ double lds[kThreads / kWave];
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    for (uint32_t p = blockIdx.x; p < a.pieces; p += gridDim.x) {
        const Entry e = entry_of(a, list, p);
        with_piece(e, p, [&](auto* grad, auto*, int n) { add_squares<std::remove_const_t<std::remove_pointer_t<decltype(grad)>>, NT>(grad, n, s); });
    }
    const double all = block_sum((s[0] + s[1]) + (s[2] + s[3]), lds);
    if (threadIdx.x == 0) a.partial[blockIdx.x] = all;
}

// The sum of squares from the blocks' sums: every block of every launch adds them in the same order.
__device__ __forceinline__ double all_squares(const double* partial, int blocks, double* lds) {
    double s = 0.0;
    for (int i = threadIdx.x; i < blocks; i += kThreads) s += partial[i];
    return block_sum(s, lds);
}

__global__ void __launch_bounds__(kThreads) grads_sum_kernel(GradsArgs a) {
    __shared__ double lds[kThreads / kWave];
    const double s = all_squares(a.partial, a.blocks, lds);
    if (threadIdx.x == 0) {
        *a.squares = s;
        if (a.norm) *a.norm = float(sqrt(s));
    }
}

template <typename L, bool NT>
__global__ void __launch_bounds__(kThreads) grads_scale_kernel(GradsArgs a, L list) {
    __shared__ double lds[kThreads / kWave];
    const double s = a.partial ? all_squares(a.partial, a.blocks, lds) : *a.squares;
    const double norm = sqrt(s), c64 = double(a.max_norm) / (norm + 1e-6);
    // (NaN stays NaN.  A factor near the least that fp32 holds, for gradients near the largest, goes in two parts that keep its bits.)
    const bool tiny = c64 < 0x1p-100;
    const float c = c64 >= 1.0 ? 1.f : float(tiny ? c64 * 0x1p100 : c64), c2 = tiny ? 0x1p-100f : 1.f;
    if (blockIdx.x == 0 && threadIdx.x == 0 && a.norm) *a.norm = float(norm);
    for (uint32_t b = blockIdx.x; b < a.pieces; b += gridDim.x) {
        const uint32_t p = a.pieces - 1 - b;
        const Entry e = entry_of(a, list, p);
        if (c == 1.f && e.grad == e.out) continue;
        with_piece(e, p, [&](auto* grad, auto* out, int n) { scale_piece<std::remove_pointer_t<decltype(out)>, NT>(grad, out, n, c, c2); });
    }
}

size_t list_bytes(int32_t count) { return count > kShort ? size_t(round_up(int64_t(count) * int64_t(sizeof(Entry)), 256)) : 0; }

// The list as the kernels take it.
struct Listed {
    List list;                  // short ones
    GradsArgs args;
    size_t bytes;
    bool is_long;
};

uint32_t pieces_of(const bns_gradient& g) {
    const int64_t per = kPiece / int64_t(dtype_bytes(g.dtype));
    return uint32_t((g.elements + per - 1) / per);      // (below 2^27)
}

// Puts the list where the kernels find it; long ones by launches on the stream.
bns_status put_list(const bns_gradient* g, int32_t count, void* workspace, hipStream_t st, Listed* l) {
    l->args = {};
    l->args.partial = static_cast<double*>(workspace);
    l->bytes = 0;
    int32_t entries = 0;
    for (int32_t i = 0; i < count; ++i) entries += g[i].elements > 0;
    l->is_long = entries > kShort;
    Entry* const room = reinterpret_cast<Entry*>(static_cast<char*>(workspace) + kMostBlocks * sizeof(double));
    uint32_t pieces = 0;        // (below 2^31 and one for every entry)
    int32_t at = 0, sent = 0;
    for (int32_t i = 0; i < count; ++i) {
        if (g[i].elements == 0) continue;
        l->list.entry[at++] = {g[i].grad, g[i].out, g[i].elements, pieces, uint32_t(g[i].dtype == BNS_F32)};
        pieces += pieces_of(g[i]);
        l->bytes += size_t(g[i].elements) * dtype_bytes(g[i].dtype);
        if (l->is_long && (at == kShort || sent + at == entries)) {
            BNS_LAUNCH(grads_list_kernel, dim3(1), dim3(kShort), 0, st, l->list, room + sent, at);
            if (hipGetLastError() != hipSuccess) return BNS_EDEVICE;
            sent += at;
            at = 0;
        }
    }
    l->args.list = l->is_long ? room : nullptr;
    l->args.entries = entries;
    l->args.pieces = pieces;
    l->args.blocks = int32_t(std::min<uint32_t>(std::max<uint32_t>(pieces, 1), kMostBlocks));
    return BNS_OK;
}

bns_status launch_norm(const Listed& l, hipStream_t st) {
    const dim3 grid{uint32_t(l.args.blocks)};
    const bool nt = l.bytes > kStreamBytes;
    if (l.is_long && nt) BNS_LAUNCH((grads_norm_kernel<ListInWorkspace, true>), grid, dim3(kThreads), 0, st, l.args, ListInWorkspace{});
    else if (l.is_long) BNS_LAUNCH((grads_norm_kernel<ListInWorkspace, false>), grid, dim3(kThreads), 0, st, l.args, ListInWorkspace{});
    else if (nt) BNS_LAUNCH((grads_norm_kernel<List, true>), grid, dim3(kThreads), 0, st, l.args, l.list);
    else BNS_LAUNCH((grads_norm_kernel<List, false>), grid, dim3(kThreads), 0, st, l.args, l.list);
    return hipGetLastError() == hipSuccess ? BNS_OK : BNS_EDEVICE;
}

bns_status launch_scale(const Listed& l, hipStream_t st) {
    const dim3 grid{std::min<uint32_t>(std::max<uint32_t>(l.args.pieces, 1), 2048)};
    const bool nt = l.bytes > kStreamBytes;
    if (l.is_long && nt) BNS_LAUNCH((grads_scale_kernel<ListInWorkspace, true>), grid, dim3(kThreads), 0, st, l.args, ListInWorkspace{});
    else if (l.is_long) BNS_LAUNCH((grads_scale_kernel<ListInWorkspace, false>), grid, dim3(kThreads), 0, st, l.args, ListInWorkspace{});
    else if (nt) BNS_LAUNCH((grads_scale_kernel<List, true>), grid, dim3(kThreads), 0, st, l.args, l.list);
    else BNS_LAUNCH((grads_scale_kernel<List, false>), grid, dim3(kThreads), 0, st, l.args, l.list);
    return hipGetLastError() == hipSuccess ? BNS_OK : BNS_EDEVICE;
}

bns_status check_call(const bns_gradient* g, int32_t count, bool scaled, const void* workspace, size_t workspace_bytes) {
    bns_status s = check_gradients(g, count, scaled);
    if (s != BNS_OK) return s;
    if (scaled && (s = gradients_apart(g, count)) != BNS_OK) return s;
    if (!workspace || !aligned16(workspace)) return BNS_EINVAL;
    return workspace_bytes < bns_grads_workspace_bytes(count) ? BNS_EWORKSPACE : BNS_OK;
}

bool fine_norm(float max_norm) { return max_norm >= 0.f && max_norm < __builtin_inff(); }

}  // namespace

extern "C" {

size_t bns_grads_workspace_bytes(int32_t count) {
    if (count < 0 || count > kMostGradients) return 0;
    return kMostBlocks * sizeof(double) + list_bytes(count);
}

bns_status bns_grads_norm(const bns_gradient* gradients, int32_t count, double* squares, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
    bns_status s = check_call(gradients, count, false, workspace, workspace_bytes);
    if (s != BNS_OK) return s;
    if (!squares || !aligned_all(8, squares) || !aligned_all(4, norm)) return BNS_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    Listed l{};
    if ((s = put_list(gradients, count, workspace, st, &l)) != BNS_OK) return s;
    if ((s = launch_norm(l, st)) != BNS_OK) return s;
    l.args.squares = squares;
    l.args.norm = norm;
    BNS_LAUNCH(grads_sum_kernel, dim3(1), dim3(kThreads), 0, st, l.args);
    return hipGetLastError() == hipSuccess ? BNS_OK : BNS_EDEVICE;
}

bns_status bns_grads_scale(const bns_gradient* gradients, int32_t count, const double* squares, float max_norm, float* norm, void* workspace, size_t workspace_bytes,
                           void* stream) {
    bns_status s = check_call(gradients, count, true, workspace, workspace_bytes);
    if (s != BNS_OK) return s;
    if (!squares || !aligned_all(8, squares) || !aligned_all(4, norm) || !fine_norm(max_norm)) return BNS_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    Listed l{};
    if ((s = put_list(gradients, count, workspace, st, &l)) != BNS_OK) return s;
    l.args.partial = nullptr;
    l.args.squares = const_cast<double*>(squares);
    l.args.norm = norm;
    l.args.max_norm = max_norm;
    return launch_scale(l, st);
}

bns_status bns_grads_clip(const bns_gradient* gradients, int32_t count, float max_norm, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
    bns_status s = check_call(gradients, count, true, workspace, workspace_bytes);
    if (s != BNS_OK) return s;
    if (!norm || !aligned_all(4, norm) || !fine_norm(max_norm)) return BNS_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    Listed l{};
    if ((s = put_list(gradients, count, workspace, st, &l)) != BNS_OK) return s;
    if ((s = launch_norm(l, st)) != BNS_OK) return s;
    l.args.norm = norm;
    l.args.max_norm = max_norm;
    return launch_scale(l, st);
}

}  // extern "C"
