// The norm of many gradients together, and their scaling down to a largest norm.  See include/bns.h for the equations.
//
// Two passes: the norm reads every element, the scaling reads and writes it; both are bound by HBM, or by their launches where elements are few.  All gradients
// are cut into pieces of 16 KB, four words a thread, numbered through; a piece is asked for while the one before it is worked on.
// Squares are formed and added in fp64 (a conversion and a fused multiply-add an element), in the same order in every call: by thread, wave, block, and at the end over the
// blocks' sums.  Every block of the scaling adds the blocks' sums up itself, while its first piece is on its way, so that a clip is two launches.  The scaling takes the pieces
// from the last to the first: what the norm has read last is still in the memory-side cache (242 MB: 117 us instead of 121).
//
// The list comes with the kernel's arguments.  A longer one goes in parts, a launch each; of a clip only the norm does, whose launches leave the parts in the workspace for one launch
// of the scaling (146 tensors of 2.2 MB 12.2 us; with more than 140 through the workspace in launches of their own 16.6, 242 tensors 16.5 against 19.5).
//
// Measured: 1.3e9 bf16 elements in 194 tensors 1282 us, 390 the norm (2.6 GB, 6.7 TB/s) and 885 the scaling (5.2 GB, 5.9 TB/s); 13.7 MB of fp32 in 34 tensors 13.4 us, two launches that
// find it in the memory-side cache.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "bns_internal.hpp"
#include "bns_lm_words.hpp"
#include "bns_step_validate.hpp"

using namespace bns;

namespace {

constexpr int kThreads = 256;
constexpr int kWords = 4;               // words of 16 bytes that a thread has of a piece
constexpr int kPiece = kThreads * kWords * 16;
constexpr int kMostBlocks = 1024;       // of the norm
// Pieces of a block of the scaling, neighbours.  Blocks start in order, so that all of them work in one stretch of memory; fewer blocks that each come by every 2048th piece
// drift apart (1.3e9 bf16 elements, both passes: 1261 us, 1 piece 1291, 4 1323, 16 1392, every 2048th 1361).
constexpr uint32_t kRun = 2;
constexpr int kShort = 200;             // entries that travel with a launch, whose arguments take 4 KB at most

// Pieces up to which the scaling of a clip has a short list with its arguments; more blocks read it faster in the workspace, where the norm left it (us, arguments against workspace:
// 864 pieces 13.5 against 14.0, 19000 166.5 against 166.2, 160000 1302 against 1282).
constexpr uint32_t kFewPieces = 16384;

// Entries: addresses, below 2^48, and the number of an entry's first piece.  Above the gradient's address: the elements of its last piece less one, and in the highest bit its type.
struct List {
    uint64_t grad[kShort], out[kShort];
    uint32_t first[kShort];
};
// The same of any length, in the workspace.
struct LongList {
    uint64_t *grad, *out;
    uint32_t* first;
};
constexpr size_t kEntry = 20;
constexpr int kAddressBits = 48;
constexpr uint64_t kIsF32 = uint64_t(1) << 63;
static_assert(kPiece / 2 <= 1 << (63 - kAddressBits), "the elements of a piece fit above an address");

struct GradsArgs {
    double* partial;                    // [blocks] sums of squares
    double* squares;                    // norm: written (may be NULL); scaling: read where `partial` is NULL
    float* norm;
    float max_norm;
    int32_t entries, blocks;            // blocks: of the norm's launch, the largest one
    uint32_t from, pieces, cold;        // pieces of the list: from `from` on; those before `cold` are not in the memory-side cache when the scaling comes to them
};
static_assert(sizeof(List) + sizeof(GradsArgs) + sizeof(LongList) + 8 <= 4096, "arguments of a launch");
static_assert(kShort <= kThreads, "a thread for each entry");

// A piece: its entry's tensors from its first element on.
struct Piece {
    const void* grad;
    void* out;
    int n;
    bool f32;
};
// Piece p belongs to the last entry whose first piece is p or less (entries have a piece at least).
template <typename L>
__device__ __forceinline__ Piece piece_of(const GradsArgs& a, const L& list, uint32_t p) {
    int lo = 0, hi = a.entries;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (list.first[mid] <= p) lo = mid;
        else hi = mid;
    }
    const uint64_t grad = list.grad[lo];
    const bool f32 = grad & kIsF32;
    const uint32_t first = list.first[lo], end = lo + 1 < a.entries ? list.first[lo + 1] : a.pieces;
    const int64_t bytes = int64_t(p - first) * kPiece;
    const int last = int(grad << 1 >> (kAddressBits + 1)) + 1;
    return {reinterpret_cast<const char*>(grad & ((uint64_t(1) << kAddressBits) - 1)) + bytes, reinterpret_cast<char*>(list.out[lo]) + bytes,
            p + 1 == end ? last : f32 ? kPiece / 4 : kPiece / 2, f32};
}

// What a thread has of a piece: words, and of the elements behind the last one, one of the first threads each one.
struct Held {
    u4 w[kWords];
    float rest;
};
template <typename T, bool NT>
__device__ __forceinline__ void ask_as(Held& h, const Piece& p) {
    constexpr int E = Words<T>::kElems;
    const T* x = static_cast<const T*>(p.grad);
#pragma unroll
    for (int j = 0; j < kWords; ++j) {
        const int at = (j * kThreads + int(threadIdx.x)) * E;
        if (at + E <= p.n) h.w[j] = get16<NT>(x + at);
        else h.w[j] = u4{0, 0, 0, 0};
    }
    const int left = p.n % E;
    h.rest = int(threadIdx.x) < left ? load_scalar<T>(x + p.n - left + threadIdx.x) : 0.f;
}
__device__ __forceinline__ void ask(Held& h, const Piece& p, bool nt) {
    if (p.f32) {
        if (nt) ask_as<float, true>(h, p);
        else ask_as<float, false>(h, p);
    } else {
        if (nt) ask_as<bf16_t, true>(h, p);
        else ask_as<bf16_t, false>(h, p);
    }
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

template <typename T>
__device__ __forceinline__ void add_squares(const Held& h, double (&s)[4]) {
    constexpr int E = Words<T>::kElems;
#pragma unroll
    for (int j = 0; j < kWords; ++j) {
        float f[E];
        Words<T>::unpack(h.w[j], f);
#pragma unroll
        for (int i = 0; i < E; ++i) s[i % 4] = fma(double(f[i]), double(f[i]), s[i % 4]);
    }
    s[0] = fma(double(h.rest), double(h.rest), s[0]);
}

template <typename T, bool NT>
__device__ __forceinline__ void put_scaled(const Held& h, const Piece& p, float c, float c2) {
    constexpr int E = Words<T>::kElems;
    T* out = static_cast<T*>(p.out);
#pragma unroll
    for (int j = 0; j < kWords; ++j) {
        const int at = (j * kThreads + int(threadIdx.x)) * E;
        if (at + E > p.n) continue;
        float f[E];
        Words<T>::unpack(h.w[j], f);
#pragma unroll
        for (int i = 0; i < E; ++i) f[i] = f[i] * c * c2;
        Words<T>::template store<NT>(out + at, E, f);
    }
    const int left = p.n % E;
    if (int(threadIdx.x) < left) Words<T>::put_one(out + p.n - left + threadIdx.x, h.rest * c * c2);
}

// One part of a list, from entry `at` on: parts behind the first add to its sums.  `keep`: where the list is left for the scaling (may be empty).
__global__ void __launch_bounds__(kThreads) grads_norm_kernel(GradsArgs a, List list, LongList keep, int at) {
    __shared__ double lds[kThreads / kWave];
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    uint32_t p = a.from + blockIdx.x;
    Held next;
    Piece piece = {};
    if (p < a.pieces) {
        piece = piece_of(a, list, p);
        ask(next, piece, p < a.cold);
    }
    while (p < a.pieces) {
        const Held now = next;
        const bool f32 = piece.f32;
        p += gridDim.x;
        if (p < a.pieces) {
            piece = piece_of(a, list, p);
            ask(next, piece, p < a.cold);
        }
        if (f32) add_squares<float>(now, s);
        else add_squares<bf16_t>(now, s);
    }
    const double all = block_sum((s[0] + s[1]) + (s[2] + s[3]), lds);
    if (threadIdx.x == 0) a.partial[blockIdx.x] = at > 0 ? a.partial[blockIdx.x] + all : all;
    if (blockIdx.x == 0 && keep.grad && int(threadIdx.x) < a.entries) {
        const int i = threadIdx.x;
        keep.grad[at + i] = list.grad[i];
        keep.out[at + i] = list.out[i];
        keep.first[at + i] = list.first[i];
    }
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

template <typename L>
__global__ void __launch_bounds__(kThreads) grads_scale_kernel(GradsArgs a, L list) {
    __shared__ double lds[kThreads / kWave];
    uint32_t b = blockIdx.x * kRun;
    const uint32_t b_end = min(b + kRun, a.pieces - a.from);
    Held next;
    Piece piece = {};
    const auto ask_for = [&]() {
        const uint32_t p = a.pieces - 1 - b;
        piece = piece_of(a, list, p);
        ask(next, piece, p < a.cold);
    };
    if (b < b_end) ask_for();
    const double s = a.partial ? all_squares(a.partial, a.blocks, lds) : *a.squares;
    const double norm = sqrt(s), c64 = double(a.max_norm) / (norm + 1e-6);
    // (NaN stays NaN.  A factor near the least that fp32 holds, for gradients near the largest, goes in two parts that keep its bits.)
    const bool tiny = c64 < 0x1p-100;
    const float c = c64 >= 1.0 ? 1.f : float(tiny ? c64 * 0x1p100 : c64), c2 = tiny ? 0x1p-100f : 1.f;
    if (blockIdx.x == 0 && threadIdx.x == 0 && a.norm) *a.norm = float(norm);
    while (b < b_end) {
        const Held now = next;
        const Piece here = piece;
        ++b;
        if (b < b_end) ask_for();
        if (c == 1.f && here.grad == here.out) continue;
        if (here.f32) {
            if (a.cold > 0) put_scaled<float, true>(now, here, c, c2);
            else put_scaled<float, false>(now, here, c, c2);
        } else {
            if (a.cold > 0) put_scaled<bf16_t, true>(now, here, c, c2);
            else put_scaled<bf16_t, false>(now, here, c, c2);
        }
    }
}

// Bytes of a long list's arrays, one behind the other in the workspace.
size_t list_bytes(int32_t count) { return size_t(round_up(int64_t(count) * int64_t(kEntry), 256)); }

uint32_t pieces_of(const bns_gradient& g) {
    const int64_t per = kPiece / int64_t(dtype_bytes(g.dtype));
    return uint32_t((g.elements + per - 1) / per);      // (below 2^28)
}

// What the launches have in common.
struct Listed {
    GradsArgs args;
    int32_t entries;
    uint32_t pieces;            // (below 2^31 and one for every entry)
    LongList long_list;         // for the scaling of a clip, where it reads it
};
Listed look_at(const bns_gradient* g, int32_t count, void* workspace) {
    Listed l{};
    size_t bytes = 0;
    for (int32_t i = 0; i < count; ++i) {
        if (g[i].elements == 0) continue;
        ++l.entries;
        l.pieces += pieces_of(g[i]);
        bytes += size_t(g[i].elements) * dtype_bytes(g[i].dtype);
    }
    char* const room = static_cast<char*>(workspace) + kMostBlocks * sizeof(double);
    if (l.entries > kShort || l.pieces > kFewPieces)
        l.long_list = {reinterpret_cast<uint64_t*>(room), reinterpret_cast<uint64_t*>(room + size_t(l.entries) * 8), reinterpret_cast<uint32_t*>(room + size_t(l.entries) * 16)};
    l.args.partial = static_cast<double*>(workspace);
    l.args.cold = bytes > kStreamBytes ? l.pieces - std::min<uint32_t>(l.pieces, uint32_t(kStreamBytes / kPiece)) : 0;
    l.args.blocks = int32_t(std::min<uint32_t>(std::max<uint32_t>(l.pieces, 1), kMostBlocks));
    return l;
}

// Calls launch(arguments, list, entries before it) for the list in parts of kShort entries (one part at least); BNS_EDEVICE if a launch fails.
template <typename Launch>
bns_status in_parts(const Listed& l, const bns_gradient* g, int32_t count, Launch launch) {
    List list{};
    GradsArgs a = l.args;
    uint32_t pieces = 0;
    int32_t at = 0, sent = 0;
    for (int32_t i = 0; i < count; ++i) {
        if (g[i].elements == 0) continue;
        const int64_t per = kPiece / int64_t(dtype_bytes(g[i].dtype));
        list.grad[at] = uint64_t(reinterpret_cast<uintptr_t>(g[i].grad)) | uint64_t((g[i].elements - 1) % per) << kAddressBits | (g[i].dtype == BNS_F32 ? kIsF32 : 0);
        list.out[at] = uint64_t(reinterpret_cast<uintptr_t>(g[i].out));
        list.first[at++] = pieces;
        pieces += pieces_of(g[i]);
        if (at < kShort || sent + at == l.entries) continue;
        a.entries = at;
        a.pieces = pieces;
        launch(a, list, sent);
        if (hipGetLastError() != hipSuccess) return BNS_EDEVICE;
        a.from = pieces;
        sent += at;
        at = 0;
    }
    a.entries = at;
    a.pieces = pieces;
    launch(a, list, sent);
    return hipGetLastError() == hipSuccess ? BNS_OK : BNS_EDEVICE;
}

bns_status launch_norm(const Listed& l, const bns_gradient* g, int32_t count, bool keep, hipStream_t st) {
    return in_parts(l, g, count, [&](const GradsArgs& a, const List& list, int at) {
        const uint32_t blocks = at > 0 ? std::min<uint32_t>(a.pieces - a.from, kMostBlocks) : uint32_t(a.blocks);      // (the first part writes all sums)
        BNS_LAUNCH(grads_norm_kernel, dim3(blocks), dim3(kThreads), 0, st, a, list, keep ? l.long_list : LongList{}, at);
    });
}

dim3 scale_grid(const GradsArgs& a) { return dim3(std::max<uint32_t>(1, (a.pieces - a.from + kRun - 1) / kRun)); }

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
    Listed l = look_at(gradients, count, workspace);
    if ((s = launch_norm(l, gradients, count, false, st)) != BNS_OK) return s;
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
    Listed l = look_at(gradients, count, workspace);
    l.args.partial = nullptr;
    l.args.squares = const_cast<double*>(squares);
    l.args.max_norm = max_norm;
    return in_parts(l, gradients, count, [&](GradsArgs a, const List& list, int at) {
        a.norm = at > 0 ? nullptr : norm;
        BNS_LAUNCH((grads_scale_kernel<List>), scale_grid(a), dim3(kThreads), 0, st, a, list);
    });
}

bns_status bns_grads_clip(const bns_gradient* gradients, int32_t count, float max_norm, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
    bns_status s = check_call(gradients, count, true, workspace, workspace_bytes);
    if (s != BNS_OK) return s;
    if (!norm || !aligned_all(4, norm) || !fine_norm(max_norm)) return BNS_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    Listed l = look_at(gradients, count, workspace);
    if ((s = launch_norm(l, gradients, count, true, st)) != BNS_OK) return s;
    l.args.norm = norm;
    l.args.max_norm = max_norm;
    if (!l.long_list.grad) {
        return in_parts(l, gradients, count, [&](const GradsArgs& a, const List& list, int) {
            BNS_LAUNCH((grads_scale_kernel<List>), scale_grid(a), dim3(kThreads), 0, st, a, list);
        });
    }
    l.args.entries = l.entries;
    l.args.pieces = l.pieces;
    BNS_LAUNCH((grads_scale_kernel<LongList>), scale_grid(l.args), dim3(kThreads), 0, st, l.args, l.long_list);
    return hipGetLastError() == hipSuccess ? BNS_OK : BNS_EDEVICE;
}

}  // extern "C"
