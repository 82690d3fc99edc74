// Softmax cross entropy from hidden states and the vocabulary's matrix, without keeping the logits, and its gradients.  See include/bns.h.
//
// Three matrix products: the logits (weight hidden^T, computed in the forward pass and again in the backward pass), dhidden = g weight and
// dweight = g^T hidden.  All of them are one kernel: C[m][n] = sum over k of A[m][k] B[n][k] with both operands k-contiguous bf16, tiles
// staged through LDS, fp32 sums on the matrix units, and an epilogue that turns a tile of logits into softmax statistics or into g.  What is not
// k-contiguous bf16 (fp32 operands, which become three bf16 parts; widths and strides that are no multiple of the tile; the
// transposes that the gradients need) is laid out in the workspace first, piece by piece of the vocabulary.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "bns_internal.hpp"
#include "bns_head_device.hpp"
#include "bns_head_direct.hpp"
#include "bns_lm_validate.hpp"

using namespace bns;

namespace {

constexpr int kDepth = 64;      // elements of k in a staged tile: 128 bytes a row

// ---- laying operands out ------------------------------------------------------------------------------------------
struct PackArgs {
    const void* src;
    uint16_t* dst;
    const int64_t* targets;     // rows whose target lies outside [0, vocab) count as zeros; NULL: none do
    int64_t src_stride;
    int32_t rows, cols;         // of src
    int32_t depth;              // elements of k in a plane of dst, padded with zeros; a row of dst holds its planes one behind the other
    int32_t vocab;
};

// Row r of src becomes row r of dst (k = the column).
template <typename T>
__global__ void __launch_bounds__(256) pack_rows_kernel(PackArgs a) {
    constexpr int P = planes_of<T>();
    const int per_row = a.depth / 8;
    const int64_t total = int64_t(a.rows) * per_row;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < total; i += int64_t(gridDim.x) * 256) {
        const int64_t row = i / per_row;
        const int col = int(i - row * per_row) * 8, left = a.cols - col;
        float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (left > 0) Row8<T>::load(static_cast<const T*>(a.src) + row * a.src_stride + col, left, f);
        uint16_t* out = a.dst + row * a.depth * P + col;
        if (P == 1) {
            *reinterpret_cast<u4*>(out) = u4{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
        } else {
            u4 w[3];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t lo[3], hi[3];
                split3(f[2 * j], lo);
                split3(f[2 * j + 1], hi);
#pragma unroll
                for (int p = 0; p < 3; ++p) w[p][j] = lo[p] | hi[p] << 16;
            }
#pragma unroll
            for (int p = 0; p < 3; ++p) *reinterpret_cast<u4*>(out + int64_t(p) * a.depth) = w[p];
        }
    }
}

// Column c of src becomes row c of dst (k = the row), in tiles of 64 x 64 through LDS.
template <typename T>
__global__ void __launch_bounds__(256) pack_columns_kernel(PackArgs a) {
    constexpr int P = planes_of<T>();
    __shared__ float tile[64][65];
    const int c0 = blockIdx.x * 64, r0 = blockIdx.y * 64;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int r = int(threadIdx.x) / 8 + 32 * j, c = int(threadIdx.x) % 8 * 8, row = r0 + r, left = a.cols - (c0 + c);
        float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        bool in = row < a.rows && left > 0;
        if (in && a.targets) {
            const int64_t target = a.targets[row];
            in = target >= 0 && target < a.vocab;
        }
        if (in) Row8<T>::load(static_cast<const T*>(a.src) + int64_t(row) * a.src_stride + c0 + c, left, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) tile[r][c + i] = f[i];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int c = int(threadIdx.x) / 8 + 32 * j, r = int(threadIdx.x) % 8 * 8;
        if (c0 + c >= a.cols) continue;
        uint16_t* out = a.dst + int64_t(c0 + c) * a.depth * P + r0 + r;
        if (P == 1) {
            u4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(tile[r + 2 * i][c], tile[r + 2 * i + 1][c]);
            *reinterpret_cast<u4*>(out) = w;
        } else {
            u4 w[3];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t lo[3], hi[3];
                split3(tile[r + 2 * i][c], lo);
                split3(tile[r + 2 * i + 1][c], hi);
#pragma unroll
                for (int p = 0; p < 3; ++p) w[p][i] = lo[p] | hi[p] << 16;
            }
#pragma unroll
            for (int p = 0; p < 3; ++p) *reinterpret_cast<u4*>(out + int64_t(p) * a.depth) = w[p];
        }
    }
}

// ---- the product --------------------------------------------------------------------------------------------------
// Operands that are k-contiguous bf16 in memory (in three planes, where they are the parts of fp32 values): a row beyond the last is read as the last.
template <int BM, int BN, int WM, int WN>
struct Tile {
    static constexpr int kThreads = WM * WN * kWave, kPerIssue = kThreads / 8;       // rows that all threads bring in at once
    static constexpr int kM = BM / WM, kN = BN / WN, MI = kM / 16, NI = kN / 16;
    static constexpr int kBytes = (BM + BN) * kDepth * 2;
    static_assert(BM % kPerIssue == 0 && BN % kPerIssue == 0, "whole issues");
};

template <typename T, int BM, int BN, int WM, int WN, int EPILOGUE>
__global__ void __launch_bounds__(WM* WN* kWave) gemm_kernel(GemmArgs a) {
#ifdef __HIP_DEVICE_COMPILE__   // (the host compiler has no buffer resources)
    using S = Tile<BM, BN, WM, WN>;
    constexpr int P = planes_of<T>(), kSegments = P == 1 ? 1 : 6;
    __shared__ __attribute__((aligned(1024))) char lds[2][S::kBytes];
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / kWave), lane = threadIdx.x % kWave;
    const int tiles = a.tiles_a * a.tiles_b, split = int(blockIdx.x) / tiles;
    int ta, tb;
    place(int(blockIdx.x) - split * tiles, tiles, a.tiles_a, a.tiles_b, ta, tb);
    const int m0 = ta * BM, n0 = tb * BN;

    // Staging: a wave brings in eight rows of 128 bytes with one instruction, which puts lane after lane into LDS; the 16-byte chunks of row r
    // are swapped by r on their way (chunk c lies at c ^ (r % 8)), so that the reads of 16 rows at one chunk spread over the banks.
    const int last_a = a.rows_a - 1 - m0, last_b = a.rows_b - 1 - n0;
    const auto ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(a.a) + int64_t(m0) * a.lda * 2), 0, -1, 0x00027000);
    const auto rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(a.b) + int64_t(n0) * a.ldb * 2), 0, -1, 0x00027000);
    uint32_t at_a[BM / S::kPerIssue], at_b[BN / S::kPerIssue];
    const int in_row = lane / 8, chunk = (lane % 8) ^ in_row;
#pragma unroll
    for (int i = 0; i < BM / S::kPerIssue; ++i) at_a[i] = uint32_t(min(i * S::kPerIssue + wave * 8 + in_row, last_a)) * uint32_t(a.lda) * 2 + chunk * 16;
#pragma unroll
    for (int i = 0; i < BN / S::kPerIssue; ++i) at_b[i] = uint32_t(min(i * S::kPerIssue + wave * 8 + in_row, last_b)) * uint32_t(a.ldb) * 2 + chunk * 16;

    const int per_plane = a.depth / kDepth, steps = per_plane * kSegments;
    const int first = int(int64_t(steps) * split / a.splits), end = int(int64_t(steps) * (split + 1) / a.splits);
    typedef __attribute__((address_space(3))) void lds_t;
    const auto stage = [&](int step, char* to) {
        int ka = step, kb = step;
        if (kSegments > 1) {
            const int segment = step / per_plane, k = step - segment * per_plane;
            ka = plane_a(segment) * per_plane + k;
            kb = plane_b(segment) * per_plane + k;
        }
#pragma unroll
        for (int i = 0; i < BM / S::kPerIssue; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_t*)(to + (i * S::kPerIssue + wave * 8) * 128), 16, at_a[i], ka * 128, 0, 0);
#pragma unroll
        for (int i = 0; i < BN / S::kPerIssue; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_t*)(to + (BM + i * S::kPerIssue + wave * 8) * 128), 16, at_b[i], kb * 128, 0, 0);
    };

    const int wm = wave / WN, wn = wave % WN, r16 = lane % 16, quarter = lane / 16;
    f32x4 acc[S::MI][S::NI];
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
#pragma unroll
        for (int j = 0; j < S::NI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    if (first < end) stage(first, lds[0]);
    for (int step = first; step < end; ++step) {
        // the tile of this step has landed, and every wave is done with the one before
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        char* const now = lds[(step - first) & 1];
        if (step + 1 < end) stage(step + 1, lds[(step + 1 - first) & 1]);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            bf16x8 fa[S::MI], fb[S::NI];
            const int at = ((kk * 4 + quarter) ^ (r16 % 8)) * 16;
#pragma unroll
            for (int j = 0; j < S::NI; ++j) fb[j] = *reinterpret_cast<const bf16x8*>(now + (BM + wn * S::kN + j * 16 + r16) * 128 + at);
#pragma unroll
            for (int i = 0; i < S::MI; ++i) fa[i] = *reinterpret_cast<const bf16x8*>(now + (wm * S::kM + i * 16 + r16) * 128 + at);
#pragma unroll
            for (int i = 0; i < S::MI; ++i)
#pragma unroll
                for (int j = 0; j < S::NI; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[i], fb[j], acc[i][j], 0, 0, 0);
        }
    }

    finish<T, EPILOGUE, BM, BN, WM, WN>(a, acc, ta, tb, split, reinterpret_cast<float2*>(lds));
#endif
}

template <typename T, int BM, int BN, int WM, int WN, int EPILOGUE>
__global__ void __launch_bounds__(WM* WN* kWave) direct_logits_kernel(GemmArgs a) {
    __shared__ __attribute__((aligned(16))) char lds[DirectTile<T, BM, BN, WM, WN>::kBytes];
    direct_tile<T, BM, BN, WM, WN, true, true, EPILOGUE>(a, int(blockIdx.x), lds);
}

// Both gradients from g in one launch: the first blocks take dhidden, whose k is the vocabulary, the others dweight, whose k is the tokens.
template <typename T, int BM, int BN, int WM, int WN, int BW, int EPILOGUE>
__global__ void __launch_bounds__(256) direct_gradients_kernel(GemmArgs h, GemmArgs w, int blocks_h) {
    constexpr int kH = DirectTile<T, BM, BN, WM, WN>::kBytes, kW = DirectTile<T, BW, BW, 2, 2>::kBytes;
    __shared__ __attribute__((aligned(16))) char lds[kH > kW ? kH : kW];
    if (int(blockIdx.x) < blocks_h) direct_tile<T, BM, BN, WM, WN, false, true, EPILOGUE>(h, int(blockIdx.x), lds);
    else direct_tile<T, BW, BW, 2, 2, false, false, kStore>(w, int(blockIdx.x) - blocks_h, lds);
}

// ---- what follows the products --------------------------------------------------------------------------------------
// loss and lse from the statistics of the tiles: 16 tokens a block, 16 threads each.
__global__ void __launch_bounds__(256) join_statistics_kernel(const float2* partial, const float* at_target, const int64_t* targets, int tiles, int tokens, int vocab,
                                                               float* loss, float* lse) {
    __shared__ float2 part[16][17];
    const int c = threadIdx.x % 16, lane = threadIdx.x / 16, token = blockIdx.x * 16 + c;
    float m = -3e38f, l = 0.f;
    if (token < tokens) {
        for (int i = lane; i < tiles; i += 16) {
            const float2 p = partial[int64_t(i) * tokens + token];
            const float most = fmaxf(m, p.x);
            l = l * __builtin_amdgcn_exp2f(m - most) + p.y * __builtin_amdgcn_exp2f(p.x - most);
            m = most;
        }
    }
    part[lane][c] = float2{m, l};
    __syncthreads();
    if (lane != 0 || token >= tokens) return;
    for (int i = 1; i < 16; ++i) m = fmaxf(m, part[i][c].x);
    l = 0.f;
    for (int i = 0; i < 16; ++i) l = fmaf(part[i][c].y, __builtin_amdgcn_exp2f(part[i][c].x - m), l);
    const float all = (m + __builtin_amdgcn_logf(l)) * kLn2;
    const int64_t target = targets[token];
    lse[token] = all;
    loss[token] = target >= 0 && target < vocab ? all - at_target[token] : 0.f;
}

// dhidden from the sums that the splits left behind.
template <typename T>
__global__ void __launch_bounds__(256) join_splits_kernel(const float* part, int64_t split_stride, int splits, int tokens, int width, int ld, T* out) {
    const int per_row = (width + 7) / 8;
    const int64_t total = int64_t(tokens) * per_row;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < total; i += int64_t(gridDim.x) * 256) {
        const int64_t row = i / per_row;
        const int col = int(i - row * per_row) * 8;
        float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int k = 0; k < splits; ++k) {
            const f32x4* p = reinterpret_cast<const f32x4*>(part + k * split_stride + row * ld + col);
            const f32x4 x = p[0], y = p[1];
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += x[e], s[4 + e] += y[e];
        }
        Row8<T>::store(out + row * width + col, width - col, s);
    }
}

__global__ void __launch_bounds__(256) fill_zero_kernel(uint16_t* p, int64_t n) {
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256) p[i] = 0;
}

// ---- the plan -------------------------------------------------------------------------------------------------------
constexpr int kTileM = 256;

struct HeadPlan {
    bool direct;                            // operands are read as they lie in memory
    int tile;                               // direct: tokens of a tile, 16, 32, 64 or 128
    int64_t piece;                          // rows of a piece of the vocabulary
    int splits;                             // of dhidden
    // laid out:
    int planes;
    int64_t depth_d, depth_t;               // padded width, tokens
    bool direct_h, direct_w;                // read where they are, without a copy
    bool narrow;                            // few tokens: tiles of 64 of them
    // offsets into the workspace
    size_t hidden, weight, partial, at_target, weight_t, hidden_t, g, gt, sums, forward_bytes, backward_bytes;
};

struct Offsets {
    size_t at = 0;
    size_t take(size_t bytes) {
        const size_t here = at;
        at += (bytes + 1023) & ~size_t(1023);
        return here;
    }
};

HeadPlan direct_plan(const HeadDims& d) {
    HeadPlan p = {};
    const size_t e = dtype_bytes(d.dtype), T = size_t(d.tokens);
    p.direct = true;
    p.tile = d.tokens <= 16 ? 16 : d.tokens <= 32 ? 32 : 64;
    if (g_tuning.head_tile == 128) p.tile = 128;
    p.depth_d = round_up(d.width, 8);
    // g of a piece takes 64 MB at most
    const int64_t piece = d.piece ? d.piece : std::max<int64_t>(1024, (int64_t(64) << 20) / int64_t(std::max<size_t>(T * e, 1)));
    p.piece = std::min(round_up(std::min<int64_t>(piece, 1 << 19), kTileM), round_up(d.vocab, kTileM));
    const int m = p.tile == 128 ? 128 : 64;
    const int64_t tiles = ((d.width + m - 1) / m) * ((d.tokens + p.tile - 1) / p.tile), steps = std::min<int64_t>(p.piece, d.vocab) / (d.dtype == BNS_F32 ? 32 : 64);
    p.splits = int(std::max<int64_t>(1, std::min<int64_t>(1024 / std::max<int64_t>(tiles, 1), steps / 4)));
    Offsets o;
    p.partial = o.take(size_t((d.vocab + m - 1) / m) * T * sizeof(float2));
    p.at_target = o.take(T * 4);
    p.forward_bytes = o.at;
    o.at = 0;
    p.g = o.take(T * p.piece * e);
    p.sums = o.take(size_t(p.splits) * T * p.depth_d * 4);
    p.backward_bytes = o.at;
    return p;
}

HeadPlan laid_out_plan(const HeadDims& d) {
    HeadPlan p = {};
    p.planes = d.dtype == BNS_F32 ? 3 : 1;
    p.depth_d = round_up(d.width, kDepth);
    p.depth_t = round_up(std::max<int64_t>(d.tokens, 1), kDepth);
    const bool fits = d.dtype == BNS_BF16 && d.width % kDepth == 0;
    p.direct_h = fits && d.hidden_stride % 8 == 0 && d.hidden_stride < (1 << 21);
    p.direct_w = fits && d.weight_stride % 8 == 0 && d.weight_stride < (1 << 21);
    p.narrow = d.tokens <= 64;
    const int64_t piece = d.piece ? d.piece : 16384;
    p.piece = std::min(round_up(std::min<int64_t>(piece, 1 << 18), kTileM), round_up(d.vocab, kTileM));
    const int64_t tiles = ((d.width + kTileM - 1) / kTileM) * ((d.tokens + (p.narrow ? 63 : 255)) / (p.narrow ? 64 : 256));
    p.splits = int(std::max<int64_t>(1, std::min<int64_t>(256 / std::max<int64_t>(tiles, 1), p.piece / 512)));
    const size_t P = size_t(p.planes) * 2, T = size_t(d.tokens), rows = size_t(p.piece);
    Offsets o;
    p.hidden = o.take(p.direct_h ? 0 : T * p.depth_d * P);
    p.weight = o.take(p.direct_w ? 0 : rows * p.depth_d * P);
    const size_t both = o.at;
    p.partial = o.take(size_t((d.vocab + kTileM - 1) / kTileM) * T * sizeof(float2));
    p.at_target = o.take(T * 4);
    p.forward_bytes = o.at;
    o.at = both;
    p.weight_t = o.take(size_t(d.width) * rows * P);
    p.hidden_t = o.take(size_t(d.width) * p.depth_t * P);
    p.g = o.take(T * rows * P);
    p.gt = o.take(rows * p.depth_t * P);
    p.sums = o.take(size_t(p.splits) * T * p.depth_d * 4);
    p.backward_bytes = o.at;
    return p;
}

HeadPlan head_plan(const HeadDims& d) {
    const int path = g_tuning.head_path;
    const bool direct = path ? path == 1 : d.tokens <= 64;
    return direct ? direct_plan(d) : laid_out_plan(d);
}

// (never 0, which stands for an invalid description)
inline size_t need(const HeadPlan& p) { return std::max<size_t>(std::max(p.forward_bytes, p.backward_bytes), 1024); }

inline bool failed() { return hipGetLastError() != hipSuccess; }

template <typename T>
bool pack_rows(const void* src, int64_t stride, int64_t rows, int width, int64_t depth, void* dst, hipStream_t st) {
    const PackArgs a = {src, static_cast<uint16_t*>(dst), nullptr, stride, int32_t(rows), width, int32_t(depth), 0};
    const int64_t blocks = (rows * (depth / 8) + 255) / 256;
    BNS_LAUNCH((pack_rows_kernel<T>), dim3(uint32_t(std::min<int64_t>(blocks, 1 << 16))), dim3(256), 0, st, a);
    return !failed();
}

template <typename T>
bool pack_columns(const void* src, int64_t stride, int64_t rows, int width, int64_t depth, const int64_t* targets, int vocab, void* dst, hipStream_t st) {
    const PackArgs a = {src, static_cast<uint16_t*>(dst), targets, stride, int32_t(rows), width, int32_t(depth), vocab};
    BNS_LAUNCH((pack_columns_kernel<T>), dim3((width + 63) / 64, uint32_t(depth / 64)), dim3(256), 0, st, a);
    return !failed();
}

template <typename T, int EPILOGUE>
bool gemm(GemmArgs a, bool narrow, hipStream_t st) {
    a.tiles_a = (a.rows_a + kTileM - 1) / kTileM;
    a.tiles_b = narrow ? (a.rows_b + 63) / 64 : (a.rows_b + 255) / 256;
    const dim3 grid(uint32_t(a.tiles_a) * a.tiles_b * a.splits);
    if (narrow) BNS_LAUNCH((gemm_kernel<T, 256, 64, 4, 2, EPILOGUE>), grid, dim3(512), 0, st, a);
    else BNS_LAUNCH((gemm_kernel<T, 256, 256, 2, 4, EPILOGUE>), grid, dim3(512), 0, st, a);
    return !failed();
}

bool join_statistics(const HeadDims& d, const HeadPlan& p, int tile, const int64_t* targets, float* loss, float* lse, char* ws, hipStream_t st) {
    BNS_LAUNCH(join_statistics_kernel, dim3(uint32_t((d.tokens + 15) / 16)), dim3(256), 0, st, reinterpret_cast<const float2*>(ws + p.partial),
               reinterpret_cast<const float*>(ws + p.at_target), targets, (d.vocab + tile - 1) / tile, int(d.tokens), d.vocab, loss, lse);
    return !failed();
}

template <typename T>
bool join_splits(const HeadDims& d, const HeadPlan& p, void* dhidden, char* ws, hipStream_t st) {
    const int64_t blocks = (d.tokens * ((d.width + 7) / 8) + 255) / 256;
    BNS_LAUNCH((join_splits_kernel<T>), dim3(uint32_t(std::min<int64_t>(blocks, 1 << 16))), dim3(256), 0, st, reinterpret_cast<const float*>(ws + p.sums),
               d.tokens * p.depth_d, p.splits, int(d.tokens), d.width, int(p.depth_d), static_cast<T*>(dhidden));
    return !failed();
}

// The operands of the logits of rows [v0, v0 + rows) of the vocabulary; packs what has to be packed.
template <typename T>
bool logits_operands(const HeadDims& d, const HeadPlan& p, const void* hidden, const void* weight, char* ws, int v0, int rows, hipStream_t st, GemmArgs* a) {
    const int64_t packed = p.depth_d * p.planes;
    a->b = p.direct_h ? hidden : ws + p.hidden;
    a->ldb = p.direct_h ? d.hidden_stride : packed;
    const void* piece = static_cast<const T*>(weight) + int64_t(v0) * d.weight_stride;
    a->a = p.direct_w ? piece : ws + p.weight;
    a->lda = p.direct_w ? d.weight_stride : packed;
    a->rows_a = rows;
    a->rows_b = int32_t(d.tokens);
    a->depth = int32_t(p.depth_d);
    a->splits = 1;
    a->v0 = v0;
    a->vocab = d.vocab;
    return p.direct_w || pack_rows<T>(piece, d.weight_stride, rows, d.width, p.depth_d, ws + p.weight, st);
}

template <typename T>
bool forward(const HeadDims& d, const HeadPlan& p, const void* hidden, const void* weight, const int64_t* targets, float* loss, float* lse, char* ws, hipStream_t st) {
    if (!p.direct_h && !pack_rows<T>(hidden, d.hidden_stride, d.tokens, d.width, p.depth_d, ws + p.hidden, st)) return false;
    // (without copies the whole vocabulary is one piece, as far as a launch goes: 2^22 blocks)
    const int64_t most = std::max<int64_t>(1, (1 << 22) / ((d.tokens + 63) / 64)) * kTileM, step = p.direct_w ? std::min<int64_t>(d.vocab, most) : p.piece;
    for (int64_t v0 = 0; v0 < d.vocab; v0 += step) {
        GemmArgs a = {};
        if (!logits_operands<T>(d, p, hidden, weight, ws, int(v0), int(std::min<int64_t>(step, d.vocab - v0)), st, &a)) return false;
        a.targets = targets;
        a.partial = reinterpret_cast<float2*>(ws + p.partial);
        a.at_target = reinterpret_cast<float*>(ws + p.at_target);
        if (!gemm<T, kStatistics>(a, p.narrow, st)) return false;
    }
    return join_statistics(d, p, kTileM, targets, loss, lse, ws, st);
}

template <typename T>
bool backward(const HeadDims& d, const HeadPlan& p, const void* hidden, const void* weight, const int64_t* targets, const float* lse, const float* dloss,
              void* dhidden, void* dweight, char* ws, hipStream_t st) {
    const int planes = p.planes;
    if (!p.direct_h && !pack_rows<T>(hidden, d.hidden_stride, d.tokens, d.width, p.depth_d, ws + p.hidden, st)) return false;
    if (!pack_columns<T>(hidden, d.hidden_stride, d.tokens, d.width, p.depth_t, targets, d.vocab, ws + p.hidden_t, st)) return false;
    for (int64_t v0 = 0; v0 < d.vocab; v0 += p.piece) {
        const int rows = int(std::min<int64_t>(p.piece, d.vocab - v0));
        const int64_t depth_v = round_up(rows, kDepth);
        GemmArgs a = {};
        if (!logits_operands<T>(d, p, hidden, weight, ws, int(v0), rows, st, &a)) return false;
        a.targets = targets;
        a.lse = lse;
        a.dloss = dloss;
        a.g = reinterpret_cast<uint16_t*>(ws + p.g);
        a.gt = reinterpret_cast<uint16_t*>(ws + p.gt);
        a.g_depth = int32_t(depth_v);
        a.gt_depth = int32_t(p.depth_t);
        if (!gemm<T, kGradientParts>(a, p.narrow, st)) return false;
        const void* piece = static_cast<const T*>(weight) + v0 * d.weight_stride;
        if (!pack_columns<T>(piece, d.weight_stride, rows, d.width, depth_v, nullptr, 0, ws + p.weight_t, st)) return false;
        // dhidden[n][m] += sum over the piece of g[n] weight[m]
        GemmArgs h = {};
        h.a = ws + p.weight_t;
        h.b = ws + p.g;
        h.lda = h.ldb = depth_v * planes;
        h.rows_a = d.width;
        h.rows_b = int32_t(d.tokens);
        h.depth = int32_t(depth_v);
        h.splits = p.splits;
        h.out = ws + p.sums;
        h.ldo = p.depth_d;
        h.split_stride = d.tokens * p.depth_d;
        h.fresh = v0 == 0;
        if (!gemm<T, kAccumulate>(h, p.narrow, st)) return false;
        // dweight[n][m] = sum over the tokens of g[n] hidden[m]
        GemmArgs w = {};
        w.a = ws + p.hidden_t;
        w.b = ws + p.gt;
        w.lda = w.ldb = p.depth_t * planes;
        w.rows_a = d.width;
        w.rows_b = rows;
        w.depth = int32_t(p.depth_t);
        w.splits = 1;
        w.out = static_cast<T*>(dweight) + v0 * d.width;
        w.ldo = d.width;
        if (!gemm<T, kStore>(w, false, st)) return false;
    }
    return join_splits<T>(d, p, dhidden, ws, st);
}

// ---- the same, operands as they lie in memory -------------------------------------------------------------------------
template <typename T, int EPILOGUE>
bool direct_logits(GemmArgs a, int tile, hipStream_t st) {
    const int m = tile == 128 ? 128 : 64;
    a.tiles_a = (a.rows_a + m - 1) / m;
    a.tiles_b = (a.rows_b + tile - 1) / tile;
    const dim3 grid(uint32_t(a.tiles_a) * a.tiles_b);
    if (tile == 16) BNS_LAUNCH((direct_logits_kernel<T, 64, 16, 4, 1, EPILOGUE>), grid, dim3(256), 0, st, a);
    else if (tile == 32) BNS_LAUNCH((direct_logits_kernel<T, 64, 32, 4, 1, EPILOGUE>), grid, dim3(256), 0, st, a);
    else if (tile == 64) BNS_LAUNCH((direct_logits_kernel<T, 64, 64, 2, 2, EPILOGUE>), grid, dim3(256), 0, st, a);
    else BNS_LAUNCH((direct_logits_kernel<T, 128, 128, 2, 2, EPILOGUE>), grid, dim3(256), 0, st, a);
    return !failed();
}

template <typename T, int EPILOGUE>
bool direct_gradients(GemmArgs h, GemmArgs w, int tile, hipStream_t st) {
    const int m = tile == 128 ? 128 : 64;
    h.tiles_a = w.tiles_a = (h.rows_a + m - 1) / m;
    h.tiles_b = (h.rows_b + tile - 1) / tile;
    w.tiles_b = (w.rows_b + m - 1) / m;
    const int blocks_h = h.tiles_a * h.tiles_b * h.splits;
    const dim3 grid(uint32_t(blocks_h) + uint32_t(w.tiles_a) * w.tiles_b);
    if (tile == 16) BNS_LAUNCH((direct_gradients_kernel<T, 64, 16, 4, 1, 64, EPILOGUE>), grid, dim3(256), 0, st, h, w, blocks_h);
    else if (tile == 32) BNS_LAUNCH((direct_gradients_kernel<T, 64, 32, 4, 1, 64, EPILOGUE>), grid, dim3(256), 0, st, h, w, blocks_h);
    else if (tile == 64) BNS_LAUNCH((direct_gradients_kernel<T, 64, 64, 2, 2, 64, EPILOGUE>), grid, dim3(256), 0, st, h, w, blocks_h);
    else BNS_LAUNCH((direct_gradients_kernel<T, 128, 128, 2, 2, 128, EPILOGUE>), grid, dim3(256), 0, st, h, w, blocks_h);
    return !failed();
}

GemmArgs direct_operands(const HeadDims& d, const void* hidden, const void* weight, const int64_t* targets, int64_t v0, int rows) {
    GemmArgs a = {};
    a.a = static_cast<const char*>(weight) + v0 * d.weight_stride * int64_t(dtype_bytes(d.dtype));
    a.b = hidden;
    a.lda = d.weight_stride;
    a.ldb = d.hidden_stride;
    a.rows_a = rows;
    a.rows_b = int32_t(d.tokens);
    a.depth = d.width;
    a.splits = 1;
    a.targets = targets;
    a.v0 = int32_t(v0);
    a.vocab = d.vocab;
    return a;
}

template <typename T>
bool forward_direct(const HeadDims& d, const HeadPlan& p, const void* hidden, const void* weight, const int64_t* targets, float* loss, float* lse, char* ws,
                    hipStream_t st) {
    const int m = p.tile == 128 ? 128 : 64;
    const int64_t most = std::max<int64_t>(1, (1 << 22) / ((d.tokens + p.tile - 1) / p.tile)) * m;
    for (int64_t v0 = 0; v0 < d.vocab; v0 += most) {
        GemmArgs a = direct_operands(d, hidden, weight, targets, v0, int(std::min<int64_t>(most, d.vocab - v0)));
        a.partial = reinterpret_cast<float2*>(ws + p.partial);
        a.at_target = reinterpret_cast<float*>(ws + p.at_target);
        if (!direct_logits<T, kStatistics>(a, p.tile, st)) return false;
    }
    return join_statistics(d, p, m, targets, loss, lse, ws, st);
}

template <typename T>
bool backward_direct(const HeadDims& d, const HeadPlan& p, const void* hidden, const void* weight, const int64_t* targets, const float* lse, const float* dloss,
                     void* dhidden, void* dweight, char* ws, hipStream_t st) {
    const bool whole = p.splits == 1 && p.piece >= d.vocab;     // dhidden needs no sums beside it
    for (int64_t v0 = 0; v0 < d.vocab; v0 += p.piece) {
        const int rows = int(std::min<int64_t>(p.piece, d.vocab - v0));
        GemmArgs a = direct_operands(d, hidden, weight, targets, v0, rows);
        a.lse = lse;
        a.dloss = dloss;
        a.out = ws + p.g;
        a.ldo = p.piece;
        if (!direct_logits<T, kGradient>(a, p.tile, st)) return false;
        GemmArgs h = {};
        h.a = a.a;
        h.lda = a.lda;
        h.b = ws + p.g;
        h.ldb = p.piece;
        h.rows_a = d.width;
        h.rows_b = int32_t(d.tokens);
        h.depth = rows;
        h.splits = p.splits;
        h.out = whole ? dhidden : ws + p.sums;
        h.ldo = whole ? d.width : p.depth_d;
        h.split_stride = d.tokens * p.depth_d;
        h.fresh = v0 == 0;
        GemmArgs w = {};
        w.a = hidden;
        w.lda = d.hidden_stride;
        w.b = ws + p.g;
        w.ldb = p.piece;
        w.rows_a = d.width;
        w.rows_b = rows;
        w.depth = int32_t(d.tokens);
        w.splits = 1;
        w.targets = targets;
        w.vocab = d.vocab;
        w.out = static_cast<T*>(dweight) + v0 * d.width;
        w.ldo = d.width;
        if (whole ? !direct_gradients<T, kStore>(h, w, p.tile, st) : !direct_gradients<T, kAccumulate>(h, w, p.tile, st)) return false;
    }
    return whole || join_splits<T>(d, p, dhidden, ws, st);
}

}  // namespace

extern "C" {

size_t bns_head_workspace_bytes(const bns_head* head) {
    HeadDims d;
    if (check_head(head, &d) != BNS_OK) return 0;
    const HeadPlan p = head_plan(d);
    return need(p);
}

bns_status bns_head_forward(const bns_head* head, const void* hidden, const void* weight, const int64_t* targets, float* loss, float* lse,
                            void* workspace, size_t workspace_bytes, void* stream) {
    HeadDims d;
    const bns_status s = check_head(head, &d);
    if (s != BNS_OK) return s;
    if (d.tokens == 0) return BNS_OK;
    if (!hidden || !weight || !targets || !loss || !lse || !workspace) return BNS_EINVAL;
    if (!aligned16(hidden) || !aligned16(weight) || !aligned16(workspace)) return BNS_EINVAL;
    const HeadPlan p = head_plan(d);
    if (workspace_bytes < need(p)) return BNS_EWORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    char* ws = static_cast<char*>(workspace);
    const auto call = d.dtype == BNS_F32 ? (p.direct ? forward_direct<float> : forward<float>) : p.direct ? forward_direct<bf16_t> : forward<bf16_t>;
    const bool ok = call(d, p, hidden, weight, targets, loss, lse, ws, st);
    return ok ? BNS_OK : BNS_EDEVICE;
}

bns_status bns_head_backward(const bns_head* head, const void* hidden, const void* weight, const int64_t* targets, const float* lse, const float* dloss,
                             void* dhidden, void* dweight, void* workspace, size_t workspace_bytes, void* stream) {
    HeadDims d;
    const bns_status s = check_head(head, &d);
    if (s != BNS_OK) return s;
    if (!weight || !dweight || !workspace || (d.tokens > 0 && (!hidden || !targets || !lse || !dloss || !dhidden))) return BNS_EINVAL;
    for (const void* q : {hidden, weight, static_cast<const void*>(dhidden), static_cast<const void*>(dweight), static_cast<const void*>(workspace)})
        if (!aligned16(q)) return BNS_EINVAL;
    const size_t e = dtype_bytes(d.dtype), row = size_t(d.width) * e;
    const Matrix mh = matrix(hidden, d.tokens, d.width, d.hidden_stride, e), mw = matrix(weight, d.vocab, d.width, d.weight_stride, e),
                 mdh = matrix(dhidden, d.tokens, d.width, d.width, e), mdw = matrix(dweight, d.vocab, d.width, d.width, e);
    for (const Matrix& out : {mdh, mdw})
        for (const Matrix& in : {mh, mw})
            if (collide(out, in, false, row, row)) return BNS_EINVAL;
    if (collide(mdh, mdw, false, row, row)) return BNS_EINVAL;
    const HeadPlan p = head_plan(d);
    if (workspace_bytes < need(p)) return BNS_EWORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    char* ws = static_cast<char*>(workspace);
    if (d.tokens == 0) {
        BNS_LAUNCH(fill_zero_kernel, dim3(4096), dim3(256), 0, st, static_cast<uint16_t*>(dweight), int64_t(d.vocab) * d.width * int64_t(e / 2));
        return failed() ? BNS_EDEVICE : BNS_OK;
    }
    const auto call = d.dtype == BNS_F32 ? (p.direct ? backward_direct<float> : backward<float>) : p.direct ? backward_direct<bf16_t> : backward<bf16_t>;
    const bool ok = call(d, p, hidden, weight, targets, lse, dloss, dhidden, dweight, ws, st);
    return ok ? BNS_OK : BNS_EDEVICE;
}

}  // extern "C"
