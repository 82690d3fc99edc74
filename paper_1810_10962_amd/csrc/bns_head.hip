// Softmax cross entropy from hidden states and the vocabulary's matrix, without keeping the logits, and its gradients.  See include/bns.h.
//
// Three matrix products: the logits (weight hidden^T, computed in the forward pass and again in the backward pass), dhidden = g weight and
// dweight = g^T hidden.  C[m][n] = sum over k of A[m][k] B[n][k] on the matrix units, bf16 operands (fp32 values as three bf16 parts) and fp32
// sums, with an epilogue that turns a tile of logits into softmax statistics or into g.  Three families of kernels, see the plan below:
// few tokens (bns_head_stream.hpp), operands as they lie in memory (bns_head_direct.hpp), operands laid out first (bns_head_laid_out.hpp).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "bns_head_direct.hpp"
#include "bns_head_laid_out.hpp"
#include "bns_head_stream.hpp"
#include "bns_internal.hpp"
#include "bns_lm_validate.hpp"

using namespace bns;

namespace {

// (Sixteen tokens stream the matrix, and seven waves on a unit that could hold six keep more of it on its way.)
template <typename T, int BM, int BN, int WM, int WN, int GROUPS, int EPILOGUE, bool NT = false>
__global__ void __launch_bounds__(256 * GROUPS, BN == 16 && GROUPS == 1 ? 7 : 1) direct_logits_kernel(GemmArgs a) {
    __shared__ __attribute__((aligned(16))) char lds[GROUPS * DirectTile<T, BM, BN, WM, WN>::kBytes];
    direct_tile<T, BM, BN, WM, WN, GROUPS, true, true, EPILOGUE, NT>(a, int(blockIdx.x), lds);
}

// Both gradients from g in one launch: `blocks_h` blocks take dhidden, whose k is the vocabulary, the others dweight, whose k is the tokens.  `ahead` of the
// latter (all or none) go first, where their chains of steps are the longer ones (700x700x7000 fp32 181 against 200 us, 1200x64x100000 bf16 232 against 253).
template <typename T, int BM, int BN, int WM, int WN, int BW, int GROUPS, int EPILOGUE>
__global__ void __launch_bounds__(256 * GROUPS) direct_gradients_kernel(GemmArgs h, GemmArgs w, int blocks_h, int ahead) {
    constexpr int kH = DirectTile<T, BM, BN, WM, WN>::kBytes, kW = DirectTile<T, BW, BW, 2, 2>::kBytes;
    __shared__ __attribute__((aligned(16))) char lds[GROUPS * (kH > kW ? kH : kW)];
    const int b = int(blockIdx.x) - ahead;
    if (b >= 0 && b < blocks_h) direct_tile<T, BM, BN, WM, WN, GROUPS, false, true, EPILOGUE>(h, b, lds);
    else direct_tile<T, BW, BW, 2, 2, GROUPS, false, false, kStore>(w, b < 0 ? int(blockIdx.x) : b - blocks_h, lds);
}

// ---- what follows the products --------------------------------------------------------------------------------------
// loss and lse from the statistics of the tiles: TOKENS tokens a block, 256 / TOKENS threads each (few tokens have many tiles each and need them all).
template <int TOKENS>
__global__ void __launch_bounds__(256) join_statistics_kernel(const float2* partial, const float* at_target, const int64_t* targets, int tiles, int tokens, int vocab,
                                                               float* loss, float* lse) {
    constexpr int kLanes = 256 / TOKENS;
    __shared__ float2 part[kLanes][TOKENS];
    const int c = threadIdx.x % TOKENS, lane = threadIdx.x / TOKENS, token = blockIdx.x * TOKENS + c;
    float m = kLowest, l = 0.f;
    if (token < tokens) {
#pragma unroll 4
        for (int i = lane; i < tiles; i += kLanes) {
            const float2 p = partial[int64_t(i) * tokens + token];
            const float most = fmaxf(m, p.x);
            l = l * __builtin_amdgcn_exp2f((m - most) * kLog2e) + p.y * __builtin_amdgcn_exp2f((p.x - most) * kLog2e);
            m = most;
        }
    }
    part[lane][c] = float2{m, l};
    for (int half = kLanes / 2; half > 0; half /= 2) {
        __syncthreads();
        if (lane >= half) continue;
        const float2 p = part[lane + half][c];
        const float most = fmaxf(m, p.x);
        l = l * __builtin_amdgcn_exp2f((m - most) * kLog2e) + p.y * __builtin_amdgcn_exp2f((p.x - most) * kLog2e);
        m = most;
        part[lane][c] = float2{m, l};
    }
    if (lane != 0 || token >= tokens) return;
    // (m is a logit, so m - z is exact near zero and never below it, and neither is the logarithm of a sum that holds exp(0))
    const float log2_l = __builtin_amdgcn_logf(l);
    const int64_t target = targets[token];
    lse[token] = fmaf(log2_l, kLn2, m);
    loss[token] = target >= 0 && target < vocab ? fmaf(log2_l, kLn2, m - at_target[token]) : 0.f;
}

// dhidden from the sums that the splits left behind: 8 columns x 32 a block and row, LANES threads each take every LANES-th split.
template <typename T, int LANES>
__global__ void __launch_bounds__(32 * LANES) join_splits_kernel(const float* part, int64_t split_stride, int splits, int tokens, int width, int64_t ld, T* out) {
    __shared__ f32x4 sums[LANES > 1 ? LANES - 1 : 1][2][32];
    const int c = threadIdx.x % 32, lane = threadIdx.x / 32, per_row = (width + 255) / 256;
    for (int64_t b = blockIdx.x; b < int64_t(tokens) * per_row; b += gridDim.x) {
        const int64_t row = b / per_row;
        const int col = (int(b - row * per_row) * 32 + c) * 8;
        f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
        if (col < width) {
#pragma unroll 4
            for (int k = lane; k < splits; k += LANES) {
                const f32x4* p = reinterpret_cast<const f32x4*>(part + k * split_stride + row * ld + col);
                x += p[0];
                y += p[1];
            }
        }
        if constexpr (LANES > 1) {
            __syncthreads();
            if (lane > 0) {
                sums[lane - 1][0][c] = x;
                sums[lane - 1][1][c] = y;
            }
            __syncthreads();
            if (lane > 0) continue;
#pragma unroll
            for (int k = 0; k < LANES - 1; ++k) {
                x += sums[k][0][c];
                y += sums[k][1][c];
            }
        }
        const float f[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
        if (col < width) Row8<T>::store(out + row * width + col, width - col, f);
    }
}

__global__ void __launch_bounds__(256) fill_zero_kernel(uint16_t* p, int64_t n) {
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256) p[i] = 0;
}

// ---- the plan -------------------------------------------------------------------------------------------------------
// Kernels of a product.
enum Kind { kStream = 1, kDirect64, kDirect128, kGemm256, kGemm128 };

inline int rows_of(Kind kind, const HeadDims& d) {      // rows of the vocabulary in a tile of logits
    switch (kind) {
        case kStream: return d.vocab < 16384 ? 16 : 32;  // (a small vocabulary needs the blocks)
        case kDirect64: return 64;
        case kGemm256: return 256;
        default: return 128;
    }
}

struct HeadPlan {
    Kind kind;                              // of the logits
    Kind gradients;
    int planes;
    int64_t piece;                          // rows of a piece of the vocabulary
    int64_t depth_d, depth_t;               // padded width, tokens
    int splits, splits_w;                   // of dhidden; of dweight's rows (kStream)
    bool copy_h, copy_w;                    // the laid-out logits need copies of hidden, weight
    // offsets into the workspace
    size_t hidden, weight, partial, at_target, weight_t, hidden_t, g, gt, sums, bytes;

    bool parts() const { return gradients == kStream || gradients >= kGemm256; }     // g as kGradientParts
};

inline int tiles_of(int64_t rows, int tile) { return int((rows + tile - 1) / tile); }

// Whether the laid-out kernels read an operand where it is.
inline bool lies_well(const HeadDims& d, int64_t stride) { return d.dtype == BNS_BF16 && d.width % kDepth == 0 && stride % 8 == 0 && stride < (1 << 21); }

// Times below: tokens x width x vocabulary, forward pass in us (best alternative behind "against").
inline Kind logits_kind(const HeadDims& d, bool backward) {
    const int chosen = backward ? g_tuning.head_logits_backward : g_tuning.head_logits;
    if (chosen) return Kind(chosen);
    const bool f32 = d.dtype == BNS_F32;
    const auto tiles = [&](int tile) { return int64_t(tiles_of(d.tokens, tile)) * tiles_of(d.vocab, tile); };
    // Fewer tiles of 64 than half of the compute units and few tokens: what counts is how long a block takes along the width, which kStream divides between
    // its waves without LDS (fp32 9x1792x1071 15 against 27, 16x4096x4000 26 against 53, 32x1024x2000 16 against 21, but 60x2048x7000 48 against 41;
    // bf16 16x4096x4000 16 against 20, 4x2048x2000 12 against 13, but 32x4096x7000 32 against 22, 2x512x8000 12 against 10).
    if (tiles(64) < 128 && (f32 ? d.tokens <= 32 && d.width >= 512 : d.tokens <= 16 && d.width >= 1536)) return kStream;
    const bool well = lies_well(d, d.hidden_stride) && lies_well(d, d.weight_stride);
    // Tiles of 256 need two rounds of blocks (bf16 4096x4096x16384 435 against 523) and tokens that fill them; copies need many uses of what they lay out
    // (fp32 4096x4096x16384 2610 against 2690, but bf16 1068x110x102656 190 against 123).
    if (tiles(256) >= 400 && (well ? d.tokens > 192 : d.tokens >= 2048 && d.width >= 1024)) return kGemm256;
    // Without copies the laid-out kernels win as soon as they have the blocks (1024x1024x8192 25 against 31, but 226x1728x1148, 18 tiles, 26 against 16).
    if (well && d.tokens > 32 && tiles(128) >= 128) return kGemm128;
    // fp32 256x512x32000 54 against 71, but 1663x128x1920, 195 tiles, 17.2 against 16.3
    return d.tokens > 64 && tiles(128) >= 256 ? kDirect128 : kDirect64;
}

// Times: whole backward pass, in us.
inline Kind gradients_kind(const HeadDims& d) {
    const int chosen = g_tuning.head_gradients;
    const bool f32 = d.dtype == BNS_F32;
    const bool few = d.tokens <= (f32 ? 32 : 64);        // what kStream holds in registers
    if (chosen && (chosen != kStream || few)) return Kind(chosen);
    const int64_t matrix = int64_t(d.width) * d.vocab;
    // bf16 16x2048x50257 160 against 192, 2x384x85765 57 against 72, 16x512x16384 23 against 26, but 40x1024x4096 30 against 23 (for 33 to 64 tokens
    // the line lies low: 51x576x14720 50 against 30, 64x1152x112896 283 against 236); fp32 1x3520x87977 917 against 1013, 8x2048x70000 472 against 506,
    // 32x1024x130000 483 against 483, 16x2048x50257 370 against 372, but 16x1024x20000 101 against 91
    if (few && matrix >= (int64_t(1) << (f32 ? 27 : 23))) return kStream;
    const double work = double(matrix) * double(d.tokens);
    // Laying operands out pays where each of them is read many times: bf16 512x2048x8192 110 against 127, 450x700x30000 178 against 195, 600x1000x9000 94
    // against 111, 1189x320x60672 352 against 357, 1130x392x39552 281 against 317, 2000x100x30000 216 against 243, but 256x4096x32000 508 against 403,
    // 1024x256x32000 145 against 125, 500x600x17000 133 against 107, 1200x64x100000 410 against 235; fp32 4096x4096x16384 7980 against 8450,
    // 2000x800x10000 702 against 803, 4000x400x6000 597 against 697, but 1024x1024x8192 327 against 304, 3000x1000x1000 331 against 213,
    // 1100x128x100000 1470 against 968.
    const bool often = f32 ? d.width >= 256 && ((d.tokens >= 1000 && work >= 1.2e10) || (d.tokens >= 2048 && work >= 5e9))
                           : (d.tokens >= 400 && d.width >= 512 && work >= (d.width >= 900 ? 5e9 : 8e9)) ||
                                 (d.tokens >= 1000 && d.width >= (d.tokens >= 1200 ? 96 : 320) && work >= 5e9) || (d.tokens >= 2048 && work >= 1e9);
    if (often) {
        // Tiles of 256 need enough of them in dweight (fp32 1500x1500x6000, 144 tiles, 617 against 640; 2500x1000x3000, 48, 566 against 400; bf16
        // 4096x4096x2048, 128, 262 against 238) and room along the others (fp32 2000x800x10000 702 against 744, 4000x500x20000 2221 against 1893; bf16
        // 450x3000x12000 226 against 208).
        const int64_t tiles = int64_t(tiles_of(d.width, 256)) * tiles_of(std::min(d.vocab, 16384), 256);
        return tiles > 128 && d.tokens >= (f32 ? 1000 : 2048) && d.width >= (f32 ? 768 : 2048) ? kGemm256 : kGemm128;
    }
    // bf16 256x4096x32000 403 against 455, but 256x512x32000 80 against 71, 400x400x100000 360 against 331; fp32 40x1024x4096 40 against 45, 374x68x130472 359
    // against 504, but 9x1792x1071 30 against 25, 2000x64x50000 1252 against 603, 520x190x8000 88 against 81 (from 100 wide on both are near: 1068x110x102656 1043
    // against 1197, 1100x128x100000 943 against 993)
    if (f32 ? matrix >= (int64_t(1) << 21) && (d.width >= 192 || d.tokens < 512) : work >= 1.5e10 && d.width >= 512) return kDirect128;
    return kDirect64;
}

// Groups of waves between which the steps of a tile of 64 are divided.  Four: no more tiles than compute units, each with steps for all groups (bf16
// 37x3712x12160 28 against 40 us, 226x1728x1148 16 against 20, but 386x3456x2389, 266 tiles, 42 against 36; gradients of 3155x68x3073 54 against 108, of 923x704x1024 fp32 62 against 71).
// Two (logits only): up to twice as many tiles with enough steps (fp32 386x3456x2389 108 against 122 us, 200x4000x8000, 500 tiles, 133 against 149,
// 16x1024x20000 26 against 33, bf16 386x3456x2389 34 against 36; but fp32 128x1024x20000, 626 tiles, 56 against 53, bf16 500x1001x4000, 16 steps, 20.0 against 19.8).
inline int groups_of(int blocks, int steps, bool logits) {
    if (g_tuning.head_groups) return g_tuning.head_groups == 1 ? 4 : g_tuning.head_groups == 3 && logits ? 2 : 1;
    return blocks <= 256 && steps >= 16 ? 4 : logits && blocks <= 512 && steps >= 32 ? 2 : 1;
}

HeadPlan head_plan(const HeadDims& d, bool backward) {
    HeadPlan p = {};
    const size_t e = dtype_bytes(d.dtype), T = size_t(d.tokens);
    const bool f32 = d.dtype == BNS_F32;
    p.kind = logits_kind(d, backward);
    p.gradients = gradients_kind(d);
    // (the laid-out kernels leave g in parts only, which is not what the direct ones read)
    if (backward && !p.parts() && p.kind >= kGemm256) p.kind = kDirect128;
    p.planes = f32 ? 3 : 1;
    p.depth_d = round_up(d.width, kDepth);
    p.depth_t = p.gradients == kStream && d.tokens <= 32 ? 32 : round_up(std::max<int64_t>(d.tokens, 1), kDepth);
    const size_t P = size_t(p.planes) * 2;
    if (p.kind >= kGemm256) {
        p.copy_h = !lies_well(d, d.hidden_stride);
        p.copy_w = !lies_well(d, d.weight_stride);
    }
    // The larger the piece, the fewer passes over dhidden's sums; 16384 rows where operands are laid out, else what keeps g at 64 MB.
    int64_t piece = d.piece;
    if (!piece) piece = p.gradients >= kGemm256 || p.copy_w ? 16384 : std::max<int64_t>(1024, (int64_t(64) << 20) / int64_t(std::max<size_t>(T * e, 1)));
    p.piece = std::min(round_up(std::min<int64_t>(piece, 1 << 18), 256), round_up(d.vocab, 256));
    const int64_t rows = std::min<int64_t>(p.piece, d.vocab);
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 1023) & ~size_t(1023);
        return here;
    };
    p.hidden = take(p.copy_h ? T * p.depth_d * P : 0);
    p.weight = take(p.copy_w ? size_t(p.piece) * p.depth_d * P : 0);
    if (!backward) {
        const int m = rows_of(p.kind, d);
        p.partial = take(size_t((d.vocab + m - 1) / m) * T * sizeof(float2));
        p.at_target = take(T * 4);
    } else {
        p.splits = p.splits_w = 1;
        if (p.gradients == kStream) {
            // blocks for half of the device's waves, each with eight steps for its waves at least
            const int64_t groups = (d.width + kStreamColumns - 1) / kStreamColumns;
            p.splits = int(std::max<int64_t>(1, std::min<int64_t>(1024 / groups, rows / 256)));
            p.splits_w = int(std::max<int64_t>(1, std::min<int64_t>(1024 / groups, rows / 128)));
        } else if (p.gradients <= kDirect128) {
            const int m = p.gradients == kDirect128 ? 128 : 64;
            const int64_t across = (d.width + m - 1) / m, tiles = across * ((d.tokens + m - 1) / m), depth = f32 ? 32 : 64, steps = rows / depth;
            // Steps enough for a block to be worth its sums: four, or four for each of four groups of waves (2870x256x1294 bf16 51 us against 68 with one for
            // each, 923x704x1024 fp32 64 against 80).  Eight instead of four: 425x1088x3328 fp32 102 against 106, but 40x1024x4096 46 against 41.
            const bool groups = m == 64 && d.tokens > 32 && groups_of(int(across * ((rows + m - 1) / m)), int(d.tokens / depth), false) == 4;
            p.splits = int(std::max<int64_t>(1, std::min<int64_t>((groups ? 512 : 1024) / std::max<int64_t>(tiles, 1), steps / (groups ? 16 : 4))));
        } else {
            const int m = p.gradients == kGemm128 ? 128 : 256;
            const int64_t tiles = ((d.width + m - 1) / m) * ((d.tokens + m - 1) / m);
            p.splits = int(std::max<int64_t>(1, std::min<int64_t>((m == 128 ? 512 : 256) / std::max<int64_t>(tiles, 1), rows / 512)));
        }
        if (p.gradients >= kGemm256) {
            p.weight_t = take(size_t(d.width) * p.piece * P);
            p.hidden_t = take(size_t(d.width) * p.depth_t * P);
        }
        p.g = take(T * p.piece * (p.parts() ? P : e));
        if (p.parts()) p.gt = take(size_t(p.piece) * p.depth_t * P);
        p.sums = take(size_t(p.splits) * T * p.depth_d * 4);
    }
    p.bytes = std::max<size_t>(at, 1024);       // (never 0, which stands for an invalid description)
    return p;
}

// What either pass needs, `other` being the plan of the one that is not `p`'s.
inline size_t workspace_of(const HeadPlan& p, const HeadPlan& other) { return std::max(p.bytes, other.bytes); }

inline bool failed() { return hipGetLastError() != hipSuccess; }

// ---- launches -------------------------------------------------------------------------------------------------------
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
bool gemm(GemmArgs a, Kind kind, hipStream_t st) {
    const int m = kind == kGemm128 ? 128 : 256;
    a.tiles_a = tiles_of(a.rows_a, m);
    a.tiles_b = tiles_of(a.rows_b, m);
    const dim3 grid(uint32_t(a.tiles_a) * a.tiles_b * a.splits);
    if (m == 128) BNS_LAUNCH((gemm_kernel<T, 128, 128, 2, 2, EPILOGUE>), grid, dim3(256), 0, st, a);
    else BNS_LAUNCH((gemm_kernel<T, 256, 256, 2, 4, EPILOGUE>), grid, dim3(512), 0, st, a);
    return !failed();
}

// Tokens of a tile in the kernels that have several sizes.
inline int token_tile(int tokens) { return tokens <= 16 ? 16 : tokens <= 32 ? 32 : 64; }

// Whether logits that read the vocabulary's matrix once do so with the non-temporal hint: more than the memory-side cache holds, in rows of whole cache lines
// (bf16 16x4096x131072 159 against 180 us, 4x1024x200000 69 against 74, fp32 3x4096x100000 322 against 341; but 16x4008x131072 260 against 215, whose rows
// share lines, and 16x2048x50257 found in the cache 51 against 38).
inline bool stream_weight(const GemmArgs& a, size_t e) {
    return a.tiles_b == 1 && size_t(a.rows_a) * size_t(a.lda) * e > kStreamBytes && size_t(a.lda) * e % 128 == 0 && reinterpret_cast<uintptr_t>(a.a) % 128 == 0;
}

template <typename T, int EPILOGUE>
bool logits(const HeadDims& d, const HeadPlan& p, GemmArgs a, hipStream_t st) {
    // (gt is written up to its depth, a multiple of 64 or 32)
    const int m = rows_of(p.kind, d), n = p.kind == kDirect128 ? 128 : EPILOGUE == kGradientParts ? std::min(a.gt_depth, 64) : token_tile(a.rows_b);
    if (p.kind >= kGemm256) {
        if constexpr (EPILOGUE != kGradient) return gemm<T, EPILOGUE>(a, p.kind, st);
        return false;       // (not planned)
    }
    a.tiles_a = tiles_of(std::max(a.rows_a, a.g_depth), m);
    a.tiles_b = tiles_of(a.rows_b, n);
    const dim3 grid(uint32_t(a.tiles_a) * a.tiles_b);
    const int groups = groups_of(a.tiles_a * a.tiles_b, a.depth / DirectTile<T, 64, 64, 2, 2>::kDepth, true);
    const bool nt = EPILOGUE == kStatistics && stream_weight(a, sizeof(T));
    if constexpr (EPILOGUE != kGradientParts) {     // (n is 32 or more there)
        if (n == 16) {
            if (p.kind == kDirect64 && groups == 4) BNS_LAUNCH((direct_logits_kernel<T, 64, 16, 4, 1, 4, EPILOGUE>), grid, dim3(1024), 0, st, a);
            else if (p.kind == kDirect64 && groups == 2) BNS_LAUNCH((direct_logits_kernel<T, 64, 16, 4, 1, 2, EPILOGUE>), grid, dim3(512), 0, st, a);
            else if (p.kind == kDirect64 && nt) BNS_LAUNCH((direct_logits_kernel<T, 64, 16, 4, 1, 1, EPILOGUE, EPILOGUE == kStatistics>), grid, dim3(256), 0, st, a);
            else if (p.kind == kDirect64) BNS_LAUNCH((direct_logits_kernel<T, 64, 16, 4, 1, 1, EPILOGUE>), grid, dim3(256), 0, st, a);
            else if (m == 16) BNS_LAUNCH((stream_logits_kernel<T, 1, 1, EPILOGUE>), grid, dim3(256), 0, st, a);
            else BNS_LAUNCH((stream_logits_kernel<T, 2, 1, EPILOGUE>), grid, dim3(256), 0, st, a);
            return !failed();
        }
    }
    if (p.kind == kDirect128) BNS_LAUNCH((direct_logits_kernel<T, 128, 128, 2, 2, 1, EPILOGUE>), grid, dim3(256), 0, st, a);
    else if (p.kind == kDirect64 && n == 32 && groups == 4) BNS_LAUNCH((direct_logits_kernel<T, 64, 32, 4, 1, 4, EPILOGUE>), grid, dim3(1024), 0, st, a);
    else if (p.kind == kDirect64 && n == 32 && groups == 2) BNS_LAUNCH((direct_logits_kernel<T, 64, 32, 4, 1, 2, EPILOGUE>), grid, dim3(512), 0, st, a);
    else if (p.kind == kDirect64 && n == 32 && nt) BNS_LAUNCH((direct_logits_kernel<T, 64, 32, 4, 1, 1, EPILOGUE, EPILOGUE == kStatistics>), grid, dim3(256), 0, st, a);
    else if (p.kind == kDirect64 && n == 32) BNS_LAUNCH((direct_logits_kernel<T, 64, 32, 4, 1, 1, EPILOGUE>), grid, dim3(256), 0, st, a);
    else if (p.kind == kDirect64 && groups == 4) BNS_LAUNCH((direct_logits_kernel<T, 64, 64, 2, 2, 4, EPILOGUE>), grid, dim3(1024), 0, st, a);
    else if (p.kind == kDirect64 && groups == 2) BNS_LAUNCH((direct_logits_kernel<T, 64, 64, 2, 2, 2, EPILOGUE>), grid, dim3(512), 0, st, a);
    else if (p.kind == kDirect64) BNS_LAUNCH((direct_logits_kernel<T, 64, 64, 2, 2, 1, EPILOGUE>), grid, dim3(256), 0, st, a);
    else if (m == 16 && n == 32) BNS_LAUNCH((stream_logits_kernel<T, 1, 2, EPILOGUE>), grid, dim3(256), 0, st, a);
    else if (m == 16) BNS_LAUNCH((stream_logits_kernel<T, 1, 4, EPILOGUE>), grid, dim3(256), 0, st, a);
    else if (n == 32) BNS_LAUNCH((stream_logits_kernel<T, 2, 2, EPILOGUE>), grid, dim3(256), 0, st, a);
    else BNS_LAUNCH((stream_logits_kernel<T, 2, 4, EPILOGUE>), grid, dim3(256), 0, st, a);
    return !failed();
}

// The operands of the logits of rows [v0, v0 + rows) of the vocabulary; copies a piece that has to be.
template <typename T>
bool logits_operands(const HeadDims& d, const HeadPlan& p, const void* hidden, const void* weight, const int64_t* targets, char* ws, int64_t v0, int rows,
                     hipStream_t st, GemmArgs* a) {
    const void* piece = static_cast<const T*>(weight) + v0 * d.weight_stride;
    const int64_t packed = p.depth_d * p.planes;
    a->a = p.copy_w ? ws + p.weight : piece;
    a->lda = p.copy_w ? packed : d.weight_stride;
    a->b = p.copy_h ? ws + p.hidden : hidden;
    a->ldb = p.copy_h ? packed : d.hidden_stride;
    a->rows_a = rows;
    a->rows_b = int32_t(d.tokens);
    a->depth = p.kind >= kGemm256 ? int32_t(p.depth_d) : d.width;
    a->splits = 1;
    a->targets = targets;
    a->v0 = int32_t(v0);
    a->vocab = d.vocab;
    if (v0 == 0 && p.copy_h && !pack_rows<T>(hidden, d.hidden_stride, d.tokens, d.width, p.depth_d, ws + p.hidden, st)) return false;
    return !p.copy_w || pack_rows<T>(piece, d.weight_stride, rows, d.width, p.depth_d, ws + p.weight, st);
}

bool join_statistics(const HeadDims& d, const HeadPlan& p, const int64_t* targets, float* loss, float* lse, char* ws, hipStream_t st) {
    const auto* partial = reinterpret_cast<const float2*>(ws + p.partial);
    const auto* at_target = reinterpret_cast<const float*>(ws + p.at_target);
    const int tiles = tiles_of(d.vocab, rows_of(p.kind, d)), tokens = int(d.tokens);
    if (tokens <= 1024) BNS_LAUNCH((join_statistics_kernel<1>), dim3(tokens), dim3(256), 0, st, partial, at_target, targets, tiles, tokens, d.vocab, loss, lse);
    else BNS_LAUNCH((join_statistics_kernel<16>), dim3((tokens + 15) / 16), dim3(256), 0, st, partial, at_target, targets, tiles, tokens, d.vocab, loss, lse);
    return !failed();
}

template <typename T>
bool join_splits(const HeadDims& d, const HeadPlan& p, void* dhidden, char* ws, hipStream_t st) {
    const dim3 grid(uint32_t(std::min<int64_t>(d.tokens * ((d.width + 255) / 256), 1 << 20)));
    const float* sums = reinterpret_cast<const float*>(ws + p.sums);
    const int64_t stride = d.tokens * p.depth_d;
    T* const out = static_cast<T*>(dhidden);
    if (p.splits > 4) BNS_LAUNCH((join_splits_kernel<T, 8>), grid, dim3(256), 0, st, sums, stride, p.splits, int(d.tokens), d.width, p.depth_d, out);
    else BNS_LAUNCH((join_splits_kernel<T, 1>), grid, dim3(32), 0, st, sums, stride, p.splits, int(d.tokens), d.width, p.depth_d, out);
    return !failed();
}

template <typename T, int EPILOGUE>
bool direct_gradients(GemmArgs h, GemmArgs w, Kind kind, hipStream_t st) {
    const int m = kind == kDirect128 ? 128 : 64, n = kind == kDirect128 ? 128 : token_tile(h.rows_b);
    h.tiles_a = w.tiles_a = tiles_of(h.rows_a, m);
    h.tiles_b = tiles_of(h.rows_b, n);
    w.tiles_b = tiles_of(w.rows_b, m);
    const int blocks_h = h.tiles_a * h.tiles_b * h.splits;
    const int blocks_w = w.tiles_a * w.tiles_b, ahead = w.depth > h.depth / h.splits ? blocks_w : 0;
    const dim3 grid(uint32_t(blocks_h) + uint32_t(blocks_w));
    const bool groups = groups_of(blocks_w, w.depth / DirectTile<T, 64, 64, 2, 2>::kDepth, false) == 4;
    if (n == 16) BNS_LAUNCH((direct_gradients_kernel<T, 64, 16, 4, 1, 64, 1, EPILOGUE>), grid, dim3(256), 0, st, h, w, blocks_h, ahead);
    else if (n == 32) BNS_LAUNCH((direct_gradients_kernel<T, 64, 32, 4, 1, 64, 1, EPILOGUE>), grid, dim3(256), 0, st, h, w, blocks_h, ahead);
    else if (n == 64 && groups) BNS_LAUNCH((direct_gradients_kernel<T, 64, 64, 2, 2, 64, 4, EPILOGUE>), grid, dim3(1024), 0, st, h, w, blocks_h, ahead);
    else if (n == 64) BNS_LAUNCH((direct_gradients_kernel<T, 64, 64, 2, 2, 64, 1, EPILOGUE>), grid, dim3(256), 0, st, h, w, blocks_h, ahead);
    else BNS_LAUNCH((direct_gradients_kernel<T, 128, 128, 2, 2, 128, 1, EPILOGUE>), grid, dim3(256), 0, st, h, w, blocks_h, ahead);
    return !failed();
}

template <typename T>
bool stream_gradients(GemmArgs h, GemmArgs w, hipStream_t st) {
    const int groups = (h.rows_a + kStreamColumns - 1) / kStreamColumns, n = token_tile(h.rows_b);
    const dim3 grid(uint32_t(groups) * uint32_t(h.splits + w.splits));
    if (n == 16) BNS_LAUNCH((stream_gradients_kernel<T, 1, 1>), grid, dim3(256), 0, st, h, w, groups);
    else if (n == 32) BNS_LAUNCH((stream_gradients_kernel<T, 2, 1>), grid, dim3(256), 0, st, h, w, groups);
    else if constexpr (sizeof(T) == 2) BNS_LAUNCH((stream_gradients_kernel<T, 4, 2>), grid, dim3(256), 0, st, h, w, groups);
    else return false;      // (not planned)
    return !failed();
}

template <typename T>
bool forward(const HeadDims& d, const HeadPlan& p, const void* hidden, const void* weight, const int64_t* targets, float* loss, float* lse, char* ws, hipStream_t st) {
    // (without copies the whole vocabulary is one piece, as far as a launch goes)
    const int64_t most = std::max<int64_t>(1, (1 << 20) / ((d.tokens + 15) / 16)) * 256, step = p.copy_w ? p.piece : std::min<int64_t>(d.vocab, most);
    for (int64_t v0 = 0; v0 < d.vocab; v0 += step) {
        GemmArgs a = {};
        if (!logits_operands<T>(d, p, hidden, weight, targets, ws, v0, int(std::min<int64_t>(step, d.vocab - v0)), st, &a)) return false;
        a.partial = reinterpret_cast<float2*>(ws + p.partial);
        a.at_target = reinterpret_cast<float*>(ws + p.at_target);
        if (!logits<T, kStatistics>(d, p, a, st)) return false;
    }
    return join_statistics(d, p, targets, loss, lse, ws, st);
}

template <typename T>
bool backward(const HeadDims& d, const HeadPlan& p, const void* hidden, const void* weight, const int64_t* targets, const float* lse, const float* dloss,
              void* dhidden, void* dweight, char* ws, hipStream_t st) {
    const bool laid_out = p.gradients >= kGemm256;
    const bool whole = p.gradients <= kDirect128 && p.gradients != kStream && p.splits == 1 && p.piece >= d.vocab;     // dhidden needs no sums beside it
    if (laid_out && !pack_columns<T>(hidden, d.hidden_stride, d.tokens, d.width, p.depth_t, targets, d.vocab, ws + p.hidden_t, st)) return false;
    for (int64_t v0 = 0; v0 < d.vocab; v0 += p.piece) {
        const int rows = int(std::min<int64_t>(p.piece, d.vocab - v0));
        const int64_t depth_v = round_up(rows, kDepth);
        GemmArgs a = {};
        if (!logits_operands<T>(d, p, hidden, weight, targets, ws, v0, rows, st, &a)) return false;
        a.lse = lse;
        a.dloss = dloss;
        if (p.parts()) {
            a.g = reinterpret_cast<uint16_t*>(ws + p.g);
            a.gt = reinterpret_cast<uint16_t*>(ws + p.gt);
            a.g_depth = int32_t(depth_v);
            a.gt_depth = int32_t(p.depth_t);
            if (!logits<T, kGradientParts>(d, p, a, st)) return false;
        } else {
            a.out = ws + p.g;
            a.ldo = p.piece;
            if (!logits<T, kGradient>(d, p, a, st)) return false;
        }
        const void* piece = static_cast<const T*>(weight) + v0 * d.weight_stride;
        if (laid_out && !pack_columns<T>(piece, d.weight_stride, rows, d.width, depth_v, nullptr, 0, ws + p.weight_t, st)) return false;
        // dhidden[n][m] += sum over the piece of g[n] weight[m]
        GemmArgs h = {};
        h.a = laid_out ? ws + p.weight_t : piece;
        h.lda = laid_out ? depth_v * p.planes : d.weight_stride;
        h.b = ws + p.g;
        h.ldb = p.parts() ? depth_v * p.planes : p.piece;
        h.rows_a = d.width;
        h.rows_b = int32_t(d.tokens);
        h.depth = laid_out ? int32_t(depth_v) : rows;
        h.g_depth = int32_t(depth_v);
        h.splits = p.splits;
        h.out = whole ? dhidden : ws + p.sums;
        h.ldo = whole ? d.width : p.depth_d;
        h.split_stride = d.tokens * p.depth_d;
        h.fresh = v0 == 0;
        // dweight[n][m] = sum over the tokens of g[n] hidden[m]
        GemmArgs w = {};
        w.a = laid_out ? ws + p.hidden_t : hidden;
        w.lda = laid_out ? p.depth_t * p.planes : d.hidden_stride;
        w.b = ws + (p.parts() ? p.gt : p.g);
        w.ldb = p.parts() ? p.depth_t * p.planes : p.piece;
        w.rows_a = d.width;
        w.rows_b = rows;
        w.depth = laid_out ? int32_t(p.depth_t) : int32_t(d.tokens);
        w.gt_depth = int32_t(p.depth_t);
        w.splits = p.splits_w;
        w.targets = targets;
        w.vocab = d.vocab;
        w.out = static_cast<T*>(dweight) + v0 * d.width;
        w.ldo = d.width;
        const bool ok = laid_out               ? gemm<T, kAccumulate>(h, p.gradients, st) && gemm<T, kStore>(w, p.gradients, st)
                        : p.gradients == kStream ? stream_gradients<T>(h, w, st)
                        : whole                  ? direct_gradients<T, kStore>(h, w, p.gradients, st)
                                                 : direct_gradients<T, kAccumulate>(h, w, p.gradients, st);
        if (!ok) return false;
    }
    return whole || join_splits<T>(d, p, dhidden, ws, st);
}

}  // namespace

extern "C" {

size_t bns_head_workspace_bytes(const bns_head* head) {
    HeadDims d;
    if (check_head(head, &d) != BNS_OK) return 0;
    return workspace_of(head_plan(d, false), head_plan(d, true));
}

bns_status bns_head_forward(const bns_head* head, const void* hidden, const void* weight, const int64_t* targets, float* loss, float* lse,
                            void* workspace, size_t workspace_bytes, void* stream) {
    HeadDims d;
    const bns_status s = check_head(head, &d);
    if (s != BNS_OK) return s;
    if (d.tokens == 0) return BNS_OK;
    if (!hidden || !weight || !targets || !loss || !lse || !workspace) return BNS_EINVAL;
    if (!aligned16(hidden) || !aligned16(weight) || !aligned16(workspace)) return BNS_EINVAL;
    const HeadPlan p = head_plan(d, false);
    if (workspace_bytes < workspace_of(p, head_plan(d, true))) return BNS_EWORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    char* ws = static_cast<char*>(workspace);
    const auto call = d.dtype == BNS_F32 ? forward<float> : forward<bf16_t>;
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
    const HeadPlan p = head_plan(d, true);
    if (workspace_bytes < workspace_of(p, head_plan(d, false))) return BNS_EWORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    char* ws = static_cast<char*>(workspace);
    if (d.tokens == 0) {
        BNS_LAUNCH(fill_zero_kernel, dim3(4096), dim3(256), 0, st, static_cast<uint16_t*>(dweight), int64_t(d.vocab) * d.width * int64_t(e / 2));
        return failed() ? BNS_EDEVICE : BNS_OK;
    }
    const auto call = d.dtype == BNS_F32 ? backward<float> : backward<bf16_t>;
    const bool ok = call(d, p, hidden, weight, targets, lse, dloss, dhidden, dweight, ws, st);
    return ok ? BNS_OK : BNS_EDEVICE;
}

}  // extern "C"
