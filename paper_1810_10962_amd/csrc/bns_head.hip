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
#include "bns_lm_device.hpp"
#include "bns_lm_validate.hpp"

using namespace bns;

namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kDepth = 64;      // elements of k in a staged tile: 128 bytes a row

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

// ---- parts of an fp32 value ---------------------------------------------------------------------------------------
// x = hi + mid + lo exactly, each of them the bf16 nearest to what is left (cut off instead where that would overflow).  Infinities and NaN are
// hi alone.  A product of two values needs the six pairs of parts whose exponents reach into an fp32 result: what is dropped is
// at most 2^-24 of it.
__device__ __forceinline__ void split3(float x, uint32_t (&part)[3]) {
    part[0] = f32_to_bf16(x);
    if (fabsf(x) > 0x1.fep127f) part[0] = __float_as_uint(x) >> 16;
    float r = x - bf16_to_f32(part[0]);
    if (!(fabsf(r) < __builtin_inff())) r = 0.f;
    part[1] = f32_to_bf16(r);
    part[2] = f32_to_bf16(r - bf16_to_f32(part[1]));
}

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

template <typename T>
constexpr int planes_of() { return sizeof(T) == 4 ? 3 : 1; }

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
enum Epilogue { kStatistics, kGradient, kAccumulate, kStore };

struct GemmArgs {
    const void *a, *b;
    int64_t lda, ldb;           // elements from row to row
    int32_t rows_a, rows_b;     // rows that exist; those beyond in a tile are read as the last one and their results left out
    int32_t depth;              // elements of k in a plane, a multiple of kDepth
    int32_t splits;             // k is divided between so many blocks (kAccumulate)
    int32_t tiles_a, tiles_b;
    // logits: m = row of the piece, n = token
    const int64_t* targets;
    const float *lse, *dloss;
    float2* partial;            // [tile of the whole vocabulary][token]: maximum and sum of a tile's logits, in powers of two
    float* at_target;           // [token]
    uint16_t *g, *gt;           // [token][planes][g_depth], [row of the piece][planes][gt_depth]
    int32_t v0, vocab, g_depth, gt_depth;
    // gradients: m = column, n = token / row of the piece
    void* out;
    int64_t ldo, split_stride;  // of out, in elements
    int32_t fresh;              // kAccumulate: out holds nothing yet
};

// Which pairs of planes an fp32 product takes, smallest first.
__device__ __forceinline__ int plane_a(int segment) { return (0x010120 >> (4 * segment)) & 3; }      // 0 2 1 0 1 0
__device__ __forceinline__ int plane_b(int segment) { return (0x001102 >> (4 * segment)) & 3; }      // 2 0 1 1 0 0

template <int BM, int BN, int WM, int WN>
struct Tile {
    static constexpr int kThreads = WM * WN * kWave, kPerIssue = kThreads / 8;       // rows that all threads bring in at once
    static constexpr int kM = BM / WM, kN = BN / WN, MI = kM / 16, NI = kN / 16;
    static constexpr int kBytes = (BM + BN) * kDepth * 2;
    static_assert(BM % kPerIssue == 0 && BN % kPerIssue == 0, "whole issues");
};

// Block -> tile.  Blocks go round robin over the eight dies, each with an L2 of its own: a die gets a contiguous range of tiles, walked in groups of
// four rows of tiles, so that the tiles in flight share their operands.
__device__ __forceinline__ void place(int block, int total, int tiles_a, int tiles_b, int& ta, int& tb) {
    const int die = block % 8, q = total / 8, r = total % 8;
    const int i = die * q + min(die, r) + block / 8;
    const int group = i / (4 * tiles_b), in = i - group * 4 * tiles_b, high = min(4, tiles_a - 4 * group);
    tb = in / high;
    ta = 4 * group + in - tb * high;
}

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

    // acc[i][j][e] is C[m][n] of m = m_base + 16 i + e, n = n_base + 16 j
    const int m_base = m0 + wm * S::kM + quarter * 4, n_base = n0 + wn * S::kN + r16;
    if constexpr (EPILOGUE == kStatistics) {
        __syncthreads();
        float2* const stat = reinterpret_cast<float2*>(lds);        // [WM][BN]
#pragma unroll
        for (int j = 0; j < S::NI; ++j) {
            const int n = n_base + 16 * j;
            const int64_t target = n < a.rows_b ? a.targets[n] : -1;
            const int aim = target >= 0 && target < a.vocab ? int(target) - a.v0 - m_base : -1;
            float m = -__builtin_inff(), l = 0.f;
#pragma unroll
            for (int i = 0; i < S::MI; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (aim == 16 * i + e) a.at_target[n] = acc[i][j][e];
                    acc[i][j][e] = m_base + 16 * i + e < a.rows_a ? acc[i][j][e] * kLog2e : -__builtin_inff();
                    m = fmaxf(m, acc[i][j][e]);
                }
            m = fmaxf(m, __shfl_xor(m, 16));
            m = fmaxf(fmaxf(m, __shfl_xor(m, 32)), -3e38f);        // (a finite number where the wave has no row)
#pragma unroll
            for (int i = 0; i < S::MI; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) l += __builtin_amdgcn_exp2f(acc[i][j][e] - m);
            l += __shfl_xor(l, 16);
            l += __shfl_xor(l, 32);
            if (quarter == 0) stat[wm * BN + wn * S::kN + 16 * j + r16] = float2{m, l};
        }
        __syncthreads();
        for (int c = threadIdx.x; c < BN; c += S::kThreads) {
            if (n0 + c >= a.rows_b) continue;
            float m = stat[c].x, l = 0.f;
#pragma unroll
            for (int w = 1; w < WM; ++w) m = fmaxf(m, stat[w * BN + c].x);
#pragma unroll
            for (int w = 0; w < WM; ++w) l = fmaf(stat[w * BN + c].y, __builtin_amdgcn_exp2f(stat[w * BN + c].x - m), l);
            a.partial[int64_t(a.v0 / BM + ta) * a.rows_b + n0 + c] = float2{m, l};
        }
    }
    if constexpr (EPILOGUE == kGradient) {
#pragma unroll
        for (int j = 0; j < S::NI; ++j) {
            const int n = n_base + 16 * j;
            int64_t target = -1;
            float lse = 0.f, scale = 0.f;
            if (n < a.rows_b) {
                target = a.targets[n];
                lse = a.lse[n];
                scale = a.dloss[n];
            }
            const bool valid = target >= 0 && target < a.vocab;
            const int aim = valid ? int(target) - a.v0 - m_base : -1;
#pragma unroll
            for (int i = 0; i < S::MI; ++i) {
                const int m = m_base + 16 * i;
                uint32_t part[4][3];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float f = __builtin_amdgcn_exp2f((acc[i][j][e] - lse) * kLog2e);
                    if (aim == 16 * i + e) f -= 1.f;
                    f = valid && m + e < a.rows_a ? f * scale : 0.f;
                    if (P == 1) part[e][0] = f32_to_bf16(f);
                    else split3(f, part[e]);
                }
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    if (n < a.gt_depth && m < a.g_depth) {
                        if (n < a.rows_b)
                            *reinterpret_cast<u2*>(a.g + int64_t(n) * a.g_depth * P + int64_t(p) * a.g_depth + m) =
                                u2{part[0][p] | part[1][p] << 16, part[2][p] | part[3][p] << 16};
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (m + e < a.rows_a) a.gt[int64_t(m + e) * a.gt_depth * P + int64_t(p) * a.gt_depth + n] = uint16_t(part[e][p]);
                    }
                }
            }
        }
    }
    if constexpr (EPILOGUE == kAccumulate) {
        float* const out = static_cast<float*>(a.out) + split * a.split_stride;
#pragma unroll
        for (int j = 0; j < S::NI; ++j) {
            const int n = n_base + 16 * j;
            if (n >= a.rows_b) continue;
#pragma unroll
            for (int i = 0; i < S::MI; ++i) {
                if (m_base + 16 * i >= a.rows_a) continue;
                f32x4* const p = reinterpret_cast<f32x4*>(out + n * a.ldo + m_base + 16 * i);
                *p = a.fresh ? acc[i][j] : *p + acc[i][j];
            }
        }
    }
    if constexpr (EPILOGUE == kStore) {
        T* const out = static_cast<T*>(a.out);
#pragma unroll
        for (int j = 0; j < S::NI; ++j) {
            const int n = n_base + 16 * j;
            if (n >= a.rows_b) continue;
#pragma unroll
            for (int i = 0; i < S::MI; ++i) {
                const int m = m_base + 16 * i;
                T* const p = out + n * a.ldo + m;
                if (m + 4 <= a.rows_a) {
                    if constexpr (P == 1) {
                        typedef u2 u2e __attribute__((aligned(2)));
                        *reinterpret_cast<u2e*>(p) = u2{pack_bf16x2(acc[i][j][0], acc[i][j][1]), pack_bf16x2(acc[i][j][2], acc[i][j][3])};
                    } else {
                        typedef f32x4 f32x4e __attribute__((aligned(4)));
                        *reinterpret_cast<f32x4e*>(p) = acc[i][j];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (m + e < a.rows_a) {
                            if constexpr (P == 1) p[e].bits = uint16_t(f32_to_bf16(acc[i][j][e]));
                            else p[e] = acc[i][j][e];
                        }
                }
            }
        }
    }
#endif
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
    int planes;
    int64_t depth_d, depth_t, piece;        // padded width, tokens, rows of a piece
    bool direct_h, direct_w;                // read where they are, without a copy
    bool narrow;                            // few tokens: tiles of 64 of them
    int splits;                             // of dhidden
    // offsets into the workspace
    size_t hidden, weight, partial, at_target, weight_t, hidden_t, g, gt, sums, forward_bytes, backward_bytes;
};

HeadPlan head_plan(const HeadDims& d) {
    HeadPlan p;
    p.planes = d.dtype == BNS_F32 ? 3 : 1;
    p.depth_d = round_up(d.width, kDepth);
    p.depth_t = round_up(std::max<int64_t>(d.tokens, 1), kDepth);
    const bool fits = d.dtype == BNS_BF16 && d.width % kDepth == 0;
    p.direct_h = fits && d.hidden_stride % 8 == 0 && d.hidden_stride < (1 << 21);
    p.direct_w = fits && d.weight_stride % 8 == 0 && d.weight_stride < (1 << 21);
    p.narrow = d.tokens <= 64;
    int64_t piece = d.piece ? d.piece : 16384;
    p.piece = std::min(round_up(std::min<int64_t>(piece, 1 << 18), kTileM), round_up(d.vocab, kTileM));
    const int64_t tiles = ((d.width + kTileM - 1) / kTileM) * ((d.tokens + (p.narrow ? 63 : 255)) / (p.narrow ? 64 : 256));
    p.splits = int(std::max<int64_t>(1, std::min<int64_t>(256 / std::max<int64_t>(tiles, 1), p.piece / 512)));
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 1023) & ~size_t(1023);
        return here;
    };
    const size_t P = size_t(p.planes) * 2, T = size_t(d.tokens), rows = size_t(p.piece);
    p.hidden = take(p.direct_h ? 0 : T * p.depth_d * P);
    p.weight = take(p.direct_w ? 0 : rows * p.depth_d * P);
    const size_t both = at;
    p.partial = take(size_t((d.vocab + kTileM - 1) / kTileM) * T * sizeof(float2));
    p.at_target = take(T * 4);
    p.forward_bytes = at;
    at = both;
    p.weight_t = take(size_t(d.width) * rows * P);
    p.hidden_t = take(size_t(d.width) * p.depth_t * P);
    p.g = take(T * rows * P);
    p.gt = take(rows * p.depth_t * P);
    p.sums = take(size_t(p.splits) * T * p.depth_d * 4);
    p.backward_bytes = at;
    return p;
}

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
    BNS_LAUNCH(join_statistics_kernel, dim3(uint32_t((d.tokens + 15) / 16)), dim3(256), 0, st, reinterpret_cast<const float2*>(ws + p.partial),
               reinterpret_cast<const float*>(ws + p.at_target), targets, int((d.vocab + kTileM - 1) / kTileM), int(d.tokens), d.vocab, loss, lse);
    return !failed();
}

template <typename T>
bool backward(const HeadDims& d, const HeadPlan& p, const void* hidden, const void* weight, const int64_t* targets, const float* lse, const float* dloss,
              void* dhidden, void* dweight, char* ws, hipStream_t st) {
    const int planes = p.planes;
    if (d.tokens == 0) {
        BNS_LAUNCH(fill_zero_kernel, dim3(4096), dim3(256), 0, st, static_cast<uint16_t*>(dweight), int64_t(d.vocab) * d.width * int64_t(sizeof(T) / 2));
        return !failed();
    }
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
        if (!gemm<T, kGradient>(a, p.narrow, st)) return false;
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
    const int64_t blocks = (d.tokens * ((d.width + 7) / 8) + 255) / 256;
    BNS_LAUNCH((join_splits_kernel<T>), dim3(uint32_t(std::min<int64_t>(blocks, 1 << 16))), dim3(256), 0, st, reinterpret_cast<const float*>(ws + p.sums),
               d.tokens * p.depth_d, p.splits, int(d.tokens), d.width, int(p.depth_d), static_cast<T*>(dhidden));
    return !failed();
}

}  // namespace

extern "C" {

size_t bns_head_workspace_bytes(const bns_head* head) {
    HeadDims d;
    if (check_head(head, &d) != BNS_OK) return 0;
    const HeadPlan p = head_plan(d);
    return std::max(p.forward_bytes, p.backward_bytes);
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
    if (workspace_bytes < std::max(p.forward_bytes, p.backward_bytes)) return BNS_EWORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    char* ws = static_cast<char*>(workspace);
    const bool ok = d.dtype == BNS_F32 ? forward<float>(d, p, hidden, weight, targets, loss, lse, ws, st)
                                       : forward<bf16_t>(d, p, hidden, weight, targets, loss, lse, ws, st);
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
    if (workspace_bytes < std::max(p.forward_bytes, p.backward_bytes)) return BNS_EWORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    char* ws = static_cast<char*>(workspace);
    const bool ok = d.dtype == BNS_F32 ? backward<float>(d, p, hidden, weight, targets, lse, dloss, dhidden, dweight, ws, st)
                                       : backward<bf16_t>(d, p, hidden, weight, targets, lse, dloss, dhidden, dweight, ws, st);
    return ok ? BNS_OK : BNS_EDEVICE;
}

}  // extern "C"
