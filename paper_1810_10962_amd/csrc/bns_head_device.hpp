// What the matrix products of the loss over the vocabulary share: parts of fp32 values, arguments, and what becomes of a tile of sums.
#pragma once
#include "bns_lm_device.hpp"

namespace bns {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

template <typename T>
constexpr int planes_of() { return sizeof(T) == 4 ? 3 : 1; }

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

// Which pairs of planes an fp32 product takes, smallest first.
__device__ __forceinline__ int plane_a(int segment) { return (0x010120 >> (4 * segment)) & 3; }      // 0 2 1 0 1 0
__device__ __forceinline__ int plane_b(int segment) { return (0x001102 >> (4 * segment)) & 3; }      // 2 0 1 1 0 0

// A product C[m][n] = sum over k of A[m][k] B[n][k].
struct GemmArgs {
    const void *a, *b;
    int64_t lda, ldb;           // elements from row to row
    int32_t rows_a, rows_b;     // m and n that exist
    int32_t depth;              // elements of k
    int32_t splits;             // k is divided between so many blocks (kAccumulate)
    int32_t tiles_a, tiles_b;
    // logits: m = row of the piece, n = token
    const int64_t* targets;     // (gradients: tokens whose rows of A count as zeros are those left out by them; NULL: none)
    const float *lse, *dloss;
    float2* partial;            // [tile of the whole vocabulary][token]: maximum and sum of a tile's logits, in powers of two
    float* at_target;           // [token]
    uint16_t *g, *gt;           // kGradientParts: [token][planes][g_depth], [row of the piece][planes][gt_depth]
    int32_t v0, vocab, g_depth, gt_depth;
    // gradients: m = column, n = token / row of the piece; kGradient: g as [token][ldo]
    void* out;
    int64_t ldo, split_stride;  // of out, in elements
    int32_t fresh;              // kAccumulate: out holds nothing yet
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

// What becomes of a tile: statistics of its logits; the gradient of its logits, as it is or laid out for the products that read it; a part of a sum that
// other tiles of k add to; a result.
enum Epilogue { kStatistics, kGradient, kGradientParts, kAccumulate, kStore };

// acc[i][j][e] is C[m][n] of m = m0 + 16 i + 4 (lane / 16) + e, n = n0 + 16 j + lane % 16, where m0, n0 are the wave's; ta: number of the tile
// along m; `stat`: LDS for WM * BN pairs, free for use.
template <typename T, int EPILOGUE, int BM, int BN, int WM, int WN>
__device__ __forceinline__ void finish(const GemmArgs& a, f32x4 (&acc)[BM / WM / 16][BN / WN / 16], int ta, int tb, int split, float2* stat) {
    constexpr int P = planes_of<T>(), kM = BM / WM, kN = BN / WN, MI = kM / 16, NI = kN / 16;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, wm = wave / WN, wn = wave % WN, r16 = lane % 16, quarter = lane / 16;
    const int n0 = tb * BN, m_base = ta * BM + wm * kM + quarter * 4, n_base = n0 + wn * kN + r16;
    if constexpr (EPILOGUE == kStatistics) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const int n = n_base + 16 * j;
            const int64_t target = n < a.rows_b ? a.targets[n] : -1;
            const int aim = target >= 0 && target < a.vocab ? int(target) - a.v0 - m_base : -1;
            float m = -__builtin_inff(), l = 0.f;
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (aim == 16 * i + e) a.at_target[n] = acc[i][j][e];
                    acc[i][j][e] = m_base + 16 * i + e < a.rows_a ? acc[i][j][e] * kLog2e : -__builtin_inff();
                    m = fmaxf(m, acc[i][j][e]);
                }
            m = fmaxf(m, __shfl_xor(m, 16));
            m = fmaxf(fmaxf(m, __shfl_xor(m, 32)), -3e38f);        // (a finite number where the wave has no row)
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) l += __builtin_amdgcn_exp2f(acc[i][j][e] - m);
            l += __shfl_xor(l, 16);
            l += __shfl_xor(l, 32);
            if (quarter == 0) stat[wm * BN + wn * kN + 16 * j + r16] = float2{m, l};
        }
        __syncthreads();
        for (int c = threadIdx.x; c < BN; c += (WM * WN * kWave)) {
            if (n0 + c >= a.rows_b) continue;
            float m = stat[c].x, l = 0.f;
#pragma unroll
            for (int w = 1; w < WM; ++w) m = fmaxf(m, stat[w * BN + c].x);
#pragma unroll
            for (int w = 0; w < WM; ++w) l = fmaf(stat[w * BN + c].y, __builtin_amdgcn_exp2f(stat[w * BN + c].x - m), l);
            a.partial[int64_t(a.v0 / BM + ta) * a.rows_b + n0 + c] = float2{m, l};
        }
    }
    if constexpr (EPILOGUE == kGradient || EPILOGUE == kGradientParts) {
#pragma unroll
        for (int j = 0; j < NI; ++j) {
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
            for (int i = 0; i < MI; ++i) {
                const int m = m_base + 16 * i;
                float f[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    f[e] = __builtin_amdgcn_exp2f((acc[i][j][e] - lse) * kLog2e);
                    if (aim == 16 * i + e) f[e] -= 1.f;
                    f[e] = valid && m + e < a.rows_a ? f[e] * scale : 0.f;
                }
                if constexpr (EPILOGUE == kGradient) {
                    if (n < a.rows_b && m < a.rows_a) {
                        T* const p = static_cast<T*>(a.out) + n * a.ldo + m;        // (ldo is a multiple of four)
                        if constexpr (P == 1) *reinterpret_cast<u2*>(p) = u2{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3])};
                        else *reinterpret_cast<f32x4*>(p) = f32x4{f[0], f[1], f[2], f[3]};
                    }
                    continue;
                }
                uint32_t part[4][3];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (P == 1) part[e][0] = f32_to_bf16(f[e]);
                    else split3(f[e], part[e]);
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
        for (int j = 0; j < NI; ++j) {
            const int n = n_base + 16 * j;
            if (n >= a.rows_b) continue;
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                if (m_base + 16 * i >= a.rows_a) continue;
                f32x4* const p = reinterpret_cast<f32x4*>(out + n * a.ldo + m_base + 16 * i);
                *p = a.fresh ? acc[i][j] : *p + acc[i][j];
            }
        }
    }
    if constexpr (EPILOGUE == kStore) {
        T* const out = static_cast<T*>(a.out);
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const int n = n_base + 16 * j;
            if (n >= a.rows_b) continue;
#pragma unroll
            for (int i = 0; i < MI; ++i) {
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
}

}  // namespace bns
