// What the matrix products of the loss over the vocabulary share: parts of fp32 values, arguments, and what becomes of a tile of sums.
#pragma once
#include "bns_lm_device.hpp"

namespace bns {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kLowest = -3.40282347e38f;      // a maximum of only -infinity is this

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

template <typename T>
constexpr int planes_of() { return sizeof(T) == 4 ? 3 : 1; }

// ---- parts of an fp32 value ---------------------------------------------------------------------------------------
// x = hi + mid + lo exactly, each of them the bf16 nearest to what is left.  A product of two values needs the six pairs of parts whose exponents reach
// into an fp32 result: what is dropped is at most 2^-24 of it.
// Two values at a time: word p holds part p of x0 in its lower half, of x1 in its upper one.
// BEYOND: values that the nearest bf16 would make infinite are among them.  The finite ones take the largest finite bf16 as their first part, the others
// carry the rest.  An infinite one is its last part alone: that part meets nothing but first parts, which are zero only where the value is, so that no
// product is infinity times a zero part and infinity times x is what it is in fp32.  (Infinity times infinity is NaN.)
constexpr float kBeyondBf16 = 0x1.ffp127f, kLargestBf16 = 0x1.fep127f;
template <bool BEYOND>
__device__ __forceinline__ void split3(float x0, float x1, uint32_t (&word)[3]) {
    const bool i0 = BEYOND && fabsf(x0) == __builtin_inff(), i1 = BEYOND && fabsf(x1) == __builtin_inff();
    const auto first = [](float x, bool infinite) { return infinite ? 0.f : BEYOND && fabsf(x) >= kBeyondBf16 ? copysignf(kLargestBf16, x) : x; };
    word[0] = pack_bf16x2(first(x0, i0), first(x1, i1));
    float r0 = x0 - __uint_as_float(word[0] << 16), r1 = x1 - __uint_as_float(word[0] & 0xffff0000u);
    word[1] = pack_bf16x2(i0 ? 0.f : r0, i1 ? 0.f : r1);
    r0 -= __uint_as_float(word[1] << 16);
    r1 -= __uint_as_float(word[1] & 0xffff0000u);
    word[2] = pack_bf16x2(r0, r1);
}
// N pairs; one look at all of them says whether some lane has a value beyond the range of bf16 (NaN needs no care).
template <int N>
__device__ __forceinline__ void split3(const float (&x0)[N], const float (&x1)[N], uint32_t (&word)[N][3]) {
    float most = 0.f;       // (one instruction a pair, where fmaxf would quiet every operand first)
#pragma unroll
    for (int j = 0; j < N; ++j) asm("v_max3_f32 %0, %0, |%1|, |%2|" : "+v"(most) : "v"(x0[j]), "v"(x1[j]));
    if (__builtin_expect(__any(most >= kBeyondBf16), 0)) {
#pragma unroll
        for (int j = 0; j < N; ++j) split3<true>(x0[j], x1[j], word[j]);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) split3<false>(x0[j], x1[j], word[j]);
    }
}
// Eight neighbours: word j of part p.
__device__ __forceinline__ void split3(const float (&f)[8], u4 (&w)[3]) {
    const float x0[4] = {f[0], f[2], f[4], f[6]}, x1[4] = {f[1], f[3], f[5], f[7]};
    uint32_t word[4][3];
    split3(x0, x1, word);
#pragma unroll
    for (int p = 0; p < 3; ++p) w[p] = u4{word[0][p], word[1][p], word[2][p], word[3][p]};
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
    float2* partial;            // [tile of the whole vocabulary][token]: maximum m of a tile's logits and sum of exp(z - m)
    float* at_target;           // [token]
    uint16_t *g, *gt;           // kGradientParts: [token][planes][g_depth], [row of the piece][planes][gt_depth]
    int32_t v0, vocab, g_depth, gt_depth;
    // gradients: m = column, n = token / row of the piece; kGradient: g as [token][ldo]
    void* out;
    int64_t ldo, split_stride;  // of out, in elements
    int32_t fresh;              // kAccumulate: out holds nothing yet
};

// Block -> split and tile.  Blocks go round robin over the eight dies, each with an L2 of its own: a die gets a contiguous range of tiles, split after split,
// walked in groups of four rows of tiles, so that the tiles in flight share their operands.
__device__ __forceinline__ void place(int block, int splits, int tiles_a, int tiles_b, int& split, int& ta, int& tb) {
    const int tiles = tiles_a * tiles_b, total = tiles * splits, die = block % 8, q = total / 8, r = total % 8;
    const int at = die * q + min(die, r) + block / 8;
    split = at / tiles;
    const int i = at - split * tiles;
    const int group = i / (4 * tiles_b), in = i - group * 4 * tiles_b, high = min(4, tiles_a - 4 * group);
    tb = in / high;
    ta = 4 * group + in - tb * high;
}

// What becomes of a tile: statistics of its logits; the gradient of its logits, as it is or laid out for the products that read it; a part of a sum that
// other tiles of k add to; a result.
enum Epilogue { kStatistics, kGradient, kGradientParts, kAccumulate, kStore };

// Which rows of a wave's part of a tile meet in a fragment of sixteen is free, as long as operands and results agree.  They are dealt out so that what a
// lane holds along m comes in runs of eight that continue from one quarter of the wave to the next (16 bytes of bf16 a lane, 64 a row of results), and
// what it holds along n is contiguous: acc[i][j][e] is C[m][n] of
//   m = m0 + 32 (i / 2) + 8 (lane / 16) + 4 (i % 2) + e  (MI even; else m0 + 16 i + 4 (lane / 16) + e)          n = n0 + NI (lane % 16) + j.
// row_m, row_n: the row that is number r (16 i + lane % 16, 16 j + lane % 16) among the fragments' rows; slot_m, slot_n: the other way round.
template <int MI>
__device__ __forceinline__ int row_m(int r) { return MI % 2 ? r : r / 32 * 32 + r % 16 / 4 * 8 + r % 32 / 16 * 4 + r % 4; }
template <int MI>
__device__ __forceinline__ int slot_m(int m) { return MI % 2 ? m : m / 32 * 32 + m % 8 / 4 * 16 + m % 32 / 8 * 4 + m % 4; }
template <int NI>
__device__ __forceinline__ int row_n(int r) { return r / (16 * NI) * (16 * NI) + r % 16 * NI + r % (16 * NI) / 16; }
template <int NI>
__device__ __forceinline__ int slot_n(int n) { return n / (16 * NI) * (16 * NI) + n % NI * 16 + n % (16 * NI) / NI; }

// COUNT neighbouring elements of a row that may begin anywhere; `left` of them exist.
template <typename T, int COUNT>
__device__ __forceinline__ void store_run(T* p, int left, const float (&f)[COUNT]) {
    if (left >= COUNT) {
        if constexpr (sizeof(T) == 2 && COUNT % 8 == 0) {
            typedef u4 u4e __attribute__((aligned(2)));
#pragma unroll
            for (int k = 0; k < COUNT; k += 8)
                *reinterpret_cast<u4e*>(p + k) = u4{pack_bf16x2(f[k], f[k + 1]), pack_bf16x2(f[k + 2], f[k + 3]), pack_bf16x2(f[k + 4], f[k + 5]), pack_bf16x2(f[k + 6], f[k + 7])};
        } else if constexpr (sizeof(T) == 2) {
            typedef u2 u2e __attribute__((aligned(2)));
#pragma unroll
            for (int k = 0; k < COUNT; k += 4) *reinterpret_cast<u2e*>(p + k) = u2{pack_bf16x2(f[k], f[k + 1]), pack_bf16x2(f[k + 2], f[k + 3])};
        } else {
            typedef f32x4 f32x4e __attribute__((aligned(4)));
#pragma unroll
            for (int k = 0; k < COUNT; k += 4) *reinterpret_cast<f32x4e*>(p + k) = f32x4{f[k], f[k + 1], f[k + 2], f[k + 3]};
        }
    } else {
#pragma unroll
        for (int k = 0; k < COUNT; ++k)
            if (k < left) {
                if constexpr (sizeof(T) == 2) p[k].bits = uint16_t(f32_to_bf16(f[k]));
                else p[k] = f[k];
            }
    }
}

// COUNT neighbouring parts at an address that is a multiple of their size.
template <int COUNT>
__device__ __forceinline__ void store_parts(uint16_t* p, const uint32_t (&v)[COUNT]) {
    if constexpr (COUNT % 8 == 0) {
#pragma unroll
        for (int k = 0; k < COUNT; k += 8)
            *reinterpret_cast<u4*>(p + k) = u4{v[k] | v[k + 1] << 16, v[k + 2] | v[k + 3] << 16, v[k + 4] | v[k + 5] << 16, v[k + 6] | v[k + 7] << 16};
    } else if constexpr (COUNT % 4 == 0) {
#pragma unroll
        for (int k = 0; k < COUNT; k += 4) *reinterpret_cast<u2*>(p + k) = u2{v[k] | v[k + 1] << 16, v[k + 2] | v[k + 3] << 16};
    } else if constexpr (COUNT == 2) {
        *reinterpret_cast<uint32_t*>(p) = v[0] | v[1] << 16;
    } else {
        static_assert(COUNT == 1, "one, two, or a multiple of four");
        *p = uint16_t(v[0]);
    }
}

// ta, tb: numbers of the tile along m and n; `stat`: LDS for WM * BN pairs, free for use once every wave has come here (WM = 1: none).
template <typename T, int EPILOGUE, int BM, int BN, int WM, int WN>
__device__ __forceinline__ void finish(const GemmArgs& a, f32x4 (&acc)[BM / WM / 16][BN / WN / 16], int ta, int tb, int split, float2* stat) {
    constexpr int P = planes_of<T>(), kM = BM / WM, kN = BN / WN, MI = kM / 16, NI = kN / 16;
    constexpr int kRun = MI % 2 ? 4 : 8, kRuns = 4 * MI / kRun, kStride = 4 * kRun;     // a lane has kRuns runs of kRun, kStride apart
    const int wave = WM * WN == 1 ? 0 : int(threadIdx.x) / kWave, lane = threadIdx.x % kWave, wm = wave / WN, wn = wave % WN, r16 = lane % 16;
    const int m_base = ta * BM + wm * kM + lane / 16 * kRun, n_base = tb * BN + wn * kN + r16 * NI, left = a.rows_a - m_base;
    // element x of run r
    const auto at = [&](int r, int j, int x) { return acc[r * (kRun / 4) + x / 4][j][x % 4]; };
    const auto put = [&](int r, int j, int x, float f) { acc[r * (kRun / 4) + x / 4][j][x % 4] = f; };
    if constexpr (EPILOGUE == kStatistics) {
        if constexpr (WM > 1) __syncthreads();
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const int n = n_base + j;
            const int64_t target = n < a.rows_b ? a.targets[n] : -1;
            const int aim = target >= 0 && target < a.vocab ? int(target) - a.v0 - m_base : -1;
            float m = -__builtin_inff(), l = 0.f;
#pragma unroll
            for (int r = 0; r < kRuns; ++r)
#pragma unroll
                for (int x = 0; x < kRun; ++x) {
                    const float z = at(r, j, x), f = r * kStride + x < left ? z : -__builtin_inff();
                    if (aim == r * kStride + x) a.at_target[n] = z;
                    put(r, j, x, f);
                    m = fmaxf(m, f);
                }
            m = fmaxf(m, __shfl_xor(m, 16));
            m = fmaxf(fmaxf(m, __shfl_xor(m, 32)), kLowest);        // (a finite number where the wave has no row)
            // (The difference is taken before it is scaled: it is exact where it counts, and does not overflow.)
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) l += __builtin_amdgcn_exp2f((acc[i][j][e] - m) * kLog2e);
            l += __shfl_xor(l, 16);
            l += __shfl_xor(l, 32);
            if (lane < 16) {
                if constexpr (WM > 1) stat[wm * BN + wn * kN + r16 * NI + j] = float2{m, l};
                else if (n < a.rows_b) a.partial[int64_t(a.v0 / BM + ta) * a.rows_b + n] = float2{m, l};
            }
        }
        if constexpr (WM > 1) {
            __syncthreads();
            for (int c = threadIdx.x; c < BN; c += WM * WN * kWave) {
                if (tb * BN + c >= a.rows_b) continue;
                float m = stat[c].x, l = 0.f;
#pragma unroll
                for (int w = 1; w < WM; ++w) m = fmaxf(m, stat[w * BN + c].x);
#pragma unroll
                for (int w = 0; w < WM; ++w) l = fmaf(stat[w * BN + c].y, __builtin_amdgcn_exp2f((stat[w * BN + c].x - m) * kLog2e), l);
                a.partial[int64_t(a.v0 / BM + ta) * a.rows_b + tb * BN + c] = float2{m, l};
            }
        }
    }
    // With bf16 operands g becomes bf16 here, as the operand that the matrix units take.  It is the one rounding between the logits and the gradients' own: at
    // 4096x4096x131072 the gradients are 1.8e-3 of their norm away from 64 bits with it, 1.7e-3 with g in fp32 (the rest is the rounding of the result to
    // bf16; single elements whose terms cancel lose more).  A second part of g would take five products where there are three, and half as long again.
    if constexpr (EPILOGUE == kGradient || EPILOGUE == kGradientParts) {
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const int n = n_base + j;
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
            for (int r = 0; r < kRuns; ++r) {
#pragma unroll
                for (int x = 0; x < kRun; ++x) {
                    float f = __builtin_amdgcn_exp2f((at(r, j, x) - lse) * kLog2e);
                    if (aim == r * kStride + x) f -= 1.f;
                    put(r, j, x, valid && r * kStride + x < left ? f * scale : 0.f);
                }
                if constexpr (EPILOGUE == kGradient) {
                    float f[kRun];
#pragma unroll
                    for (int x = 0; x < kRun; ++x) f[x] = at(r, j, x);
                    if (n < a.rows_b) store_run<T, kRun>(static_cast<T*>(a.out) + n * a.ldo + m_base + r * kStride, left - r * kStride, f);
                }
            }
        }
        if constexpr (EPILOGUE == kGradientParts) {
            // g with zeros behind the rows of the piece, gt with zeros behind the tokens: their k is a whole number of steps
#pragma unroll
            for (int r = 0; r < kRuns; ++r) {
                const int m = m_base + r * kStride;
                uint32_t part[kRun][NI][P];
#pragma unroll
                for (int j = 0; j < NI; ++j) {
                    float even[kRun / 2], odd[kRun / 2];
                    uint32_t word[kRun / 2][3];
#pragma unroll
                    for (int x = 0; x < kRun / 2; ++x) even[x] = at(r, j, 2 * x), odd[x] = at(r, j, 2 * x + 1);
                    if constexpr (P == 1) {
#pragma unroll
                        for (int x = 0; x < kRun / 2; ++x) word[x][0] = pack_bf16x2(even[x], odd[x]);
                    } else {
                        split3(even, odd, word);
                    }
#pragma unroll
                    for (int x = 0; x < kRun / 2; ++x)
#pragma unroll
                        for (int p = 0; p < P; ++p) part[2 * x][j][p] = word[x][p] & 0xffffu, part[2 * x + 1][j][p] = word[x][p] >> 16;
                }
#pragma unroll
                for (int p = 0; p < P; ++p) {
#pragma unroll
                    for (int j = 0; j < NI; ++j) {
                        uint32_t v[kRun];
#pragma unroll
                        for (int x = 0; x < kRun; ++x) v[x] = part[x][j][p];
                        if (n_base + j < a.rows_b && m < a.g_depth) store_parts<kRun>(a.g + int64_t(n_base + j) * a.g_depth * P + int64_t(p) * a.g_depth + m, v);
                    }
#pragma unroll
                    for (int x = 0; x < kRun; ++x) {
                        uint32_t v[NI];
#pragma unroll
                        for (int j = 0; j < NI; ++j) v[j] = part[x][j][p];
                        if (r * kStride + x < left && n_base < a.gt_depth) store_parts<NI>(a.gt + int64_t(m + x) * a.gt_depth * P + int64_t(p) * a.gt_depth + n_base, v);
                    }
                }
            }
        }
    }
    if constexpr (EPILOGUE == kAccumulate) {
        float* const out = static_cast<float*>(a.out) + split * a.split_stride;
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            if (n_base + j >= a.rows_b) continue;
#pragma unroll
            for (int r = 0; r < kRuns; ++r)
#pragma unroll
                for (int x = 0; x < kRun; x += 4) {
                    if (r * kStride + x >= left) continue;
                    const f32x4 sum = {at(r, j, x), at(r, j, x + 1), at(r, j, x + 2), at(r, j, x + 3)};
                    f32x4* const p = reinterpret_cast<f32x4*>(out + (n_base + j) * a.ldo + m_base + r * kStride + x);
                    *p = a.fresh ? sum : *p + sum;
                }
        }
    }
    if constexpr (EPILOGUE == kStore) {
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            if (n_base + j >= a.rows_b) continue;
#pragma unroll
            for (int r = 0; r < kRuns; ++r) {
                float f[kRun];
#pragma unroll
                for (int x = 0; x < kRun; ++x) f[x] = at(r, j, x);
                store_run<T, kRun>(static_cast<T*>(a.out) + (n_base + j) * a.ldo + m_base + r * kStride, left - r * kStride, f);
            }
        }
    }
}

}  // namespace bns
