// The products of the loss over the vocabulary for few tokens, which read the vocabulary's matrix (or write its gradient) at the rate of memory and do little
// else: every wave streams rows of the matrix from memory straight into the fragments of the matrix units, with the loads of the next steps on
// their way, and no exchange through LDS but one sum at the end.  Operands are read as they lie in memory, as in bns_head_direct.hpp.
// Measured: gradients of 16x2048x50257 in bf16 with the logits before them 158 us (618 MB: the matrix read twice, its gradient written: 3.9 TB/s), in fp32 370;
// logits of 16x4096x4000 bf16 16 us, 9x1792x1071 fp32 15 us, where the length of a chain of loads along the width counts.
#pragma once
#include "bns_head_device.hpp"

namespace bns {

constexpr int kStreamColumns = 128;     // columns of a block in the gradients: sixteen lanes, eight neighbours each

template <typename T>
__device__ __forceinline__ void fetch_left(Raw8<T>& r, const T* p, int left) {
    if (left >= 8) r.load(p);
    else r.load_left(p, left);
}

__device__ __forceinline__ f32x4 multiply(u4 x, u4 y, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
}
template <int P>
__device__ __forceinline__ f32x4 multiply(const u4 (&x)[P], const u4 (&y)[P], f32x4 c) {
#pragma unroll
    for (int s = P == 1 ? 5 : 0; s < 6; ++s) c = multiply(x[plane_a(s)], y[plane_b(s)], c);
    return c;
}

// Eight neighbours along k as operands of the matrix units.
__device__ __forceinline__ void to_parts(const Raw8<bf16_t>& r, u4 (&w)[1]) { w[0] = r.a; }
__device__ __forceinline__ void to_parts(const Raw8<float>& r, u4 (&w)[3]) {
    float f[8];
    r.unpack(f);
    split3(f, w);
}
// Column f of eight rows, the rows being neighbours along k.
__device__ __forceinline__ void column_parts(const Raw8<bf16_t> (&r)[8], int f, u4 (&w)[1]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t even = r[2 * j].a[f / 2], odd = r[2 * j + 1].a[f / 2];
        w[0][j] = f % 2 ? even >> 16 | (odd & 0xffff0000u) : (even & 0xffffu) | odd << 16;
    }
}
__device__ __forceinline__ void column_parts(const Raw8<float> (&r)[8], int f, u4 (&w)[3]) {
    float column[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) column[j] = __uint_as_float(f < 4 ? r[j].a[f % 4] : r[j].b[f % 4]);
    split3(column, w);
}

// Logits of 16 MI rows of the vocabulary and 16 NI tokens.  The four waves of a block take every fourth step of k each.
template <typename T, int MI, int NI, int EPILOGUE>
__global__ void __launch_bounds__(256) stream_logits_kernel(GemmArgs a) {
    constexpr int P = planes_of<T>(), kRaws = P == 1 ? 2 : 1, kStep = 32 * kRaws, kAhead = MI + NI <= 3 ? 4 : MI + NI <= 4 ? 3 : 2;
    __shared__ f32x4 sums[3][MI * NI][kWave];
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / kWave), lane = threadIdx.x % kWave, r16 = lane % 16;
    const int ta = int(blockIdx.x) / a.tiles_b, tb = int(blockIdx.x) - ta * a.tiles_b, m0 = ta * 16 * MI, n0 = tb * 16 * NI, k_lane = lane / 16 * 8 * kRaws, steps = (a.depth + kStep - 1) / kStep;
    const T *x[MI], *y[NI];
#pragma unroll
    for (int i = 0; i < MI; ++i) x[i] = static_cast<const T*>(a.a) + min(m0 + row_m<MI>(16 * i + r16), a.rows_a - 1) * a.lda + k_lane;
#pragma unroll
    for (int j = 0; j < NI; ++j) y[j] = static_cast<const T*>(a.b) + min(n0 + row_n<NI>(16 * j + r16), a.rows_b - 1) * a.ldb + k_lane;
    Raw8<T> rx[kAhead][MI][kRaws], ry[kAhead][NI][kRaws];
    const auto ask = [&](Raw8<T> (&qx)[MI][kRaws], Raw8<T> (&qy)[NI][kRaws], int step) {
        const int k = step * kStep;
        if (k + kStep <= a.depth) {
#pragma unroll
            for (int h = 0; h < kRaws; ++h) {
#pragma unroll
                for (int i = 0; i < MI; ++i) qx[i][h].load(x[i] + k + 8 * h);
#pragma unroll
                for (int j = 0; j < NI; ++j) qy[j][h].load(y[j] + k + 8 * h);
            }
        } else {
#pragma unroll
            for (int h = 0; h < kRaws; ++h) {
                const int left = a.depth - k - k_lane - 8 * h;
#pragma unroll
                for (int i = 0; i < MI; ++i) fetch_left(qx[i][h], x[i] + k + 8 * h, left);
#pragma unroll
                for (int j = 0; j < NI; ++j) fetch_left(qy[j][h], y[j] + k + 8 * h, left);
            }
        }
    };
    f32x4 acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < kAhead; ++u) ask(rx[u], ry[u], wave + 4 * u);
    for (int step = wave; step < steps; step += 4 * kAhead) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {      // (steps beyond the last hold zeros)
#pragma unroll
            for (int h = 0; h < kRaws; ++h) {
                u4 px[MI][P], py[NI][P];
#pragma unroll
                for (int i = 0; i < MI; ++i) to_parts(rx[u][i][h], px[i]);
#pragma unroll
                for (int j = 0; j < NI; ++j) to_parts(ry[u][j][h], py[j]);
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int j = 0; j < NI; ++j) acc[i][j] = multiply<P>(px[i], py[j], acc[i][j]);
            }
            ask(rx[u], ry[u], step + 4 * (u + kAhead));
        }
    }
    if (wave > 0) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) sums[wave - 1][i * NI + j][lane] = acc[i][j];
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 0; w < 3; ++w)
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] += sums[w][i * NI + j][lane];
    finish<T, EPILOGUE, 16 * MI, 16 * NI, 1, 1>(a, acc, ta, tb, 0, nullptr);
}

// The gradients of all tokens (16 NI at most; gt holds 32 KT of them) from g, gt as kGradientParts leaves them, both in one launch.  h: a = weight, b = g,
// out = sums [split][token][ldo]; w: a = hidden, b = gt, out = dweight, `splits` parts of the vocabulary.  A block has
// kStreamColumns columns and one split; its waves take every fourth step each.
template <typename T, int NI, int KT>
__global__ void __launch_bounds__(256) stream_gradients_kernel(GemmArgs h, GemmArgs w, int groups) {
    constexpr int P = planes_of<T>();
    __shared__ f32x4 sums[8 * NI][kWave];
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / kWave), lane = threadIdx.x % kWave, r16 = lane % 16, quarter = lane / 16;
    // (row r of a fragment has eight columns from (4 (r % 4) + r / 4) 8 on, so that results of neighbouring quarters of a wave lie side by side)
    const int c0 = int(blockIdx.x) % groups * kStreamColumns, col = c0 + (r16 % 4 * 4 + r16 / 4) * 8, part = int(blockIdx.x) / groups;
    const int width = h.rows_a;
    const bool whole = c0 + kStreamColumns <= width;
    if (part < h.splits) {
        // dhidden: 32 rows of the vocabulary a step
        const int rows = h.depth, steps = (rows + 31) / 32, first = int(int64_t(steps) * part / h.splits), end = int(int64_t(steps) * (part + 1) / h.splits);
        const T* const x = static_cast<const T*>(h.a) + col;
        const uint16_t* y[NI];
#pragma unroll
        for (int j = 0; j < NI; ++j) y[j] = static_cast<const uint16_t*>(h.b) + int64_t(min(16 * j + r16, h.rows_b - 1)) * h.ldb + quarter * 8;
        Raw8<T> rx[2][8];
        u4 ry[2][NI][P];
        const auto ask = [&](Raw8<T> (&qx)[8], u4 (&qy)[NI][P], int step) {
            const int v = step * 32 + quarter * 8;
            if (step >= end) return;
            if (whole && step * 32 + 32 <= rows) {
#pragma unroll
                for (int r = 0; r < 8; ++r) qx[r].load(x + int64_t(v + r) * h.lda);
            } else {
#pragma unroll
                for (int r = 0; r < 8; ++r) fetch_left(qx[r], x + int64_t(v + r) * h.lda, v + r < rows ? width - col : 0);
            }
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int p = 0; p < P; ++p) qy[j][p] = *reinterpret_cast<const u4*>(y[j] + p * h.g_depth + step * 32);
        };
        f32x4 acc[8][NI];
#pragma unroll
        for (int f = 0; f < 8; ++f)
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[f][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        ask(rx[0], ry[0], first + wave);
        ask(rx[1], ry[1], first + wave + 4);
        for (int step = first + wave; step < end; step += 8) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (step + 4 * u >= end) break;
#pragma unroll
                for (int f = 0; f < 8; ++f) {
                    u4 px[P];
                    column_parts(rx[u], f, px);
#pragma unroll
                    for (int j = 0; j < NI; ++j) acc[f][j] = multiply<P>(px, ry[u][j], acc[f][j]);
                }
                ask(rx[u], ry[u], step + 4 * (u + 2));
            }
        }
        for (int from = 1; from < 4; ++from) {      // in a fixed order
            __syncthreads();
            if (wave == from) {
#pragma unroll
                for (int f = 0; f < 8; ++f)
#pragma unroll
                    for (int j = 0; j < NI; ++j) sums[f * NI + j][lane] = acc[f][j];
            }
            __syncthreads();
            if (wave == 0) {
#pragma unroll
                for (int f = 0; f < 8; ++f)
#pragma unroll
                    for (int j = 0; j < NI; ++j) acc[f][j] += sums[f * NI + j][lane];
            }
        }
        if (wave > 0) return;
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const int n = 16 * j + r16;
            if (n >= h.rows_b) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int m = c0 + e * 32 + quarter * 8;
                if (m >= width) continue;
                f32x4* const out = reinterpret_cast<f32x4*>(static_cast<float*>(h.out) + part * h.split_stride + n * h.ldo + m);
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const f32x4 s = {acc[4 * q][j][e], acc[4 * q + 1][j][e], acc[4 * q + 2][j][e], acc[4 * q + 3][j][e]};
                    out[q] = h.fresh ? s : out[q] + s;
                }
            }
        }
    } else {
        // dweight: 16 rows of the vocabulary a step, the tokens' columns stay in registers
        const int at = part - h.splits, rows = w.rows_b, steps = (rows + 15) / 16;
        const int first = int(int64_t(steps) * at / w.splits), end = int(int64_t(steps) * (at + 1) / w.splits);
        u4 px[KT][8][P];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            Raw8<T> r[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int t = kt * 32 + quarter * 8 + i;
                const int64_t target = t < w.depth ? w.targets[t] : -1;
                fetch_left(r[i], static_cast<const T*>(w.a) + int64_t(t) * w.lda + col, target >= 0 && target < w.vocab ? width - col : 0);
            }
#pragma unroll
            for (int f = 0; f < 8; ++f) column_parts(r, f, px[kt][f]);
        }
        const uint16_t* const y = static_cast<const uint16_t*>(w.b) + quarter * 8;
        u4 ry[2][KT][P];
        const auto ask = [&](u4 (&q)[KT][P], int step) {
            if (step >= end) return;
            const uint16_t* const p0 = y + int64_t(min(step * 16 + r16, rows - 1)) * w.ldb;
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int p = 0; p < P; ++p) q[kt][p] = *reinterpret_cast<const u4*>(p0 + p * w.gt_depth + kt * 32);
        };
        ask(ry[0], first + wave);
        ask(ry[1], first + wave + 4);
        for (int step = first + wave; step < end; step += 8) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (step + 4 * u >= end) break;
                float f[4][8];
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt) acc = multiply<P>(px[kt][c], ry[u][kt], acc);
#pragma unroll
                    for (int e = 0; e < 4; ++e) f[e][c] = acc[e];
                }
                const int n = (step + 4 * u) * 16 + r16, m = c0 + quarter * 8;
                ask(ry[u], step + 4 * (u + 2));
                if (n >= rows) continue;
#pragma unroll
                for (int e = 0; e < 4; ++e) store_run<T, 8>(static_cast<T*>(w.out) + n * w.ldo + m + e * 32, width - m - e * 32, f[e]);
            }
        }
    }
}

}  // namespace bns
