// Root-mean-square norm of the residual stream: forward with the residual's addition and an output in 8 bits, and backward.
// See include/bns.h for the equations.
//
// Both passes read every element once and write once, so HBM bounds them (a handful of operations per element); a row stays in registers between its
// sum of squares and its output.  A row belongs to TPR threads (a wave, 256, 512 or 1024), each of which holds VPT vectors of eight neighbouring
// elements: 16 bytes of bf16 a lane, a whole kilobyte a wave.  A wave per row needs no exchange through LDS, more threads per row leave fewer registers
// to each and keep more of a long row on its way; one row of one token takes as many threads as it has vectors.
// Measured: 8192x5120 bf16 with residual to 8 bits 54 us (5.5 TB/s; a large copy on the same device 5.2), one row of 4096 4.5 us, which is a launch;
// backward 16384x4096 bf16 90 us (6.0 TB/s), 777x1001 fp32 9.5 us: two launches, the first with one row a wave, whose vectors of a ragged width are asked
// for in branches one after another, and the sums of three waves through LDS behind it.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "bns_internal.hpp"
#include "bns_lm_device.hpp"
#include "bns_lm_validate.hpp"

using namespace bns;

namespace {

struct RmsArgs {
    const void *x, *residual, *weight;
    void *sum, *y;
    float *scales, *rstd;
    int64_t rows, x_stride, residual_stride, sum_stride, y_stride;
    int32_t width, groups, group;
    int32_t weight_bf16, e4m3, pow2;
    float eps, inv_width;
};

struct RmsBackwardArgs {
    const void *x, *weight, *dy, *dsum;
    const float* rstd;
    void* dx;
    float* partial;     // [blocks][width]
    int64_t rows, x_stride, dsum_stride, dx_stride, dy_stride;
    int32_t width, weight_bf16;
    float inv_width;
};

__device__ __forceinline__ void load_weight(const void* w, int bf16, int col, int left, float (&f)[8]) {
    if (bf16) Row8<bf16_t>::load(static_cast<const bf16_t*>(w) + col, left, f);
    else Row8<float>::load(static_cast<const float*>(w) + col, left, f);
}

// Sum / maximum over the TPR threads of a row; `lds` holds a float for every wave, and two calls in a row are given two different ones.
template <int TPR, typename F>
__device__ __forceinline__ F row_sum(F v, F* lds) {
    v = wave_sum(v);
    if (TPR == kWave) return v;
    if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = v;
    __syncthreads();
    F s = 0;
#pragma unroll
    for (int i = 0; i < TPR / kWave; ++i) s += lds[i];
    return s;
}
template <int TPR>
__device__ __forceinline__ float row_max(float v, float* lds) {
    v = wave_max(v);
    if (TPR == kWave) return v;
    if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = v;
    __syncthreads();
    float s = lds[0];
#pragma unroll
    for (int i = 1; i < TPR / kWave; ++i) s = fmaxf(s, lds[i]);
    return s;
}

// The vectors of a row that a thread holds.  RAGGED: the width is no multiple of eight, so the last vector goes element by element.  Otherwise
// a vector lies in the row or behind it, and what lies behind is read from the row's last vector and cleared: the loads stand in no branch,
// so that all of them are on their way at once.
template <typename T, int TPR, int VPT, bool RAGGED, bool NT>
struct RowOf {
    Raw8<T> raw[RAGGED ? 1 : VPT];
    float f[RAGGED ? VPT : 1][8];

    __device__ __forceinline__ void load(const T* p, int t, int width) {
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int col = (j * TPR + t) * 8;
            if constexpr (RAGGED) {
                if (col < width) {
                    Row8<T>::load(p + col, width - col, f[j]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[j][i] = 0.f;
                }
            } else {
                raw[j].template load<NT>(p + min(col, width - 8));
            }
        }
    }
    __device__ __forceinline__ void get(int j, int t, int width, float (&out)[8]) const {
        if constexpr (RAGGED) {
#pragma unroll
            for (int i = 0; i < 8; ++i) out[i] = f[j][i];
        } else {
            const bool in = (j * TPR + t) * 8 < width;
            raw[j].unpack(out);
#pragma unroll
            for (int i = 0; i < 8; ++i) out[i] = in ? out[i] : 0.f;
        }
    }
};

// Mean and eps with a rounding each, as the formula is written: scales that are rounded up to powers of two hang on the last bit of rstd, and an implementation of it by
// elementary operations comes to the same one.
__device__ __forceinline__ float mean_and_eps(float sum, float inv_width, float eps) {
#pragma clang fp contract(off)
    const float mean = sum * inv_width;
    return mean + eps;
}

// a / b to nearest, as a division gives it, from inv = 1 / b to nearest: the remainder of the product is exact (for a from 2^-102 on), one step takes it in.
__device__ __forceinline__ float quotient(float a, float b, float inv) {
    const float q = a * inv;
    return fmaf(fmaf(-q, b, a), inv, q);
}

// The scale of values whose largest magnitude is `most`: see include/bns.h.
__device__ __forceinline__ float e4m3_scale(float most, int pow2) {
    const float by = quotient(most, 448.f, 1.f / 448.f), s = most < __builtin_inff() ? fmaxf(by, 0x1p-126f) : most;
    if (!pow2) return s;
    const uint32_t bits = __float_as_uint(s);
    return __uint_as_float((bits + 0x7fffffu) & 0x7f800000u);
}

template <int TPR>
constexpr int block_of() { return TPR == kWave ? 256 : TPR; }

template <typename T, int TPR, int VPT, bool RAGGED, bool NT>
__global__ void __launch_bounds__(block_of<TPR>()) rms_forward_kernel(RmsArgs a) {
    constexpr int kRows = block_of<TPR>() / TPR;
    __shared__ double sums[block_of<TPR>() / kWave];
    __shared__ float maxima[block_of<TPR>() / kWave];
    const int t = threadIdx.x % TPR;
    for (int64_t row = int64_t(blockIdx.x) * kRows + threadIdx.x / TPR; row < a.rows; row += int64_t(gridDim.x) * kRows) {
        RowOf<T, TPR, VPT, RAGGED, NT> x, r;
        x.load(static_cast<const T*>(a.x) + row * a.x_stride, t, a.width);
        if (a.residual) r.load(static_cast<const T*>(a.residual) + row * a.residual_stride, t, a.width);
        float s[VPT][8];
        // (the squares of a vector are added in fp32, the vectors in fp64: the mean is as good as exact, for a dozen instructions)
        double squares = 0.0;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            x.get(j, t, a.width, s[j]);
            if (a.residual) {
                float f[8];
                r.get(j, t, a.width, f);
#pragma unroll
                for (int i = 0; i < 8; ++i) s[j][i] += f[i];
            }
            float square = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) square = fmaf(s[j][i], s[j][i], square);
            squares += double(square);
        }
        const float rstd = rsqrtf(mean_and_eps(float(row_sum<TPR>(squares, sums)), a.inv_width, a.eps));
        if (a.rstd && t == 0) a.rstd[row] = rstd;
        if (a.sum) {
            T* out = static_cast<T*>(a.sum) + row * a.sum_stride;
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                const int col = (j * TPR + t) * 8;
                if (col < a.width) Row8<T>::template store<NT>(out + col, RAGGED ? a.width - col : 8, s[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int col = (j * TPR + t) * 8;
            if (col < a.width) {
                float w[8];
                load_weight(a.weight, a.weight_bf16, col, RAGGED ? a.width - col : 8, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) s[j][i] = s[j][i] * rstd * w[i];
            }
        }
        if (!a.e4m3) {
            T* y = static_cast<T*>(a.y) + row * a.y_stride;
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                const int col = (j * TPR + t) * 8;
                if (col < a.width) Row8<T>::template store<NT>(y + col, RAGGED ? a.width - col : 8, s[j]);
            }
            if (TPR > kWave) __syncthreads();       // (the sums have been read)
            continue;
        }
        float most[VPT], whole = 0.f;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            most[j] = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) most[j] = fmaxf(most[j], fabsf(s[j][i]));
            whole = fmaxf(whole, most[j]);
        }
        if (a.group == 0) {
            whole = row_max<TPR>(whole, maxima);
#pragma unroll
            for (int j = 0; j < VPT; ++j) most[j] = whole;
        } else {
            // the vectors of a group lie in 4, 8 or 16 neighbouring lanes
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                most[j] = fmaxf(most[j], __shfl_xor(most[j], 1));
                most[j] = fmaxf(most[j], __shfl_xor(most[j], 2));
                if (a.group > 32) most[j] = fmaxf(most[j], __shfl_xor(most[j], 4));
                if (a.group > 64) most[j] = fmaxf(most[j], __shfl_xor(most[j], 8));
            }
        }
        uint8_t* y = static_cast<uint8_t*>(a.y) + row * a.y_stride;
        float* scales = a.scales + row * a.groups;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int col = (j * TPR + t) * 8, left = RAGGED ? a.width - col : 8;
            if (col >= a.width) continue;
            const float scale = e4m3_scale(most[j], a.pow2);
            if (a.group == 0 ? col == 0 : col % a.group == 0) scales[a.group == 0 ? 0 : col / a.group] = scale;
            // Quotients, not products with the reciprocal, whose rounding would decide what lies halfway between two numbers of the type (divisions instead: 8192x5120
            // bf16 57.6 against 54.2 us, 2000x2048 9.6 against 8.6).
            const float inv = 1.f / scale, finite = fminf(scale, 0x1.fffffep127f);
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = quotient(s[j][i], finite, inv);
            uint32_t q[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                int v = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * h], f[4 * h + 1], 0, false);
                q[h] = uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * h + 2], f[4 * h + 3], v, true));
            }
            if (left >= 8) {
                typedef uint32_t u2 __attribute__((ext_vector_type(2)));
                typedef u2 u2e __attribute__((aligned(1)));
                if constexpr (NT) __builtin_nontemporal_store((u2{q[0], q[1]}), reinterpret_cast<u2e*>(y + col));
                else *reinterpret_cast<u2e*>(y + col) = u2{q[0], q[1]};
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < left) y[col + i] = uint8_t(q[i / 4] >> (8 * (i % 4)));
            }
        }
        if (TPR > kWave) __syncthreads();
    }
}

// dx of every row, and dweight as one partial sum for each block (512 blocks at most, added by column_sum_kernel in a fixed order, without atomics): a
// thread meets the same columns in every row, so their sums stay in its registers.  The next row is asked for before the present one is worked on, where the registers hold both.
template <typename T, int TPR, int VPT, bool RAGGED, bool NT>
__global__ void __launch_bounds__(block_of<TPR>()) rms_backward_kernel(RmsBackwardArgs a) {
    constexpr int kRows = block_of<TPR>() / TPR;
    constexpr bool kAhead = TPR < 1024;
    __shared__ float lds[2][block_of<TPR>() / kWave];
    const int t = threadIdx.x % TPR;
    const int64_t first = int64_t(blockIdx.x) * kRows + threadIdx.x / TPR, step = int64_t(gridDim.x) * kRows;
    float dw[VPT][8];
#pragma unroll
    for (int j = 0; j < VPT; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[j][i] = 0.f;
    RowOf<T, TPR, VPT, RAGGED, NT> next_x, next_dy, next_ds;
    float next_rstd = 0.f;
    const auto ask = [&](int64_t row) {
        next_rstd = a.rstd[row];
        next_x.load(static_cast<const T*>(a.x) + row * a.x_stride, t, a.width);
        next_dy.load(static_cast<const T*>(a.dy) + row * a.dy_stride, t, a.width);
        if (a.dsum) next_ds.load(static_cast<const T*>(a.dsum) + row * a.dsum_stride, t, a.width);
    };
    if (kAhead && first < a.rows) ask(first);
    int turn = 0;
    for (int64_t row = first; row < a.rows; row += step, turn ^= 1) {
        if (!kAhead) ask(row);
        const RowOf<T, TPR, VPT, RAGGED, NT> x = next_x, dy = next_dy, ds = next_ds;
        const float rstd = next_rstd;
        if (kAhead && row + step < a.rows) ask(row + step);
        float xh[VPT][8], g[VPT][8];
        float dot = 0.f;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int col = (j * TPR + t) * 8;
            x.get(j, t, a.width, xh[j]);
            dy.get(j, t, a.width, g[j]);
            float w[8];
            if (RAGGED) {
                if (col < a.width) {
                    load_weight(a.weight, a.weight_bf16, col, a.width - col, w);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] = 0.f;
                }
            } else {
                load_weight(a.weight, a.weight_bf16, min(col, a.width - 8), 8, w);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                xh[j][i] *= rstd;
                dw[j][i] = fmaf(g[j][i], xh[j][i], dw[j][i]);
                g[j][i] *= w[i];
                dot = fmaf(g[j][i], xh[j][i], dot);
            }
        }
        const float mean = row_sum<TPR>(dot, lds[turn]) * a.inv_width;
        T* dx = static_cast<T*>(a.dx) + row * a.dx_stride;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int col = (j * TPR + t) * 8;
            if (col >= a.width) continue;
            float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (a.dsum) ds.get(j, t, a.width, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = fmaf(rstd, fmaf(-xh[j][i], mean, g[j][i]), f[i]);
            Row8<T>::template store<NT>(dx + col, RAGGED ? a.width - col : 8, f);
        }
    }
    if constexpr (kRows > 1) {                      // the waves of a block add theirs up first
        __shared__ float sums[kRows - 1][VPT * 8][TPR];
        const int group = threadIdx.x / TPR;
        if (group > 0) {
#pragma unroll
            for (int j = 0; j < VPT; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) sums[group - 1][j * 8 + i][t] = dw[j][i];
        }
        __syncthreads();
        if (group > 0) return;
#pragma unroll
        for (int k = 0; k < kRows - 1; ++k)
#pragma unroll
            for (int j = 0; j < VPT; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) dw[j][i] += sums[k][j * 8 + i][t];
    }
    float* out = a.partial + int64_t(blockIdx.x) * a.width;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int col = (j * TPR + t) * 8;
        if (col < a.width) Row8<float>::store(out + col, RAGGED ? a.width - col : 8, dw[j]);
    }
}

// Adds the partial sums of a column in a fixed order: 32 threads take every 32nd of them, then one adds the 32.
constexpr int kSumColumns = 32, kSumLanes = 32;
__global__ void __launch_bounds__(kSumColumns * kSumLanes) column_sum_kernel(const float* partial, int count, int width, float* out) {
    __shared__ float lds[kSumLanes][kSumColumns];
    const int c = threadIdx.x % kSumColumns, l = threadIdx.x / kSumColumns, col = blockIdx.x * kSumColumns + c;
    float s = 0.f;
    if (col < width) {
#pragma unroll 8
        for (int i = l; i < count; i += kSumLanes) s += partial[int64_t(i) * width + col];
    }
    lds[l][c] = s;
    __syncthreads();
    if (l == 0 && col < width) {
        for (int i = 1; i < kSumLanes; ++i) s += lds[i][c];
        out[col] = s;
    }
}

// Threads per row and vectors per thread.
struct RmsPlan {
    int tpr, vpt;
};
RmsPlan forward_plan(int64_t rows, int width) {
    const int vectors = (width + 7) / 8;
    // Few rows leave compute units idle: as many threads as the row has vectors.  Many rows: a wave each as far as its registers go, which
    // needs no exchange through LDS.
    const bool few = rows < 1024;
    const int tpr = vectors <= (few ? 64 : 256) ? 64 : vectors <= (few ? 256 : 1024) ? 256 : few && vectors <= 1024 ? 1024 : 512;
    int vpt = (vectors + tpr - 1) / tpr;
    if (tpr == 64 && vpt == 3) vpt = 4;
    if (tpr == 512) vpt = 4;
    return {tpr, vpt};
}

// The backward pass holds five values of an element where the forward pass holds two: two vectors per thread at most.
RmsPlan backward_plan(int width) {
    const int vectors = (width + 7) / 8;
    const int tpr = vectors <= 128 ? 64 : vectors <= 512 ? 256 : vectors <= 1024 ? 512 : 1024;
    return {tpr, tpr > 256 ? 2 : (vectors + tpr - 1) / tpr};
}

// Blocks of the backward pass: enough to fill the device, each of which leaves a row of partial sums behind.
int64_t backward_blocks(const RmsPlan& p, int64_t rows) {
    const int per_block = p.tpr == kWave ? 4 : 1;
    return std::min<int64_t>(std::max<int64_t>((rows + per_block - 1) / per_block, 1), 512);
}

// nt: with the non-temporal hint (8192x5120 bf16 to 8 bits 53.5 against 59.5 us, backward of 16384x4096 bf16 91 against 99; small calls lose, 777x1001 fp32
// 10.2 against 9.4).
#define BNS_RMS_CASE(T, KERNEL, TPR, VPT, THREADS)                                                                    \
    if (a.width % 8) BNS_LAUNCH((KERNEL<T, TPR, VPT, true, false>), grid, dim3(THREADS), 0, st, a);                   \
    else if (nt) BNS_LAUNCH((KERNEL<T, TPR, VPT, false, true>), grid, dim3(THREADS), 0, st, a);                       \
    else BNS_LAUNCH((KERNEL<T, TPR, VPT, false, false>), grid, dim3(THREADS), 0, st, a);                              \
    break;
// (plans of few rows, which never move that much)
#define BNS_RMS_FEW(T, KERNEL, TPR, VPT, THREADS)                                                                     \
    if (a.width % 8) BNS_LAUNCH((KERNEL<T, TPR, VPT, true, false>), grid, dim3(THREADS), 0, st, a);                   \
    else BNS_LAUNCH((KERNEL<T, TPR, VPT, false, false>), grid, dim3(THREADS), 0, st, a);                              \
    break;
#define BNS_RMS_FORWARD(T)                                              \
    switch (p.tpr * 10 + p.vpt) {                                       \
        case 641: BNS_RMS_CASE(T, rms_forward_kernel, 64, 1, 256)       \
        case 642: BNS_RMS_CASE(T, rms_forward_kernel, 64, 2, 256)       \
        case 644: BNS_RMS_CASE(T, rms_forward_kernel, 64, 4, 256)       \
        case 2561: BNS_RMS_FEW(T, rms_forward_kernel, 256, 1, 256)      \
        case 2562: BNS_RMS_CASE(T, rms_forward_kernel, 256, 2, 256)     \
        case 2563: BNS_RMS_CASE(T, rms_forward_kernel, 256, 3, 256)     \
        case 2564: BNS_RMS_CASE(T, rms_forward_kernel, 256, 4, 256)     \
        case 10241: BNS_RMS_FEW(T, rms_forward_kernel, 1024, 1, 1024)   \
        default: BNS_RMS_CASE(T, rms_forward_kernel, 512, 4, 512)       \
    }
#define BNS_RMS_BACKWARD(T)                                             \
    switch (p.tpr * 10 + p.vpt) {                                       \
        case 641: BNS_RMS_CASE(T, rms_backward_kernel, 64, 1, 256)      \
        case 642: BNS_RMS_CASE(T, rms_backward_kernel, 64, 2, 256)      \
        case 2561: BNS_RMS_CASE(T, rms_backward_kernel, 256, 1, 256)    \
        case 2562: BNS_RMS_CASE(T, rms_backward_kernel, 256, 2, 256)    \
        case 5122: BNS_RMS_CASE(T, rms_backward_kernel, 512, 2, 512)    \
        default: BNS_RMS_CASE(T, rms_backward_kernel, 1024, 2, 1024)    \
    }

constexpr int64_t kMostBlocks = int64_t(1) << 20;      // (a launch holds fewer than 2^32 threads; rows beyond are taken in turn)

}  // namespace

extern "C" {

bns_status bns_rms_forward(const bns_rms* rms, const void* x, const void* residual, const void* weight, void* sum, void* y, float* scales,
                           float* rstd, void* stream) {
    RmsDims d;
    const bns_status s = check_rms(rms, &d);
    if (s != BNS_OK) return s;
    const bool e4m3 = rms->out == BNS_OUT_E4M3;
    if (sum && !residual) return BNS_EINVAL;
    if (!e4m3 && scales) return BNS_EINVAL;
    if (d.rows == 0) return BNS_OK;
    if (!x || !weight || !y || (e4m3 && !scales)) return BNS_EINVAL;
    for (const void* p : {x, residual, weight, static_cast<const void*>(sum), static_cast<const void*>(y)})
        if (!aligned16(p)) return BNS_EINVAL;
    const size_t e = dtype_bytes(rms->dtype), ye = e4m3 ? 1 : e, row = size_t(d.width) * e, yrow = size_t(d.width) * ye;
    const Matrix mx = matrix(x, d.rows, d.width, d.x_stride, e), mr = matrix(residual, d.rows, d.width, d.residual_stride, e),
                 ms = matrix(sum, d.rows, d.width, d.sum_stride, e), my = matrix(y, d.rows, d.width, d.y_stride, ye);
    if (collide(ms, mx, true, row, row) || collide(ms, mr, true, row, row) || collide(my, mx, !e4m3, yrow, row) || collide(my, mr, false, yrow, row) ||
        collide(my, ms, false, yrow, row))
        return BNS_EINVAL;
    const RmsArgs a = {x, residual, weight, sum, y, scales, rstd, d.rows, d.x_stride, d.residual_stride, d.sum_stride, d.y_stride,
                       d.width, d.groups, rms->group, rms->weight_dtype == BNS_BF16, e4m3, rms->pow2_scales, rms->eps, 1.f / float(d.width)};
    const RmsPlan p = forward_plan(d.rows, d.width);
    const bool nt = size_t(d.rows) * (row * (residual ? sum ? 3 : 2 : 1) + yrow) > kStreamBytes;
    const int per_block = p.tpr == kWave ? 4 : 1;
    const dim3 grid(uint32_t(std::min<int64_t>((d.rows + per_block - 1) / per_block, kMostBlocks)));
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (rms->dtype == BNS_F32) {
        BNS_RMS_FORWARD(float)
    } else {
        BNS_RMS_FORWARD(bf16_t)
    }
    return hipGetLastError() == hipSuccess ? BNS_OK : BNS_EDEVICE;
}

size_t bns_rms_workspace_bytes(const bns_rms* rms) {
    RmsDims d;
    if (check_rms(rms, &d) != BNS_OK) return 0;
    return size_t(round_up(backward_blocks(backward_plan(d.width), d.rows) * d.width * 4, 256));
}

bns_status bns_rms_backward(const bns_rms* rms, const void* x, const void* weight, const float* rstd, const void* dy, const void* dsum, void* dx,
                            float* dweight, void* workspace, size_t workspace_bytes, void* stream) {
    RmsDims d;
    const bns_status s = check_rms(rms, &d);
    if (s != BNS_OK) return s;
    if (!weight || !dweight || !workspace || (d.rows > 0 && (!x || !rstd || !dy || !dx))) return BNS_EINVAL;
    for (const void* p : {x, weight, dy, dsum, static_cast<const void*>(dx), static_cast<const void*>(workspace)})
        if (!aligned16(p)) return BNS_EINVAL;
    const size_t e = dtype_bytes(rms->dtype), row = size_t(d.width) * e;
    const Matrix mx = matrix(x, d.rows, d.width, d.x_stride, e), mdy = matrix(dy, d.rows, d.width, d.y_stride, e),
                 mds = matrix(dsum, d.rows, d.width, d.residual_stride, e), mdx = matrix(dx, d.rows, d.width, d.sum_stride, e);
    if (collide(mdx, mx, false, row, row) || collide(mdx, mdy, true, row, row) || collide(mdx, mds, true, row, row)) return BNS_EINVAL;
    if (workspace_bytes < bns_rms_workspace_bytes(rms)) return BNS_EWORKSPACE;
    const RmsBackwardArgs a = {x, weight, dy, dsum, rstd, dx, static_cast<float*>(workspace), d.rows, d.x_stride, d.residual_stride, d.sum_stride,
                               d.y_stride, d.width, rms->weight_dtype == BNS_BF16, 1.f / float(d.width)};
    const RmsPlan p = backward_plan(d.width);
    const bool nt = size_t(d.rows) * row * (dsum ? 4 : 3) > kStreamBytes;
    const int64_t blocks = backward_blocks(p, d.rows);
    const dim3 grid{uint32_t(blocks)};
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (rms->dtype == BNS_F32) {
        BNS_RMS_BACKWARD(float)
    } else {
        BNS_RMS_BACKWARD(bf16_t)
    }
    if (hipGetLastError() != hipSuccess) return BNS_EDEVICE;
    BNS_LAUNCH(column_sum_kernel, dim3((d.width + kSumColumns - 1) / kSumColumns), dim3(kSumColumns * kSumLanes), 0, st,
               static_cast<const float*>(workspace), int(blocks), d.width, dweight);
    return hipGetLastError() == hipSuccess ? BNS_OK : BNS_EDEVICE;
}

}  // extern "C"
