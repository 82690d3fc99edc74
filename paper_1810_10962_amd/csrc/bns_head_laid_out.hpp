// The products of the loss over the vocabulary for large sizes: operands that are k-contiguous bf16 in memory go into LDS without passing through registers.
// What is not (fp32 values, which become three planes of bf16 parts; widths and strides that are no whole steps; the transposes
// that the gradients need) is laid out in the workspace first, piece by piece of the vocabulary.
#pragma once
#include "bns_head_device.hpp"

namespace bns {

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

// Row r of src becomes row r of dst (k = the column).  Bound by HBM.
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
            split3(f, w);
#pragma unroll
            for (int p = 0; p < 3; ++p) *reinterpret_cast<u4*>(out + int64_t(p) * a.depth) = w[p];
        }
    }
}

// Column c of src becomes row c of dst (k = the row), in tiles of 64 x 64 through LDS.  Bound by HBM: 16384x4096 bf16 56 us (4.8 TB/s), 4 % of a backward
// pass of 4096 tokens.
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
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = tile[r + i][c];
            u4 w[3];
            split3(f, w);
#pragma unroll
            for (int p = 0; p < 3; ++p) *reinterpret_cast<u4*>(out + int64_t(p) * a.depth) = w[p];
        }
    }
}

// ---- the product --------------------------------------------------------------------------------------------------
// Operands that are k-contiguous bf16 in memory (in three planes, where they are the parts of fp32 values): a row beyond the last is read as the last.
// The matrix units bound it.  A tile of 256 x 256 belongs to eight waves, 128 x 64 each, so that a step of 64 along k reads 24 fragments from LDS for
// 64 matrix instructions; two steps lie in LDS (128 KB), the next on its way past the registers while the present one is multiplied, one barrier a step.
// Tiles of 128 (four waves, 64 x 64) take over where those of 256 leave compute units idle.
// Measured: logits of 4096x4096x131072 bf16 with their statistics 3.45 to 3.52 ms (1.25 to 1.27 PFLOP/s; a large library product on the same device 1.27 to 1.38 with the same
// kind of values, more with zeros: power bounds both), as part of the backward pass 1.19 (g in two layouts) and 1.25 to 1.29 (the gradients); the six products of
// fp32 parts at 1021x1000x32003 1.00 to 1.12 PFLOP/s of bf16, one round of 256 tiles that nothing overlaps.
// Other forms were not faster: rings of four and five steps of 32 (422 and 434 us against 415 at 4096x4096x16384), halves of a block in turn (415), 32x32x16
// instructions (445), four waves of 128 x 128 (488).
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
    int split, ta, tb;
    place(int(blockIdx.x), a.splits, a.tiles_a, a.tiles_b, split, ta, tb);
    const int m0 = ta * BM, n0 = tb * BN;

    // Staging: a wave brings in eight rows of 128 bytes with one instruction, which puts lane after lane into LDS; the 16-byte chunks of row r
    // are swapped by r on their way (chunk c lies at c ^ (r % 8)), so that the reads of 16 rows at one chunk spread over the banks.
    const int last_a = a.rows_a - 1 - m0, last_b = a.rows_b - 1 - n0;
    const auto ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(a.a) + int64_t(m0) * a.lda * 2), 0, -1, 0x00027000);
    const auto rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(a.b) + int64_t(n0) * a.ldb * 2), 0, -1, 0x00027000);
    uint32_t at_a[BM / S::kPerIssue], at_b[BN / S::kPerIssue];
    const int in_row = lane / 8, chunk = (lane % 8) ^ in_row;
#pragma unroll
    for (int i = 0; i < BM / S::kPerIssue; ++i) at_a[i] = uint32_t(min(row_m<S::MI>(i * S::kPerIssue + wave * 8 + in_row), last_a)) * uint32_t(a.lda) * 2 + chunk * 16;
#pragma unroll
    for (int i = 0; i < BN / S::kPerIssue; ++i) at_b[i] = uint32_t(min(row_n<S::NI>(i * S::kPerIssue + wave * 8 + in_row), last_b)) * uint32_t(a.ldb) * 2 + chunk * 16;

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

}  // namespace bns
