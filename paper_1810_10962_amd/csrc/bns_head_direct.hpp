// Matrix products whose operands are read as they lie in memory: fp32 or bf16, rows or columns along k, any stride, any size.  On their way
// into LDS fp32 values become three bf16 parts and columns become rows, so nothing is laid out beforehand; that work is done again in every tile that
// reads an element, which is why large products prefer operands laid out once.
//
// A tile of BM x BN belongs to four waves, or, where there are few tiles, to GROUPS times four, each of which takes every GROUPS-th step of k; their sums are added at the
// end, in a fixed order.  The operands of the next steps of k are on their way from memory into registers while the present one is
// multiplied; LDS holds one step, so that several blocks share a compute unit and hide each other's waits.
//
// Few tokens: HBM bounds it (bf16 16x4096x131072 160 us, 6.7 TB/s; 16x2048x50257 57 us cold, 38 where the matrix lies in the memory-side cache; fp32 3x4096x100000
// 324 us, 5.1 TB/s).  More tokens: the way into LDS does, and for fp32 the splitting (some seven vector instructions for each element of a tile, nearly as long as the matrix
// instructions take at 64 x 64): fp32 386x3456x2389 108 us (0.35 PFLOP/s of bf16), 617x2752x7296 209 us, logits of 1021x1000x32003 as part of the backward pass 0.85.
#pragma once
#include "bns_head_device.hpp"

namespace bns {

// The elements of one operand's tile that a thread brings in: eight neighbours along k of a row (K_ROWS), or eight neighbouring rows at two
// neighbouring k, which together give whole 32-bit words of LDS.  ROW, SLOT: which row of the tile lies at which place in LDS (row_m, slot_m, ...).
// NT: with the non-temporal hint.
template <typename T, int ROWS, int DEPTH, bool K_ROWS, int THREADS, int (*ROW)(int), int (*SLOT)(int), bool NT = false>
struct Feed {
    static constexpr int P = planes_of<T>(), kRowBytes = DEPTH * 2, kPlane = ROWS * kRowBytes, kChunks = DEPTH / 8;
    static constexpr int kUnits = K_ROWS ? ROWS * DEPTH / 8 : (DEPTH / 2) * (ROWS / 8), kPer = (kUnits + THREADS - 1) / THREADS, kRaw = K_ROWS ? 1 : 2;
    Raw8<T> raw[kPer][kRaw];
    int64_t target[K_ROWS ? 1 : kPer][2];

    // Where 16-byte chunk c of row r lies: the chunks of a row change places with the row, so that neither the writes nor the reads of
    // sixteen rows at one chunk meet in a bank more often than they have to.
    static __device__ __forceinline__ int at(int r, int c) {
        const int s = kChunks == 8 ? (r ^ (r >> 3)) & 7 : ((r >> 1) ^ (r >> 3)) & 3;
        return r * kRowBytes + ((c ^ s) << 4);
    }

    static __device__ __forceinline__ void fetch(Raw8<T>& r, const T* p, int left) {
        if (left >= 8) r.load(p);
        else r.load_left(p, left);
    }

    // Rows [row0, row0 + ROWS) of `rows`, k in [k0, k0 + DEPTH) of `depth`; what lies outside is zero (rows of a K_ROWS operand: any row, their
    // results are left out).
    __device__ __forceinline__ void ask(int tid, const T* base, int64_t ld, int row0, int rows, int k0, int depth, const int64_t* targets) {
        const bool inside = k0 + DEPTH <= depth && (K_ROWS || row0 + ROWS <= rows);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int unit = i * THREADS + tid;
            if (kUnits % THREADS != 0 && unit >= kUnits) break;
            if constexpr (K_ROWS) {
                const int row = min(row0 + ROW(unit / kChunks), rows - 1), k = k0 + unit % kChunks * 8;
                const T* p = base + row * ld + k;
                if (inside) raw[i][0].template load<NT>(p);
                else fetch(raw[i][0], p, depth - k);
            } else {
                const int row = row0 + unit % (ROWS / 8) * 8, k = k0 + unit / (ROWS / 8) * 2;
                const T* p = base + k * ld + row;
                if (inside) {
                    raw[i][0].load(p);
                    raw[i][1].load(p + ld);
                } else {
                    fetch(raw[i][0], p, k < depth ? rows - row : 0);
                    fetch(raw[i][1], p + ld, k + 1 < depth ? rows - row : 0);
                }
                if (targets) {
                    target[i][0] = targets[min(k, depth - 1)];
                    target[i][1] = targets[min(k + 1, depth - 1)];
                }
            }
        }
    }

    __device__ __forceinline__ void put(int tid, char* lds, const int64_t* targets, int vocab) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int unit = i * THREADS + tid;
            if (kUnits % THREADS != 0 && unit >= kUnits) break;
            if constexpr (K_ROWS) {
                const int to = at(unit / kChunks, unit % kChunks);
                if constexpr (P == 1) {
                    *reinterpret_cast<u4*>(lds + to) = raw[i][0].a;
                } else {
                    float f[8];
                    raw[i][0].unpack(f);
                    u4 w[3];
                    split3(f, w);
#pragma unroll
                    for (int p = 0; p < 3; ++p) *reinterpret_cast<u4*>(lds + p * kPlane + to) = w[p];
                }
            } else {
                if (targets) {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        if (!(target[i][h] >= 0 && target[i][h] < vocab)) raw[i][h].clear();
                }
                const int row = unit % (ROWS / 8) * 8, pair = unit / (ROWS / 8);
                if constexpr (P == 1) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const uint32_t even = raw[i][0].a[j / 2], odd = raw[i][1].a[j / 2];
                        *reinterpret_cast<uint32_t*>(lds + at(SLOT(row + j), pair / 4) + pair % 4 * 4) =
                            j % 2 ? even >> 16 | (odd & 0xffff0000u) : (even & 0xffffu) | odd << 16;
                    }
                } else {
                    float even[8], odd[8];
                    raw[i][0].unpack(even);
                    raw[i][1].unpack(odd);
                    uint32_t word[8][3];
                    split3(even, odd, word);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
#pragma unroll
                        for (int p = 0; p < 3; ++p)
                            *reinterpret_cast<uint32_t*>(lds + p * kPlane + at(SLOT(row + j), pair / 4) + pair % 4 * 4) = word[j][p];
                }
            }
        }
    }
};

template <typename T, int BM, int BN, int WM, int WN>
struct DirectTile {
    static constexpr int P = planes_of<T>(), kThreads = WM * WN * kWave, kDepth = P == 1 ? 64 : 32, kBytes = (BM + BN) * kDepth * 2 * P;
    static_assert(WM * BN * 8 <= kBytes, "room for the statistics");
};

// One tile of a product.  A_ROWS, B_ROWS: whether that operand's rows run along k (else m, n are its columns, and a.lda, a.ldb lead from one k to the next).
// `lds`: GROUPS times DirectTile::kBytes.  NT: A, which nobody reads again, with the non-temporal hint.
template <typename T, int BM, int BN, int WM, int WN, int GROUPS, bool A_ROWS, bool B_ROWS, int EPILOGUE, bool NT = false>
__device__ __forceinline__ void direct_tile(const GemmArgs& a, int block, char* lds) {
    using S = DirectTile<T, BM, BN, WM, WN>;
    constexpr int P = S::P, D = S::kDepth, MI = BM / WM / 16, NI = BN / WN / 16;
    static_assert(S::kThreads == 256 && MI * NI * int(sizeof(f32x4)) * 256 <= S::kBytes * (GROUPS > 1 ? 1 : 1000), "a group's sums fit its part of LDS");
    using FeedA = Feed<T, BM, D, A_ROWS, S::kThreads, row_m<MI>, slot_m<MI>, NT>;
    using FeedB = Feed<T, BN, D, B_ROWS, S::kThreads, row_n<NI>, slot_n<NI>>;
    const int group = GROUPS > 1 ? __builtin_amdgcn_readfirstlane(int(threadIdx.x) / 256) : 0, tid = GROUPS > 1 ? int(threadIdx.x) % 256 : int(threadIdx.x);
    char* const lds_a = lds + group * S::kBytes;
    char* const lds_b = lds_a + FeedA::kPlane * P;
    int split, ta, tb;
    place(block, a.splits, a.tiles_a, a.tiles_b, split, ta, tb);
    const int m0 = ta * BM, n0 = tb * BN;
    const int steps = (a.depth + D - 1) / D, first = int(int64_t(steps) * split / a.splits), end = int(int64_t(steps) * (split + 1) / a.splits);
    const T *pa = static_cast<const T*>(a.a), *pb = static_cast<const T*>(a.b);
    const int64_t* const targets = A_ROWS ? nullptr : a.targets;
    const int lane = tid % kWave, wave = tid / kWave, wm = wave / WN, wn = wave % WN, r16 = lane % 16, quarter = lane / 16;
    constexpr int kAhead = BM * BN > 64 * 64 || (GROUPS > 1 && P > 1) ? 1 : 2;      // steps on their way, as far as registers go
    FeedA fa[kAhead];
    FeedB fb[kAhead];
    f32x4 acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const auto ask = [&](int u, int step) {
        fa[u].ask(tid, pa, a.lda, m0, a.rows_a, step * D, a.depth, targets);
        fb[u].ask(tid, pb, a.ldb, n0, a.rows_b, step * D, a.depth, nullptr);
    };
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
        if (first + group + GROUPS * u < end) ask(u, first + group + GROUPS * u);
    for (int at = first; at < end; at += GROUPS * kAhead) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int base = at + GROUPS * u, step = base + group;
            if (base >= end) break;                 // (the same for all groups, which meet twice a step)
            __syncthreads();                        // (the step before has been read)
            if (step < end) {
                fa[u].put(tid, lds_a, targets, a.vocab);
                fb[u].put(tid, lds_b, nullptr, 0);
            }
            __syncthreads();
            if (step >= end) continue;
            if (step + GROUPS * kAhead < end) ask(u, step + GROUPS * kAhead);
#pragma unroll
            for (int kk = 0; kk < D / 32; ++kk) {
                bf16x8 x[MI][P], y[NI][P];
#pragma unroll
                for (int p = 0; p < P; ++p) {
#pragma unroll
                    for (int j = 0; j < NI; ++j)
                        y[j][p] = *reinterpret_cast<const bf16x8*>(lds_b + p * FeedB::kPlane + FeedB::at(wn * (BN / WN) + j * 16 + r16, kk * 4 + quarter));
#pragma unroll
                    for (int i = 0; i < MI; ++i)
                        x[i][p] = *reinterpret_cast<const bf16x8*>(lds_a + p * FeedA::kPlane + FeedA::at(wm * (BM / WM) + i * 16 + r16, kk * 4 + quarter));
                }
#pragma unroll
                for (int s = P == 1 ? 5 : 0; s < 6; ++s)
#pragma unroll
                    for (int i = 0; i < MI; ++i)
#pragma unroll
                        for (int j = 0; j < NI; ++j)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[i][plane_a(s)], y[j][plane_b(s)], acc[i][j], 0, 0, 0);
            }
        }
    }
    if constexpr (GROUPS > 1) {
        __syncthreads();
        if (group > 0) {
            f32x4* const sums = reinterpret_cast<f32x4*>(lds_a);
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j) sums[(i * NI + j) * 256 + tid] = acc[i][j];
        }
        __syncthreads();
        if (group > 0) {
            if constexpr (EPILOGUE == kStatistics && WM > 1) {      // finish() meets twice
                __syncthreads();
                __syncthreads();
            }
            return;
        }
        for (int g = 1; g < GROUPS; ++g) {
            const f32x4* const sums = reinterpret_cast<const f32x4*>(lds + g * S::kBytes);
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j) acc[i][j] += sums[(i * NI + j) * 256 + tid];
        }
    }
    finish<T, EPILOGUE, BM, BN, WM, WN>(a, acc, ta, tb, split, reinterpret_cast<float2*>(lds));
}

}  // namespace bns
