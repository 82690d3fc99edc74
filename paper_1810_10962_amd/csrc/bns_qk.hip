// Queries and keys: the root-mean-square norm of every head and the rotation by position behind it, forward and backward.  See include/bns.h for the
// equations.
//
// Both read every element once and write once, so HBM bounds them where tokens are many and a launch where they are few.  A head of `width` elements belongs
// to a group of G lanes; a lane holds one unit of it, two chunks of 16 bytes that contain both elements of every pair that it rotates (chunks
// rotated / 2 apart, or neighbours), so that the rotation needs no exchange and the sums one of log2 G steps.  The lanes of a wave take hs heads each of
// 64 / (G hs) tokens at a time, go on to the next heads with the same angles, and queries and keys go to different blocks, so that a wave holds one weight.
//
// Angles: position * frequency is formed in quarter turns in fp64 and reduced exactly (the remainder of a fused multiply-add with the nearest whole
// number); what is left, at most an eighth of a turn, is exact enough in fp32, and Taylor's series to x^9 and x^10 leave 2e-9 there.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "bns_internal.hpp"
#include "bns_lm_device.hpp"
#include "bns_step_validate.hpp"

using namespace bns;

namespace {

// Queries, or keys.
struct Heads {
    const void *x, *dy, *weight;
    void* out;          // forward: y; backward: dx
    float* partial;     // backward: [blocks][width]
    HeadStrides xs, ds, os;
    FastDiv splits;     // waves that share the heads of a token
    int64_t jobs;       // pieces of work of a wave: groups of tokens times splits
    int32_t heads, turns;   // turns: steps of a wave over the heads of its tokens
    int32_t log_hs;     // heads of a token that a wave takes at a time
    int32_t blocks;
};

struct QkArgs {
    Heads part[2];
    const int64_t* positions;
    const double* frequencies;
    int64_t tokens;
    int32_t width, rotated, weight_bf16, interleaved;
    float eps, inv_width;
};

// Elements of a lane: a chunk of E as it is stored, or a single element.
template <typename T, int E>
struct Chunk;
template <typename T>
struct Chunk<T, 1> {
    float f = 0.f;
    __device__ __forceinline__ void load(const T* p) { f = load_scalar<T>(p); }
    __device__ __forceinline__ void clear() { f = 0.f; }
    __device__ __forceinline__ void unpack(float (&v)[1]) const { v[0] = f; }
    template <bool NT>
    static __device__ __forceinline__ void store(T* p, const float (&v)[1]) { Vec<T, 1>{{v[0]}}.store(p); }
};
template <>
struct Chunk<float, 4> {
    words4_t w;
    __device__ __forceinline__ void load(const float* p) { w = get16<false>(p); }
    __device__ __forceinline__ void clear() { w = words4_t{0, 0, 0, 0}; }
    __device__ __forceinline__ void unpack(float (&v)[4]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
    }
    template <bool NT>
    static __device__ __forceinline__ void store(float* p, const float (&v)[4]) {
        put16<NT>(p, words4_t{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])});
    }
};
template <>
struct Chunk<bf16_t, 8> {
    words4_t w;
    __device__ __forceinline__ void load(const bf16_t* p) { w = get16<false>(p); }
    __device__ __forceinline__ void clear() { w = words4_t{0, 0, 0, 0}; }
    __device__ __forceinline__ void unpack(float (&v)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    template <bool NT>
    static __device__ __forceinline__ void store(bf16_t* p, const float (&v)[8]) {
        put16<NT>(p, words4_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])});
    }
};

// Sum over groups of G neighbouring lanes, in every one of them.
template <int CTRL>
__device__ __forceinline__ float dpp_move(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
template <int G>
__device__ __forceinline__ float group_sum(float v) {
    static_assert(G >= 4 && G <= 64, "groups of lanes");
    v += dpp_move<0xb1>(v);                     // quad_perm: lane ^ 1
    v += dpp_move<0x4e>(v);                     // quad_perm: lane ^ 2
    if (G >= 8) v += dpp_move<0x141>(v);        // row_half_mirror: the other four of eight
    if (G >= 16) v += dpp_move<0x140>(v);       // row_mirror: the other eight of sixteen
    if (G >= 32) v += __shfl_xor(v, 16);
    if (G >= 64) v += __shfl_xor(v, 32);
    return v;
}

// cos and sin of `position` times an angle given in quarter turns.
__device__ __forceinline__ void turn(double position, double quarters, float* c, float* s) {
    const double n = rint(position * quarters);
    const float x = float(fma(position, quarters, -n)) * 1.57079632679489662f;      // |x| <= pi / 4
    const int quadrant = int(fma(-4.0, rint(n * 0.25), n));                        // -2 .. 2
    const float x2 = x * x;
    const float sine = x * fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), 1.f);
    const float cosine = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
    const bool odd = quadrant & 1;
    const float a = odd ? sine : cosine, b = odd ? cosine : sine;
    *c = (quadrant + 1) & 2 ? -a : a;       // 1, 2, -2 (as 2): negative; -1 gives 0 & 2
    *s = quadrant & 2 ? -b : b;             // 2, -2, -1 (as 3): negative
}

// What a lane holds of a head, the same for every head.
template <typename T, int E, int G, int UPL, bool NEIGHBOURS>
struct Lane {
    int at[UPL][2];             // first elements of its chunks; -1: none
    bool turned[UPL][2];
    float w[UPL][2][E];
    double quarters[UPL][E];    // NEIGHBOURS: E / 2 of each chunk

    __device__ __forceinline__ void set(const QkArgs& a, const Heads& p, int l) {
#pragma unroll
        for (int k = 0; k < UPL; ++k) {
            const int u = k * G + l;
            int angle[2];
            if (NEIGHBOURS) {
                at[k][0] = 2 * u * E;
                at[k][1] = at[k][0] + E;
                angle[0] = at[k][0] / 2;
                angle[1] = at[k][1] / 2;
                turned[k][0] = at[k][0] < a.rotated;
                turned[k][1] = at[k][1] < a.rotated;
            } else {
                const int units = a.rotated / (2 * E), rest = u - units;
                const bool t = rest < 0;
                if (E == 1 && a.interleaved) {
                    at[k][0] = 2 * u;
                    at[k][1] = 2 * u + 1;
                } else {
                    at[k][0] = t ? u * E : a.rotated + 2 * rest * E;
                    at[k][1] = t ? a.rotated / 2 + u * E : at[k][0] + E;
                }
                angle[0] = angle[1] = u * E;
                turned[k][0] = turned[k][1] = t;
            }
#pragma unroll
            for (int c = 0; c < 2; ++c)
                if (at[k][c] >= a.width) at[k][c] = -1;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const int c = NEIGHBOURS ? i / (E / 2 > 0 ? E / 2 : 1) : 0, j = NEIGHBOURS ? i % (E / 2 > 0 ? E / 2 : 1) : i;
                quarters[k][i] = turned[k][c] && at[k][c] >= 0 ? a.frequencies[angle[c] + j] * 0.63661977236758134308 : 0.0;    // 2 / pi
            }
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const int e = at[k][c] + i;
                    w[k][c][i] = at[k][c] < 0 ? 0.f : !p.weight ? 1.f : a.weight_bf16 ? load_scalar<bf16_t>(static_cast<const bf16_t*>(p.weight) + e) : static_cast<const float*>(p.weight)[e];
                }
        }
    }
    __device__ __forceinline__ void load(Chunk<T, E> (&c)[UPL][2], const T* head) const {
#pragma unroll
        for (int k = 0; k < UPL; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (at[k][i] >= 0) c[k][i].load(head + at[k][i]);
                else c[k][i].clear();
            }
    }
    template <bool NT>
    __device__ __forceinline__ void store(T* head, const float (&v)[UPL][2][E]) const {
#pragma unroll
        for (int k = 0; k < UPL; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (at[k][i] >= 0) Chunk<T, E>::template store<NT>(head + at[k][i], v[k][i]);
    }
    // BACK: by the negative angle
    template <bool BACK>
    __device__ __forceinline__ void rotate(float (&v)[UPL][2][E], const float (&cs)[UPL][E], const float (&sn)[UPL][E]) const {
#pragma unroll
        for (int k = 0; k < UPL; ++k)
#pragma unroll
            for (int i = 0; i < E; ++i) {
                constexpr int H = E / 2 > 0 ? E / 2 : 1;
                const int c = NEIGHBOURS ? i / H : 0, j = NEIGHBOURS ? i % H : i;
                float &x = NEIGHBOURS ? v[k][c][2 * j] : v[k][0][i], &y = NEIGHBOURS ? v[k][c][2 * j + 1] : v[k][1][i];
                const float s = BACK ? -sn[k][i] : sn[k][i];
                const float xr = fmaf(x, cs[k][i], -(y * s)), yr = fmaf(x, s, y * cs[k][i]);
                x = turned[k][c] ? xr : x;
                y = turned[k][c] ? yr : y;
            }
    }
};

// The work of a wave: one piece after another, each a group of tokens and some of their heads.  `step(token, head)` is called for one head at a time by
// all lanes of it, or for none (head < 0).
template <typename T, int E, int G, int UPL, bool NEIGHBOURS, bool NT>
__global__ void __launch_bounds__(256) qk_forward_kernel(QkArgs a) {
    const int which = int(blockIdx.x) >= a.part[0].blocks;
    const Heads& p = a.part[which];
    const int lane = threadIdx.x % kWave, slot = lane / G;
    const int hs = 1 << p.log_hs, tokens_at_once = (kWave / G) >> p.log_hs;
    Lane<T, E, G, UPL, NEIGHBOURS> mine;
    mine.set(a, p, lane % G);
    const int64_t first = int64_t(int(blockIdx.x) - (which ? a.part[0].blocks : 0)) * 4 + threadIdx.x / kWave;
    for (int64_t job = first; job < p.jobs; job += int64_t(p.blocks) * 4) {
        const uint32_t group = fdiv(uint32_t(job), p.splits), split = uint32_t(job) - group * p.splits.d;
        const int64_t token = int64_t(group) * tokens_at_once + (slot >> p.log_hs);
        if (token >= a.tokens) continue;
        const int from = int(int64_t(p.turns) * split / p.splits.d), to = int(int64_t(p.turns) * (split + 1) / p.splits.d);
        const int h0 = slot & (hs - 1);
        const T* x = static_cast<const T*>(p.x) + token * p.xs.token;
        T* out = static_cast<T*>(p.out) + token * p.os.token;
        Chunk<T, E> next[UPL][2];
        int h = from * hs + h0;
        if (h < p.heads) mine.load(next, x + int64_t(h) * p.xs.head);
        float cs[UPL][E], sn[UPL][E];
        const double position = a.positions ? double(a.positions[token]) : 0.0;
#pragma unroll
        for (int k = 0; k < UPL; ++k)
#pragma unroll
            for (int i = 0; i < E; ++i) turn(position, mine.quarters[k][i], &cs[k][i], &sn[k][i]);
        for (int t = from; t < to; ++t, h += hs) {
            if (h >= p.heads) break;
            float v[UPL][2][E];
#pragma unroll
            for (int k = 0; k < UPL; ++k)
#pragma unroll
                for (int c = 0; c < 2; ++c) next[k][c].unpack(v[k][c]);
            if (t + 1 < to && h + hs < p.heads) mine.load(next, x + int64_t(h + hs) * p.xs.head);
            if (p.weight) {
                float squares = 0.f;
#pragma unroll
                for (int k = 0; k < UPL; ++k)
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int i = 0; i < E; ++i) squares = fmaf(v[k][c][i], v[k][c][i], squares);
                const float rstd = rsqrtf(fmaf(group_sum<G>(squares), a.inv_width, a.eps));
#pragma unroll
                for (int k = 0; k < UPL; ++k)
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int i = 0; i < E; ++i) v[k][c][i] *= rstd * mine.w[k][c][i];
            }
            mine.template rotate<false>(v, cs, sn);
            mine.template store<NT>(out + int64_t(h) * p.os.head, v);
        }
    }
}

template <typename T, int E, int G, int UPL, bool NEIGHBOURS, bool NT>
__global__ void __launch_bounds__(256) qk_backward_kernel(QkArgs a) {
    const int which = int(blockIdx.x) >= a.part[0].blocks;
    const Heads& p = a.part[which];
    const int lane = threadIdx.x % kWave, slot = lane / G;
    const int hs = 1 << p.log_hs, tokens_at_once = (kWave / G) >> p.log_hs;
    Lane<T, E, G, UPL, NEIGHBOURS> mine;
    mine.set(a, p, lane % G);
    float dw[UPL][2][E];
#pragma unroll
    for (int k = 0; k < UPL; ++k)
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < E; ++i) dw[k][c][i] = 0.f;
    const int block = int(blockIdx.x) - (which ? a.part[0].blocks : 0);
    for (int64_t job = int64_t(block) * 4 + threadIdx.x / kWave; job < p.jobs; job += int64_t(p.blocks) * 4) {
        const uint32_t group = fdiv(uint32_t(job), p.splits), split = uint32_t(job) - group * p.splits.d;
        const int64_t token = int64_t(group) * tokens_at_once + (slot >> p.log_hs);
        if (token >= a.tokens) continue;
        const int from = int(int64_t(p.turns) * split / p.splits.d), to = int(int64_t(p.turns) * (split + 1) / p.splits.d);
        const int h0 = slot & (hs - 1);
        const T *x = static_cast<const T*>(p.x) + token * p.xs.token, *dy = static_cast<const T*>(p.dy) + token * p.ds.token;
        T* out = static_cast<T*>(p.out) + token * p.os.token;
        Chunk<T, E> next_x[UPL][2], next_g[UPL][2];
        int h = from * hs + h0;
        const auto ask = [&](int head) {
            mine.load(next_g, dy + int64_t(head) * p.ds.head);
            if (p.weight) mine.load(next_x, x + int64_t(head) * p.xs.head);
        };
        if (h < p.heads) ask(h);
        float cs[UPL][E], sn[UPL][E];
        const double position = a.positions ? double(a.positions[token]) : 0.0;
#pragma unroll
        for (int k = 0; k < UPL; ++k)
#pragma unroll
            for (int i = 0; i < E; ++i) turn(position, mine.quarters[k][i], &cs[k][i], &sn[k][i]);
        for (int t = from; t < to; ++t, h += hs) {
            if (h >= p.heads) break;
            float g[UPL][2][E], v[UPL][2][E];
#pragma unroll
            for (int k = 0; k < UPL; ++k)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    next_g[k][c].unpack(g[k][c]);
                    if (p.weight) next_x[k][c].unpack(v[k][c]);
                }
            if (t + 1 < to && h + hs < p.heads) ask(h + hs);
            mine.template rotate<true>(g, cs, sn);
            if (p.weight) {
                float squares = 0.f, dot = 0.f;
#pragma unroll
                for (int k = 0; k < UPL; ++k)
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int i = 0; i < E; ++i) {
                            squares = fmaf(v[k][c][i], v[k][c][i], squares);
                            dot = fmaf(g[k][c][i] * mine.w[k][c][i], v[k][c][i], dot);
                        }
                const float rstd = rsqrtf(fmaf(group_sum<G>(squares), a.inv_width, a.eps));
                const float mean = group_sum<G>(dot) * rstd * a.inv_width;       // of weight * g * x^
#pragma unroll
                for (int k = 0; k < UPL; ++k)
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int i = 0; i < E; ++i) {
                            const float xh = v[k][c][i] * rstd;
                            dw[k][c][i] = fmaf(g[k][c][i], xh, dw[k][c][i]);
                            g[k][c][i] = rstd * fmaf(g[k][c][i], mine.w[k][c][i], -xh * mean);
                        }
            }
            mine.template store<NT>(out + int64_t(h) * p.os.head, g);
        }
    }
    if (!p.weight) return;
    // The block's sums: the lanes that hold the same elements, in their order.
    constexpr int kSlots = 256 / G;
    __shared__ float sums[UPL * 2 * E][256];
#pragma unroll
    for (int k = 0; k < UPL; ++k)
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < E; ++i) sums[(k * 2 + c) * E + i][threadIdx.x] = dw[k][c][i];
    __syncthreads();
    float* partial = p.partial + int64_t(block) * a.width;
    // (element r of lane l: written by that lane's place among the first G threads, which knows where it goes)
    for (int r = threadIdx.x / G; r < UPL * 2 * E; r += kSlots) {
        const int l = threadIdx.x % G;
        float s = 0.f;
        for (int j = 0; j < kSlots; ++j) s += sums[r][j * G + l];
        const int k = r / (2 * E), c = r / E % 2, i = r % E;
        int at = -1;
#pragma unroll
        for (int kk = 0; kk < UPL; ++kk)
#pragma unroll
            for (int cc = 0; cc < 2; ++cc)
                if (kk == k && cc == c) at = mine.at[kk][cc];
        if (at >= 0) partial[at + i] = s;
    }
}

// Adds the blocks' sums of an element in a fixed order: 32 threads take every 32nd of them, then one adds the 32.  Row 0 of the grid: queries; 1: keys.
constexpr int kSumColumns = 32, kSumLanes = 32;
struct SumArgs {
    const float* partial[2];
    float* out[2];
    int32_t count[2], width;
};
__global__ void __launch_bounds__(kSumColumns * kSumLanes) qk_weight_sum_kernel(SumArgs a) {
    __shared__ float lds[kSumLanes][kSumColumns];
    const int which = blockIdx.y;
    if (!a.out[which]) return;
    const float* partial = a.partial[which];
    const int c = threadIdx.x % kSumColumns, l = threadIdx.x / kSumColumns, col = blockIdx.x * kSumColumns + c;
    float s = 0.f;
    if (col < a.width) {
#pragma unroll 8
        for (int i = l; i < a.count[which]; i += kSumLanes) s += partial[int64_t(i) * a.width + col];
    }
    lds[l][c] = s;
    __syncthreads();
    if (l == 0 && col < a.width) {
        for (int i = 1; i < kSumLanes; ++i) s += lds[i][c];
        a.out[which][col] = s;
    }
}

// How a head lies in lanes.
struct QkPlan {
    int chunk, group, per_lane;
};
QkPlan qk_plan(const QkDims& d, int32_t dtype, bool interleaved) {
    const int e = dtype == BNS_F32 ? 4 : 8;
    if (d.width % e || d.rotated % (interleaved ? e : 2 * e)) return (d.width + 1) / 2 <= 64 ? QkPlan{1, 16, 4} : QkPlan{1, 64, 4};
    const int units = interleaved ? (d.width / e + 1) / 2 : d.rotated / (2 * e) + ((d.width - d.rotated) / e + 1) / 2;
    int g = 4;
    while (g < units) g *= 2;
    return {e, g, 1};
}

constexpr int kMostForwardBlocks = 256 * 8, kMostBackwardBlocks = 512;

// Shares the tokens and heads of one tensor out: `most` blocks of four waves.
void share_out(Heads* p, const QkPlan& plan, int64_t tokens, int heads, int most) {
    const int slots = kWave / plan.group;
    p->heads = heads;
    p->log_hs = 0;
    while ((1 << p->log_hs) < heads && (2 << p->log_hs) <= slots) ++p->log_hs;
    const int hs = 1 << p->log_hs, tokens_at_once = slots / hs;
    p->turns = (heads + hs - 1) / hs;
    const int64_t groups = (tokens + tokens_at_once - 1) / tokens_at_once;
    // Few tokens: the turns over their heads go to different waves.  (Jobs are numbered in 32 bits: splits only where tokens are few.)
    const int64_t splits = std::max<int64_t>(1, std::min<int64_t>(p->turns, groups > 0 ? int64_t(most) * 4 / groups : 1));
    p->splits = make_fastdiv(uint32_t(splits));
    p->jobs = heads > 0 ? groups * splits : 0;
    p->blocks = int32_t(std::min<int64_t>((p->jobs + 3) / 4, most));
}

void fill(QkArgs* a, const bns_qk* qk, const QkDims& d, const QkPlan& plan, int most) {
    a->tokens = d.tokens;
    a->width = d.width;
    a->rotated = d.rotated;
    a->weight_bf16 = qk->weight_dtype == BNS_BF16;
    a->interleaved = qk->interleaved;
    a->eps = qk->eps;
    a->inv_width = 1.f / float(d.width);
    for (int i = 0; i < 2; ++i) share_out(&a->part[i], plan, d.tokens, d.heads[i], most);
}

#define BNS_QK_ONE(KERNEL, T, E, G, UPL, NB)                                                                                   \
    do {                                                                                                                       \
        if (nt) BNS_LAUNCH((KERNEL<T, E, G, UPL, NB, true>), grid, dim3(256), 0, st, a);                                       \
        else BNS_LAUNCH((KERNEL<T, E, G, UPL, NB, false>), grid, dim3(256), 0, st, a);                                         \
    } while (0)
#define BNS_QK_CASE(KERNEL, T, E, G)                                    \
    do {                                                                \
        if (a.interleaved) BNS_QK_ONE(KERNEL, T, E, G, 1, true);        \
        else BNS_QK_ONE(KERNEL, T, E, G, 1, false);                     \
    } while (0)
#define BNS_QK_LAUNCH(KERNEL)                                                                       \
    do {                                                                                            \
        if (f32 && plan.chunk == 1 && plan.group == 16) BNS_LAUNCH((KERNEL<float, 1, 16, 4, false, false>), grid, dim3(256), 0, st, a); \
        else if (f32 && plan.chunk == 1) BNS_LAUNCH((KERNEL<float, 1, 64, 4, false, false>), grid, dim3(256), 0, st, a);                \
        else if (plan.chunk == 1 && plan.group == 16) BNS_LAUNCH((KERNEL<bf16_t, 1, 16, 4, false, false>), grid, dim3(256), 0, st, a);  \
        else if (plan.chunk == 1) BNS_LAUNCH((KERNEL<bf16_t, 1, 64, 4, false, false>), grid, dim3(256), 0, st, a);                      \
        else if (f32 && plan.group == 4) BNS_QK_CASE(KERNEL, float, 4, 4);                          \
        else if (f32 && plan.group == 8) BNS_QK_CASE(KERNEL, float, 4, 8);                          \
        else if (f32 && plan.group == 16) BNS_QK_CASE(KERNEL, float, 4, 16);                        \
        else if (f32 && plan.group == 32) BNS_QK_CASE(KERNEL, float, 4, 32);                        \
        else if (f32) BNS_QK_CASE(KERNEL, float, 4, 64);                                            \
        else if (plan.group == 4) BNS_QK_CASE(KERNEL, bf16_t, 8, 4);                                \
        else if (plan.group == 8) BNS_QK_CASE(KERNEL, bf16_t, 8, 8);                                \
        else if (plan.group == 16) BNS_QK_CASE(KERNEL, bf16_t, 8, 16);                              \
        else BNS_QK_CASE(KERNEL, bf16_t, 8, 32);                                                    \
    } while (0)

// What both directions take: the weights, positions and frequencies.
bns_status check_common(const bns_qk* qk, const QkDims& d, const void* q_weight, const void* k_weight, const void* positions, const void* frequencies) {
    if (d.rotated > 0 && d.tokens > 0 && (!positions || !frequencies)) return BNS_EINVAL;
    return aligned_all(dtype_bytes(qk->weight_dtype), q_weight, k_weight) && aligned_all(8, positions, frequencies) ? BNS_OK : BNS_EINVAL;
}

}  // namespace

extern "C" {

bns_status bns_qk_forward(const bns_qk* qk, const void* q, const void* k, const void* q_weight, const void* k_weight, const int64_t* positions,
                          const double* frequencies, void* q_out, void* k_out, void* stream) {
    QkDims d;
    bns_status s = check_qk(qk, &d);
    if (s != BNS_OK) return s;
    if (d.tokens == 0 || (d.heads[0] == 0 && d.heads[1] == 0)) return BNS_OK;
    if ((s = check_common(qk, d, q_weight, k_weight, positions, frequencies)) != BNS_OK) return s;
    const void* in[2] = {q, k};
    void* out[2] = {q_out, k_out};
    const void* weight[2] = {q_weight, k_weight};
    const size_t e = dtype_bytes(qk->dtype);
    HeadMatrix mi[2], mo[2];
    for (int i = 0; i < 2; ++i) {
        if (d.heads[i] > 0 && (!in[i] || !out[i])) return BNS_EINVAL;
        mi[i] = head_matrix(in[i], d.tokens, d.heads[i], d.width, d.x[i], e);
        mo[i] = head_matrix(out[i], d.tokens, d.heads[i], d.width, d.out[i], e);
    }
    if (!aligned_all(e, q, k, q_out, k_out)) return BNS_EINVAL;
    if (collide(mo[0], mi[0], true) || collide(mo[1], mi[1], true) || collide(mo[0], mi[1], false) || collide(mo[1], mi[0], false) || collide(mo[0], mo[1], false))
        return BNS_EINVAL;
    QkArgs a{};
    const QkPlan plan = qk_plan(d, qk->dtype, qk->interleaved);
    fill(&a, qk, d, plan, kMostForwardBlocks);
    a.positions = d.rotated > 0 ? positions : nullptr;
    a.frequencies = frequencies;
    for (int i = 0; i < 2; ++i) {
        a.part[i].x = in[i];
        a.part[i].out = out[i];
        a.part[i].weight = weight[i];
        a.part[i].xs = d.x[i];
        a.part[i].os = d.out[i];
    }
    const bool f32 = qk->dtype == BNS_F32, nt = size_t(d.tokens) * (size_t(d.heads[0]) + d.heads[1]) * d.width * e * 2 > kStreamBytes;
    const dim3 grid{uint32_t(a.part[0].blocks + a.part[1].blocks)};
    hipStream_t st = static_cast<hipStream_t>(stream);
    BNS_QK_LAUNCH(qk_forward_kernel);
    return hipGetLastError() == hipSuccess ? BNS_OK : BNS_EDEVICE;
}

size_t bns_qk_workspace_bytes(const bns_qk* qk) {
    QkDims d;
    if (check_qk(qk, &d) != BNS_OK) return 0;
    return size_t(round_up(int64_t(2) * kMostBackwardBlocks * d.width * 4, 256));
}

bns_status bns_qk_backward(const bns_qk* qk, const void* q, const void* k, const void* q_weight, const void* k_weight, const int64_t* positions,
                           const double* frequencies, const void* dq_out, const void* dk_out, void* dq, void* dk, float* dq_weight, float* dk_weight,
                           void* workspace, size_t workspace_bytes, void* stream) {
    QkDims d;
    bns_status s = check_qk(qk, &d);
    if (s != BNS_OK) return s;
    if ((s = check_common(qk, d, q_weight, k_weight, positions, frequencies)) != BNS_OK) return s;
    const void* x[2] = {q, k};
    const void* dy[2] = {dq_out, dk_out};
    void* out[2] = {dq, dk};
    const void* weight[2] = {q_weight, k_weight};
    float* dweight[2] = {dq_weight, dk_weight};
    const size_t e = dtype_bytes(qk->dtype);
    HeadMatrix mx[2], mg[2], mo[2];
    for (int i = 0; i < 2; ++i) {
        if (!weight[i] != !dweight[i]) return BNS_EINVAL;
        if (d.tokens > 0 && d.heads[i] > 0 && (!dy[i] || !out[i] || (weight[i] && !x[i]))) return BNS_EINVAL;
        mx[i] = head_matrix(weight[i] ? x[i] : nullptr, d.tokens, d.heads[i], d.width, d.x[i], e);
        mg[i] = head_matrix(dy[i], d.tokens, d.heads[i], d.width, d.out[i], e);
        mo[i] = head_matrix(out[i], d.tokens, d.heads[i], d.width, d.dx[i], e);
    }
    if (!aligned_all(e, q, k, dq_out, dk_out, dq, dk) || !aligned_all(4, dq_weight, dk_weight)) return BNS_EINVAL;
    if (!workspace || !aligned16(workspace)) return BNS_EINVAL;
    for (int i = 0; i < 2; ++i)
        if (collide(mo[i], mg[i], true) || collide(mo[i], mg[1 - i], false) || collide(mo[i], mx[0], false) || collide(mo[i], mx[1], false)) return BNS_EINVAL;
    if (collide(mo[0], mo[1], false)) return BNS_EINVAL;
    if (workspace_bytes < bns_qk_workspace_bytes(qk)) return BNS_EWORKSPACE;
    QkArgs a{};
    const QkPlan plan = qk_plan(d, qk->dtype, qk->interleaved);
    fill(&a, qk, d, plan, kMostBackwardBlocks);
    a.positions = d.rotated > 0 ? positions : nullptr;
    a.frequencies = frequencies;
    for (int i = 0; i < 2; ++i) {
        a.part[i].x = x[i];
        a.part[i].dy = dy[i];
        a.part[i].out = out[i];
        a.part[i].weight = weight[i];
        a.part[i].partial = static_cast<float*>(workspace) + int64_t(i) * kMostBackwardBlocks * d.width;
        a.part[i].xs = d.x[i];
        a.part[i].ds = d.out[i];
        a.part[i].os = d.dx[i];
    }
    const bool f32 = qk->dtype == BNS_F32, nt = size_t(d.tokens) * (size_t(d.heads[0]) + d.heads[1]) * d.width * e * 3 > kStreamBytes;
    const dim3 grid{uint32_t(a.part[0].blocks + a.part[1].blocks)};
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (grid.x > 0) {
        BNS_QK_LAUNCH(qk_backward_kernel);
        if (hipGetLastError() != hipSuccess) return BNS_EDEVICE;
    }
    if (!dq_weight && !dk_weight) return BNS_OK;
    SumArgs sum{};
    for (int i = 0; i < 2; ++i) {
        sum.partial[i] = a.part[i].partial;
        sum.out[i] = dweight[i];
        sum.count[i] = a.part[i].blocks;
    }
    sum.width = d.width;
    BNS_LAUNCH(qk_weight_sum_kernel, dim3((d.width + kSumColumns - 1) / kSumColumns, 2), dim3(kSumColumns * kSumLanes), 0, st, sum);
    return hipGetLastError() == hipSuccess ? BNS_OK : BNS_EDEVICE;
}

}  // extern "C"
