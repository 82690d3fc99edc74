// Queries and keys: the root-mean-square norm of every head and the rotation by position behind it, forward and backward.  See include/bns.h for the
// equations.
//
// Both read every element once and write once, so HBM bounds them where tokens are many and a launch where they are few.  A head of `width` elements belongs
// to a group of G lanes; a lane holds one unit of it, two chunks of up to 16 bytes that contain both elements of every pair that it rotates (chunks
// rotated / 2 apart, or neighbours), so that the rotation needs no exchange and the sums one of log2 G steps.  The lanes of a wave take hs heads each of
// 64 / (G hs) tokens at a time: a turn.  A wave walks a range of turns, one head group of a token after the other and one token after the other, and asks for the next turn's
// elements before it works on those of this one.  Queries and keys go to different blocks, the queries' first.
//
// Angles: each of the lanes that share a token works out a part of its angles, and all of them get them through LDS.  position * frequency is formed in quarter turns in fp64
// and reduced exactly (the remainder of a fused multiply-add with the nearest whole number); what frequency * 2 / pi loses as a number of 53 bits, times 2^31 as much as fp32
// tells apart, is a second, small factor.  What is left, at most an eighth of a turn, is exact enough in fp32, and Taylor's series to x^9 and x^10 leave 2e-9 there.
//
// Measured: 8192 tokens of (32 + 8) heads of 128, bf16, 37.5 us (168 MB, 4.5 TB/s; a large copy moves 5.1 TB/s), 46 without the next turn's elements on their way; backward of 16 384
// tokens 105 us (503 MB, 4.8 TB/s); a single token 4.4 to 5 us, what one launch takes; a small backward 8.1 us, two launches, of one or two tokens 5 to 6, in one.
// Heads that are no whole chunks: 9109 x (48 + 6) x 83 bf16 44.5 us (164 MB), by single elements 102; backward of 9537 x (23 + 23) x 46, of which 10 turn, 44.9 (121 MB),
// by single elements 198; backward of 2905 x (119 + 17) x 16, of which 4 turn, 16.6, by chunks of two elements 77,
// with four lanes at least for a head 32.5.
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
    int64_t units;      // turns of all tokens
    int32_t run;        // turns that a wave takes one after the other, then as many behind those of all others
    FastDiv turns;      // of a wave over the heads of its tokens
    int32_t heads;
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

constexpr int kThreads = 256, kWaves = kThreads / kWave, kMostWidth = 512;

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
struct Chunk<float, 2> {
    typedef uint32_t u2 __attribute__((ext_vector_type(2)));
    typedef u2 u2e __attribute__((aligned(4)));
    u2 w;
    __device__ __forceinline__ void load(const float* p) { w = *reinterpret_cast<const u2e*>(p); }
    __device__ __forceinline__ void clear() { w = u2{0, 0}; }
    __device__ __forceinline__ void unpack(float (&v)[2]) const { v[0] = __uint_as_float(w.x), v[1] = __uint_as_float(w.y); }
    template <bool NT>
    static __device__ __forceinline__ void store(float* p, const float (&v)[2]) { *reinterpret_cast<u2e*>(p) = u2{__float_as_uint(v[0]), __float_as_uint(v[1])}; }
};
template <>
struct Chunk<bf16_t, 2> {
    typedef uint32_t u1e __attribute__((aligned(2)));
    uint32_t w;
    __device__ __forceinline__ void load(const bf16_t* p) { w = *reinterpret_cast<const u1e*>(p); }
    __device__ __forceinline__ void clear() { w = 0; }
    __device__ __forceinline__ void unpack(float (&v)[2]) const { v[0] = __uint_as_float(w << 16), v[1] = __uint_as_float(w & 0xffff0000u); }
    template <bool NT>
    static __device__ __forceinline__ void store(bf16_t* p, const float (&v)[2]) { *reinterpret_cast<u1e*>(p) = pack_bf16x2(v[0], v[1]); }
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
struct Chunk<bf16_t, 4> {
    typedef uint32_t u2 __attribute__((ext_vector_type(2)));
    typedef u2 u2e __attribute__((aligned(2)));
    u2 w;
    __device__ __forceinline__ void load(const bf16_t* p) { w = *reinterpret_cast<const u2e*>(p); }
    __device__ __forceinline__ void clear() { w = u2{0, 0}; }
    __device__ __forceinline__ void unpack(float (&v)[4]) const {
        v[0] = __uint_as_float(w.x << 16), v[1] = __uint_as_float(w.x & 0xffff0000u);
        v[2] = __uint_as_float(w.y << 16), v[3] = __uint_as_float(w.y & 0xffff0000u);
    }
    template <bool NT>
    static __device__ __forceinline__ void store(bf16_t* p, const float (&v)[4]) { *reinterpret_cast<u2e*>(p) = u2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])}; }
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
    static_assert(G >= 1 && G <= 64, "groups of lanes");
    if (G >= 2) v += dpp_move<0xb1>(v);         // quad_perm: lane ^ 1
    if (G >= 4) v += dpp_move<0x4e>(v);         // quad_perm: lane ^ 2
    if (G >= 8) v += dpp_move<0x141>(v);        // row_half_mirror: the other four of eight
    if (G >= 16) v += dpp_move<0x140>(v);       // row_mirror: the other eight of sixteen
    if (G >= 32) v += __shfl_xor(v, 16);
    if (G >= 64) v += __shfl_xor(v, 32);
    return v;
}

// cos and sin of `position` (`near` in fp32: `less` is 2^-53 of `quarters`, so its product needs no more) times an angle of `quarters` + `less` quarter turns.
__device__ __forceinline__ void turn_by(double position, float near, double quarters, float less, float* c, float* s) {
    const double n = rint(position * quarters);
    const float x = fmaf(near, less, float(fma(position, quarters, -n))) * 1.57079632679489662f;      // |x| <= pi / 4
    const int quadrant = int(fma(-4.0, rint(n * 0.25), n));                        // -2 .. 2
    const float x2 = x * x;
    const float sine = x * fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), 1.f);
    const float cosine = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
    const bool odd = quadrant & 1;
    const float a = odd ? sine : cosine, b = odd ? cosine : sine;
    *c = (quadrant + 1) & 2 ? -a : a;       // 1, 2, -2 (as 2): negative; -1 gives 0 & 2
    *s = quadrant & 2 ? -b : b;             // 2, -2, -1 (as 3): negative
}

// What a lane holds of a head, the same for every head.  RAGGED: what is rotated (its halves; all of it, for neighbours) and the rest need not be whole chunks.  The last chunk
// of each begins further down, so that it ends where they do, and its first elements are another lane's too: both work them out and write the same, one counts them.
// Where that is not so, a rest shorter than a chunk that begins among the rotated elements, it writes its own only.  Neighbours' last chunk goes on into the rest instead, where the
// head is long enough.  INNER: halves that lie in one chunk together are rotated there.
enum Form { WHOLE = 0, RAGGED = 1, INNER = 2 };
template <typename T, int E, int G, int UPL, bool NEIGHBOURS, int FORM>
struct Lane {
    static constexpr bool kOverlap = FORM != WHOLE, kInner = FORM == INNER;
    int at[UPL][2];             // first elements of its chunks; -1: none
    int own[UPL][2];            // from which one on they count
    bool turned[UPL][2];
    bool alone;                 // the last chunk writes its own elements only

    // Chunk q of what lies behind `begin` and is not rotated.
    __device__ __forceinline__ void set_rest(const QkArgs& a, int k, int c, int q, int begin) {
        const int from = begin + q * E;
        at[k][c] = from >= a.width ? -1 : !kOverlap ? from : min(from, a.width - E);
        own[k][c] = kOverlap ? from - at[k][c] : 0;
        turned[k][c] = false;
    }
    __device__ __forceinline__ void set(const QkArgs& a, int l) {
        const int half = a.rotated / 2;
        const int chunks = kInner ? 0 : ((NEIGHBOURS ? a.rotated : half) + E - 1) / E;       // that are rotated (halves: each)
        int begin = kInner ? 0 : a.rotated;
        if (kOverlap && NEIGHBOURS && chunks * E <= a.width) begin = chunks * E;
        alone = kOverlap && a.width - E < a.rotated && (a.width - begin) % E != 0;
#pragma unroll
        for (int k = 0; k < UPL; ++k) {
            const int u = k * G + l;
            if (NEIGHBOURS) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int j = 2 * u + c;
                    if (j < chunks) {
                        at[k][c] = kOverlap ? min(j * E, begin - E) : j * E;
                        own[k][c] = j * E - at[k][c];
                        turned[k][c] = true;
                    } else {
                        set_rest(a, k, c, j - chunks, begin);
                    }
                }
            } else if (u < chunks) {
                const int o = kOverlap ? min(u * E, half - E) : u * E;
                at[k][0] = o;
                at[k][1] = half + o;
                own[k][0] = own[k][1] = u * E - o;
                turned[k][0] = turned[k][1] = true;
            } else {
                set_rest(a, k, 0, 2 * (u - chunks), begin);
                set_rest(a, k, 1, 2 * (u - chunks) + 1, begin);
            }
        }
        if (kInner && l == 0) turned[0][0] = true;
    }
    // Whether element i of a chunk counts here.
    __device__ __forceinline__ bool counts(int k, int c, int i) const { return !kOverlap || i >= own[k][c]; }
    // Whether a chunk may be written as a whole.
    __device__ __forceinline__ bool whole(const QkArgs& a, int k, int c) const { return !(alone && !turned[k][c] && at[k][c] < a.rotated); }
    // Place of the first angle of chunk c (0, or halves) among a token's angles (0 where it is not turned).
    __device__ __forceinline__ int angle(const QkArgs& a, int k, int c) const { return !turned[k][c] ? 0 : NEIGHBOURS ? at[k][c] / 2 : at[k][c]; }
    // Its elements' weights (0 for a chunk that is not there, behind the last one).
    __device__ __forceinline__ void weights(float (&w)[UPL][2][E], const float* weight) const {
#pragma unroll
        for (int k = 0; k < UPL; ++k)
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int i = 0; i < E; ++i) w[k][c][i] = weight[(at[k][c] < 0 ? kMostWidth : at[k][c]) + i];
    }
    // Elements from a turn's base to the lane's chunks.
    struct Offsets {
        int64_t to[UPL][2];
    };
    __device__ __forceinline__ Offsets offsets(int64_t of_lane) const {
        Offsets o;
#pragma unroll
        for (int k = 0; k < UPL; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) o.to[k][i] = of_lane + at[k][i];
        return o;
    }
    __device__ __forceinline__ void load(Chunk<T, E> (&c)[UPL][2], const T* base, const Offsets& o) const {
#pragma unroll
        for (int k = 0; k < UPL; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (at[k][i] >= 0) c[k][i].load(base + o.to[k][i]);
                else c[k][i].clear();
            }
    }
    template <bool NT>
    __device__ __forceinline__ void store(const QkArgs& a, T* base, const Offsets& o, const float (&v)[UPL][2][E]) const {
#pragma unroll
        for (int k = 0; k < UPL; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (at[k][i] >= 0 && whole(a, k, i)) Chunk<T, E>::template store<NT>(base + o.to[k][i], v[k][i]);
        if (!alone) return;
#pragma unroll
        for (int k = 0; k < UPL; ++k)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                if (at[k][c] < 0 || whole(a, k, c)) continue;
#pragma unroll
                for (int i = 0; i < E; ++i)
                    if (i >= own[k][c]) Vec<T, 1>{{v[k][c][i]}}.store(base + o.to[k][c] + i);
            }
    }
    // Whether every chunk is turned.  (A chunk that is not there has no angles: behind those of the head lies what an earlier kernel left, NaN perhaps.)
    static __device__ __forceinline__ bool all_turned(const QkArgs& a) { return !kOverlap && a.rotated == a.width && !(NEIGHBOURS && a.width % (2 * E)); }
    // BACK: by the negative angle.  `all`: every chunk is turned.
    template <bool BACK>
    __device__ __forceinline__ void rotate(const QkArgs& a, float (&v)[UPL][2][E], const float (&cs)[UPL][E], const float (&sn)[UPL][E], bool all) const {
        const auto turn = [](float& x, float& y, float c, float s, bool here) {
            s = BACK ? -s : s;
            const float xr = fmaf(x, c, -(y * s)), yr = fmaf(x, s, y * c);
            x = here ? xr : x;
            y = here ? yr : y;
        };
        if constexpr (kInner) {     // (the first chunk's pairs: i and i + half)
            const auto turn_all = [&](auto half) {
#pragma unroll
                for (int i = 0; i < half.value; ++i) turn(v[0][0][i], v[0][0][i + half.value], cs[0][i], sn[0][i], turned[0][0]);
            };
            if (a.rotated == 2) turn_all(std::integral_constant<int, 1>());
            if constexpr (E >= 4) {
                if (a.rotated == 4) turn_all(std::integral_constant<int, 2>());
            }
            if constexpr (E >= 8) {
                if (a.rotated == 6) turn_all(std::integral_constant<int, 3>());
                if (a.rotated == 8) turn_all(std::integral_constant<int, 4>());
            }
            return;
        }
#pragma unroll
        for (int k = 0; k < UPL; ++k)
#pragma unroll
            for (int i = 0; i < E; ++i) {
                constexpr int H = E / 2 > 0 ? E / 2 : 1;
                const int c = NEIGHBOURS ? i / H : 0, j = NEIGHBOURS ? i % H : i;
                const bool here = all || (turned[k][c] && (!(kOverlap && NEIGHBOURS) || at[k][c] + 2 * j < a.rotated));
                if (NEIGHBOURS) turn(v[k][c][2 * j], v[k][c][2 * j + 1], cs[k][i], sn[k][i], here);
                else turn(v[k][0][i], v[k][1][i], cs[k][i], sn[k][i], here);
            }
    }
};

// What stays in LDS, as registers decide how many waves there are: the weight, angles in quarter turns by position, and cos and sin of those of the tokens that
// a wave works on.
template <int E, int UPL>
struct Angles {
    alignas(16) float cosine[kWaves][kWave * E * UPL], sine[kWaves][kWave * E * UPL];
    alignas(16) float weight[kMostWidth + 8];
    struct alignas(16) {
        double quarters;
        float less;         // what is left of them
    } angle[kMostWidth / 2];
};

// The walk of a wave over its turns: runs of neighbouring ones, so that all waves work in one stretch of memory.
template <typename T, int E, int G, int UPL, bool NEIGHBOURS>
struct Walk {
    const QkArgs& a;
    const Heads& p;
    Angles<E, UPL>& angles;
    int lane, wave, block;
    int hs, tokens_at_once, sharing;        // sharing: lanes of a token
    int64_t unit, skip, group;              // skip: from the end of a run to the next one
    int turn, left;                         // left: turns of the run
    bool there;                             // whether this lane has a head in this turn
    int64_t position;                       // of the next group of tokens, asked for early (as it is: a conversion would wait for it)

    __device__ __forceinline__ Walk(const QkArgs& args, Angles<E, UPL>& lds)
        : a(args), p(args.part[int(blockIdx.x) >= args.part[0].blocks]), angles(lds) {
        lane = threadIdx.x % kWave;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        block = int(blockIdx.x) - (int(blockIdx.x) >= a.part[0].blocks ? a.part[0].blocks : 0);
        hs = 1 << p.log_hs;
        tokens_at_once = (kWave / G) >> p.log_hs;
        sharing = G << p.log_hs;
        const int64_t waves = int64_t(p.blocks) * kWaves;
        unit = (int64_t(block) * kWaves + wave) * p.run;
        skip = (waves - 1) * p.run;
        left = p.run;
        group = group_of(unit);
        turn = int(unit - group * p.turns.d);
        for (int i = threadIdx.x; i < a.rotated / 2; i += kThreads) {
            constexpr double kUpper = 0.63661977236758138, kLower = -3.9357353350364971e-17;        // 2 / pi
            const double f = a.frequencies[i], quarters = f * kUpper;
            angles.angle[i].quarters = quarters;
            angles.angle[i].less = float(fma(f, kLower, fma(f, kUpper, -quarters)));
        }
        if (p.weight) {
            for (int i = threadIdx.x; i < a.width; i += kThreads)
                angles.weight[i] = a.weight_bf16 ? load_scalar<bf16_t>(static_cast<const bf16_t*>(p.weight) + i) : static_cast<const float*>(p.weight)[i];
            if (threadIdx.x < 8) angles.weight[kMostWidth + threadIdx.x] = 0.f;
        }
        __syncthreads();
        ask_position(group);
        look();
    }
    __device__ __forceinline__ int64_t group_of(int64_t u) const { return u < (int64_t(1) << 31) ? int64_t(fdiv(uint32_t(u), p.turns)) : u / p.turns.d; }
    __device__ __forceinline__ bool more() const { return unit < p.units; }
    __device__ __forceinline__ void look() {
        const int tokens_left = int(max(int64_t(0), min(a.tokens - group * tokens_at_once, int64_t(kWave))));
        there = more() && lane / sharing < tokens_left && turn * hs + lane / G % hs < p.heads;
    }
    // Where the lane's head lies: the same for all lanes, and what the lane adds to that in every turn.
    __device__ __forceinline__ int64_t base(const HeadStrides& s) const { return group * (tokens_at_once * s.token) + turn * (hs * s.head); }
    __device__ __forceinline__ int64_t of_lane(const HeadStrides& s) const { return lane / sharing * s.token + lane / G % hs * s.head; }
    __device__ __forceinline__ void ask_position(int64_t g) {
        const int64_t t = g * tokens_at_once + lane / sharing;
        position = 0;
        if (a.rotated > 0 && t < a.tokens) position = a.positions[t];
    }
    __device__ __forceinline__ void next() {
        ++unit;
        if (--left == 0) {
            unit += skip;
            left = p.run;
            group = group_of(unit);
            turn = int(unit - group * p.turns.d);
        } else if (++turn == int(p.turns.d)) {
            turn = 0;
            ++group;
        }
        look();
    }
    // The angles of the group whose position was asked for; asks for the next one's.
    __device__ __forceinline__ void work_out() {
        const int each = a.rotated / 2, base = lane / sharing * each;
        float *c = angles.cosine[wave], *s = angles.sine[wave];
        const double here = double(position);
        const float near = float(here);
        asm volatile("" ::: "memory");      // (a wave's accesses to LDS are in order)
        for (int i = lane % sharing; i < each; i += sharing) {
            const auto angle = angles.angle[i];
            turn_by(here, near, angle.quarters, angle.less, c + base + i, s + base + i);
        }
        asm volatile("" ::: "memory");
        ask_position(left > int(p.turns.d) - turn ? group + 1 : group_of(unit + left + skip));
    }
    template <typename Lane>
    __device__ __forceinline__ void get(float (&cs)[UPL][E], float (&sn)[UPL][E], const Lane& mine) const {
        const int base = lane / sharing * (a.rotated / 2);
        const float *c = angles.cosine[wave], *s = angles.sine[wave];
#pragma unroll
        for (int k = 0; k < UPL; ++k) {
            // (chunks that are not turned read the first angles and use none)
            const int first = base + mine.angle(a, k, 0), second = NEIGHBOURS ? base + mine.angle(a, k, 1) - E / 2 : first;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const int from = NEIGHBOURS && i >= E / 2 ? second : first;
                cs[k][i] = c[from + i];
                sn[k][i] = s[from + i];
            }
        }
    }
};

template <typename T, int E, int G, int UPL, bool NEIGHBOURS, int FORM, bool NT>
__global__ void __launch_bounds__(kThreads) qk_forward_kernel(QkArgs a) {
    __shared__ Angles<E, UPL> angles;
    Walk<T, E, G, UPL, NEIGHBOURS> at(a, angles);
    const Heads& p = at.p;
    Lane<T, E, G, UPL, NEIGHBOURS, FORM> mine;
    Chunk<T, E> next[UPL][2];
    mine.set(a, at.lane % G);
    const auto x_to = mine.offsets(at.of_lane(p.xs)), out_to = mine.offsets(at.of_lane(p.os));
    const auto ask = [&]() {
        if (at.there) mine.load(next, static_cast<const T*>(p.x) + at.base(p.xs), x_to);
    };
    ask();
    const bool all = mine.all_turned(a);
    int64_t group = -1;
    while (at.more()) {
        if (a.rotated > 0 && at.group != group) at.work_out();
        group = at.group;
        float v[UPL][2][E];
#pragma unroll
        for (int k = 0; k < UPL; ++k)
#pragma unroll
            for (int c = 0; c < 2; ++c) next[k][c].unpack(v[k][c]);
        T* out = static_cast<T*>(p.out) + at.base(p.os);
        const bool there = at.there;
        at.next();
        ask();
        asm volatile("" ::: "memory");      // (nothing from LDS is kept in registers from turn to turn)
        if (!there) continue;
        if (p.weight) {
            float squares = 0.f, w[UPL][2][E];
            mine.weights(w, angles.weight);
#pragma unroll
            for (int k = 0; k < UPL; ++k)
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int i = 0; i < E; ++i) {
                        const float x = mine.counts(k, c, i) ? v[k][c][i] : 0.f;
                        squares = fmaf(x, x, squares);
                    }
            const float rstd = rsqrtf(fmaf(group_sum<G>(squares), a.inv_width, a.eps));
#pragma unroll
            for (int k = 0; k < UPL; ++k)
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int i = 0; i < E; ++i) v[k][c][i] *= rstd * w[k][c][i];
        }
        if (a.rotated > 0) {
            float cs[UPL][E], sn[UPL][E];
            at.get(cs, sn, mine);
            mine.template rotate<false>(a, v, cs, sn, all);
        }
        mine.template store<NT>(a, out, out_to, v);
    }
}

template <typename T, int E, int G, int UPL, bool NEIGHBOURS, int FORM, bool NT>
__global__ void __launch_bounds__(kThreads, UPL == 1 ? 4 : 1) qk_backward_kernel(QkArgs a) {       // (four waves a SIMD: 128 registers)
    __shared__ union {
        Angles<E, UPL> angles;
        float sums[UPL * 2 * E][kThreads];
    } lds;
    Walk<T, E, G, UPL, NEIGHBOURS> at(a, lds.angles);
    const Heads& p = at.p;
    Lane<T, E, G, UPL, NEIGHBOURS, FORM> mine;
    Chunk<T, E> next_x[UPL][2], next_g[UPL][2];
    mine.set(a, at.lane % G);
    const auto x_to = mine.offsets(at.of_lane(p.xs)), dy_to = mine.offsets(at.of_lane(p.ds)), out_to = mine.offsets(at.of_lane(p.os));
    const auto ask = [&]() {
        if (!at.there) return;
        mine.load(next_g, static_cast<const T*>(p.dy) + at.base(p.ds), dy_to);
        if (p.weight) mine.load(next_x, static_cast<const T*>(p.x) + at.base(p.xs), x_to);
    };
    ask();
    const bool all = mine.all_turned(a);
    float dw[UPL][2][E];
#pragma unroll
    for (int k = 0; k < UPL; ++k)
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < E; ++i) dw[k][c][i] = 0.f;
    int64_t group = -1;
    while (at.more()) {
        if (a.rotated > 0 && at.group != group) at.work_out();
        group = at.group;
        float g[UPL][2][E], v[UPL][2][E];
#pragma unroll
        for (int k = 0; k < UPL; ++k)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                next_g[k][c].unpack(g[k][c]);
                if (p.weight) next_x[k][c].unpack(v[k][c]);
            }
        T* out = static_cast<T*>(p.out) + at.base(p.os);
        const bool there = at.there;
        at.next();
        ask();
        asm volatile("" ::: "memory");      // (nothing from LDS is kept in registers from turn to turn)
        if (!there) continue;
        if (a.rotated > 0) {
            float cs[UPL][E], sn[UPL][E];
            at.get(cs, sn, mine);
            mine.template rotate<true>(a, g, cs, sn, all);
        }
        if (p.weight) {
            float squares = 0.f, dot = 0.f, w[UPL][2][E];
            mine.weights(w, lds.angles.weight);
#pragma unroll
            for (int k = 0; k < UPL; ++k)
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int i = 0; i < E; ++i) {
                        const float x = mine.counts(k, c, i) ? v[k][c][i] : 0.f;
                        squares = fmaf(x, x, squares);
                        dot = fmaf(mine.counts(k, c, i) ? g[k][c][i] * w[k][c][i] : 0.f, x, dot);
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
                        g[k][c][i] = rstd * fmaf(g[k][c][i], w[k][c][i], -xh * mean);
                    }
        }
        mine.template store<NT>(a, out, out_to, g);
    }
    if (!p.weight) return;
    // The block's sums: the lanes that hold the same elements, in their order; in fp64 and rounded once, as those of the blocks are.  (A lane's own terms, one for each of its turns, are added in fp32.)
    constexpr int kSlots = kThreads / G;
    __syncthreads();        // (the angles are no longer needed)
#pragma unroll
    for (int k = 0; k < UPL; ++k)
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < E; ++i) lds.sums[(k * 2 + c) * E + i][threadIdx.x] = dw[k][c][i];
    __syncthreads();
    float* partial = p.partial + int64_t(at.block) * a.width;
    // (element r of lane l: written by that lane's place among the first G threads of its parts, which knows where it goes; threads beyond one for each element take parts of
    // the sum: 15425 x (32 + 8) x 16 bf16 20.2 us, by one 22.3)
    constexpr int kElements = UPL * 2 * E, kParts = kElements * G < kThreads ? kThreads / (kElements * G) : 1;
    static_assert(kParts * G <= kWave && kParts <= kSlots, "the parts of a sum lie in a wave");
    for (int r = threadIdx.x / (G * kParts); r < kElements; r += kThreads / (G * kParts)) {
        const int l = threadIdx.x % G, part = threadIdx.x / G % kParts;
        double s = 0.0;
#pragma unroll 16
        for (int j = 0; j < kSlots / kParts; ++j) s += double(lds.sums[r][(j * kParts + part) * G + l]);
#pragma unroll
        for (int o = G; o < G * kParts; o *= 2) s += __shfl_xor(s, o);
        const int k = r / (2 * E), c = r / E % 2, i = r % E;
        int place = -1, own = 0;
#pragma unroll
        for (int kk = 0; kk < UPL; ++kk)
#pragma unroll
            for (int cc = 0; cc < 2; ++cc)
                if (kk == k && cc == c) place = mine.at[kk][cc], own = mine.own[kk][cc];
        if (part == 0 && place >= 0 && i >= own) partial[place + i] = float(s);
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
    __shared__ double lds[kSumLanes][kSumColumns];
    const int which = blockIdx.y;
    if (!a.out[which]) return;
    const float* partial = a.partial[which];
    const int c = threadIdx.x % kSumColumns, l = threadIdx.x / kSumColumns, col = blockIdx.x * kSumColumns + c;
    double s = 0.0;
    if (col < a.width) {
#pragma unroll 16
        for (int i = l; i < a.count[which]; i += kSumLanes) s += double(partial[int64_t(i) * a.width + col]);
    }
    lds[l][c] = s;
    __syncthreads();
    if (l == 0 && col < a.width) {
        for (int i = 1; i < kSumLanes; ++i) s += lds[i][c];
        a.out[which][col] = float(s);
    }
}

// How a head lies in lanes: chunks of 16 bytes, RAGGED where what is rotated and the rest are not whole ones; of fewer elements where halves are shorter and too long to
// lie in one together, and where ragged heads would need more lanes than there are.
struct QkPlan {
    int chunk, group, form;
};
QkPlan qk_plan(const QkDims& d, int32_t dtype, bool interleaved) {
    const int half = d.rotated / 2, largest = dtype == BNS_F32 ? 4 : 8;
    for (int e = largest; e > 1; e /= 2) {
        const bool inner = !interleaved && d.rotated > 0 && d.rotated <= e;
        if (d.width < e || (!interleaved && !inner && d.rotated > 0 && half < e)) continue;
        const int turned = inner ? 0 : ((interleaved ? d.rotated : half) + e - 1) / e;
        const int begin = inner ? 0 : interleaved && turned * e <= d.width ? turned * e : d.rotated, others = (d.width - begin + e - 1) / e;
        const int units = interleaved ? (turned + others + 1) / 2 : turned + (others + 1) / 2;
        if (units > kWave * (e == 2 ? 2 : 1)) continue;
        if (e < largest) return {e, e == 4 && units <= 8 ? 8 : units <= (e == 2 ? 32 : 16) ? 16 : 64, inner ? INNER : RAGGED};
        int g = 1;
        while (g < units) g *= 2;
        return {e, g, inner ? INNER : d.width % e != 0 || d.rotated % (interleaved ? e : 2 * e) != 0 ? RAGGED : WHOLE};
    }
    return {1, (d.width + 1) / 2 <= 64 ? 16 : 64, WHOLE};
}

// Blocks of the queries and of the keys, each.  (us: forward, 16384 x (32 + 8) x 128 bf16, 512 blocks 68.5, 1024 65.1, 2048 64.3; backward 384 112, 448 111, 512 106, 768 108.)
constexpr int kMostForwardBlocks = 2048, kMostBackwardBlocks = 512;
// Turns that make a wave worth its beginning, where that leaves enough waves (2048 x (32 + 8) x 128 bf16 forward, a turn a wave 11.5 us, two 9.7).
constexpr int64_t kTurnsOfWave = 2, kEnoughTurns = 4096;

// Backward: turns of a tensor that one block takes, so that there are no other blocks' sums to add and no second launch: two a wave.  (us, in one launch against two: (32 + 8) x 128
// bf16, 1 token 4.9 against 8.2, 2 tokens, 8 turns, 6.0 against 9.4, 4 tokens 8.4 against 8.3, 8 tokens 13.5 against 9.2; (4 + 4) x 16, 32 tokens, 8 turns, 7.0 against 8.8.)
constexpr int64_t kTurnsAtOnce = 2 * kWaves;

// Shares the turns of a tensor out over at most `most` blocks.
void share_out(Heads* p, const QkPlan& plan, int64_t tokens, int heads, int most) {
    const int slots = kWave / plan.group;
    p->heads = heads;
    p->log_hs = 0;
    while ((1 << p->log_hs) < heads && (2 << p->log_hs) <= slots) ++p->log_hs;
    const int hs = 1 << p->log_hs, tokens_at_once = slots / hs, turns = std::max(1, (heads + hs - 1) / hs);
    p->turns = make_fastdiv(uint32_t(turns));
    p->units = heads > 0 ? (tokens + tokens_at_once - 1) / tokens_at_once * int64_t(turns) : 0;
    // Runs: all turns of a token, so that its angles are worked out once, unless tokens are few.
    const int64_t waves = int64_t(most) * kWaves, whole = turns * ((kTurnsOfWave + turns - 1) / turns);
    p->run = int32_t(std::min(whole, std::max<int64_t>((p->units + waves - 1) / waves, p->units >= kEnoughTurns ? kTurnsOfWave : 1)));
    const int64_t of_block = int64_t(p->run) * kWaves;
    p->blocks = int32_t(std::min<int64_t>((p->units + of_block - 1) / of_block, most));
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

#define BNS_QK_ONE(KERNEL, T, E, G, UPL, NB, FORM, NT) BNS_LAUNCH((KERNEL<T, E, G, UPL, NB, FORM, NT>), grid, dim3(kThreads), 0, st, a)
// Chunks of 16 bytes, E of the largest.
#define BNS_QK_CASE(KERNEL, T, E, G)                                                                                            \
    do {                                                                                                                        \
        if (plan.group != G) break;                                                                                             \
        if (plan.form == INNER) BNS_QK_ONE(KERNEL, T, E, G, 1, false, INNER, false);                                            \
        else if (plan.form == RAGGED && a.interleaved) BNS_QK_ONE(KERNEL, T, E, G, 1, true, RAGGED, false);                     \
        else if (plan.form == RAGGED) BNS_QK_ONE(KERNEL, T, E, G, 1, false, RAGGED, false);                                     \
        else if (a.interleaved && nt) BNS_QK_ONE(KERNEL, T, E, G, 1, true, WHOLE, true);                                        \
        else if (a.interleaved) BNS_QK_ONE(KERNEL, T, E, G, 1, true, WHOLE, false);                                             \
        else if (nt) BNS_QK_ONE(KERNEL, T, E, G, 1, false, WHOLE, true);                                                        \
        else BNS_QK_ONE(KERNEL, T, E, G, 1, false, WHOLE, false);                                                               \
    } while (0)
// One kernel, if the plan is its.
#define BNS_QK_IF(KERNEL, T, E, G, UPL, NB, FORM)                                                                               \
    do {                                                                                                                        \
        if (plan.chunk == E && plan.group == G && plan.form == FORM && (NB == bool(a.interleaved) || E == 1))                   \
            BNS_QK_ONE(KERNEL, T, E, G, UPL, NB, FORM, false);                                                                  \
    } while (0)
#define BNS_QK_SMALL(KERNEL, T)                                                                                                 \
    do {                                                                                                                        \
        BNS_QK_IF(KERNEL, T, 2, 16, 2, false, RAGGED);                                                                          \
        BNS_QK_IF(KERNEL, T, 2, 64, 2, false, RAGGED);                                                                          \
        BNS_QK_IF(KERNEL, T, 2, 16, 2, true, RAGGED);                                                                           \
        BNS_QK_IF(KERNEL, T, 2, 16, 2, false, INNER);                                                                           \
        BNS_QK_IF(KERNEL, T, 1, 16, 4, false, WHOLE);                                                                           \
        BNS_QK_IF(KERNEL, T, 1, 64, 4, false, WHOLE);                                                                           \
    } while (0)
#define BNS_QK_LAUNCH(KERNEL)                                                                                                   \
    do {                                                                                                                        \
        if (plan.chunk <= 2 && f32) {                                                                                           \
            BNS_QK_SMALL(KERNEL, float);                                                                                        \
            BNS_QK_IF(KERNEL, float, 2, 64, 2, true, RAGGED);                                                                   \
        } else if (plan.chunk <= 2) {                                                                                           \
            BNS_QK_SMALL(KERNEL, bf16_t);                                                                                       \
        } else if (f32) {                                                                                                       \
            BNS_QK_CASE(KERNEL, float, 4, 1);                                                                                   \
            BNS_QK_CASE(KERNEL, float, 4, 2);                                                                                   \
            BNS_QK_CASE(KERNEL, float, 4, 4);                                                                                   \
            BNS_QK_CASE(KERNEL, float, 4, 8);                                                                                   \
            BNS_QK_CASE(KERNEL, float, 4, 16);                                                                                  \
            BNS_QK_CASE(KERNEL, float, 4, 32);                                                                                  \
            BNS_QK_CASE(KERNEL, float, 4, 64);                                                                                  \
        } else if (plan.chunk == 4) {                                                                                           \
            BNS_QK_IF(KERNEL, bf16_t, 4, 8, 1, false, RAGGED);                                                                  \
            BNS_QK_IF(KERNEL, bf16_t, 4, 16, 1, false, RAGGED);                                                                 \
            BNS_QK_IF(KERNEL, bf16_t, 4, 64, 1, false, RAGGED);                                                                 \
            BNS_QK_IF(KERNEL, bf16_t, 4, 8, 1, true, RAGGED);                                                                   \
            BNS_QK_IF(KERNEL, bf16_t, 4, 8, 1, false, INNER);                                                                   \
        } else {                                                                                                                \
            BNS_QK_CASE(KERNEL, bf16_t, 8, 1);                                                                                  \
            BNS_QK_CASE(KERNEL, bf16_t, 8, 2);                                                                                  \
            BNS_QK_CASE(KERNEL, bf16_t, 8, 4);                                                                                  \
            BNS_QK_CASE(KERNEL, bf16_t, 8, 8);                                                                                  \
            BNS_QK_CASE(KERNEL, bf16_t, 8, 16);                                                                                 \
            BNS_QK_CASE(KERNEL, bf16_t, 8, 32);                                                                                 \
            BNS_QK_IF(KERNEL, bf16_t, 8, 64, 1, false, RAGGED);                                                                 \
            BNS_QK_IF(KERNEL, bf16_t, 8, 64, 1, true, RAGGED);                                                                  \
        }                                                                                                                       \
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
    if (dq_weight && dk_weight && dq_weight < dk_weight + d.width && dk_weight < dq_weight + d.width) return BNS_EINVAL;
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
    // (without tokens there is nothing but the sums, of no rows: positions and frequencies may be NULL then and are not read)
    const bool at_once = d.tokens > 0 && std::max(a.part[0].units, a.part[1].units) <= kTurnsAtOnce;
    if (at_once) {
        for (int i = 0; i < 2; ++i) {
            Heads& p = a.part[i];
            if (!dweight[i]) continue;
            p.run = std::max(1, int(p.units + kWaves - 1) / kWaves);
            p.blocks = 1;           // (of no heads, too: its sums are zero)
            p.partial = dweight[i];
        }
    }
    const dim3 grid{uint32_t(a.part[0].blocks + a.part[1].blocks)};
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (grid.x > 0) {
        BNS_QK_LAUNCH(qk_backward_kernel);
        if (hipGetLastError() != hipSuccess) return BNS_EDEVICE;
    }
    if (at_once || (!dq_weight && !dk_weight)) return BNS_OK;
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
