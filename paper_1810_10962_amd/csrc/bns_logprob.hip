// Log probabilities of given tokens, entropy and the most probable alternatives from rows of logits, and their gradient.  See include/bns.h for the
// equations.
//
// Both passes read every logit once (backward writes as much), so HBM bounds them; beside it the forward pass has an exponential and ten more
// operations for each.  Forward: a thread keeps, over all chunks of its row that go by, the largest logit m, l = sum exp((x - m) / tau) and
// d = sum exp((x - m) / tau) (x - m), which are moved to a new m when a chunk has a larger one, so that a row needs one pass and few registers, and other
// blocks' loads go on while it is worked on.  entropy = log l - d / (l tau) has two terms of one sign.
//
// Alternatives: what a thread has as its largest logit so far bounds the k-th largest of the row from below, if enough threads have such a one: the j-th largest of
// each wave's 64, j = ceil(k / waves), the least of all waves' taken.  The first chunk sets that bound, larger parts of the row raise it, and what reaches it goes to a
// list, some 2 k elements of each doubling of what was seen; in the end a few times k are left, whose places come from counting the larger ones.  Rows that
// put more on the list than it holds (rising logits, many equal ones) are searched by halving the range of values instead.
//
// Few rows are cut into segments, one block each, and joined by a second launch.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "bns_internal.hpp"
#include "bns_lm_words.hpp"
#include "bns_step_validate.hpp"

using namespace bns;

namespace {

constexpr int kList = 2048;             // entries of a block's list
constexpr int kMostSegments = 64;

struct LogprobArgs {
    const void* logits;
    const int64_t* targets;
    float *logp, *entropy, *stats;
    int64_t* top_ids;
    float* top_logp;
    float4* parts;                      // [rows][segments] {m, l, d, -}
    uint64_t* candidates;               // [rows][segments][top], falling, 0 behind the last
    int64_t tokens, stride;
    int32_t vocab, top, segments, segment;      // segment: elements, a multiple of 8
    float tau;
};

struct LogprobBackwardArgs {
    const void* logits;
    const int64_t* targets;
    const float *stats, *entropy, *dlogp, *dentropy;
    void* dlogits;
    int64_t tokens, stride, dstride;
    int32_t vocab, segments, segment;
    float tau;
};

// A logit above -infinity and its place as one number: larger logits first, then lower indices; never 0.
__device__ __forceinline__ uint64_t rank_of(float x, int index) {
    const uint32_t b = __float_as_uint(x + 0.f);        // (one zero)
    return uint64_t(b >> 31 ? ~b : b | 0x80000000u) << 32 | uint32_t(~index);
}
__device__ __forceinline__ float logit_of(uint64_t r) {
    const uint32_t k = uint32_t(r >> 32);
    return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k);
}
__device__ __forceinline__ int index_of(uint64_t r) { return int(~uint32_t(r)); }

// The j-th largest of the 64 lanes' values, equal ones counted as often as they come.
__device__ __forceinline__ float wave_jth(float v, int j) {
    const int lane = threadIdx.x % kWave;
    float most = wave_max(v);
    for (int i = 1; i < j; ++i) {
        const uint64_t who = __ballot(v == most);
        if (who == 0) break;                            // (only NaN left)
        if (lane == __builtin_ctzll(who)) v = -__builtin_inff();
        most = wave_max(v);
    }
    return most;
}

// What a block knows of the alternatives.
struct Top {
    uint64_t list[kList];
    uint64_t best[kList];
    float bound[1024 / kWave];
    int count, left;
};

// Sum over the block (all threads), in `scratch` of a word per wave.
template <int THREADS>
__device__ __forceinline__ int block_count(int n, int* scratch) {
    constexpr int kWaves = THREADS / kWave;
#pragma unroll
    for (int o = 1; o < kWave; o *= 2) n += __shfl_xor(n, o);
    __syncthreads();
    if (threadIdx.x % kWave == 0) scratch[threadIdx.x / kWave] = n;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) all += scratch[i];
    return all;
}

// Exact search of the elements [v0, v1) of a row for its k largest, with as many passes over them as it takes: leaves at most kList entries in top.list that
// hold the k largest, top.count of them.  `most`: the largest one (finite or infinite, not NaN).
template <typename T, int THREADS>
__device__ void search(Top& top, int* scratch, const T* z, int v0, int v1, int k, float most) {
    const auto key = [](float x) { return uint32_t(rank_of(x, 0) >> 32); };
    const uint32_t none = key(-__builtin_inff());       // keys of interest lie above
    const auto count_from = [&](uint32_t at_least) {
        int n = 0;
        for (int v = v0 + int(threadIdx.x); v < v1; v += THREADS) {
            const float x = load_scalar<T>(z + v);
            n += x > -__builtin_inff() && key(x) >= at_least;
        }
        return block_count<THREADS>(n, scratch);
    };
    // lo: at least k elements reach it (or it is the least of all keys); hi: fewer do
    uint32_t lo = none + 1, hi = key(most) + 1;
    bool fits = false;
    int above = 0;                                      // elements that reach hi
    while (hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        const int n = count_from(mid);
        if (n >= k) {
            lo = mid;
            if (n <= kList) {
                fits = true;
                break;
            }
        } else {
            hi = mid;
            above = n;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) top.count = 0;
    __syncthreads();
    const uint32_t from = fits ? lo : hi;
    for (int v = v0 + int(threadIdx.x); v < v1; v += THREADS) {
        const float x = load_scalar<T>(z + v);
        if (x > -__builtin_inff() && key(x) >= from) {
            const int at = atomicAdd(&top.count, 1);
            if (at < kList) top.list[at] = rank_of(x, v);
        }
    }
    __syncthreads();
    if (fits) return;
    // More elements have the key lo than there is room for: the first of them by index, as many as are needed.
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    int have = above;
    for (int v = v0; v < v1 && have < k; v += THREADS) {
        const int at = v + int(threadIdx.x);
        const float x = at < v1 ? load_scalar<T>(z + at) : 0.f;
        const bool mine = at < v1 && x > -__builtin_inff() && key(x) == lo;
        const uint64_t who = __ballot(mine);
        __syncthreads();
        if (lane == 0) scratch[wave] = __popcll(who);
        __syncthreads();
        int before = have, all = have;
#pragma unroll
        for (int i = 0; i < THREADS / kWave; ++i) {
            if (i < wave) before += scratch[i];
            all += scratch[i];
        }
        before += __popcll(who & ((uint64_t(1) << lane) - 1));
        if (mine && before < k) top.list[before] = rank_of(x, at);
        have = all;
    }
    __syncthreads();
    if (threadIdx.x == 0) top.count = min(have, k);
    __syncthreads();
}

// Puts the k largest entries of top.list[0, n) in falling order: calls put(place, entry).  `bound`: at least k entries reach it (or all count).
template <int THREADS, typename Put>
__device__ __forceinline__ void place(Top& top, int n, int k, uint64_t bound, Put put) {
    if (threadIdx.x == 0) top.left = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += THREADS) {
        const uint64_t r = top.list[i];
        if (r >= bound) top.best[atomicAdd(&top.left, 1)] = r;
    }
    __syncthreads();
    const int left = top.left;
    for (int i = threadIdx.x; i < left; i += THREADS) {
        const uint64_t r = top.best[i];
        int larger = 0;
        for (int j = 0; j < left; ++j) larger += top.best[j] > r;
        if (larger < k) put(larger, r);
    }
}

// Alternatives behind the last one above -infinity: the other elements (-infinity, NaN) by index.
template <typename T, int THREADS>
__device__ void fill_up(int* scratch, const T* z, int vocab, int have, int k, int64_t* ids, float* logp, float value) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    for (int v = 0; v < vocab && have < k; v += THREADS) {
        const int at = v + int(threadIdx.x);
        const bool mine = at < vocab && !(load_scalar<T>(z + at) > -__builtin_inff());
        const uint64_t who = __ballot(mine);
        __syncthreads();
        if (lane == 0) scratch[wave] = __popcll(who);
        __syncthreads();
        int before = have, all = have;
#pragma unroll
        for (int i = 0; i < THREADS / kWave; ++i) {
            if (i < wave) before += scratch[i];
            all += scratch[i];
        }
        before += __popcll(who & ((uint64_t(1) << lane) - 1));
        if (mine && before < k) {
            ids[before] = at;
            logp[before] = value;
        }
        have = all;
    }
}

// m, l, d of two parts of a row as those of both.
struct Sums {
    float m, l, d;
};
__device__ __forceinline__ void move_to(Sums& s, float m, float c) {
    const float down = s.m - m, scale = __builtin_amdgcn_exp2f(down * c);
    s.d = scale > 0.f ? (s.d + s.l * down) * scale : 0.f;       // (0 where everything is far below m, or nothing was there)
    s.l *= scale;
    s.m = m;
}

// What is reported of a row.
struct Row {
    float m, s, inv_tau;
    bool empty;
    __device__ __forceinline__ float logp(float x) const { return empty ? -__builtin_inff() : (x - m) * inv_tau - s; }
};
template <typename T>
__device__ __forceinline__ Row finish_row(const LogprobArgs& a, int64_t row, const T* z, const Sums& all, bool write) {
    Row r;
    r.inv_tau = 1.f / a.tau;
    r.empty = all.l == 0.f;
    r.m = r.empty ? -__builtin_inff() : all.m;
    r.s = r.empty ? 0.f : logf(all.l);
    if (write) {
        if (a.stats) {
            a.stats[2 * row] = r.m;
            a.stats[2 * row + 1] = r.s;
        }
        if (a.entropy) a.entropy[row] = r.empty ? 0.f : r.s - all.d / all.l * r.inv_tau;
        if (a.logp) {
            const int64_t t = a.targets[row];
            a.logp[row] = t >= 0 && t < a.vocab ? r.logp(load_scalar<T>(z + t)) : 0.f;
        }
    }
    return r;
}

// One segment of a row, or all of it (segments = 1).
template <typename T, int THREADS, bool TOP, bool NT>
__global__ void __launch_bounds__(THREADS) logprob_forward_kernel(LogprobArgs a) {
    constexpr int E = Words<T>::kElems, kAtOnce = 4, kWaves = THREADS / kWave, kStep = THREADS * E * kAtOnce;
    __shared__ float part[3][kWaves];
    __shared__ int scratch[kWaves];
    __shared__ typename std::conditional<TOP, Top, int>::type top_storage;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const float c = kLog2e / a.tau;
    for (int64_t b = blockIdx.x; b < a.tokens * a.segments; b += gridDim.x) {
        const int64_t row = a.segments == 1 ? b : b / a.segments;
        const int seg = a.segments == 1 ? 0 : int(b - row * a.segments), v0 = seg * a.segment, v1 = min(v0 + a.segment, a.vocab);
        const T* z = static_cast<const T*>(a.logits) + row * a.stride;
        const int per_wave = (a.top + kWaves - 1) / kWaves;
        Sums s = {kLeast, 0.f, 0.f};
        u4 w[kAtOnce];
        const auto ask = [&](int v) {
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) w[j] = Words<T>::template load<NT>(z + v + j * THREADS * E, v1 - v - j * THREADS * E);
        };
        float bound = -__builtin_inff();
        if constexpr (TOP) {
            if (threadIdx.x == 0) top_storage.count = 0;
        }
        const auto least_bound = [&]() {
            float f = -__builtin_inff();
            if constexpr (TOP) {
                f = reinterpret_cast<volatile float*>(top_storage.bound)[0];
#pragma unroll
                for (int i = 1; i < kWaves; ++i) f = fminf(f, reinterpret_cast<volatile float*>(top_storage.bound)[i]);
            }
            return f;
        };
        // (all threads take the first step, the elements behind the end are -infinity)
        int v = v0 + int(threadIdx.x) * E;
        ask(v);
        const int steps = max(1, (v1 - v0 + kStep - 1) / kStep);
        for (int step = 0; step < steps; ++step, v += kStep) {
            float f[kAtOnce][E], most = -__builtin_inff();
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                Words<T>::unpack(w[j], f[j]);
#pragma unroll
                for (int i = 0; i < E; ++i) most = fmaxf(most, f[j][i]);
            }
            if (step + 1 < steps) ask(v + kStep);
            if (most > s.m) move_to(s, most, c);
            float l = 0.f, d = 0.f;
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const float down = f[j][i] - s.m, e = __builtin_amdgcn_exp2f(down * c);
                    l += e;
                    d = fmaf(e, fmaxf(down, kLeast), d);        // (e = 0 where the logit is -infinity)
                }
            s.l += l;
            s.d += d;
            if constexpr (TOP) {
                if ((step & (step - 1)) == 0) {                 // 0, 1, 2, 4, 8: what was seen has doubled
                    const float mine = wave_jth(s.l > 0.f || s.m > kLeast ? s.m : -__builtin_inff(), per_wave);
                    if (step == 0) __syncthreads();
                    if (lane == 0) reinterpret_cast<volatile float*>(top_storage.bound)[wave] = mine;
                    if (step == 0) __syncthreads();
                    bound = least_bound();
                }
                if (most >= bound && most > -__builtin_inff()) {
#pragma unroll
                    for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
                        for (int i = 0; i < E; ++i)
                            if (f[j][i] >= bound && f[j][i] > -__builtin_inff()) {
                                const int at = atomicAdd(&top_storage.count, 1);
                                if (at < kList) top_storage.list[at] = rank_of(f[j][i], v + j * THREADS * E + i);
                            }
                }
            }
        }
        // the block's sums
        const float mine = s.l > 0.f || s.m > kLeast ? s.m : -__builtin_inff();
        {
            const float m = wave_max(s.m);
            move_to(s, m, c);
            s.l = wave_sum(s.l);
            s.d = wave_sum(s.d);
            if (lane == 0) {
                part[0][wave] = s.m;
                part[1][wave] = s.l;
                part[2][wave] = s.d;
            }
        }
        if constexpr (TOP) {
            const float f = wave_jth(mine, per_wave);
            if (lane == 0) top_storage.bound[wave] = f;
        }
        __syncthreads();
        Sums all = {kLeast, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kWaves; ++i) all.m = fmaxf(all.m, part[0][i]);
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            Sums p = {part[0][i], part[1][i], part[2][i]};
            move_to(p, all.m, c);
            all.l += p.l;
            all.d += p.d;
        }
        Row r;
        if (a.segments == 1) r = finish_row<T>(a, row, z, all, threadIdx.x == 0);
        else if (threadIdx.x == 0) a.parts[b] = float4{all.m, all.l, all.d, 0.f};
        if constexpr (TOP) {
            Top& top = top_storage;
            int n = top.count;
            uint64_t from = 0;
            if (n > kList) {
                search<T, THREADS>(top, scratch, z, v0, v1, a.top, all.m);
                n = top.count;
            } else {
                const float f = least_bound();
                if (f > -__builtin_inff()) from = rank_of(f, -1);       // (the last of all indices)
            }
            const int k = min(n, a.top);
            if (a.segments == 1) {
                int64_t* ids = a.top_ids + row * a.top;
                float* logp = a.top_logp + row * a.top;
                place<THREADS>(top, n, k, from, [&](int at, uint64_t e) {
                    ids[at] = index_of(e);
                    logp[at] = r.logp(logit_of(e));
                });
                if (k < a.top) fill_up<T, THREADS>(scratch, z, a.vocab, k, a.top, ids, logp, r.logp(-__builtin_inff()));
            } else {
                uint64_t* out = a.candidates + b * a.top;
                place<THREADS>(top, n, k, from, [&](int at, uint64_t e) { out[at] = e; });
                for (int i = k + int(threadIdx.x); i < a.top; i += THREADS) out[i] = 0;
            }
        }
        __syncthreads();        // (what the block holds in common is free again)
    }
}

// Joins the segments of a row.
constexpr int kJoin = 256;
template <typename T>
__global__ void __launch_bounds__(kJoin) logprob_join_kernel(LogprobArgs a) {
    __shared__ int scratch[kJoin / kWave];
    __shared__ Top top;
    const float c = kLog2e / a.tau;
    for (int64_t row = blockIdx.x; row < a.tokens; row += gridDim.x) {
        const T* z = static_cast<const T*>(a.logits) + row * a.stride;
        Sums all = {kLeast, 0.f, 0.f};
        const float4* parts = a.parts + row * a.segments;
        for (int i = 0; i < a.segments; ++i) all.m = fmaxf(all.m, parts[i].x);
        for (int i = 0; i < a.segments; ++i) {
            Sums p = {parts[i].x, parts[i].y, parts[i].z};
            move_to(p, all.m, c);
            all.l += p.l;
            all.d += p.d;
        }
        const Row r = finish_row<T>(a, row, z, all, threadIdx.x == 0);
        if (a.top > 0) {
            // Every segment's j-th largest, j = ceil(k / segments): k elements reach the least of them.
            const uint64_t* in = a.candidates + row * a.segments * a.top;
            const int j = (a.top + a.segments - 1) / a.segments;
            uint64_t from = ~uint64_t(0);
            for (int i = 0; i < a.segments; ++i) from = min(from, in[int64_t(i) * a.top + j - 1]);
            if (threadIdx.x == 0) top.count = 0;
            __syncthreads();
            for (int i = threadIdx.x; i < a.segments * a.top; i += kJoin) {
                const uint64_t e = in[i];
                if (e != 0 && e >= from) {
                    const int at = atomicAdd(&top.count, 1);
                    top.list[at] = e;       // (at most segments * top <= kList)
                }
            }
            __syncthreads();
            const int n = top.count, k = min(n, a.top);
            int64_t* ids = a.top_ids + row * a.top;
            float* logp = a.top_logp + row * a.top;
            place<kJoin>(top, n, k, 0, [&](int at, uint64_t e) {
                ids[at] = index_of(e);
                logp[at] = r.logp(logit_of(e));
            });
            if (k < a.top) fill_up<T, kJoin>(scratch, z, a.vocab, k, a.top, ids, logp, r.logp(-__builtin_inff()));
            __syncthreads();
        }
    }
}

// One segment of a row.
template <typename T, bool NT>
__global__ void __launch_bounds__(256) logprob_backward_kernel(LogprobBackwardArgs a) {
    constexpr int E = Words<T>::kElems, kAtOnce = 4;
    const float inv_tau = 1.f / a.tau;
    for (int64_t b = blockIdx.x; b < a.tokens * a.segments; b += gridDim.x) {
        const int64_t row = b / a.segments;
        const int v0 = int(b - row * a.segments) * a.segment, v1 = min(v0 + a.segment, a.vocab);
        const T* z = static_cast<const T*>(a.logits) + row * a.stride;
        T* out = static_cast<T*>(a.dlogits) + row * a.dstride;
        u4 w[kAtOnce];
        const auto ask = [&](int v) {
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) w[j] = Words<T>::template load<NT>(z + v + j * 256 * E, v1 - v - j * 256 * E);
        };
        int v = v0 + int(threadIdx.x) * E;
        ask(v);
        const int64_t target = a.targets ? a.targets[row] : -1;
        const bool given = a.dlogp && target >= 0 && target < a.vocab;
        const float g = given ? a.dlogp[row] : 0.f, dh = a.dentropy ? a.dentropy[row] : 0.f;
        const float m = a.stats[2 * row], s = a.stats[2 * row + 1];
        const bool none = (g == 0.f && dh == 0.f) || m == -__builtin_inff();
        // -p (g + dh (log p + H)) / tau = p (base + slope log p)
        const float base = -inv_tau * (dh == 0.f ? g : fmaf(dh, a.entropy[row], g)), slope = -inv_tau * dh;
        const auto gradient = [&](float x) {
            const float logp = fmaf(x - m, inv_tau, -s), p = __builtin_amdgcn_exp2f(logp * kLog2e);
            return none || p == 0.f ? 0.f : p * fmaf(slope, logp, base);
        };
        // (the target's logit, before anything is written where it may be read)
        const bool here = given && !none && target >= v0 && target < v1;
        const float at_target = here ? load_scalar<T>(z + target) : 0.f;
        __syncthreads();
        while (v < v1) {
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                float f[E];
                Words<T>::unpack(w[j], f);
#pragma unroll
                for (int i = 0; i < E; ++i) f[i] = gradient(f[i]);
                if (v + j * 256 * E < v1) Words<T>::template store<NT>(out + v + j * 256 * E, v1 - v - j * 256 * E, f);
            }
            v += 256 * E * kAtOnce;
            if (v < v1) ask(v);
        }
        __syncthreads();
        if (here && threadIdx.x == 0) Words<T>::put_one(out + target, fmaf(g, inv_tau, gradient(at_target)));
        __syncthreads();
    }
}

constexpr int64_t kMostBlocks = int64_t(1) << 20;

struct LogprobPlan {
    int threads, segments, segment;
};
LogprobPlan logprob_plan(const LogprobDims& d, int32_t dtype) {
    const int e = dtype == BNS_F32 ? 4 : 8;
    LogprobPlan p = {256, 1, d.vocab};
    // Segments where rows alone leave compute units idle, down to what a block takes at a time.
    int64_t segments = std::min<int64_t>(std::max<int64_t>(1, 1024 / std::max<int64_t>(d.tokens, 1)), (d.vocab + 256 * 4 * e - 1) / (256 * 4 * e));
    segments = std::min<int64_t>(segments, kMostSegments);
    if (d.top > 0) segments = std::min<int64_t>(segments, kList / d.top);
    p.segment = int(round_up((d.vocab + segments - 1) / segments, 8));
    p.segments = (d.vocab + p.segment - 1) / p.segment;
    return p;
}

size_t parts_bytes(const LogprobDims& d, const LogprobPlan& p) { return p.segments > 1 ? size_t(round_up(d.tokens * p.segments * 16, 256)) : 0; }

template <typename T>
void launch_forward(const LogprobArgs& a, const LogprobPlan& p, hipStream_t st) {
    const dim3 grid(uint32_t(std::min(a.tokens * p.segments, kMostBlocks)));
    const bool nt = size_t(a.tokens) * a.vocab * sizeof(T) > kStreamBytes;
    if (a.top > 0 && nt) BNS_LAUNCH((logprob_forward_kernel<T, 256, true, true>), grid, dim3(256), 0, st, a);
    else if (a.top > 0) BNS_LAUNCH((logprob_forward_kernel<T, 256, true, false>), grid, dim3(256), 0, st, a);
    else if (nt) BNS_LAUNCH((logprob_forward_kernel<T, 256, false, true>), grid, dim3(256), 0, st, a);
    else BNS_LAUNCH((logprob_forward_kernel<T, 256, false, false>), grid, dim3(256), 0, st, a);
    if (p.segments > 1 && hipPeekAtLastError() == hipSuccess)
        BNS_LAUNCH((logprob_join_kernel<T>), dim3(uint32_t(std::min(a.tokens, kMostBlocks))), dim3(kJoin), 0, st, a);
}

template <typename T>
void launch_backward(LogprobBackwardArgs a, hipStream_t st) {
    const int64_t least = 256 * 2 * Words<T>::kElems, want = std::max<int64_t>(1, 2048 / std::max<int64_t>(a.tokens, 1));
    const int64_t segments = std::max<int64_t>(1, std::min<int64_t>(want, (a.vocab + least - 1) / least));
    a.segment = int32_t(round_up((a.vocab + segments - 1) / segments, 8));
    a.segments = (a.vocab + a.segment - 1) / a.segment;
    const dim3 grid(uint32_t(std::min(a.tokens * a.segments, kMostBlocks)));
    if (size_t(a.tokens) * a.vocab * sizeof(T) * 2 > kStreamBytes) BNS_LAUNCH((logprob_backward_kernel<T, true>), grid, dim3(256), 0, st, a);
    else BNS_LAUNCH((logprob_backward_kernel<T, false>), grid, dim3(256), 0, st, a);
}

}  // namespace

extern "C" {

size_t bns_logprob_workspace_bytes(const bns_logprob* logprob) {
    LogprobDims d;
    if (check_logprob(logprob, &d) != BNS_OK) return 0;
    const LogprobPlan p = logprob_plan(d, logprob->dtype);
    const size_t n = parts_bytes(d, p);
    return n == 0 ? 256 : n + size_t(round_up(d.tokens * p.segments * d.top * 8, 256));
}

bns_status bns_logprob_forward(const bns_logprob* logprob, const void* logits, const int64_t* targets, float* logp, float* entropy, float* stats,
                               int64_t* top_ids, float* top_logp, void* workspace, size_t workspace_bytes, void* stream) {
    LogprobDims d;
    const bns_status s = check_logprob(logprob, &d);
    if (s != BNS_OK) return s;
    if (!targets && logp) return BNS_EINVAL;
    if (d.top == 0 && (top_ids || top_logp)) return BNS_EINVAL;
    if (d.tokens == 0) return BNS_OK;
    if (!logits || !workspace || (targets && !logp) || (d.top > 0 && (!top_ids || !top_logp))) return BNS_EINVAL;
    if (!aligned_all(dtype_bytes(logprob->dtype), logits) || !aligned_all(8, targets, top_ids) || !aligned_all(4, logp, entropy, stats, top_logp) || !aligned16(workspace))
        return BNS_EINVAL;
    if (workspace_bytes < bns_logprob_workspace_bytes(logprob)) return BNS_EWORKSPACE;
    const LogprobPlan p = logprob_plan(d, logprob->dtype);
    const LogprobArgs a = {logits, targets, logp, entropy, stats, top_ids, top_logp, static_cast<float4*>(workspace),
                           reinterpret_cast<uint64_t*>(static_cast<char*>(workspace) + parts_bytes(d, p)), d.tokens, d.logits_stride, d.vocab, d.top, p.segments,
                           p.segment, logprob->temperature};
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (logprob->dtype == BNS_F32) launch_forward<float>(a, p, st);
    else launch_forward<bf16_t>(a, p, st);
    return hipGetLastError() == hipSuccess ? BNS_OK : BNS_EDEVICE;
}

bns_status bns_logprob_backward(const bns_logprob* logprob, const void* logits, const int64_t* targets, const float* stats, const float* entropy,
                                const float* dlogp, const float* dentropy, void* dlogits, void* stream) {
    LogprobDims d;
    const bns_status s = check_logprob(logprob, &d);
    if (s != BNS_OK) return s;
    if (d.tokens == 0) return BNS_OK;
    if (!logits || !stats || !dlogits || !targets != !dlogp || (dentropy && !entropy)) return BNS_EINVAL;
    if (!aligned_all(dtype_bytes(logprob->dtype), logits, dlogits) || !aligned_all(8, targets) || !aligned_all(4, stats, entropy, dlogp, dentropy)) return BNS_EINVAL;
    const size_t e = dtype_bytes(logprob->dtype), row = size_t(d.vocab) * e;
    if (collide(matrix(dlogits, d.tokens, d.vocab, d.dlogits_stride, e), matrix(logits, d.tokens, d.vocab, d.logits_stride, e), true, row, row)) return BNS_EINVAL;
    const LogprobBackwardArgs a = {logits, targets, stats, entropy, dlogp, dentropy, dlogits, d.tokens, d.logits_stride, d.dlogits_stride, d.vocab, 1, d.vocab,
                                   logprob->temperature};
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (logprob->dtype == BNS_F32) launch_backward<float>(a, st);
    else launch_backward<bf16_t>(a, st);
    return hipGetLastError() == hipSuccess ? BNS_OK : BNS_EDEVICE;
}

}  // extern "C"
