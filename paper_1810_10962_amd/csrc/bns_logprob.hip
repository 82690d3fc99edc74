// Log probabilities of given tokens, entropy and the most probable alternatives from rows of logits, and their gradient.  See include/bns.h for the
// equations.
//
// Both passes read every logit once (backward writes as much), so HBM bounds them; beside it the forward pass has an exponential and ten more
// operations for each.  Forward: a thread keeps, over all chunks of its row that go by, the largest logit m, l = sum exp((x - m) / tau) and
// d = sum exp((x - m) / tau) (x - m), which are moved to a new m when a chunk has a larger one, so that a row needs one pass and few registers, and other
// blocks' loads go on while it is worked on.  entropy = log l - d / (l tau) has two terms of one sign.
//
// Alternatives: what a thread has as its largest logit bounds the k-th largest of the row from below, if enough threads have such a one: the j-th largest of
// each wave's 64, j = ceil(k / waves), the least of all waves' taken.  On the way each thread leaves the largest logit of every chunk of its words in LDS (its upper 16
// bits), nothing else.  Afterwards the chunks that reach the bound, some two for each alternative, are read again (from the L2), and their elements that do go to the wave's
// list, where the place of one is the number of larger ones.  Rows that put more on the lists than they hold (many equal logits) are searched by halving the range of values,
// some 25 passes over the row by single elements: one row of 131072 equal bf16 logits 340 us, 4096 of them 23 ms.
//
// Few rows are cut into segments, one block each, and joined by a second launch.
//
// Measured: 4096 rows of 131072 bf16 forward 172 to 177 us (1.07 GB, 6.1 TB/s), backward 404 us (2.1 GB, 5.3 TB/s); 333 x 50257 fp32 with 5 alternatives 16.8 us (67 MB, from the
// memory-side cache); one row of 131072 bf16 with 20 alternatives 12.2 to 12.6 us, of which some 4 are the join's launch.  With alternatives kept in a sorted list by
// every thread on the way the same row took 22.7 us, and 4000 x 1500 with 5 alternatives 705 us instead of 10.3.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "bns_internal.hpp"
#include "bns_lm_words.hpp"
#include "bns_step_validate.hpp"

using namespace bns;

namespace {

constexpr int kRegion = 512;            // entries of a wave's list
constexpr int kWords = 4;               // words of 16 bytes that a thread has of a row at a time
constexpr int kSlots = 16;              // chunks of its words that a thread tells apart
constexpr int kPending = 256;           // chunks that a wave looks through
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

__device__ __forceinline__ int lanes_below(uint64_t who) { return int(__builtin_amdgcn_mbcnt_hi(uint32_t(who >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(who), 0))); }

// Words of a row, of elements [.., end): one that would go beyond is moved back so that it ends there, which needs no branch; what it holds of
// the words before it is masked where it counts.  `end` is at least a word, but for rows shorter than one (BRIEF), whose elements are asked for one by one.
template <typename T, bool NT>
__device__ __forceinline__ u4 word_at(const T* z, int v, int end, bool brief) {
    constexpr int E = Words<T>::kElems;
    return brief ? Words<T>::template load<NT>(z, v == 0 ? end : 0) : get16<NT>(z + min(v, end - E));
}
// Elements of word v that are those of the words before it.
template <typename T>
__device__ __forceinline__ int shared_of(int v, int end, bool brief) { return brief ? 0 : v - min(v, end - Words<T>::kElems); }
// -infinity in the place of a word's first n elements.
__device__ __forceinline__ u4 masked(const float*, u4 w, int n) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = i < n ? 0xff800000u : w[i];
    return w;
}
__device__ __forceinline__ u4 masked(const bf16_t*, u4 w, int n) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[i] = 2 * i < n ? (w[i] & 0xffff0000u) | 0xff80u : w[i];
        w[i] = 2 * i + 1 < n ? (w[i] & 0xffffu) | 0xff800000u : w[i];
    }
    return w;
}

// The upper half of a float's bits in the order of the floats; that of +0 is one above that of -0.
constexpr uint32_t kNoKey = 0x007f;     // of -infinity
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x);
    return (b >> 31 ? ~b : b | 0x80000000u) >> 16;
}

// A value that at least j of the 64 lanes reach: the j-th largest without its last 16 bits (-infinity where fewer than j lanes have more).  The range of the lanes' values is cut
// into four again and again: compares and counts of lanes, whatever j is.
__device__ __forceinline__ float wave_reach(float v, int j) {
    if (j > kWave) return -__builtin_inff();
    const uint32_t key = key_of(v);
    const auto enough = [&](uint32_t at) { return int(__popcll(__ballot(key >= at))) >= j; };
    uint32_t lo = kNoKey, hi = key_of(wave_max(v)) + 1;         // lo: j lanes reach it (or it is that of -infinity), hi: fewer do
    // (lanes' largest logits lie close together: less than a factor of two apart, or of sixteen, or of any size)
    for (uint32_t span = 0x80; span <= 0x2000 && hi > lo + span; span *= 8) {
        if (enough(hi - span)) {
            lo = hi - span;
            break;
        }
        hi -= span;
    }
    while (hi - lo > 1) {
        const uint32_t quarter = (hi - lo + 3) / 4, a = lo + quarter, b = min(a + quarter, hi), c = min(b + quarter, hi);
        const bool at_a = enough(a), at_b = enough(b), at_c = enough(c);       // (not at hi)
        lo = at_c ? c : at_b ? b : at_a ? a : lo;
        hi = !at_a ? a : !at_b ? b : !at_c ? c : hi;
    }
    if (lo <= kNoKey) return -__builtin_inff();
    const uint32_t k = lo << 16;
    return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k);
}

// What a block knows of the alternatives: a list for each wave, of which it writes its own without asking the others.
template <int THREADS>
struct Top {
    static constexpr int kWaves = THREADS / kWave, kList = kWaves * kRegion;
    alignas(16) uint64_t list[kList];       // (a wave's keys lie where its list will be: [kSlots][kWave])
    uint16_t pending[kWaves][kPending];     // lane and slot of a chunk
    float bound[kWaves];
    int count[kWaves];                      // (more than kRegion: not all of them are there)
    int found;

    __device__ __forceinline__ int all() const {
        int n = 0;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) n += count[i];
        return n;
    }
    // The largest element of the chunk that the lane has as its slot-th.
    __device__ __forceinline__ void leave_key(int w, int slot, float most) {
        reinterpret_cast<uint16_t*>(list + w * kRegion)[slot * kWave + int(threadIdx.x % kWave)] = uint16_t(key_of(most));
    }
    // What all waves' largest elements say, behind a barrier.
    __device__ __forceinline__ float least(int waves) const {
        float f = bound[0];
#pragma unroll
        for (int i = 1; i < kWaves; ++i) f = i < waves ? fminf(f, bound[i]) : f;
        return f;
    }
    // Adds the entries of the lanes for which `hit` holds to wave w's list, which holds n.
    __device__ __forceinline__ void add(int w, int& n, bool hit, uint64_t entry) {
        const uint64_t who = __ballot(hit);
        const int at = n + lanes_below(who);
        if (hit & (at < kRegion)) list[w * kRegion + at] = entry;
        n += __popcll(who);
    }
    // Says how many entries wave w's list has (all lanes of that wave).
    __device__ __forceinline__ void close(int w, int n) {
        if (threadIdx.x % kWave == 0) {
            count[w] = n;
            if (n % 2 && n < kRegion) list[w * kRegion + n] = 0;        // (they are read two at a time)
        }
    }
    // The wave's chunks whose largest element reaches `at_least`; the number of them.
    __device__ __forceinline__ int find_chunks(int w, int slots, float at_least) {
        const uint16_t* keys = reinterpret_cast<const uint16_t*>(list + w * kRegion);
        const int lane = threadIdx.x % kWave;
        const uint32_t least_key = key_of(at_least) - (at_least == 0.f);        // (-0 reaches +0, as ranks have one zero)
        int n = 0;
        asm volatile("" ::: "memory");      // (a wave's accesses to LDS are in order; nothing is exchanged with other waves)
        for (int i = 0; i < slots; ++i) {
            const bool hit = keys[i * kWave + lane] >= least_key;
            const uint64_t who = __ballot(hit);
            const int at = n + lanes_below(who);
            if (hit & (at < kPending)) pending[w][at] = uint16_t(i * kWave + lane);
            n += __popcll(who);
        }
        asm volatile("" ::: "memory");
        return n;
    }
    // Reads `chunks` of them again, of 2^log_words words, and puts their elements that reach `at_least` on the list; the number of those.
    template <typename T>
    __device__ __forceinline__ int look_through(int w, int chunks, int log_words, float at_least, const T* z, int v0, int v1, bool brief) {
        constexpr int E = Words<T>::kElems;
        const int lane = threadIdx.x % kWave;
        int n = 0;
        struct Item {
            u4 x;
            int at, shared;
            bool there;
        };
        const auto ask = [&](int i) {
            const int item = i + lane, chunk = min(item >> log_words, chunks - 1), which = pending[w][chunk];
            const int word = (which / kWave << log_words) + (item & ((1 << log_words) - 1));
            int at = v0 + (word * THREADS + w * kWave + which % kWave) * E;
            const bool there = item < chunks << log_words && at < v1;
            if (!there) at = v0;
            const int shared = shared_of<T>(at, v1, brief);
            return Item{word_at<T, false>(z, at, v1, brief), at - shared, shared, there};
        };
        if (chunks == 0) return 0;
        Item next = ask(0);
        for (int i = 0; i < chunks << log_words; i += kWave) {
            const Item now = next;
            if (i + kWave < chunks << log_words) next = ask(i + kWave);
            float f[E];
            Words<T>::unpack(now.x, f);
            uint32_t hits = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) hits |= uint32_t(f[e] >= at_least) << e;
            hits = now.there ? hits >> now.shared << now.shared : 0;
            // (a word has one or two of them, if any)
            while (const uint64_t who = __ballot(hits != 0)) {
                const int e = __builtin_ctz(hits | 1u << 31), place = n + lanes_below(who);
                if ((hits != 0) & (place < kRegion)) list[w * kRegion + place] = rank_of(Words<T>::element(now.x, e), now.at + e);
                n += __popcll(who);
                hits &= hits - 1;
            }
        }
        return n;
    }
    // Calls put(place, entry) for the k largest entries; the place of one is the number of larger ones.
    template <typename Put>
    __device__ __forceinline__ void place(int k, Put put) const {
        typedef uint64_t two_t __attribute__((ext_vector_type(2)));
        const int w = threadIdx.x / kWave, mine = count[w];
        for (int i = threadIdx.x % kWave; i < mine; i += kWave) {
            const uint64_t r = list[w * kRegion + i];
            int larger = 0;
#pragma unroll 1
            for (int o = 0; o < kWaves; ++o) {
                const int n = count[o];
#pragma unroll 8
                for (int j = 0; j < n; j += 2) {
                    const two_t e = *reinterpret_cast<const two_t*>(list + o * kRegion + j);
                    larger += (e.x > r) + (e.y > r);
                }
            }
            if (larger < k) put(larger, r);
        }
    }
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

// Exact search of the elements [v0, v1) of a row for its k largest, with as many passes over them as it takes: leaves no more entries than the lists hold, the k largest
// among them.  `most`: the largest element (not NaN); more than k are above -infinity.
template <typename T, int THREADS>
__device__ void search(Top<THREADS>& top, int* scratch, const T* z, int v0, int v1, int k, float most) {
    constexpr int kList = Top<THREADS>::kList, kWaves = THREADS / kWave;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const auto key = [](float x) { return uint32_t(rank_of(x, 0) >> 32); };
    // lo: more than the lists hold or at least k elements reach it; hi: fewer than k do
    uint32_t lo = key(-__builtin_inff()) + 1, hi = key(most) + 1;
    bool fits = false;
    int above = 0;                                      // elements that reach hi
    while (hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        int n = 0;
        for (int v = v0 + int(threadIdx.x); v < v1; v += THREADS) {
            const float x = load_scalar<T>(z + v);
            n += x > -__builtin_inff() && key(x) >= mid;
        }
        n = block_count<THREADS>(n, scratch);
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
    if (threadIdx.x == 0) top.found = 0;
    __syncthreads();
    const uint32_t from = fits ? lo : hi;
    for (int v = v0 + int(threadIdx.x); v < v1; v += THREADS) {
        const float x = load_scalar<T>(z + v);
        if (x > -__builtin_inff() && key(x) >= from) {
            const int at = atomicAdd(&top.found, 1);
            if (at < kList) top.list[at] = rank_of(x, v);
        }
    }
    __syncthreads();
    int have = fits ? top.found : above;
    if (!fits) {
        // More elements have the key lo than there is room for: the first of them by index, as many as are needed.
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
            for (int i = 0; i < kWaves; ++i) {
                if (i < wave) before += scratch[i];
                all += scratch[i];
            }
            before += lanes_below(who);
            if (mine && before < k) top.list[before] = rank_of(x, at);
            have = all;
        }
        have = min(have, k);
    }
    __syncthreads();
    top.close(wave, max(0, min(have - wave * kRegion, kRegion)));
    __syncthreads();
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
        before += lanes_below(who);
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

// The logit of a row's target, asked for early; `there`: the target is one.
struct Target {
    float x = 0.f;
    bool there = false;
    template <typename T>
    __device__ __forceinline__ void ask(const LogprobArgs& a, int64_t row, const T* z) {
        const int64_t t = a.logp ? a.targets[row] : -1;
        there = t >= 0 && t < a.vocab;
        if (there) x = load_scalar<T>(z + t);
    }
};

// What is reported of a row.
struct Row {
    float m, s, inv_tau;
    bool empty;
    __device__ __forceinline__ float logp(float x) const { return empty ? -__builtin_inff() : (x - m) * inv_tau - s; }
};
__device__ __forceinline__ Row finish_row(const LogprobArgs& a, int64_t row, const Target& target, const Sums& all, bool write) {
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
        if (a.logp) a.logp[row] = target.there ? r.logp(target.x) : 0.f;
    }
    return r;
}

// One segment of a row, or all of it (segments = 1).
template <typename T, int THREADS, bool TOP, bool NT>
__global__ void __launch_bounds__(THREADS) logprob_forward_kernel(LogprobArgs a) {
    constexpr int E = Words<T>::kElems, kAtOnce = kWords, kWaves = THREADS / kWave, kStep = THREADS * E * kAtOnce;
    __shared__ float part[3][kWaves];
    __shared__ int scratch[kWaves];
    __shared__ typename std::conditional<TOP, Top<THREADS>, int>::type top;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const float c = kLog2e / a.tau;
    for (int64_t b = blockIdx.x; b < a.tokens * a.segments; b += gridDim.x) {
        const int64_t row = a.segments == 1 ? b : b / a.segments;
        const int seg = a.segments == 1 ? 0 : int(b - row * a.segments), v0 = seg * a.segment, v1 = min(v0 + a.segment, a.vocab);
        const T* z = static_cast<const T*>(a.logits) + row * a.stride;
        // waves whose 64 lanes all have elements (at least one wave counts), and how many of the k each answers for
        const int steps = max(1, (v1 - v0 + kStep - 1) / kStep);
        const int full = steps > 1 ? kWaves : min(kWaves, max(1, (v1 - v0 + E - 1) / (E * kWave))), per_wave = (a.top + full - 1) / full;
        const bool brief = a.vocab < E;
        Sums s = {kLeast, 0.f, 0.f};
        u4 w[kAtOnce];
        const auto ask = [&](int v) {
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) w[j] = word_at<T, NT>(z, v + j * THREADS * E, v1, brief);
        };
        // (all threads take the first step, the elements behind the end are -infinity)
        int v = v0 + int(threadIdx.x) * E;
        ask(v);
        Target target;
        if (a.segments == 1 && threadIdx.x == 0) target.ask(a, row, z);
        // chunks: of 1, 2, 4 .. steps, as many as it takes
        const int log_chunk = steps <= kSlots ? 0 : 32 - __builtin_clz((steps - 1) / kSlots);
        float chunk_most = -__builtin_inff();
        for (int step = 0; step < steps; ++step, v += kStep) {
            u4 now[kAtOnce];
            float most = -__builtin_inff();
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                float f[E];
                now[j] = w[j];
                if (step + 1 == steps) now[j] = masked(z, now[j], shared_of<T>(v + j * THREADS * E, v1, brief));
                Words<T>::unpack(now[j], f);
#pragma unroll
                for (int i = 0; i < E; ++i) most = fmaxf(most, f[i]);
            }
            if (step + 1 < steps) ask(v + kStep);
            if constexpr (TOP) {
                chunk_most = fmaxf(chunk_most, most);
                if (((step + 1) & ((1 << log_chunk) - 1)) == 0 || step + 1 == steps) {
                    top.leave_key(wave, step >> log_chunk, chunk_most);
                    chunk_most = -__builtin_inff();
                }
            }
            if (most > s.m) move_to(s, most, c);
            keep_packed(now);
            float l = 0.f, d = 0.f;
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                if (v0 + step * kStep + (j * kWaves + wave) * kWave * E >= v1) break;       // (nothing of the wave's is left)
                float f[E];
                Words<T>::unpack(now[j], f);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const float down = f[i] - s.m, e = __builtin_amdgcn_exp2f(down * c);
                    l += e;
                    d = fmaf(e, fmaxf(down, kLeast), d);        // (e = 0 where the logit is -infinity)
                }
            }
            s.l += l;
            s.d += d;
        }
        if constexpr (TOP) {
            const float f = wave_reach(s.l > 0.f || s.m > kLeast ? s.m : -__builtin_inff(), per_wave);
            if (lane == 0) top.bound[wave] = f;
        }
        // the block's sums
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
        if (a.segments == 1) r = finish_row(a, row, target, all, threadIdx.x == 0);
        else if (threadIdx.x == 0) a.parts[b] = float4{all.m, all.l, all.d, 0.f};
        if constexpr (TOP) {
            const float bound = fmaxf(top.least(full), kLeast);         // (finite: -infinity and NaN are no alternatives)
            const int chunks = top.find_chunks(wave, ((steps - 1) >> log_chunk) + 1, bound);
            const int listed = chunks > kPending ? kRegion + 1 : top.template look_through<T>(wave, chunks, 2 + log_chunk, bound, z, v0, v1, brief);
            top.close(wave, listed);
            __syncthreads();
            bool over = false;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) over |= top.count[i] > kRegion;
            if (over) search<T, THREADS>(top, scratch, z, v0, v1, a.top, all.m);
            const int k = min(top.all(), a.top);
            if (a.segments == 1) {
                int64_t* ids = a.top_ids + row * a.top;
                float* logp = a.top_logp + row * a.top;
                top.place(k, [&](int at, uint64_t e) {
                    ids[at] = index_of(e);
                    logp[at] = r.logp(logit_of(e));
                });
                if (k < a.top) fill_up<T, THREADS>(scratch, z, a.vocab, k, a.top, ids, logp, r.logp(-__builtin_inff()));
            } else {
                uint64_t* out = a.candidates + b * a.top;
                top.place(k, [&](int at, uint64_t e) { out[at] = e; });
                for (int i = k + int(threadIdx.x); i < a.top; i += THREADS) out[i] = 0;
            }
        }
        __syncthreads();        // (what the block holds in common is free again)
    }
}

// Joins the segments of a row: a lane takes a segment's sums, in every wave, and a thread some of the alternatives.
constexpr int kMostJoined = 512;        // alternatives of all segments of a row
// (with alternatives four waves, without a single one, which has no barriers to wait at: one row of 131072 bf16, 64 alternatives 15.2 us against 16.7 by one wave, 20 12.8 against
// 13.0, none 8.4 against 7.9)
template <typename T, bool TOP>
__global__ void __launch_bounds__(TOP ? 256 : 64) logprob_join_kernel(LogprobArgs a) {
    constexpr int JOIN = TOP ? 256 : 64, kEach = kMostJoined / JOIN;
    static_assert(kMostSegments <= kWave && kEach * kWave <= kRegion, "a lane for each segment, room for all that a wave has");
    __shared__ int scratch[JOIN / kWave];
    __shared__ typename std::conditional<TOP, Top<JOIN>, int>::type top;
    __shared__ uint64_t entries[TOP ? kMostJoined : 1];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const float c = kLog2e / a.tau;
    for (int64_t row = blockIdx.x; row < a.tokens; row += gridDim.x) {
        const T* z = static_cast<const T*>(a.logits) + row * a.stride;
        const float4 mine = lane < a.segments ? a.parts[row * a.segments + lane] : float4{kLeast, 0.f, 0.f, 0.f};
        const uint64_t* in = a.candidates + row * a.segments * a.top;
        const int n = a.segments * a.top;           // (at most kMostJoined)
        uint64_t e[kEach];
        if constexpr (TOP) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int at = i * JOIN + int(threadIdx.x);
                e[i] = at < n ? in[at] : 0;
            }
        }
        Target target;
        if (threadIdx.x == 0) target.ask(a, row, z);
        Sums all = {mine.x, mine.y, mine.z};
        move_to(all, wave_max(all.m), c);
        all.l = wave_sum(all.l);
        all.d = wave_sum(all.d);
        const Row r = finish_row(a, row, target, all, threadIdx.x == 0);
        if constexpr (TOP) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int at = i * JOIN + int(threadIdx.x);
                if (at < n) entries[at] = e[i];
            }
            __syncthreads();
            // Every segment's j-th largest, j = ceil(k / segments): k elements reach the least of them.
            const int j = (a.top + a.segments - 1) / a.segments;
            uint64_t one = 0;
            if (lane < a.segments) one = entries[lane * a.top + j - 1];
            const float least = -wave_max(lane >= a.segments ? -__builtin_inff() : one ? -logit_of(one) : __builtin_inff());
            const uint64_t from = least > -__builtin_inff() ? rank_of(least, -1) : 0;
            int listed = 0;
#pragma unroll
            for (int i = 0; i < kEach; ++i) top.add(wave, listed, e[i] != 0 && e[i] >= from, e[i]);
            top.close(wave, listed);
            __syncthreads();
            const int k = min(top.all(), a.top);
            int64_t* ids = a.top_ids + row * a.top;
            float* logp = a.top_logp + row * a.top;
            top.place(k, [&](int at, uint64_t best) {
                ids[at] = index_of(best);
                logp[at] = r.logp(logit_of(best));
            });
            if (k < a.top) fill_up<T, JOIN>(scratch, z, a.vocab, k, a.top, ids, logp, r.logp(-__builtin_inff()));
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
        const bool brief = a.vocab < E;
        u4 w[kAtOnce];
        const auto ask = [&](int v) {
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) w[j] = word_at<T, NT>(z, v + j * 256 * E, v1, brief);
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
                // (of a word that was moved back only its own elements: in place, the others may have been the gradient already)
                const int at = v + j * 256 * E;
                if (at + E <= v1) {
                    Words<T>::template store<NT>(out + at, E, f);
                } else if (at < v1) {
                    const int shared = shared_of<T>(at, v1, brief);
#pragma unroll
                    for (int i = 0; i < E; ++i)
                        if (i >= shared && at + i - shared < v1) Words<T>::put_one(out + at + i - shared, f[i]);
                }
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
    const int64_t words = (d.vocab + (dtype == BNS_F32 ? 3 : 7)) / (dtype == BNS_F32 ? 4 : 8), steps = (words + 256 * kWords - 1) / (256 * kWords);
    LogprobPlan p = {256, 1, d.vocab};
    // A wave for each row, which needs no barriers, where rows are short or many.  (us, a wave against four: bf16 with 20 alternatives 512x1500 7.1 against 8.7, 1000x8000 10.9 against
    // 12.8, 1000x16000 15.2 against 16.0, 1000x32000 22 against 21, 4000x32000 53 against 60, 4000x64000 99 against 98; a bound for more alternatives takes more lanes.)
    if (d.top <= 32 && words <= std::max<int64_t>(512, std::min<int64_t>(4096, d.tokens * d.tokens / 512))) {
        p.threads = 64;
        return p;
    }
    // Segments of two steps at least where rows leave compute units idle, which a second launch joins.  (bf16 with 20 alternatives: 1x131072 13.1 in eight against 20.9 in one, 1x64000 12.5
    // against 13.7, 1x32000 11.3 against 9.7; 64x131072 16.0 in four against 22.0, 128x131072 18.7 against 22.2, 128x64000 15.9 against 14.9, 256x131072 26 against 23.)
    if (d.tokens <= 128 && steps >= 8 && (d.tokens <= 64 || d.vocab >= 100000)) {
        int64_t segments = std::min<int64_t>(steps / 2, std::max<int64_t>(4, 256 / std::max<int64_t>(d.tokens, 1)));
        segments = std::min<int64_t>(segments, kMostSegments);
        if (d.top > 0) segments = std::min<int64_t>(segments, kMostJoined / d.top);
        p.segment = int(round_up((d.vocab + segments - 1) / segments, 8));
        p.segments = (d.vocab + p.segment - 1) / p.segment;
    }
    return p;
}

size_t parts_bytes(const LogprobDims& d, const LogprobPlan& p) { return p.segments > 1 ? size_t(round_up(d.tokens * p.segments * 16, 256)) : 0; }

template <typename T, int THREADS>
void launch_rows(const LogprobArgs& a, const dim3& grid, bool nt, hipStream_t st) {
    if (a.top > 0 && nt) BNS_LAUNCH((logprob_forward_kernel<T, THREADS, true, true>), grid, dim3(THREADS), 0, st, a);
    else if (a.top > 0) BNS_LAUNCH((logprob_forward_kernel<T, THREADS, true, false>), grid, dim3(THREADS), 0, st, a);
    else if (nt) BNS_LAUNCH((logprob_forward_kernel<T, THREADS, false, true>), grid, dim3(THREADS), 0, st, a);
    else BNS_LAUNCH((logprob_forward_kernel<T, THREADS, false, false>), grid, dim3(THREADS), 0, st, a);
}

template <typename T>
void launch_forward(const LogprobArgs& a, const LogprobPlan& p, hipStream_t st) {
    const dim3 grid(uint32_t(std::min(a.tokens * p.segments, kMostBlocks)));
    const bool nt = size_t(a.tokens) * a.vocab * sizeof(T) > kStreamBytes;
    if (p.threads == 64) launch_rows<T, 64>(a, grid, nt, st);
    else launch_rows<T, 256>(a, grid, nt, st);
    if (p.segments == 1 || hipPeekAtLastError() != hipSuccess) return;
    const dim3 rows(uint32_t(a.tokens));
    if (a.top > 0) BNS_LAUNCH((logprob_join_kernel<T, true>), rows, dim3(256), 0, st, a);
    else BNS_LAUNCH((logprob_join_kernel<T, false>), rows, dim3(64), 0, st, a);
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
