// Distillation from a teacher's top logits: the loss with the logits' gradient from the same pass, and the gradient on its own.  See
// include/bns.h for the equations.
//
// Softmax of both sides in powers of two: p = exp2((z - m) log2(e) / tau - log2 sum), all of it in fp32 (a word of bf16 is unpacked where it is used).
// Both read every logit once and write every gradient once, so HBM bounds them.  Forward: a block takes a row and keeps it in registers
// as it is stored (256 KB of the 512 KB of a compute unit), so that maximum, sum and gradient come from one read; of longer rows the
// rest is read again, which the memory-side cache serves.  Wave 0 works the teacher's distribution out while the row is on its way.  The gradient is
// written as if the teacher were not there, then the few elements that it touches once more.  Backward needs no sum, so a row is cut into segments where
// rows are few.
// Measured: 4096x131072 bf16 with gradient 401 us (5.4 TB/s, a large copy 5.1), 1630x77568 fp32 181 us, 64x50257 bf16 11 us (one block per row: launch, load,
// two exchanges, store); the gradient alone 2048x50304 fp32 162 us (5.1 TB/s), 7x100003 bf16 6.4 us, which is a launch.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "bns_internal.hpp"
#include "bns_lm_validate.hpp"
#include "bns_lm_words.hpp"

using namespace bns;

namespace {

constexpr int kMostEntries = 1024;

struct DistillArgs {
    const void* logits;
    const int64_t* ids;
    const float *teacher, *dloss;
    const float* lse_in;        // backward
    float *loss, *lse;          // forward
    void* dlogits;
    int64_t tokens, logits_stride, dlogits_stride;
    int32_t vocab, k;
    int32_t segment;            // backward: elements per block, a multiple of 8
    float tau;
};

// The teacher's part of a row, worked out by one wave.
struct Teacher {
    alignas(16) int32_t id[kMostEntries];   // -1: no entry
    alignas(16) float q[kMostEntries];      // (0 from entry k on to a multiple of four)
    float z[kMostEntries];                  // the student's logit there (only of ids in [v0, v1))
    float cross;                            // sum q (log q - (z - z0) / tau)
    float z0;                               // the student's largest logit at the entries
    int32_t some;                           // whether the row has an entry
    float one;                              // 1; NaN where a teacher's logit is NaN or +infinity, which makes all of the row's gradient so
};

// An entry that its lane has asked for; the first kWave of them are asked for before the row is, so that they arrive first.
struct Entry {
    int64_t id = -1;
    float u = 0.f;
    __device__ __forceinline__ void ask(const DistillArgs& a, int64_t row, int j) {
        if (j < a.k) {
            id = a.ids[row * a.k + j];
            u = a.teacher[row * a.k + j];
        }
    }
};

template <typename T>
__device__ __forceinline__ void work_teacher(Teacher& s, const DistillArgs& a, int64_t row, const Entry& first, const T* logits, int v0, int v1, bool cross) {
    const int lane = threadIdx.x;
    const float c = kLog2e / a.tau;
    float most = -__builtin_inff(), z0 = kLeast;
    bool some = false;
    for (int j = lane; j < (a.k + 3) / 4 * 4; j += kWave) {
        Entry e = first;
        if (j >= kWave) {
            e.id = -1;
            e.ask(a, row, j);
        }
        const bool valid = j < a.k && e.id >= 0 && e.id < a.vocab && !(e.u == -__builtin_inff());
        s.id[j] = valid ? int32_t(e.id) : -1;
        s.q[j] = e.u;
        if (valid) {
            if (e.id >= v0 && e.id < v1) {
                s.z[j] = load_scalar<T>(logits + e.id);
                z0 = fmaxf(z0, s.z[j]);
            }
            some = true;
            most = fmaxf(most, e.u);
        }
    }
    most = fmaxf(wave_max(most), kLeast);
    if (cross) z0 = wave_max(z0);
    float sum = 0.f;
    for (int j = lane; j < a.k; j += kWave)
        if (s.id[j] >= 0) sum += __builtin_amdgcn_exp2f((s.q[j] - most) * c);
    const float total = wave_sum(sum), inv = 1.f / total, log2_total = __builtin_amdgcn_logf(total);
    float x = 0.f;
    for (int j = lane; j < (a.k + 3) / 4 * 4; j += kWave) {
        if (s.id[j] < 0) {
            s.q[j] = 0.f;
            continue;
        }
        const float e = (s.q[j] - most) * c, q = __builtin_amdgcn_exp2f(e) * inv;
        s.q[j] = q;
        if (cross && !(q == 0.f)) x += q * ((e - log2_total) * kLn2 - (s.z[j] - z0) / a.tau);
    }
    x = cross ? wave_sum(x) : 0.f;
    const bool any = __any(some);
    if (lane == 0) {
        s.cross = x;
        s.z0 = z0;
        s.some = any;
        s.one = total == total ? 1.f : total;
    }
}

// The gradient where the teacher has entries: what all entries of one id add up to is taken off the student's probability.
template <typename T, typename P>
__device__ __forceinline__ void fix_entries(const Teacher& s, const DistillArgs& a, T* dlogits, int v0, int v1, float scale, P probability) {
    for (int j = threadIdx.x; j < a.k; j += blockDim.x) {
        const int id = s.id[j];
        if (id < v0 || id >= v1) continue;
        float q = 0.f;
        for (int i = 0; i < a.k; i += 4) {
            const int4 ids = *reinterpret_cast<const int4*>(s.id + i);
            const float4 qs = *reinterpret_cast<const float4*>(s.q + i);
            q += (ids.x == id ? qs.x : 0.f) + (ids.y == id ? qs.y : 0.f) + (ids.z == id ? qs.z : 0.f) + (ids.w == id ? qs.w : 0.f);
        }
        Words<T>::put_one(dlogits + id, scale * (probability(s.z[j]) - q));
    }
}

// NV: 16-byte words per thread that hold the row, or with REST its beginning; what lies behind is read again (NV = 0: rows shorter than a word).  NT: with
// the non-temporal hint (4096x131072 bf16 with its gradient 400 against 416 us, gradient of 2048x50304 fp32 162 against 172; 7x100003 bf16 6.7 against 6.4).
template <typename T, int THREADS, int NV, bool REST, bool NT>
__global__ void __launch_bounds__(THREADS) distill_forward_kernel(DistillArgs a) {
    constexpr int E = Words<T>::kElems, kWaves = THREADS / kWave, kHeld = NV * THREADS * E;
    static_assert(NV > 0 || REST, "somebody takes the row");
    __shared__ Teacher teacher;
    __shared__ float part[2][kWaves];
    const int tid = threadIdx.x, wave = tid / kWave;
    const float inv_tau = 1.f / a.tau, c = kLog2e / a.tau;
    for (int64_t row = blockIdx.x; row < a.tokens; row += gridDim.x) {
        const T* z = static_cast<const T*>(a.logits) + row * a.logits_stride;
        Entry entry;
        if (wave == 0) entry.ask(a, row, tid);
        u4 held[NV > 0 ? NV : 1];
        // Without REST the row's last word is moved back so that it ends with the row, and so are those behind it: all are on their way before any is
        // looked at.  What they hold twice does not change a maximum, is left out of the sum and written twice with the same bits.
        int t = tid;        // (opaque, here and before each use: nothing that follows from it is kept in registers from row to row)
        asm volatile("" : "+v"(t));
        if (NV > 0) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int v = (j * THREADS + t) * E;
                held[j] = Words<T>::template load<NT>(z + (REST ? v : min(v, a.vocab - E)), E);
            }
        }
        if (wave == 0) work_teacher(teacher, a, row, entry, z, 0, a.vocab, true);
        // Maximum, and sum of exp2 of what lies below it.  The difference is taken before it is scaled, so that logits of the type's lowest value, which a
        // mask may hold everywhere, do not overflow.
        float m = kLeast, l = 0.f;
        if (REST) {
            for (int v = kHeld + tid * E; v < a.vocab; v += THREADS * E) {
                float f[E], most = -__builtin_inff();
                Words<T>::unpack(Words<T>::template load<false>(z + v, a.vocab - v), f);
#pragma unroll
                for (int i = 0; i < E; ++i) most = fmaxf(most, f[i]);
                most = fmaxf(m, most);
                l *= __builtin_amdgcn_exp2f((m - most) * c);
                m = most;
#pragma unroll
                for (int i = 0; i < E; ++i) l += __builtin_amdgcn_exp2f((f[i] - m) * c);
            }
        }
        float most = -__builtin_inff();
        if (NV > 0) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float f[E];
                Words<T>::unpack(held[j], f);
#pragma unroll
                for (int i = 0; i < E; ++i) most = fmaxf(most, f[i]);
                __builtin_amdgcn_sched_barrier(0);      // (registers: one word's values at a time)
            }
        }
        most = wave_max(fmaxf(most, m));
        l *= __builtin_amdgcn_exp2f((m - most) * c);
        m = most;
        if (NV > 0) {
            keep_packed(held);
            asm volatile("" : "+v"(t));
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float f[E];
                Words<T>::unpack(held[j], f);
#pragma unroll
                for (int i = 0; i < E; ++i) f[i] = __builtin_amdgcn_exp2f((f[i] - m) * c);
                if (!REST && (j + 1) * THREADS * E > a.vocab) {
                    const int twice = (j * THREADS + t + 1) * E - a.vocab;
#pragma unroll
                    for (int i = 0; i < E; ++i) f[i] = i < twice ? 0.f : f[i];
                }
#pragma unroll
                for (int i = 0; i < E; ++i) l += f[i];
                asm volatile("" : "+v"(l));             // (added here and now, for the same reason)
            }
        }
        l = wave_sum(l);
        if (tid % kWave == 0) {
            part[0][wave] = m;
            part[1][wave] = l;
        }
        __syncthreads();
        m = part[0][0];
#pragma unroll
        for (int i = 1; i < kWaves; ++i) m = fmaxf(m, part[0][i]);
        l = 0.f;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) l = fmaf(part[1][i], __builtin_amdgcn_exp2f((part[0][i] - m) * c), l);
        const float log2_l = __builtin_amdgcn_logf(l), ln_l = log2_l * kLn2;
        const bool some = teacher.some;
        if (tid == 0) {
            a.lse[row] = fmaf(m, inv_tau, ln_l);
            a.loss[row] = some ? a.tau * a.tau * (teacher.cross + fmaf(m - teacher.z0, inv_tau, ln_l)) : 0.f;
        }
        if (a.dlogits) {
            T* out = static_cast<T*>(a.dlogits) + row * a.dlogits_stride;
            const float scale = some ? a.tau * a.dloss[row] * teacher.one : 0.f;
            const auto probability = [&](float f) { return __builtin_amdgcn_exp2f(fmaf(f - m, c, -log2_l)); };
            const auto write = [&](int v, u4 w, int left) {
                float f[E];
                Words<T>::unpack(w, f);
#pragma unroll
                for (int i = 0; i < E; ++i) f[i] = some ? scale * probability(f[i]) : 0.f;
                Words<T>::template store<NT>(out + v, left, f);
            };
            if (NV > 0) {
                keep_packed(held);
                asm volatile("" : "+v"(t));
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const int v = (j * THREADS + t) * E;
                    if (REST || v < a.vocab) write(REST ? v : min(v, a.vocab - E), held[j], E);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if (REST) {
                for (int v = kHeld + tid * E; v < a.vocab; v += THREADS * E) write(v, Words<T>::template load<false>(z + v, a.vocab - v), a.vocab - v);
            }
            __syncthreads();
            if (some) fix_entries(teacher, a, out, 0, a.vocab, scale, probability);
        }
        __syncthreads();        // (the teacher's part is free again)
    }
}

// One segment of a row.
template <typename T, bool NT>
__global__ void __launch_bounds__(256) distill_backward_kernel(DistillArgs a, int segments) {
    constexpr int E = Words<T>::kElems, kAtOnce = 4;
    __shared__ Teacher teacher;
    const float inv_tau = 1.f / a.tau;
    for (int64_t b = blockIdx.x; b < a.tokens * segments; b += gridDim.x) {
        const int64_t row = b / segments;
        const int v0 = int(b % segments) * a.segment, v1 = min(v0 + a.segment, a.vocab);
        const T* z = static_cast<const T*>(a.logits) + row * a.logits_stride;
        T* out = static_cast<T*>(a.dlogits) + row * a.dlogits_stride;
        Entry entry;
        if (threadIdx.x < kWave) entry.ask(a, row, threadIdx.x);
        const float lse = a.lse_in[row], dloss = a.dloss[row];
        const auto probability = [&](float f) { return __builtin_amdgcn_exp2f(fmaf(f, inv_tau, -lse) * kLog2e); };
        // (the first words are on their way while the teacher is worked out; nothing is written before the teacher has read)
        u4 w[kAtOnce];
        const auto ask = [&](int v) {
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) w[j] = Words<T>::template load<NT>(z + v + j * 256 * E, v1 - v - j * 256 * E);
        };
        int v = v0 + int(threadIdx.x) * E;
        ask(v);
        if (threadIdx.x < kWave) work_teacher(teacher, a, row, entry, z, v0, v1, false);
        __syncthreads();
        const bool some = teacher.some;
        const float scale = some ? a.tau * dloss * teacher.one : 0.f;
        while (v < v1) {
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                float f[E];
                Words<T>::unpack(w[j], f);
#pragma unroll
                for (int i = 0; i < E; ++i) f[i] = some ? scale * probability(f[i]) : 0.f;
                if (v + j * 256 * E < v1) Words<T>::template store<NT>(out + v + j * 256 * E, v1 - v - j * 256 * E, f);
            }
            v += 256 * E * kAtOnce;
            if (v < v1) ask(v);
        }
        __syncthreads();
        if (some) fix_entries(teacher, a, out, v0, v1, scale, probability);
        __syncthreads();
    }
}

constexpr int64_t kMostBlocks = int64_t(1) << 20;

template <typename T, int THREADS, int NV, bool REST = false>
void launch_rows(const DistillArgs& a, hipStream_t st) {
    const dim3 grid(uint32_t(std::min(a.tokens, kMostBlocks)));
    if (size_t(a.tokens) * a.vocab * sizeof(T) * (a.dlogits ? 2 : 1) > kStreamBytes)
        BNS_LAUNCH((distill_forward_kernel<T, THREADS, NV, REST, true>), grid, dim3(THREADS), 0, st, a);
    else BNS_LAUNCH((distill_forward_kernel<T, THREADS, NV, REST, false>), grid, dim3(THREADS), 0, st, a);
}

// The smallest block that holds a row.
template <typename T>
void launch_forward(const DistillArgs& a, hipStream_t st) {
    const int64_t words = (a.vocab + Words<T>::kElems - 1) / Words<T>::kElems;
    if (a.vocab < Words<T>::kElems) launch_rows<T, 64, 0, true>(a, st);
    else if (words <= 256 * 2) launch_rows<T, 256, 2>(a, st);
    else if (words <= 256 * 4) launch_rows<T, 256, 4>(a, st);
    else if (words <= 512 * 4) launch_rows<T, 512, 4>(a, st);
    else if (words <= 1024 * 4) launch_rows<T, 1024, 4>(a, st);
    else if (words <= 1024 * 8) launch_rows<T, 1024, 8>(a, st);
    else if (words <= 1024 * 12) launch_rows<T, 1024, 12>(a, st);
    else if (words <= 1024 * 16) launch_rows<T, 1024, 16>(a, st);
    else launch_rows<T, 1024, 16, true>(a, st);
}

template <typename T>
void launch_backward(DistillArgs a, hipStream_t st) {
    // Segments of a whole row where the rows alone fill the device, else shorter ones, down to half of the 256 x 4 words that a block takes at a time.
    const int64_t least = 256 * 2 * Words<T>::kElems, want = std::max<int64_t>(1, 2048 / std::max<int64_t>(a.tokens, 1));
    const int64_t segments = std::max<int64_t>(1, std::min<int64_t>(want, (a.vocab + least - 1) / least));
    a.segment = int32_t(round_up((a.vocab + segments - 1) / segments, 8));
    const int count = int((a.vocab + a.segment - 1) / a.segment);
    const dim3 grid(uint32_t(std::min(a.tokens * count, kMostBlocks)));
    if (size_t(a.tokens) * a.vocab * sizeof(T) * 2 > kStreamBytes) BNS_LAUNCH((distill_backward_kernel<T, true>), grid, dim3(256), 0, st, a, count);
    else BNS_LAUNCH((distill_backward_kernel<T, false>), grid, dim3(256), 0, st, a, count);
}

bns_status check_tensors(const bns_distill* distill, const DistillDims& d, const void* logits, const void* ids, const void* teacher, const void* dlogits) {
    if (!logits || !ids || !teacher) return BNS_EINVAL;
    for (const void* p : {logits, ids, teacher, dlogits})
        if (!aligned16(p)) return BNS_EINVAL;
    const size_t e = dtype_bytes(distill->dtype), row = size_t(d.vocab) * e;
    const Matrix out = matrix(dlogits, d.tokens, d.vocab, d.dlogits_stride, e), in = matrix(logits, d.tokens, d.vocab, d.logits_stride, e);
    if (collide(out, in, true, row, row) || collide(out, matrix(ids, d.tokens, d.k, d.k, 8), false, row, size_t(d.k) * 8) ||
        collide(out, matrix(teacher, d.tokens, d.k, d.k, 4), false, row, size_t(d.k) * 4))
        return BNS_EINVAL;
    return BNS_OK;
}

}  // namespace

extern "C" {

bns_status bns_distill_forward(const bns_distill* distill, const void* logits, const int64_t* ids, const float* teacher, const float* dloss,
                               float* loss, float* lse, void* dlogits, void* stream) {
    DistillDims d;
    bns_status s = check_distill(distill, &d);
    if (s != BNS_OK) return s;
    if (d.tokens == 0) return BNS_OK;
    if (!loss || !lse || (dlogits && !dloss)) return BNS_EINVAL;
    if ((s = check_tensors(distill, d, logits, ids, teacher, dlogits)) != BNS_OK) return s;
    const DistillArgs a = {logits, ids, teacher, dloss, nullptr, loss, lse, dlogits, d.tokens, d.logits_stride, d.dlogits_stride,
                           d.vocab, d.k, 0, distill->temperature};
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (distill->dtype == BNS_F32) launch_forward<float>(a, st);
    else launch_forward<bf16_t>(a, st);
    return hipGetLastError() == hipSuccess ? BNS_OK : BNS_EDEVICE;
}

bns_status bns_distill_backward(const bns_distill* distill, const void* logits, const int64_t* ids, const float* teacher, const float* lse,
                                const float* dloss, void* dlogits, void* stream) {
    DistillDims d;
    bns_status s = check_distill(distill, &d);
    if (s != BNS_OK) return s;
    if (d.tokens == 0) return BNS_OK;
    if (!lse || !dloss || !dlogits) return BNS_EINVAL;
    if ((s = check_tensors(distill, d, logits, ids, teacher, dlogits)) != BNS_OK) return s;
    const DistillArgs a = {logits, ids, teacher, dloss, lse, nullptr, nullptr, dlogits, d.tokens, d.logits_stride, d.dlogits_stride,
                           d.vocab, d.k, 0, distill->temperature};
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (distill->dtype == BNS_F32) launch_backward<float>(a, st);
    else launch_backward<bf16_t>(a, st);
    return hipGetLastError() == hipSuccess ? BNS_OK : BNS_EDEVICE;
}

}  // extern "C"
