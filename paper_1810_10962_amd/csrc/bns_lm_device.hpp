// Device-side building blocks of the language-model operators: rows that begin at any element, maxima over a wave.
#pragma once
#include "bns_device.hpp"

namespace bns {

// Accesses with the non-temporal hint, for calls that move more than the memory-side cache holds anyway: lines that nobody will find there are not
// kept (see kStreamBytes).
typedef uint32_t words4_t __attribute__((ext_vector_type(4)));
typedef words4_t words4_f32_t __attribute__((aligned(4)));
typedef words4_t words4_bf16_t __attribute__((aligned(2)));
template <bool NT>
__device__ __forceinline__ words4_t get16(const float* p) {
    if constexpr (NT) return __builtin_nontemporal_load(reinterpret_cast<const words4_f32_t*>(p));
    else return *reinterpret_cast<const words4_f32_t*>(p);
}
template <bool NT>
__device__ __forceinline__ words4_t get16(const bf16_t* p) {
    if constexpr (NT) return __builtin_nontemporal_load(reinterpret_cast<const words4_bf16_t*>(p));
    else return *reinterpret_cast<const words4_bf16_t*>(p);
}
template <bool NT>
__device__ __forceinline__ void put16(float* p, words4_t v) {
    if constexpr (NT) __builtin_nontemporal_store(v, reinterpret_cast<words4_f32_t*>(p));
    else *reinterpret_cast<words4_f32_t*>(p) = v;
}
template <bool NT>
__device__ __forceinline__ void put16(bf16_t* p, words4_t v) {
    if constexpr (NT) __builtin_nontemporal_store(v, reinterpret_cast<words4_bf16_t*>(p));
    else *reinterpret_cast<words4_bf16_t*>(p) = v;
}

// Eight neighbouring elements of a row, as floats.  A row may begin at any element, so the accesses are declared for element alignment: the
// hardware takes 128 bits from any address, and those that happen to be aligned cost nothing extra.  The last vector of a row that is no
// multiple of eight goes element by element.
template <typename T>
struct Row8;

template <>
struct Row8<float> {
    typedef float v4 __attribute__((ext_vector_type(4)));
    typedef v4 v4e __attribute__((aligned(4)));
    static __device__ __forceinline__ void load(const float* p, int left, float (&f)[8]) {
        if (left >= 8) {
            const v4 a = *reinterpret_cast<const v4e*>(p), b = *reinterpret_cast<const v4e*>(p + 4);
            f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = i < left ? p[i] : 0.f;
        }
    }
    template <bool NT = false>
    static __device__ __forceinline__ void store(float* p, int left, const float (&f)[8]) {
        if (left >= 8) {
            put16<NT>(p, __builtin_bit_cast(words4_t, v4{f[0], f[1], f[2], f[3]}));
            put16<NT>(p + 4, __builtin_bit_cast(words4_t, v4{f[4], f[5], f[6], f[7]}));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) p[i] = f[i];
        }
    }
};

template <>
struct Row8<bf16_t> {
    typedef uint32_t u4 __attribute__((ext_vector_type(4)));
    typedef u4 u4e __attribute__((aligned(2)));
    static __device__ __forceinline__ void load(const bf16_t* p, int left, float (&f)[8]) {
        if (left >= 8) {
            Vec<bf16_t, 8> v;
            v.unpack(*reinterpret_cast<const u4e*>(p));
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = v.f[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = i < left ? bf16_to_f32(p[i].bits) : 0.f;
        }
    }
    template <bool NT = false>
    static __device__ __forceinline__ void store(bf16_t* p, int left, const float (&f)[8]) {
        if (left >= 8) {
            put16<NT>(p, u4{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])});
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) p[i].bits = uint16_t(f32_to_bf16(f[i]));
        }
    }
};

// The same eight elements as they are stored, so that a row that is asked for ahead of its turn takes no more registers than memory.
template <typename T>
struct Raw8;
template <>
struct Raw8<float> {
    typedef uint32_t u4 __attribute__((ext_vector_type(4)));
    u4 a, b;
    template <bool NT = false>
    __device__ __forceinline__ void load(const float* p) {
        a = get16<NT>(p);
        b = get16<NT>(p + 4);
    }
    __device__ __forceinline__ void load_left(const float* p, int left) {       // the first `left` elements, zeros behind them
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a[i] = i < left ? __float_as_uint(p[i]) : 0u;
            b[i] = 4 + i < left ? __float_as_uint(p[4 + i]) : 0u;
        }
    }
    __device__ __forceinline__ void clear() { a = b = u4{0, 0, 0, 0}; }
    __device__ __forceinline__ void unpack(float (&f)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(a[i]), f[4 + i] = __uint_as_float(b[i]);
    }
};
template <>
struct Raw8<bf16_t> {
    typedef uint32_t u4 __attribute__((ext_vector_type(4)));
    u4 a;
    template <bool NT = false>
    __device__ __forceinline__ void load(const bf16_t* p) { a = get16<NT>(p); }
    __device__ __forceinline__ void load_left(const bf16_t* p, int left) {
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = uint32_t(2 * i < left ? p[2 * i].bits : 0) | uint32_t(2 * i + 1 < left ? p[2 * i + 1].bits : 0) << 16;
    }
    __device__ __forceinline__ void clear() { a = u4{0, 0, 0, 0}; }
    __device__ __forceinline__ void unpack(float (&f)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[2 * i] = __uint_as_float(a[i] << 16), f[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
    }
};

// Maximum over the 64 lanes of a wave, as a wave-uniform value; as wave_sum, NaN counting for nothing.
__device__ __forceinline__ float wave_max(float v) {
#define BNS_MAX_STEP(ctrl, rows) \
    v = fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, v), __builtin_bit_cast(int, v), ctrl, rows, 0xf, false)))
    BNS_MAX_STEP(0x111, 0xf);
    BNS_MAX_STEP(0x112, 0xf);
    BNS_MAX_STEP(0x114, 0xf);
    BNS_MAX_STEP(0x118, 0xf);
    BNS_MAX_STEP(0x142, 0xa);
    BNS_MAX_STEP(0x143, 0xc);
#undef BNS_MAX_STEP
    return last_lane(v);
}

}  // namespace bns
