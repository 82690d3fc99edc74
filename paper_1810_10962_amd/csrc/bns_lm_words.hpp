// Rows of logits as words of 16 bytes, for the operators that read them from memory.
#pragma once
#include "bns_lm_device.hpp"

namespace bns {

constexpr float kLeast = -3.40282347e38f;      // the lowest finite value: a maximum of only -infinity is this, one of rows masked with it is exact
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

typedef uint32_t u4 __attribute__((ext_vector_type(4)));

// 16 bytes of a row as they are stored; elements behind its end are -infinity.
template <typename T>
struct Words;
template <>
struct Words<float> {
    static constexpr int kElems = 4;
    template <bool NT>
    static __device__ __forceinline__ u4 load(const float* p, int left) {
        if (left >= 4) return get16<NT>(p);
        const uint32_t* w = reinterpret_cast<const uint32_t*>(p);
        const uint32_t none = 0xff800000u;
        return u4{left > 0 ? w[0] : none, left > 1 ? w[1] : none, left > 2 ? w[2] : none, none};
    }
    static __device__ __forceinline__ void unpack(u4 w, float (&f)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(w[i]);
    }
    static __device__ __forceinline__ float element(u4 w, int i) {
        const uint32_t a = i & 1 ? w[1] : w[0], b = i & 1 ? w[3] : w[2];
        return __uint_as_float(i & 2 ? b : a);
    }
    template <bool NT>
    static __device__ __forceinline__ void store(float* p, int left, const float (&f)[4]) {
        if (left >= 4) {
            put16<NT>(p, u4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])});
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < left) p[i] = f[i];
        }
    }
    static __device__ __forceinline__ void put_one(float* p, float f) { *p = f; }
};
template <>
struct Words<bf16_t> {
    static constexpr int kElems = 8;
    template <bool NT>
    static __device__ __forceinline__ u4 load(const bf16_t* p, int left) {
        if (left >= 8) return get16<NT>(p);
        u4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = 2 * i < left ? p[2 * i].bits : 0xff80u, hi = 2 * i + 1 < left ? p[2 * i + 1].bits : 0xff80u;
            w[i] = lo | hi << 16;
        }
        return w;
    }
    static __device__ __forceinline__ void unpack(u4 w, float (&f)[8]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ float element(u4 w, int i) {
        const uint32_t a = i & 2 ? w[1] : w[0], b = i & 2 ? w[3] : w[2], both = i & 4 ? b : a;
        return __uint_as_float(i & 1 ? both & 0xffff0000u : both << 16);
    }
    template <bool NT>
    static __device__ __forceinline__ void store(bf16_t* p, int left, const float (&f)[8]) { Row8<bf16_t>::store<NT>(p, left, f); }
    static __device__ __forceinline__ void put_one(bf16_t* p, float f) { p->bits = uint16_t(f32_to_bf16(f)); }
};

// Keeps the compiler from carrying the words' values, twice their size in bf16, from one use of the row to the next.
template <int N>
__device__ __forceinline__ void keep_packed(u4 (&w)[N]) {
#pragma unroll
    for (int j = 0; j < N; ++j) asm volatile("" : "+v"(w[j]));
}

}  // namespace bns
