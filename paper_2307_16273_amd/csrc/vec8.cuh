// Eight adjacent items at any address, held as they lie in memory (k_loss.hip, k_update.hip).
#pragma once
#include "layer8.cuh"

// Eight adjacent items as they lie in memory, two of 16 bits to a register, and as floats.
typedef uint32_t Quad __attribute__((ext_vector_type(4)));
typedef uint32_t QuadAnywhere __attribute__((ext_vector_type(4), aligned(1)));
template <class T>
struct Raw8 {
    Quad q[sizeof(T) / 2];
    __device__ __forceinline__ uint32_t operator[](int i) const { return q[i / 4][i % 4]; }
};
template <class T>
static __device__ __forceinline__ Raw8<T> load8(const T* p) {
    Raw8<T> v;
#pragma unroll
    for (int h = 0; h < (int)sizeof(T) / 2; ++h) v.q[h] = ((const QuadAnywhere*)p)[h];
    return v;
}
static __device__ __forceinline__ void floats8(const Raw8<float>& v, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(v[i]);
}
static __device__ __forceinline__ void floats8(const Raw8<bf16_t>& v, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(v[i] << 16);
        f[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
    }
}
static __device__ __forceinline__ void floats8(const Raw8<__half>& v, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 x = __half22float2(__builtin_bit_cast(__half2, v[i]));
        f[2 * i] = x.x;
        f[2 * i + 1] = x.y;
    }
}
// Eight floats as they leave for memory, two of 16 bits rounded by one instruction.
static __device__ __forceinline__ void pack8(const float (&f)[8], Raw8<float>& v) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v.q[i / 4][i % 4] = __float_as_uint(f[i]);
}
static __device__ __forceinline__ void pack8(const float (&f)[8], Raw8<bf16_t>& v) {
    typedef float F2 __attribute__((ext_vector_type(2)));
    typedef __bf16 B2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const F2 x = {f[2 * i], f[2 * i + 1]};
        v.q[0][i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, B2));
    }
}
static __device__ __forceinline__ void pack8(const float (&f)[8], Raw8<__half>& v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        __half lo, hi;
        l8_put(f[2 * i], lo);
        l8_put(f[2 * i + 1], hi);
        v.q[0][i] = (uint32_t)__half_as_ushort(lo) | (uint32_t)__half_as_ushort(hi) << 16;
    }
}
// PAST: past the caches, whose lines go on holding what was there.
template <bool PAST = false, class T>
static __device__ __forceinline__ void store8(T* p, const float (&f)[8]) {
    Raw8<T> w;
    pack8(f, w);
#pragma unroll
    for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
        if (PAST) __builtin_nontemporal_store(w.q[h], (QuadAnywhere*)p + h);
        else ((QuadAnywhere*)p)[h] = w.q[h];
    }
}
// What follows takes the floats of v from its registers again: without this they would stay in registers of their own, twice as many.
template <class T>
static __device__ __forceinline__ void keep_packed(Raw8<T>& v) {
#pragma unroll
    for (int h = 0; h < (int)sizeof(T) / 2; ++h) asm("" : "+v"(v.q[h]));
}
