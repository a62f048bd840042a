// What the expert-layer operators share: element types, 8-bit conversions, scales, small wave helpers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/hgemm.h"

namespace hgemm {

bool current_device_is_gfx950();        // of the calling thread's current device
int64_t compute_units();
bool wait_for_clearing(bool& clearing, hipStream_t stream);      // before a run: false if the counters of the plan could not be waited for

constexpr int kScaleBlock = HGEMM_SCALE_BLOCK;
typedef float f4 __attribute__((ext_vector_type(4)));
typedef int i4 __attribute__((ext_vector_type(4)));
typedef int i8 __attribute__((ext_vector_type(8)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));
typedef unsigned u2 __attribute__((ext_vector_type(2)));
typedef unsigned short bf16_bits;

inline int64_t blocks_of(int64_t n) { return (n + kScaleBlock - 1) / kScaleBlock; }
inline int64_t round_up(int64_t n, int64_t step) { return (n + step - 1) / step * step; }
inline int type_size(hgemm_type_t t) { return t == HGEMM_F32 ? 4 : 2; }
inline bool fits_grid(int64_t workgroups, int64_t threads) { return workgroups <= 0xffffffffLL / threads; }      // a launch has fewer than 2^32 threads along x
inline bool aligned(const void* p, size_t to) { return (uintptr_t)p % to == 0; }

// An e8m0 scale is the biased exponent of a power of two: 0 stands for 2^-127, 255 for NaN.
__device__ __forceinline__ float e8m0_value(unsigned e) { return __builtin_bit_cast(float, e == 0 ? 0x400000u : e == 255 ? 0x7fc00000u : e << 23); }
__device__ __forceinline__ float load_scale(const void* s, int64_t at, bool e8m0)
{
    return e8m0 ? e8m0_value(((const uint8_t*)s)[at]) : ((const float*)s)[at];
}

// Elements of X as fp32, and back with one rounding to nearest even (bf16: NaN stays NaN).
__device__ __forceinline__ float as_float(_Float16 x) { return (float)x; }
__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(__bf16 x) { return (float)x; }
template <class T> __device__ __forceinline__ T from_float(float x) { return (T)x; }

// Four consecutive fp32 values as the type of C, packed.
template <class T> struct Packed4;
template <> struct Packed4<float> { typedef f4 type; };
template <> struct Packed4<_Float16> { typedef _Float16 type __attribute__((ext_vector_type(4))); };
template <> struct Packed4<__bf16> { typedef __bf16 type __attribute__((ext_vector_type(4))); };
template <class T> __device__ __forceinline__ typename Packed4<T>::type pack4(f4 v)
{
    typename Packed4<T>::type o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (T)v[e];
    return o;
}

// The first `left` of four consecutive elements at p, whatever p is aligned to: global memory takes 8- and 16-byte
// accesses at any element's address.
template <class T> __device__ __forceinline__ void store4(T* p, f4 v, int64_t left)
{
    const auto o = pack4<T>(v);
    if (left >= 4) {
        __builtin_memcpy(p, &o, sizeof o);
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < left) p[e] = o[e];
    }
}

// Eight consecutive elements: loaded and stored as 16-byte words at any element's address, the last of a row, where it has fewer (`left`), one by one
// (8191 x 11003 in bf16, quantised both ways: 85 us, one by one throughout 180).  `wide`: they lie on 16 bytes and are all there.  Such stores bypass
// what they can of the caches (combine and its gradients, 8191 x 4 rows of 4096: 196 us without, 180).
template <class T> struct Eight;
template <class T> struct Eight16 {
    u4 v;
    __device__ __forceinline__ unsigned bits(int e) const { return e & 1 ? v[e >> 1] >> 16 : v[e >> 1] & 0xffffu; }
    __device__ __forceinline__ void set(int e, T x)
    {
        const unsigned b = __builtin_bit_cast(unsigned short, x);
        v[e >> 1] = e & 1 ? (v[e >> 1] & 0xffffu) | b << 16 : (v[e >> 1] & 0xffff0000u) | b;
    }
    __device__ __forceinline__ void load(const T* p, int64_t left, bool wide)
    {
        if (wide) {
            v = *(const u4*)p;
        } else if (left >= 8) {
            __builtin_memcpy(&v, p, sizeof v);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < left) set(e, p[e]);
        }
    }
    __device__ __forceinline__ void store(T* p, int64_t left, bool wide) const
    {
        if (wide) {
            __builtin_nontemporal_store(v, (u4*)p);
        } else if (left >= 8) {
            __builtin_memcpy(p, &v, sizeof v);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < left) p[e] = __builtin_bit_cast(T, (unsigned short)bits(e));
        }
    }
};
template <> struct Eight<_Float16> : Eight16<_Float16> {
    static constexpr unsigned FINITE = 0x7bff;          // bits of the largest finite magnitude
    __device__ __forceinline__ float value(int e) const { return (float)__builtin_bit_cast(_Float16, (unsigned short)bits(e)); }
};
template <> struct Eight<__bf16> : Eight16<__bf16> {
    static constexpr unsigned FINITE = 0x7f7f;
    __device__ __forceinline__ float value(int e) const { return __builtin_bit_cast(float, e & 1 ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16); }
};
template <> struct Eight<float> {
    u4 v[2];
    static constexpr unsigned FINITE = 0x7f7fffff;
    __device__ __forceinline__ unsigned bits(int e) const { return v[e >> 2][e & 3]; }
    __device__ __forceinline__ float value(int e) const { const unsigned b = bits(e); return __builtin_bit_cast(float, b); }
    __device__ __forceinline__ void set(int e, float x) { v[e >> 2][e & 3] = __builtin_bit_cast(unsigned, x); }
    __device__ __forceinline__ void load(const float* p, int64_t left, bool wide)
    {
        if (wide) {
            v[0] = *(const u4*)p;
            v[1] = *(const u4*)(p + 4);
        } else if (left >= 8) {
            __builtin_memcpy(&v, p, sizeof v);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < left) set(e, p[e]);
        }
    }
    __device__ __forceinline__ void store(float* p, int64_t left, bool wide) const
    {
        if (wide) {
            __builtin_nontemporal_store(v[0], (u4*)p);
            __builtin_nontemporal_store(v[1], (u4*)(p + 4));
        } else if (left >= 8) {
            __builtin_memcpy(p, &v, sizeof v);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < left) p[e] = value(e);
        }
    }
};

}  // namespace hgemm
