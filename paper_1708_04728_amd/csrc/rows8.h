// Eight consecutive elements of a row, the unit in which the dropout, loss and adapter kernels read: 16 bytes of bf16, 32 of fp32, at any element's address.
#pragma once
#include "dr_store.h"

namespace dr {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// (16-byte loads and stores need no alignment beyond an element's; the types say so to the compiler)
typedef unsigned int u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ void unpack8(const u32x4& t, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(t[i] << 16);
        v[2 * i + 1] = __uint_as_float(t[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ u32x4 pack8(const float (&v)[8])
{
    u32x4 t;
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
    return t;
}

__device__ __forceinline__ void load8(const uint16_t* p, float (&v)[8]) 
{
    const u32x4 t = *reinterpret_cast<const u32x4_any*>(p);
    unpack8(t, v);
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8])
{
    const f32x4 a = *reinterpret_cast<const f32x4_any*>(p), b = *reinterpret_cast<const f32x4_any*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) { *reinterpret_cast<u32x4_any*>(p) = pack8(v); }
__device__ __forceinline__ void store8(float* p, const float (&v)[8])
{
    *reinterpret_cast<f32x4_any*>(p) = f32x4{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4_any*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ void store4(uint16_t* p, const float (&v)[4])
{
    typedef unsigned int u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
    *reinterpret_cast<u32x2_any*>(p) = u32x2_any{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
}
__device__ __forceinline__ void store4(float* p, const float (&v)[4]) { *reinterpret_cast<f32x4_any*>(p) = f32x4{v[0], v[1], v[2], v[3]}; }
// ... of which `n` exist (n <= 0: none; 8 and more: all), `none` in the place of the others
template <typename T>
__device__ __forceinline__ void load8(const T* p, int n, float none, float (&v)[8])
{
    if (n >= 8) return load8(p, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? Store<T>::ld(p + i) : none;
}
template <typename T>
__device__ __forceinline__ void store8(T* p, int n, const float (&v)[8])
{
    if (n >= 8) return store8(p, v);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) Store<T>::st(p + i, v[i]);
}

}  // namespace
}  // namespace dr
