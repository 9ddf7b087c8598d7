// Element types of the operators that take more than one: 16 bytes of them as binary32 values and back, one rounding to nearest even.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "flash3d.h"

namespace f3d {

namespace {

template <int TYPE>
struct Elems;

template <>
struct Elems<F3D_F32> {
    typedef float one;
    static constexpr int W = 4;                       // in 16 bytes
    static __device__ __forceinline__ float to_f32(one x) { return x; }
    static __device__ __forceinline__ one from_f32(float x) { return x; }
    static __device__ __forceinline__ void unpack(const uint4& u, float (&x)[W])
    {
        x[0] = __uint_as_float(u.x);
        x[1] = __uint_as_float(u.y);
        x[2] = __uint_as_float(u.z);
        x[3] = __uint_as_float(u.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&x)[W])
    {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
};

template <class T, int TYPE>
struct Elems16 {
    typedef T one;
    typedef __attribute__((ext_vector_type(2))) T two;
    typedef __attribute__((ext_vector_type(2))) float f2;
    static constexpr int W = 8;
    static __device__ __forceinline__ float to_f32(one x) { return (float)x; }
    static __device__ __forceinline__ one from_f32(float x) { return (one)x; }
    static __device__ __forceinline__ uint32_t pack2(float lo, float hi)
    {
        const f2 x = {lo, hi};
        const two y = __builtin_convertvector(x, two);
        return *reinterpret_cast<const uint32_t*>(&y);
    }
    static __device__ __forceinline__ void unpack(const uint4& u, float (&x)[W])
    {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (TYPE == F3D_BF16) {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            } else {
                const two h = *reinterpret_cast<const two*>(&w[i]);
                x[2 * i] = (float)h[0];
                x[2 * i + 1] = (float)h[1];
            }
        }
    }
    static __device__ __forceinline__ uint4 pack(const float (&x)[W])
    {
        return make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
    }
};

template <>
struct Elems<F3D_BF16> : Elems16<__bf16, F3D_BF16> {};
template <>
struct Elems<F3D_F16> : Elems16<_Float16, F3D_F16> {};

constexpr int elem_bytes(int type) { return type == F3D_F32 ? 4 : 2; }

}  // namespace

}  // namespace f3d
