// What the kernels of a stage's operators share: element types, rounding, sums over a wavefront.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "harp.h"

namespace harp {
namespace ops {

constexpr int kWave = 64;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Elements as they are stored and as they are computed with.  Conversions round to nearest, ties to even.
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__bf16 x) { return float(x); }
__device__ __forceinline__ float to_f32(_Float16 x) { return float(x); }

template <typename T> struct Vec4 {                   // 4 elements as one load, where an element may lie
    typedef T type __attribute__((ext_vector_type(4)));
    typedef type loose __attribute__((aligned(sizeof(T))));
};

// Four neighbouring elements.  Memory takes them at any alignment of the elements, with the same instruction.
template <typename T> __device__ __forceinline__ f32x4 load4(const T *p) {
    const typename Vec4<T>::type v = *reinterpret_cast<const typename Vec4<T>::loose *>(p);
    return f32x4{to_f32(v.x), to_f32(v.y), to_f32(v.z), to_f32(v.w)};
}
// `past`: not kept in the caches, for what is larger than they are.  The empty statements keep the compiler from making one
// store of the two, which it does by dropping what tells them apart.
template <int ALIGN, typename V> __device__ __forceinline__ void store_as(void *to, V v, bool past) {
    typedef V Loose __attribute__((aligned(ALIGN)));
    Loose *p = static_cast<Loose *>(to);
    if (past) {
        asm volatile("");
        __builtin_nontemporal_store(v, p);
        asm volatile("");
    } else {
        *p = v;
    }
}
template <typename T> __device__ __forceinline__ void store4(T *p, f32x4 v, bool past = false) {
    const typename Vec4<T>::type o = {T(v.x), T(v.y), T(v.z), T(v.w)};
    store_as<int(sizeof(T))>(p, o, past);
}

// A value of 16 lanes that a rotation of theirs brings (DPP), and one lane's value for all.
template <int CTRL> __device__ __forceinline__ uint32_t rotated(uint32_t x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xF, 0xF, true); }
template <int CTRL> __device__ __forceinline__ float rotated(float x) { return __uint_as_float(rotated<CTRL>(__float_as_uint(x))); }
__device__ __forceinline__ uint32_t lane_of(uint32_t x, int lane) { return __builtin_amdgcn_readlane(x, lane); }
__device__ __forceinline__ float lane_of(float x, int lane) { return __uint_as_float(lane_of(__float_as_uint(x), lane)); }
constexpr int kRotate8 = 0x128, kRotate4 = 0x124, kRotate2 = 0x122, kRotate1 = 0x121;      // row_ror

// Sum over 16 lanes, the same bits in each: a tree of rotations.
__device__ __forceinline__ float sum16(float x) {
    x += rotated<kRotate8>(x);
    x += rotated<kRotate4>(x);
    x += rotated<kRotate2>(x);
    return x + rotated<kRotate1>(x);
}
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }
// Largest of a wavefront's values.
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
    x = larger(x, rotated<kRotate8>(x));
    x = larger(x, rotated<kRotate4>(x));
    x = larger(x, rotated<kRotate2>(x));
    x = larger(x, rotated<kRotate1>(x));
    return larger(larger(lane_of(x, 0), lane_of(x, 16)), larger(lane_of(x, 32), lane_of(x, 48)));
}

// Bytes of an element, 0 for a type that there is none of.
inline int type_bytes(int type) { return type == HARP_F32 ? 4 : type == HARP_BF16 || type == HARP_F16 ? 2 : 0; }
inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

}  // namespace ops
}  // namespace harp
