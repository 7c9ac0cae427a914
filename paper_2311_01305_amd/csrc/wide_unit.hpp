// Eight consecutive values of a row in any of the float types: one unit of 16 bytes (binary32: two).
#pragma once
#include "common.hpp"

namespace aweq {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

template <class E> struct UnitOf;
template <> struct UnitOf<_Float16> { typedef f16x8 type; };
template <> struct UnitOf<__bf16> { typedef bf16x8 type; };
template <> struct UnitOf<float> { typedef f32x8 type; };
template <class E> using Unit = typename UnitOf<E>::type;

// (16-byte alignment is all that a row promises: binary32 units are two quads)
template <class E>
__device__ __forceinline__ Unit<E> load_unit(const E* p)
{
    if constexpr (sizeof(E) == 4) {
        const Float4 a = *reinterpret_cast<const Float4*>(p), b = *reinterpret_cast<const Float4*>(p + 4);
        return f32x8{a.f[0], a.f[1], a.f[2], a.f[3], b.f[0], b.f[1], b.f[2], b.f[3]};
    } else {
        return *reinterpret_cast<const Unit<E>*>(p);
    }
}

template <class E>
__device__ __forceinline__ void store_unit(E* p, const float x[8])
{
    if constexpr (sizeof(E) == 4) {
        *reinterpret_cast<Float4*>(p) = Float4{{x[0], x[1], x[2], x[3]}};
        *reinterpret_cast<Float4*>(p + 4) = Float4{{x[4], x[5], x[6], x[7]}};
    } else {
        Unit<E> u;
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = (E)x[i];
        *reinterpret_cast<Unit<E>*>(p) = u;
    }
}

// The same past the caches (16-bit types): for calls whose data does not fit them anyway
template <class E>
__device__ __forceinline__ Unit<E> stream_unit(const E* p)
{
    typedef int v4 __attribute__((ext_vector_type(4)));
    if constexpr (sizeof(E) == 4) return load_unit(p);
    else return __builtin_bit_cast(Unit<E>, __builtin_nontemporal_load(reinterpret_cast<const v4*>(p)));
}
template <class E>
__device__ __forceinline__ void stream_unit(E* p, const float x[8])
{
    typedef int v4 __attribute__((ext_vector_type(4)));
    if constexpr (sizeof(E) == 4) {
        store_unit(p, x);
    } else {
        Unit<E> u;
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = (E)x[i];
        __builtin_nontemporal_store(__builtin_bit_cast(v4, u), reinterpret_cast<v4*>(p));
    }
}

template <class E>
__device__ __forceinline__ void widen(const Unit<E>& u, float x[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)u[i];
}

}  // namespace aweq
