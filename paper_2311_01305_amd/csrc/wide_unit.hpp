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

template <class E>
__device__ __forceinline__ void widen(const Unit<E>& u, float x[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)u[i];
}

}  // namespace aweq
