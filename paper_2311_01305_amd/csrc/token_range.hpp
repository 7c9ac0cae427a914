// A token's range, its Step and Z, and the codes of eight of its values: shared by the token quantizer and the few-token int8 GEMM that
// quantises its own input.
#pragma once
#include "act_unit.hpp"
#include "wide_unit.hpp"

namespace aweq {

// 1 / s of eight channels, widened values times them where there are any (FOLD)
template <bool FOLD>
__device__ __forceinline__ void load_scales(const float* inv_s, int unit, float is[8])
{
    if constexpr (FOLD) {
        const f32x8 v = load_unit(inv_s + (int64_t)unit * 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) is[e] = v[e];
    }
}
template <bool FOLD, class E>
__device__ __forceinline__ float token_value(const Unit<E>& u, const float is[8], int e)
{
    // (with + 0 a binary16 value is widened by the same instruction; it changes nothing but the sign of a zero)
    if constexpr (FOLD) return __builtin_fmaf((float)u[e], is[e], 0.0f);
    return (float)u[e];
}

// Extremes of eight values and what was seen before.  IEEE maximum and minimum: a NaN stays one, so that the token's range tells of it
template <bool FOLD, class E>
__device__ __forceinline__ void token_extremes(const Unit<E>& u, const float is[8], float& lo, float& hi)
{
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const float a = token_value<FOLD, E>(u, is, e), b = token_value<FOLD, E>(u, is, e + 1);
        lo = __builtin_elementwise_minimum(__builtin_elementwise_minimum(lo, a), b);
        hi = __builtin_elementwise_maximum(__builtin_elementwise_maximum(hi, a), b);
    }
}

// Eq. 2 for a range that contains 0.  A range so small that its 255th part is subnormal would leave steps of too few digits for a zero point in
// [0, 255]: clamped (its values are below 1e-36)
__device__ __forceinline__ void token_params(float lo, float hi, float& step, int& zero, uint32_t& st)
{
    if (!(fabsf(lo) < INFINITY && fabsf(hi) < INFINITY)) st |= AWEQ_ST_NONFINITE;
    float s = (hi - lo) / 255.0f;
    if (isinf(s)) s = hi / 255.0f - lo / 255.0f;   // (binary32 values whose range is beyond it)
    if (!(s > 0.0f) || isinf(s)) s = 1.0f;
    step = s;
    zero = (int)fminf(fmaxf(-rintf(lo / s), 0.0f), 255.0f);
}

// Eq. 1 on eight values: packed codes u - 128, their sum added to rs.  Quotients are at most 255 or so, so the screened quotient of the activation
// quantizer (whose header explains it) holds wherever Step's exponent allows its reciprocal; its test for a tie decides between that and the division.
template <bool FOLD, class E>
__device__ __forceinline__ uint2 token_unit(const Unit<E>& u, const float is[8], const ActParams& p, int& rs)
{
    const float zf = (float)p.zero;
    float n[8], dmax = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float q = __builtin_fmaf(token_value<FOLD, E>(u, is, e), p.rstep, zf);
        n[e] = rintf(q);
        dmax = fmaxf(dmax, fabsf(q - n[e]));
    }
    if (!p.screen || !(dmax <= p.thr)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) n[e] = rintf(token_value<FOLD, E>(u, is, e) / p.step) + zf;
    }
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e >> 2] = __builtin_amdgcn_cvt_pk_u8_f32(n[e], e & 3, w[e >> 2]);   // (clamps to 0 .. 255)
    w[0] ^= 0x80808080u;
    w[1] ^= 0x80808080u;
    rs = __builtin_amdgcn_sdot4((int)w[0], 0x01010101, rs, false);
    rs = __builtin_amdgcn_sdot4((int)w[1], 0x01010101, rs, false);
    return make_uint2(w[0], w[1]);
}

}  // namespace aweq
