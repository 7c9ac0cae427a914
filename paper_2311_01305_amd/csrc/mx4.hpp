// Microscaled 4-bit floating point (the header defines format and layout): places of codes and scales, and a block's codes, shared by the quantizer and by
// the products that quantise their tokens.
#pragma once
#include "wide_unit.hpp"

namespace aweq {

constexpr int kMxBlock = 32;                      // values of a scale
constexpr int kMxPanel = 128;                     // values of a panel: 64 bytes of codes a row
constexpr int kMxGroup = 4;                       // panels whose scales are 16 bytes a row
__host__ __device__ inline int64_t mx_panels(int64_t K) { return (K + kMxPanel - 1) / kMxPanel; }
__host__ __device__ inline int64_t mx_groups(int64_t K) { return (K + kMxPanel * kMxGroup - 1) / (kMxPanel * kMxGroup); }
// byte of block b of a panel in a row's 16 (and p % 4 on top)
__host__ __device__ inline int mx_scale_place(int b) { return ((b & 1) * 2 + (b >> 1)) * 4; }

inline bool mx_shape_ok(int64_t rows, int64_t K) { return rows > 0 && rows < (1ll << 31) && K > 0 && K <= (1 << 20) && K % kMxBlock == 0; }

// e + 127 of a block whose largest magnitude has these bits; 255: not finite
__device__ __forceinline__ uint32_t mx_scale(uint32_t most)
{
    const uint32_t e = most >> 23;
    return e == 255u ? 255u : e > 2u ? e - 2u : 0u;
}

// Eight values x times `factor`, a quarter of a block whose other quarters the lane's neighbours in a group of four have: their codes, and the block's scale
template <bool FACTOR, class E>
__device__ __forceinline__ uint32_t mx_unit(const Unit<E>& u, const float factor[8], uint32_t& scale)
{
    float x[8], top = 0.0f;       // (a NaN stays one)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        x[e] = FACTOR ? (float)u[e] * factor[e] : (float)u[e];
        top = __builtin_elementwise_maximum(top, __builtin_fabsf(x[e]));
    }
    uint32_t most = __float_as_uint(top) & 0x7fffffffu;
    most = max(most, (uint32_t)partner<0>((int)most));
    most = max(most, (uint32_t)partner<1>((int)most));
    scale = mx_scale(most);
    uint32_t by = scale << 23;
    if (__builtin_amdgcn_ballot_w64(most < (27u << 23)) != 0) {
        // subnormal numbers among values or scales (below 2^-100 there may be some): both brought up by 2^64
        const bool low = most < (27u << 23);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = low ? x[e] * 0x1p64f : x[e];
        by = low ? (scale + 64u) << 23 : by;
    }
    // v_cvt_scalef32_pk_fp4_f32: x over the scale, to the nearest, ties to the even code, at most 6
    const float step = __uint_as_float(by);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], step, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], step, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], step, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], step, 3);
    return scale == 255u ? 0u : w;
}

// What the products read and write
struct MxArgs {
    const uint8_t *a, *a_scale;    // tokens
    const uint8_t *b, *b_scale;    // weight
    int64_t T, N, K;
    const float* bias;
    void* out;
    int out_kind;                  // kMx*
    int64_t ldo;
    uint32_t* status;
};
enum { kMxF32 = 0, kMxF16 = 1, kMxBf16 = 2 };

// four consecutive outputs of a token
__device__ __forceinline__ void mx_store(const MxArgs& g, int64_t t, int64_t n, const float y[4])
{
    if (g.out_kind == kMxF16) {
        typedef _Float16 h4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<h4*>(reinterpret_cast<_Float16*>(g.out) + t * g.ldo + n) = h4{(_Float16)y[0], (_Float16)y[1], (_Float16)y[2], (_Float16)y[3]};
    } else if (g.out_kind == kMxBf16) {
        typedef __bf16 b4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<b4*>(reinterpret_cast<__bf16*>(g.out) + t * g.ldo + n) = b4{(__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]};
    } else {
        *reinterpret_cast<Float4*>(reinterpret_cast<float*>(g.out) + t * g.ldo + n) = Float4{{y[0], y[1], y[2], y[3]}};
    }
}

int check_quant_mx4(const void* X, aweq_dtype dt, int64_t rows, int64_t K, int64_t ldx, const float* factor, const uint8_t* codes, const uint8_t* scales);
int launch_quant_mx4(const void* X, aweq_dtype dt, int64_t rows, int64_t K, int64_t ldx, const float* factor, uint8_t* codes, uint8_t* scales,
                     uint32_t* status, hipStream_t st);

}  // namespace aweq
