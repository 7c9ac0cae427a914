// Product in microscaled 4-bit floating point  out[t,n] = sum_k x[t,k] w[n,k] + bias[n]: the entry point and its choice among the forms.
#include "gemm_mx4.hpp"

using namespace aweq;

extern "C" int aweq_mx4_gemm_tokens(const void* X, aweq_dtype x_dt, int64_t T, int64_t K, int64_t ldx, const float* factor, uint8_t* xq, uint8_t* x_scale,
                                    const uint8_t* wq, const uint8_t* w_scale, int64_t N, const float* bias, void* out, aweq_dtype out_dt, int64_t ldo,
                                    uint32_t* status, void* stream)
{
    if (!xq || !x_scale || !wq || !w_scale || !out) return AWEQ_ERR_NULL;
    if (out_dt != AWEQ_F32 && out_dt != AWEQ_F16 && out_dt != AWEQ_BF16) return AWEQ_ERR_DTYPE;
    if (!mx_shape_ok(T, K) || !mx_shape_ok(N, K) || (N % 4) != 0 || ldo < N || (ldo % 4) != 0) return AWEQ_ERR_SHAPE;
    if (X) {
        const int rc = check_quant_mx4(X, x_dt, T, K, ldx, factor, xq, x_scale);
        if (rc != AWEQ_OK) return rc;
    }
    if (!aligned16(xq) || !aligned16(x_scale) || !aligned16(wq) || !aligned16(w_scale) || !aligned16(out) || (bias && !aligned16(bias))) return AWEQ_ERR_ALIGN;
    MxArgs g = {};
    g.a = xq; g.a_scale = x_scale; g.b = wq; g.b_scale = w_scale;
    g.T = T; g.N = N; g.K = K;
    g.bias = bias; g.out = out; g.ldo = ldo; g.status = status;
    g.out_kind = out_dt == AWEQ_F16 ? kMxF16 : out_dt == AWEQ_BF16 ? kMxBf16 : kMxF32;
    hipStream_t st = as_stream(stream);
    if (X && T <= kMxQuantTokens && T * mx_panels(K) * 64 <= kMxQuantBytes) return launch_mx4_few_quant(g, MxIn{X, ldx, factor, xq, x_scale}, x_dt, st);
    if (X) {
        const int rc = launch_quant_mx4(X, x_dt, T, K, ldx, factor, xq, x_scale, status, st);
        if (rc != AWEQ_OK) return rc;
    }
    const MxTiledPlan tiled = plan_mx4_tiled(T, N, K);
    if (T > 64 && tiled.rc == AWEQ_OK) return launch_mx4_tiled(g, tiled, st);
    return launch_mx4_few(g, st);
}
