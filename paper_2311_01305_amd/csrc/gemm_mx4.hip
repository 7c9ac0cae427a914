// Product in microscaled 4-bit floating point  out[t,n] = sum_k x[t,k] w[n,k] + bias[n]: the entry point and its choice among the forms.
#include "gemm_mx4.hpp"

namespace aweq {

// What each form is modelled to take (us), from its time with a workgroup on few and on all of the 256 compute units; all are near a constant and a share of the
// panels.  No form is below the read of the weight.  us, codes given, bfloat16 output, weights that are in no cache:
//   tokens          1     16    32    64     128    256    333    512    1024   2048   4096
//   4096 x 4096     4.3   4.5   5.0   6.1    7.3   10.4   11.6   12.6    16.5   21.6   34.1
//   11008 x 4096    6.9   7.5   9.4  10.7   13.2   17.1   19.1   19.7    27.4   51.4   93.0
//   8192 x 8192     8.3   8.5   9.9  11.9   19.7   20.9   26.3   27.4    36.6   59.7   114
//   22016 x 8192   19.0  19.6  21.4  23.5   32.3   36.1   43.2   48.0    102    176    331      (96 MB: 5 TB/s at one token; 4.5 PFLOP/s at 4096)
struct MxPlan {
    enum { kFew, kMid, kTiled } form;
    int a, b;          // few: tt, nt; mid: square; tiled: mi
    double us;
};

static MxPlan plan_mx4(int64_t T, int64_t N, int64_t K)
{
    const double panels = (double)mx_panels(K), read = 2.2 + (double)N * (double)K * (17.0 / 32.0) / 5.2e6;
    MxPlan best = {MxPlan::kFew, 4, 4, 1e300};
    auto offer = [&](int form, int a, int b, double us) {
        if (us < read) us = read;
        if (us < best.us) best = {static_cast<decltype(best.form)>(form), a, b, us};
    };
    auto rounds = [&](int bm, int bn) { return (double)cdiv(cdiv(T, bm) * cdiv(N, bn), 256); };
    // few tokens: a round of workgroups in us a panel; two or more share a compute unit (one token's, two tokens' tiles)
    struct { int tt, nt; double us; } const few[] = {{1, 2, 0.085}, {1, 1, 0.045}, {2, 1, 0.066}, {2, 2, 0.1}, {4, 2, 0.14}, {4, 4, 0.22}};
    for (const auto& f : few)
        if (T <= 16 * f.tt * 8 && N < (1 << 26)) offer(MxPlan::kFew, f.tt, f.nt, 2.2 + panels * f.us * rounds(16 * f.tt, 16 * f.nt));
    // some hundred: rounds after the first take longer, since nothing of one overlaps with the next
    if (T > 16 && T <= 2048 && N < (1 << 23)) {
        offer(MxPlan::kMid, 0, 0, 5.0 + panels * (0.19 + 0.26 * (rounds(64, 128) - 1.0)));
        offer(MxPlan::kMid, 1, 0, 5.0 + panels * (0.33 + 0.42 * (rounds(128, 128) - 1.0)));
    }
    // many: a tile takes 0.11 + 0.105 mi us a panel with most compute units idle, 1.74 times that with none
    for (int mi = 4; mi >= 1; --mi) {
        int64_t tiles = 0, turns = 0;
        if (!plan_mx4_tiled(T, N, K, mi, tiles, turns)) continue;
        const double last = (double)(tiles - (turns - 1) * 256) / 256.0, busy = last > 0.4 ? 1.0 + 0.74 * (last - 0.4) / 0.6 : 1.0;
        offer(MxPlan::kTiled, mi, 0, 5.0 + panels * (0.11 + 0.105 * mi) * (1.74 * (double)(turns - 1) + (busy < 1.74 ? busy : 1.74)));
    }
    return best;
}

// 100 form + 10 a + b of the form that a shape is given to (the tests name the one that each of their shapes is meant for)
int mx4_form(int64_t T, int64_t N, int64_t K)
{
    const MxPlan p = plan_mx4(T, N, K);
    return 100 * p.form + 10 * p.a + p.b;
}

}  // namespace aweq

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
    const MxPlan p = plan_mx4(T, N, K);
    if (X && p.form == MxPlan::kFew && p.a == 1 && mx4_few_quantises(T, N, K, p.b))
        return launch_mx4_few_quant(g, MxIn{X, ldx, factor, xq, x_scale}, x_dt, p.b, st);
    if (X) {
        const int rc = launch_quant_mx4(X, x_dt, T, K, ldx, factor, xq, x_scale, status, st);
        if (rc != AWEQ_OK) return rc;
    }
    if (p.form == MxPlan::kFew) return launch_mx4_few(g, p.a, p.b, st);
    if (p.form == MxPlan::kMid) return launch_mx4_mid(g, p.a != 0, st);
    return launch_mx4_tiled(g, p.a, st);
}
