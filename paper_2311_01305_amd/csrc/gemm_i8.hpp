// Arguments of the int8 GEMM kernels, and the forms for fewer tokens (gemm_i8_few.hip, gemm_i8_mid.hip) that
// aweq_w8a8_gemm chooses from.
#pragma once
#include "tile_walk.hpp"

namespace aweq {

enum { kOutF32 = 0, kOutF16 = 1, kOutBf16 = 2 };   // (bfloat16: products with a quantizer a token only)

struct GemmArgs : TileWalk {
    const int8_t* A;   // xq [T x K], K-panel layout
    const int8_t* B;   // wq [N x K], K-panel layout
    int64_t T, N, K;
    int32_t* out_i32;
    void* out_deq;
    int out_f16;       // kOut*
    int64_t ldo;
    long long* colsum_acc;
    const float* act_step;    // one, or one for each token
    const int32_t* act_zero;
    const float* step_w;
    const int32_t* zero_w;
    const int32_t* rowsum_x;
    const int32_t* rowsum_w;
    const float* bias;
    int w_per_tensor;  // step_w / zero_w hold one entry for the whole weight instead of one per output channel
    // fused epilogues on the de-quantised binary16 output y (the next layer's calibration input)
    int act;                    // 0: none, 1: ReLU before y is rounded
    uint32_t* ykeys;            // [2 N] order-preserving keys of the column minimum / maximum of y
    long long* yfix;            // [N] column sums of y in units of 2^-24 (exact: y is binary16)
    const float* next_inv_s;    // [N] the next layer's 1 / s, Step and Z: y is quantised with them
    const float* next_step;
    const int32_t* next_zero;
    int8_t* yq;                 // [T x N] codes of y, K-panel layout (panels of 64 output channels)
    int32_t* rowsum_y;          // [T]
    long long* colsum_yq;       // [N]
    uint32_t* status;
};

// Several weights of N channels each that multiply the same codes, in one launch of the tiled kernel: the tile columns of one after the other's
// (TileWalk's), each weight with its own operands and output; B, out_deq, step_w, zero_w, rowsum_w and bias above are not read.
constexpr int kGroupMost = 4;
struct GroupArgs : GemmArgs {
    struct Member {
        const int8_t* B;
        void* out_deq;
        const float* step_w;
        const int32_t* zero_w;
        const int32_t* rowsum_w;
        const float* bias;
    } m[kGroupMost];
    int member_tiles;   // tile columns of a weight
};

// The binary16 outputs of n weights of N channels (g: what they share; K, T and A among it) in one launch, where it is modelled to take less than a
// launch each; AWEQ_ERR_SHAPE, and nothing launched, where not
int launch_gemm_i8_group(GroupArgs& g, int n, hipStream_t st);

// The few-token kernel's tile for a shape, and what it is modelled to take in the unit of kTiledRoundCost
struct FewPlan {
    int tile;      // index of the instantiation
    double cost;
};
FewPlan plan_few(int64_t T, int64_t N);
int launch_gemm_i8_few(const GemmArgs& g, const FewPlan& p, hipStream_t st, bool tokens = false);   // tokens: act_step and act_zero for each token

// The same for at most kQuantTokens binary16 / binary32 tokens that the launch quantises itself (what the activation quantizer would
// write goes to xq and rowsum_x; g.A and g.rowsum_x are not read)
struct QuantIn {
    const void* X;
    int64_t ldx;
    const float* inv_s;
    int8_t* xq;
    int32_t* rowsum_x;
};
struct TokenIn : QuantIn {   // a quantizer a token, which the launch finds; inv_s may be null
    float* step;
    int32_t* zero;
};
int launch_gemm_i8_few_quant(const GemmArgs& g, const FewPlan& p, const QuantIn& in, bool f16, hipStream_t st);
int launch_gemm_i8_few_tokens(const GemmArgs& g, const FewPlan& p, const TokenIn& in, bool f16, hipStream_t st);   // binary16 or bfloat16 tokens
constexpr int kQuantTokens = 4;
constexpr int64_t kQuantFewBytes = 16384;   // codes such a launch may hold

// The same of the kernel for some hundred tokens (gemm_i8_mid.hip)
struct MidPlan {
    bool square;   // 128 x 128 tiles instead of 64 x 128
    double cost;
};
MidPlan plan_mid(int64_t T, int64_t N);
int launch_gemm_i8_mid(const GemmArgs& g, const MidPlan& p, hipStream_t st, bool tokens = false);

// The output of a product whose tokens have scales of their own: acc - Z'x A - Z'w rowsum_x, A = rowsum_w - K Z'w, in wrap-around 32 bits (nzw
// = -Z'w), and its scaling, the same in every form: in fp64 (the steps' product is exact there, and a bias may cancel what it is added to), rounded to fp32 and
// from there to a 16-bit output
__device__ __forceinline__ int token_integer(int acc, int zx, unsigned a, int nzw, int rowsum_x)
{
    return (int)((unsigned)acc - (unsigned)zx * a + (unsigned)nzw * (unsigned)rowsum_x);
}
// a token's Z' = Z - 128; Z outside [0, 255] is reported and clamped
__device__ __forceinline__ int token_zero(int zero, uint32_t& est)
{
    const int z = min(max(zero, 0), 255);
    if (z != zero) est |= AWEQ_ST_ZEROPOINT;
    return z - 128;
}
__device__ __forceinline__ float token_scaled(int i, float sx, float sw, float bias) { return (float)__builtin_fma((double)i, (double)sx * (double)sw, (double)bias); }

// Time of one round of workgroups at K = 8192 (us; every kernel's time is close to proportional to K): 256 tiles of 256 x 256
constexpr double kTiledRoundCost = 100.0;
constexpr double kHalfTileCost = 0.57;   // the same of 128 x 256 tiles, against that (0.55 - 0.58 from K = 256 to 16384)

}  // namespace aweq
