// Forms of the product in microscaled 4-bit floating point that aweq_mx4_gemm_tokens chooses from.
#pragma once
#include "mx4.hpp"
#include "tile_walk.hpp"

namespace aweq {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));

// A matrix instruction takes eight registers of an operand; a 4-bit one is in the first four, and the others are not read
__device__ __forceinline__ v8i mx_operand(const v4i& v) { return __builtin_shufflevector(v, v, 0, 1, 2, 3, -1, -1, -1, -1); }

// Tokens that a launch quantises itself: at most kMxQuantTokens, of kMxQuantBytes of codes in all
struct MxIn {
    const void* X;
    int64_t ldx;
    const float* factor;
    uint8_t *xq, *x_scale;
};
constexpr int kMxQuantTokens = 4;
constexpr int64_t kMxQuantBytes = 16384;

// Tiles of 256 tokens (half: 128) x 256 channels; rounds of 256 workgroups with the larger ones
struct MxTiledPlan {
    bool half;
    double rounds;
    int rc;
};
MxTiledPlan plan_mx4_tiled(int64_t T, int64_t N, int64_t K);
int launch_mx4_tiled(const MxArgs& g, const MxTiledPlan& p, hipStream_t st);

int launch_mx4_few(const MxArgs& g, hipStream_t st);
int launch_mx4_few_quant(const MxArgs& g, const MxIn& in, aweq_dtype dt, hipStream_t st);

}  // namespace aweq
