// Forms of the product in microscaled 4-bit floating point that aweq_mx4_gemm_tokens chooses from.
#pragma once
#include "mx4.hpp"
#include "tile_walk.hpp"

namespace aweq {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));

// A matrix instruction takes eight registers of an operand; a 4-bit one is in the first four, and the others are not read
__device__ __forceinline__ v8i mx_operand(const v4i& v) { return __builtin_shufflevector(v, v, 0, 1, 2, 3, -1, -1, -1, -1); }

// Tokens that a launch quantises itself
struct MxIn {
    const void* X;
    int64_t ldx;
    const float* factor;
    uint8_t *xq, *x_scale;
};

// Tiles of 64 mi tokens x 256 channels: how many, and in how many rounds of 256 workgroups; false: too many for a launch
bool plan_mx4_tiled(int64_t T, int64_t N, int64_t K, int mi, int64_t& tiles, int64_t& rounds);
int launch_mx4_tiled(const MxArgs& g, int mi, hipStream_t st);
// Some hundred tokens: tiles of 64 x 128, or 128 x 128
int launch_mx4_mid(const MxArgs& g, bool square, hipStream_t st);

// Few tokens: tiles of 16 tt tokens x 16 nt channels
int launch_mx4_few(const MxArgs& g, int tt, int nt, hipStream_t st);
// whether the launch for tiles of 16 tokens quantises them itself
bool mx4_few_quantises(int64_t T, int64_t N, int64_t K, int nt);
int launch_mx4_few_quant(const MxArgs& g, const MxIn& in, aweq_dtype dt, int nt, hipStream_t st);

int mx4_form(int64_t T, int64_t N, int64_t K);

}  // namespace aweq
