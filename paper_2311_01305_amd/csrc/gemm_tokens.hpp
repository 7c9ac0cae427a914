// The token quantizer's launch and argument checks (quant_token.hip), for the product that runs it first.
#pragma once
#include "gemm_i8.hpp"

namespace aweq {

int check_quant_tokens(const void* X, aweq_dtype dt, int64_t T, int64_t K, int64_t ldx, const float* inv_s, const int8_t* xq, const float* step,
                       const int32_t* zero, const int32_t* rowsum);
int launch_quant_tokens(const void* X, aweq_dtype dt, int64_t T, int64_t K, int64_t ldx, const float* inv_s, int8_t* xq, float* step, int32_t* zero,
                        int32_t* rowsum, uint32_t* status, hipStream_t st);

}  // namespace aweq
