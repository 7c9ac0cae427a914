// Attention of drafted tokens that form trees: the entry point, and the kernels whose new tokens see what their masks say.
#include "attention.hpp"

using namespace aweq;

extern "C" int aweq_tree_attention(const void* q, aweq_dtype dt, int64_t T, int64_t Hq, int64_t D, int64_t ldq,
                                   const void* k_cache, const void* v_cache, const float* k_step, const float* v_step, aweq_dtype cache_dt,
                                   int64_t pages, int64_t page_size, int64_t Hk, const int32_t* prefix_table, int64_t prefix_len,
                                   const int32_t* table, int64_t table_ld, const int32_t* lens, const int32_t* q_start, int64_t B,
                                   int64_t max_len, int64_t max_q, const uint64_t* mask, int64_t mask_ld, float scale, void* out, int64_t ldo, float* lse,
                                   void* ws, size_t ws_bytes, uint32_t* status, void* stream)
{
    return attn::attend_call<true>(q, dt, T, Hq, D, ldq, k_cache, v_cache, k_step, v_step, cache_dt, pages, page_size, Hk, prefix_table, prefix_len, table, table_ld,
                                   lens, q_start, B, max_len, max_q, mask, mask_ld, scale, out, ldo, lse, ws, ws_bytes, status, stream);
}
