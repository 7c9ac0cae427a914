// Attention behind a shared prefix: the entry point, its scratch memory, and the kernels whose new tokens see those before them.
#include "attention.hpp"

using namespace aweq;

extern "C" size_t aweq_prefix_attention_ws(int64_t T, int64_t Hq, int64_t Hk, int64_t D, int64_t B, int64_t max_q, int64_t prefix_len, int64_t max_len)
{
    if (!attn::shapes_ok(T, Hq, Hk, D, B, max_q, prefix_len, max_len)) return 0;
    max_q = max_q < T ? max_q : T;
    int parts = 1;
    for (const bool codes : {false, true}) {
        const int n = attn::plan(D, codes, T, Hq, Hk, B, max_q, prefix_len, max_len).parts();
        if (n > parts) parts = n;
    }
    return parts > 1 ? (size_t)parts * (size_t)(T * Hq) * (size_t)(D * 4 + 8) : 0;
}

extern "C" size_t aweq_prefix_attention_ws_most(int64_t T, int64_t Hq, int64_t Hk, int64_t D, int64_t B, int64_t max_q, int64_t prefix_len, int64_t max_len)
{
    if (!attn::shapes_ok(T, Hq, Hk, D, B, max_q, prefix_len, max_len)) return 0;
    if (prefix_len == 0 && max_len <= attn::kWideLeast) return 0;
    const int64_t rows = T * Hq, own = attn::most_parts(rows, max_len + prefix_len);   // (a sequence's rows may take the prefix along)
    return (size_t)(attn::most_parts(rows, prefix_len) + (own > rows ? own : rows)) * (size_t)(D * 4 + 8);
}

extern "C" int aweq_prefix_attention(const void* q, aweq_dtype dt, int64_t T, int64_t Hq, int64_t D, int64_t ldq,
                                     const void* k_cache, const void* v_cache, const float* k_step, const float* v_step, aweq_dtype cache_dt,
                                     int64_t pages, int64_t page_size, int64_t Hk, const int32_t* prefix_table, int64_t prefix_len,
                                     const int32_t* table, int64_t table_ld, const int32_t* lens, const int32_t* q_start, int64_t B,
                                     int64_t max_len, int64_t max_q, float scale, void* out, int64_t ldo, float* lse,
                                     void* ws, size_t ws_bytes, uint32_t* status, void* stream)
{
    return attn::attend_call<false>(q, dt, T, Hq, D, ldq, k_cache, v_cache, k_step, v_step, cache_dt, pages, page_size, Hk, prefix_table, prefix_len, table, table_ld,
                                    lens, q_start, B, max_len, max_q, nullptr, 0, scale, out, ldo, lse, ws, ws_bytes, status, stream);
}
