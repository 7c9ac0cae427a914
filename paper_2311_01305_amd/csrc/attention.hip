// Attention of a batch over a shared prefix and over each sequence's own pages of the cache.
//
//   out = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q k_j - m),  m the running maximum: one pass over the keys, any range of them by itself.
//
// A range of keys belongs to all tokens (the prefix) or to one sequence's.  For a key head the rows that multiply it are its G = Hq / Hk query heads
// of each of those tokens, row r = token r / G, head r % G: the prefix is read once for all rows of the batch.
//
// A wavefront has 16 MT rows and takes the keys in tiles.  It forms S^T = K Q^T and O^T = V^T P^T with v_mfma_f32_16x16x32: the weights' side of
// both products comes from the cache, a lane has one row of Q in its column, so that maximum and sum of a row need two exchanges across the
// wavefront, and the four consecutive keys that a lane holds of a 16 x 16 tile of S^T are, two tiles at a time, the eight it has to supply of P^T: the order
// of the keys inside a product is free as long as V^T's is the same.  V^T's is made by the transposing LDS reads.
//
// Tiles of K and V are filled by LDS-DMA loads, 16 bytes a lane, two tiles in turn.  16 neighbouring tokens lie in one page (its size is a
// multiple of 16), so a group of 16 rows has one base address.  Chunks of 16 bytes are XOR swizzled by choosing which one a lane fetches.
// A tile's rows past the range repeat its last token: what a page holds past the range is never read.
//
// WR = wavefronts that share a tile and have rows of their own (many rows: the prefix, prompts); WR = 1: every wavefront has tiles of its own and all
// have the same 16 rows (decoding: one token's heads), whose results meet in LDS at the end.
//
// An 8-bit cache is multiplied as binary16 codes.  The step of a key goes to its score.  The step of a value goes into the exponent:
// p' = exp(s + log step - m') is at most 1 and is what multiplies the codes; the sum takes p' / step back.
#include "wide_unit.hpp"

#include <cmath>
#include <type_traits>

namespace aweq {
namespace attn {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

struct Args {
    const void *q, *k_cache, *v_cache;
    const float *k_step, *v_step;
    const int32_t *prefix_table, *table, *lens, *q_start;
    void* out;
    float* lse;
    float* part_o;      // [part][T Hq][D], not divided by the sum
    float2* part_ml;    // [part][T Hq]: maximum (log2), sum
    uint32_t* status;
    int64_t T, ldq, ldo, table_ld;
    int64_t prefix_len, max_len;
    int64_t page_elts;  // values of one page: Hk page_size D
    int pages, page_size, page_shift;
    int Hq, Hk, G, B, max_q;
    int q_bf16;         // type of q and out (an 8-bit cache: any)
    int parts;          // of a row: 1: the result itself
    int first_part;     // this launch's first part
    int splits;         // this launch's ranges
    int row_tiles;
    float scale_log2e;
};

template <int N>
__device__ __forceinline__ void wait_vm()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// lane i's 16 bytes (4 bytes) land at lds_addr + 16 i (4 i); lds_addr and base wave-uniform
__device__ __forceinline__ void dma16(const char* base, uint32_t off, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds_addr), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void dma4(const float* at, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds_addr), "v"(at) : "memory");
}

// E: type of the cache (int8_t: codes).  M: type of the products
template <class E> struct Mfma;
template <> struct Mfma<_Float16> {
    typedef f16x8 V;
    typedef _Float16 S;
    static __device__ __forceinline__ f32x4 mul(V a, V b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <> struct Mfma<int8_t> : Mfma<_Float16> {};
template <> struct Mfma<__bf16> {
    typedef bf16x8 V;
    typedef __bf16 S;
    static __device__ __forceinline__ f32x4 mul(V a, V b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};

// 8 codes to binary16: the byte u = code + 128 under the exponent of 1024 is 1024 + u
__device__ __forceinline__ f16x8 codes_to_f16(i32x2 w)
{
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    union { uint32_t u[4]; h2 h[4]; f16x8 v; } r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t u = (uint32_t)w[i] ^ 0x80808080u;
        r.u[2 * i] = __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u);
        r.u[2 * i + 1] = __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) r.h[i] = r.h[i] - h2{(_Float16)1152.0f, (_Float16)1152.0f};
    return r.v;
}

template <class E, int D, int WR>
struct Tile {
    static constexpr int kWaves = WR > 1 ? WR : (D == 256 && sizeof(E) == 2 ? 2 : 4);
    static constexpr int kThreads = kWaves * kWave;
    static constexpr int kKeys = WR > 1 ? 64 : 32;
    static constexpr int kRow = D * (int)sizeof(E);            // bytes of a token's head
    static constexpr int kChunks = kRow / 16;
    static constexpr int kHalf = kKeys * kRow;                 // K, then V
    static constexpr bool kSteps = sizeof(E) == 1;
    static constexpr int kStepBytes = kSteps ? kKeys / 16 * 256 : 0;   // of a group of 16 keys: 16 steps of K, 16 of V (and 32 unused)
    static constexpr int kSlot = 2 * kHalf + kStepBytes;
    static constexpr int kStages = 2;
    static constexpr int kRing = kStages * kSlot;              // of the wavefronts that share tiles
    static constexpr int kGroups = kKeys / 16;
    static constexpr int kMine = WR > 1 ? kGroups / WR : kGroups;      // groups of 16 keys that a wavefront fetches
    static constexpr int kLoads = kRow * 16 / 1024;            // load instructions for 16 rows
    static constexpr int kMerge = WR > 1 ? 0 : kWaves * (16 * D * 4 + 128);
    static constexpr int kLds = WR > 1 ? kRing : (kWaves * kRing > kMerge ? kWaves * kRing : kMerge);
};

// Swizzles of the 16-byte chunks of a row: reads of one chunk of 16 rows (K), and the transposing reads of V (binary16: 8 rows x 2 chunks,
// codes: rows 0 - 7 and 16 - 23 of one chunk) fall on different banks
template <int C>
__device__ __forceinline__ int swz_k(int row)
{
    return C >= 16 ? (row & 15) : (row / (16 / C)) & (C - 1);
}
template <int C, bool CODES>
__device__ __forceinline__ int swz_v(int row)
{
    if constexpr (CODES) {
        constexpr int span = C >= 16 ? 1 : 16 / C, low = 8 / span;
        return ((row / span) & (low - 1)) + low * ((row >> 4) & 1);
    } else {
        constexpr int span = C >= 16 ? 1 : 16 / C;
        return 2 * ((row / span) & (8 / span - 1));
    }
}

// PREFIX: the range is the prefix and rows are those of all tokens; else the sequence's own keys.
template <class E, int D, int WR, int MT, bool PREFIX>
__global__ __launch_bounds__((Tile<E, D, WR>::kThreads)) void attention_kernel(Args g)
{
    using TL = Tile<E, D, WR>;
    using M = Mfma<E>;
    using V = typename M::V;
    constexpr int C = TL::kChunks;
    constexpr bool kCodes = TL::kSteps;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
    const int col = lane & 15, grp = lane >> 4;

    // ---- which rows and keys
    unsigned id = blockIdx.x;
    const int split = id % (unsigned)g.splits; id /= (unsigned)g.splits;
    const int row_tile = id % (unsigned)g.row_tiles; id /= (unsigned)g.row_tiles;
    const int kvh = id % (unsigned)g.Hk;
    const int b = id / (unsigned)g.Hk;
    uint32_t est = 0;
    int64_t t0 = 0;
    int tokens, len;
    const int32_t* table;
    if constexpr (PREFIX) {
        tokens = (int)g.T;
        len = (int)g.prefix_len;
        table = g.prefix_table;
    } else {
        int64_t t1;
        if (g.q_start) {
            t0 = g.q_start[b];
            t1 = g.q_start[b + 1];
            if (t0 < 0 || t1 < t0 || t1 > g.T || t1 - t0 > g.max_q) est |= AWEQ_ST_INDEX;
            t0 = min(max(t0, (int64_t)0), g.T);
            t1 = min(max(t1, t0), min(g.T, t0 + g.max_q));
        } else {
            t0 = b;
            t1 = b + 1;
        }
        tokens = (int)(t1 - t0);
        len = g.lens[b];
        const int most = (int)min(g.max_len, g.table_ld * g.page_size);
        if (len < 0 || len > most) est |= AWEQ_ST_INDEX;
        len = min(max(len, 0), most);
        table = g.table + (int64_t)b * g.table_ld;
    }
    const int rows = tokens * g.G;
    const int row0 = row_tile * (16 * MT * WR) + (WR > 1 ? wave * 16 * MT : 0);   // this wavefront's first row
    if (row_tile * (16 * MT * WR) >= rows) {
        if (threadIdx.x == 0) raise_status(g.status, est);
        return;
    }
    // the keys of this range: an equal number of tiles of the splits, up to what the tile's last row sees
    const int last_token = min(((row_tile + 1) * (16 * MT * WR) - 1) / g.G, tokens - 1);
    const int seen = PREFIX ? len : min(len, len - tokens + 1 + last_token);    // (not positive: the row sees none)
    const int per = ((len + g.splits - 1) / g.splits + TL::kKeys - 1) / TL::kKeys * TL::kKeys;
    const int begin = split * per, end = min(min(begin + per, len), seen);

    // ---- Q: column `col` of the wavefront's row tile i, eight values of its head at a time
    V qf[MT][D / 32];
    float row_scale[MT];
    int limit[MT];      // keys that the row sees
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int r = min(row0 + 16 * i + col, rows - 1);
        const int64_t t = t0 + r / g.G;
        limit[i] = PREFIX ? len : min(len, len - tokens + 1 + r / g.G);
        const char* src = reinterpret_cast<const char*>(g.q) + (t * g.ldq + (int64_t)(kvh * g.G + r % g.G) * D) * 2;
        row_scale[i] = g.scale_log2e;
        if (kCodes && g.q_bf16) {
            // bfloat16 queries as binary16: scaled by a power of two, the largest value below 2^15
            float x[D / 32][8], big = 0.0f;
#pragma unroll
            for (int kk = 0; kk < D / 32; ++kk) {
                widen<__bf16>(*reinterpret_cast<const bf16x8*>(src + (kk * 32 + grp * 8) * 2), x[kk]);
#pragma unroll
                for (int j = 0; j < 8; ++j) big = fmaxf(big, fabsf(x[kk][j]));
            }
            big = fmaxf(big, partner<5>(big));
            big = fmaxf(big, partner<4>(big));
            const int e = big > 0.0f ? 14 - ilogbf(big) : 0;
#pragma unroll
            for (int kk = 0; kk < D / 32; ++kk)
#pragma unroll
                for (int j = 0; j < 8; ++j) qf[i][kk][j] = (typename M::S)ldexpf(x[kk][j], e);
            row_scale[i] = ldexpf(g.scale_log2e, -e);
        } else {
#pragma unroll
            for (int kk = 0; kk < D / 32; ++kk) qf[i][kk] = *reinterpret_cast<const V*>(src + (kk * 32 + grp * 8) * 2);
        }
    }

    f32x4 o[MT][D / 16];
    float m[MT], l[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        m[i] = -INFINITY;
        l[i] = 0.0f;
#pragma unroll
        for (int d = 0; d < D / 16; ++d) o[i][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    // ---- the ring
    const int tile_step = WR > 1 ? TL::kKeys : TL::kKeys * TL::kWaves;           // between this wavefront's tiles
    const int first = begin + (WR > 1 ? 0 : wave * TL::kKeys);
    const int tiles = end > first ? (end - first + tile_step - 1) / tile_step : 0;
    char* const ring = lds + (WR > 1 ? 0 : wave * TL::kRing);
    const uint32_t ring_addr = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)ring);
    constexpr int kRowsPerLoad = 1024 / TL::kRow;    // rows of one load instruction
    auto fetch = [&](int tile) {
        const uint32_t slot = ring_addr + (uint32_t)(tile % TL::kStages) * TL::kSlot;
#pragma unroll
        for (int q = 0; q < TL::kMine; ++q) {
            const int group = (WR > 1 ? wave * TL::kMine : 0) + q;
            const int key0 = first + tile * tile_step + group * 16;              // a multiple of 16: the group lies in one page
            const int base_key = min(key0, end - 1);
            int page = __builtin_amdgcn_readfirstlane(table[base_key >> g.page_shift]);
            if ((unsigned)page >= (unsigned)g.pages) { est |= AWEQ_ST_INDEX; page = 0; }
            const int64_t head_row = ((int64_t)page * g.Hk + kvh) << g.page_shift;   // row of the cache where this head's page begins
            const char* const kb = reinterpret_cast<const char*>(g.k_cache) + head_row * TL::kRow;
            const char* const vb = reinterpret_cast<const char*>(g.v_cache) + head_row * TL::kRow;
            const int in_page = g.page_size - 1;
#pragma unroll
            for (int j = 0; j < TL::kLoads; ++j) {
                const int sub = j * kRowsPerLoad + lane / C;                         // row of the 16
                const int row = min(key0 + sub, end - 1) & in_page;
                const int trow = group * 16 + sub;                                   // of the tile: the swizzle's
                const uint32_t at = slot + (uint32_t)(group * 16 * TL::kRow + j * 1024);
                dma16(kb, (uint32_t)(row * TL::kRow + ((lane % C) ^ swz_k<C>(trow)) * 16), at);
                dma16(vb, (uint32_t)(row * TL::kRow + ((lane % C) ^ swz_v<C, kCodes>(trow)) * 16), at + TL::kHalf);
            }
            if constexpr (kCodes) {
                const int row = min(key0 + col, end - 1) & in_page;
                dma4((grp & 1 ? g.v_step : g.k_step) + head_row + row, slot + 2 * TL::kHalf + (uint32_t)group * 256);
            }
        }
    };

    if (tiles > 0) fetch(0);
    for (int tile = 0; tile < tiles; ++tile) {
        wait_vm<0>();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");        // this wavefront's reads of the tile before are done: its slot is filled next
        if constexpr (WR > 1) __builtin_amdgcn_s_barrier();       // and everyone's, and the tile has landed for everyone
        if (tile + 1 < tiles) fetch(tile + 1);
        const char* const kt = ring + (tile % TL::kStages) * TL::kSlot;
        const char* const vt = kt + TL::kHalf;
        const int key0 = first + tile * tile_step;

        // S^T: 16 keys x 16 rows at a time
        f32x4 s[MT][TL::kGroups];
#pragma unroll
        for (int n = 0; n < TL::kGroups; ++n) {
#pragma unroll
            for (int i = 0; i < MT; ++i) s[i][n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            const int row = n * 16 + col;
#pragma unroll
            for (int kk = 0; kk < D / 32; ++kk) {
                V kf;
                if constexpr (kCodes) {
                    const int chunk = kk * 2 + (grp >> 1);
                    kf = codes_to_f16(*reinterpret_cast<const i32x2*>(kt + row * TL::kRow + ((chunk ^ swz_k<C>(row)) * 16) + (grp & 1) * 8));
                } else {
                    kf = *reinterpret_cast<const V*>(kt + row * TL::kRow + (((kk * 4 + grp) ^ swz_k<C>(row)) * 16));
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) s[i][n] = M::mul(kf, qf[i][kk], s[i][n]);
            }
        }

        // scores in units of log2, those past the row's keys minus infinity; the running maximum and sum
        float lv[TL::kGroups][4], rv[TL::kGroups][4], ks[TL::kGroups][4];
        if constexpr (kCodes) {
#pragma unroll
            for (int n = 0; n < TL::kGroups; ++n) {
                const Float4 a = *reinterpret_cast<const Float4*>(kt + 2 * TL::kHalf + n * 256 + grp * 16);
                const Float4 c = *reinterpret_cast<const Float4*>(kt + 2 * TL::kHalf + n * 256 + 64 + grp * 16);
#pragma unroll
                for (int v = 0; v < 4; ++v) { ks[n][v] = a.f[v]; lv[n][v] = __builtin_amdgcn_logf(c.f[v]); rv[n][v] = 1.0f / c.f[v]; }
            }
        }
        V pf[MT][TL::kGroups / 2];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const bool edge = key0 + TL::kKeys > end || (!PREFIX && key0 + TL::kKeys > limit[i]);
            float top = -INFINITY;
#pragma unroll
            for (int n = 0; n < TL::kGroups; ++n)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    float x = s[i][n][v] * row_scale[i];
                    if constexpr (kCodes) x = __builtin_fmaf(x, ks[n][v], lv[n][v]);
                    if (edge) {
                        const int key = key0 + n * 16 + grp * 4 + v;
                        if (key >= end || key >= limit[i]) x = -INFINITY;
                    }
                    s[i][n][v] = x;
                    top = fmaxf(top, x);
                }
            top = fmaxf(top, partner<4>(top));
            top = fmaxf(top, partner<5>(top));
            const float m_new = fmaxf(m[i], top);
            const float m_use = m_new == -INFINITY ? 0.0f : m_new;
            const float alpha = __builtin_amdgcn_exp2f(m[i] - m_use);
            m[i] = m_new;
            float sum = 0.0f;
#pragma unroll
            for (int n = 0; n < TL::kGroups; ++n)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const float p = __builtin_amdgcn_exp2f(s[i][n][v] - m_use);
                    if constexpr (kCodes) sum = __builtin_fmaf(p, rv[n][v], sum);
                    else sum += p;
                    pf[i][n / 2][(n & 1) * 4 + v] = (typename M::S)p;
                }
            l[i] = l[i] * alpha + sum;      // (of this lane's keys: added up across the wavefront at the end)
#pragma unroll
            for (int d = 0; d < D / 16; ++d) o[i][d] *= alpha;
        }

        // O^T: 16 values x 16 rows at a time, 32 keys to a product
#pragma unroll
        for (int u = 0; u < TL::kGroups / 2; ++u)
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
                V vf;
                if constexpr (kCodes) {
                    const int r = col >> 1, row = u * 32 + 16 * (r >> 2) + 4 * grp + (r & 3);
                    const char* const at = vt + row * TL::kRow + ((d ^ swz_v<C, true>(row)) * 16) + (col & 1) * 8;
                    vf = codes_to_f16(__builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2*)at));
                } else {
                    union { s16x4 h[2]; V v; } f;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int row = u * 32 + half * 16 + 4 * grp + (col >> 2);
                        const char* const at = vt + row * TL::kRow + (((2 * d + ((col & 3) >> 1)) ^ swz_v<C, false>(row)) * 16) + (col & 1) * 8;
                        f.h[half] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
                    }
                    vf = f.v;
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) o[i][d] = M::mul(vf, pf[i][u], o[i][d]);
            }
    }
    if (est && lane == 0) raise_status(g.status, est);

#pragma unroll
    for (int i = 0; i < MT; ++i) {
        l[i] += partner<4>(l[i]);
        l[i] += partner<5>(l[i]);
    }

    const int64_t all_rows = g.T * g.Hq;
    // four consecutive values of one row: the result, or a part's share of it
    auto store = [&](int r, int d, const f32x4& v, float mm, float ll) {
        const int64_t t = t0 + r / g.G;
        const int h = kvh * g.G + r % g.G;
        if (g.parts == 1) {
            const float inv = ll > 0.0f ? 1.0f / ll : 0.0f;
            if (g.q_bf16) {
                typedef __bf16 b4 __attribute__((ext_vector_type(4)));
                *reinterpret_cast<b4*>(reinterpret_cast<__bf16*>(g.out) + t * g.ldo + (int64_t)h * D + d) =
                    b4{(__bf16)(v[0] * inv), (__bf16)(v[1] * inv), (__bf16)(v[2] * inv), (__bf16)(v[3] * inv)};
            } else {
                *reinterpret_cast<f16x4*>(reinterpret_cast<_Float16*>(g.out) + t * g.ldo + (int64_t)h * D + d) =
                    f16x4{(_Float16)(v[0] * inv), (_Float16)(v[1] * inv), (_Float16)(v[2] * inv), (_Float16)(v[3] * inv)};
            }
            if (d == 0 && g.lse) g.lse[t * g.Hq + h] = ll > 0.0f ? (mm + __builtin_amdgcn_logf(ll)) * kLn2 : -INFINITY;
        } else {
            const int64_t at = (int64_t)(g.first_part + split) * all_rows + t * g.Hq + h;
            *reinterpret_cast<f32x4*>(g.part_o + at * D + d) = v;
            if (d == 0) g.part_ml[at] = make_float2(mm, ll);
        }
    };

    if constexpr (WR > 1) {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int r = row0 + 16 * i + col;
            if (r < rows) {
#pragma unroll
                for (int d = 0; d < D / 16; ++d) store(r, d * 16 + grp * 4, o[i][d], m[i], l[i]);
            }
        }
    } else {
        // the wavefronts' ranges of the same 16 rows
        __syncthreads();   // (every wavefront is done with its ring)
        float* const so = reinterpret_cast<float*>(lds);                         // [wave][row][D]
        float* const sm = so + TL::kWaves * 16 * D;                              // [wave][row][2]
#pragma unroll
        for (int d = 0; d < D / 16; ++d) *reinterpret_cast<f32x4*>(so + (wave * 16 + col) * D + d * 16 + grp * 4) = o[0][d];
        if (grp == 0) { sm[(wave * 16 + col) * 2] = m[0]; sm[(wave * 16 + col) * 2 + 1] = l[0]; }
        __syncthreads();
        for (int e = threadIdx.x; e < 16 * D / 4; e += TL::kThreads) {
            const int r = e / (D / 4), d = e % (D / 4) * 4;
            if (row0 + r >= rows) continue;
            float mm = -INFINITY, ll = 0.0f;
#pragma unroll
            for (int w = 0; w < TL::kWaves; ++w) mm = fmaxf(mm, sm[(w * 16 + r) * 2]);
            const float use = mm == -INFINITY ? 0.0f : mm;
            f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < TL::kWaves; ++w) {
                const float a = __builtin_amdgcn_exp2f(sm[(w * 16 + r) * 2] - use);
                ll += a * sm[(w * 16 + r) * 2 + 1];
                v += a * *reinterpret_cast<const f32x4*>(so + (w * 16 + r) * D + d);
            }
            store(row0 + r, d, v, mm, ll);
        }
    }
}

// A row's parts joined: one wavefront each
template <int D>
__global__ __launch_bounds__(256) void join_kernel(Args g)
{
    const int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave, all_rows = g.T * g.Hq;
    if (row >= all_rows) return;
    const int lane = threadIdx.x & (kWave - 1);
    float mm = -INFINITY;
    for (int p = 0; p < g.parts; ++p) mm = fmaxf(mm, g.part_ml[p * all_rows + row].x);
    const float use = mm == -INFINITY ? 0.0f : mm;
    constexpr int N = D / kWave;
    float ll = 0.0f, v[N] = {};
    for (int p = 0; p < g.parts; ++p) {
        const float2 ml = g.part_ml[p * all_rows + row];
        if (!(ml.y > 0.0f)) continue;
        const float a = __builtin_amdgcn_exp2f(ml.x - use);
        ll += a * ml.y;
        const float* const src = g.part_o + (p * all_rows + row) * D + lane * N;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += a * src[i];
    }
    const float inv = ll > 0.0f ? 1.0f / ll : 0.0f;
    const int64_t t = row / g.Hq, at = t * g.ldo + row % g.Hq * D + lane * N;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (g.q_bf16) reinterpret_cast<__bf16*>(g.out)[at + i] = (__bf16)(v[i] * inv);
        else reinterpret_cast<_Float16*>(g.out)[at + i] = (_Float16)(v[i] * inv);
    }
    if (lane == 0 && g.lse) g.lse[row] = ll > 0.0f ? (mm + __builtin_amdgcn_logf(ll)) * kLn2 : -INFINITY;
}

// How a call is cut up
struct Plan {
    int prefix_rows, own_rows;        // rows of a workgroup: 16, 64 or 128
    int prefix_splits, own_splits;    // 0: no such keys
    int parts() const { return prefix_splits + own_splits; }
};

static int tile_rows(int64_t rows) { return rows <= 16 ? 16 : rows <= 64 ? 64 : 128; }

static int split_count(int64_t items, int64_t len, int64_t least)
{
    const int64_t want = cdiv(512, items), most = cdiv(len, least);
    const int64_t n = want < most ? want : most;
    return (int)(n < 1 ? 1 : n > 64 ? 64 : n);
}

static Plan plan(int64_t T, int64_t Hq, int64_t Hk, int64_t B, int64_t max_q, int64_t prefix_len, int64_t max_len)
{
    const int64_t G = Hq / Hk;
    Plan p = {16, 16, 0, 0};
    if (prefix_len > 0) {
        p.prefix_rows = tile_rows(T * G);
        p.prefix_splits = split_count(Hk * cdiv(T * G, p.prefix_rows), prefix_len, 256);
    }
    if (max_len > 0 || prefix_len == 0) {
        p.own_rows = tile_rows(max_q * G);
        p.own_splits = split_count(B * Hk * cdiv(max_q * G, p.own_rows), max_len, 256);
    }
    return p;
}

template <class E, int D, int WR, int MT, bool PREFIX>
static int launch_one(Args g, int64_t blocks, hipStream_t st)
{
    using TL = Tile<E, D, WR>;
    const void* fn = reinterpret_cast<const void*>(attention_kernel<E, D, WR, MT, PREFIX>);
    int dev = 0, cus = 0;
    if (device_cus(dev, cus) != AWEQ_OK || raise_lds_limit(fn, dev, TL::kLds) != AWEQ_OK) return AWEQ_ERR_LAUNCH;
    void* args[] = {&g};
    if (hipLaunchKernel(fn, dim3((unsigned)blocks), dim3(TL::kThreads), args, TL::kLds, st) != hipSuccess) return AWEQ_ERR_LAUNCH;
    return AWEQ_OK;
}

template <class E, int D, bool PREFIX>
static int launch_rows(Args g, int rows, int64_t most_rows, int splits, int first_part, hipStream_t st)
{
    g.splits = splits;
    g.first_part = first_part;
    g.row_tiles = (int)cdiv(most_rows, rows);
    const int64_t blocks = (int64_t)splits * g.row_tiles * g.Hk * (PREFIX ? 1 : g.B);
    if (blocks > (1 << 24) - 1) return AWEQ_ERR_SHAPE;
    if (rows == 16) return launch_one<E, D, 1, 1, PREFIX>(g, blocks, st);
    if (rows == 64) return launch_one<E, D, 4, 1, PREFIX>(g, blocks, st);
    return launch_one<E, D, 4, 2, PREFIX>(g, blocks, st);
}

template <class E, int D>
static int launch(const Args& g, const Plan& p, hipStream_t st)
{
    int rc = AWEQ_OK;
    if (p.prefix_splits) rc = launch_rows<E, D, true>(g, p.prefix_rows, g.T * g.G, p.prefix_splits, 0, st);
    if (rc == AWEQ_OK && p.own_splits) rc = launch_rows<E, D, false>(g, p.own_rows, (int64_t)g.max_q * g.G, p.own_splits, p.prefix_splits, st);
    if (rc == AWEQ_OK && p.parts() > 1) join_kernel<D><<<(unsigned)cdiv(g.T * g.Hq, 4), 256, 0, st>>>(g);
    return rc != AWEQ_OK ? rc : launch_status();
}

template <class E>
static int launch_head(const Args& g, const Plan& p, int64_t D, hipStream_t st)
{
    if (D == 64) return launch<E, 64>(g, p, st);
    if (D == 128) return launch<E, 128>(g, p, st);
    return launch<E, 256>(g, p, st);
}

static bool shapes_ok(int64_t T, int64_t Hq, int64_t Hk, int64_t D, int64_t B, int64_t max_q, int64_t prefix_len, int64_t max_len)
{
    if (T <= 0 || Hq <= 0 || Hk <= 0 || Hq % Hk != 0 || (D != 64 && D != 128 && D != 256) || B <= 0 || max_q <= 0) return false;
    if (prefix_len < 0 || max_len < 0 || prefix_len > (1 << 30) || max_len > (1 << 30)) return false;
    return T <= (1 << 24) && B <= (1 << 24) && Hq <= (1 << 16) && T * Hq <= (1 << 25);
}

}  // namespace attn
}  // namespace aweq

using namespace aweq;

extern "C" size_t aweq_prefix_attention_ws(int64_t T, int64_t Hq, int64_t Hk, int64_t D, int64_t B, int64_t max_q, int64_t prefix_len, int64_t max_len)
{
    if (!attn::shapes_ok(T, Hq, Hk, D, B, max_q, prefix_len, max_len)) return 0;
    max_q = max_q < T ? max_q : T;
    const int parts = attn::plan(T, Hq, Hk, B, max_q, prefix_len, max_len).parts();
    return parts > 1 ? (size_t)parts * (size_t)(T * Hq) * (size_t)(D * 4 + 8) : 0;
}

extern "C" int aweq_prefix_attention(const void* q, aweq_dtype dt, int64_t T, int64_t Hq, int64_t D, int64_t ldq,
                                     const void* k_cache, const void* v_cache, const float* k_step, const float* v_step, aweq_dtype cache_dt,
                                     int64_t pages, int64_t page_size, int64_t Hk, const int32_t* prefix_table, int64_t prefix_len,
                                     const int32_t* table, int64_t table_ld, const int32_t* lens, const int32_t* q_start, int64_t B,
                                     int64_t max_len, int64_t max_q, float scale, void* out, int64_t ldo, float* lse,
                                     void* ws, size_t ws_bytes, uint32_t* status, void* stream)
{
    if (!q || !out || !k_cache || !v_cache || !lens || (max_len > 0 && !table) || (prefix_len > 0 && !prefix_table)) return AWEQ_ERR_NULL;
    if ((dt != AWEQ_F16 && dt != AWEQ_BF16) || (cache_dt != dt && cache_dt != AWEQ_I8)) return AWEQ_ERR_DTYPE;
    if (cache_dt == AWEQ_I8 && (!k_step || !v_step)) return AWEQ_ERR_NULL;
    if (!attn::shapes_ok(T, Hq, Hk, D, B, max_q, prefix_len, max_len)) return AWEQ_ERR_SHAPE;
    max_q = max_q < T ? max_q : T;
    if (pages <= 0 || pages > 0x7fffffff || page_size < 16 || page_size > 256 || (page_size & (page_size - 1)) != 0) return AWEQ_ERR_SHAPE;
    if (ldq < Hq * D || ldo < Hq * D || (!q_start && (T != B || max_q != 1)) || (max_len > 0 && table_ld < 1)) return AWEQ_ERR_SHAPE;
    if (!aligned16(q) || !aligned16(out) || (ldq % 8) != 0 || (ldo % 8) != 0 || !aligned16(k_cache) || !aligned16(v_cache) ||
        (cache_dt == AWEQ_I8 && (!aligned16(k_step) || !aligned16(v_step))))
        return AWEQ_ERR_ALIGN;
    const attn::Plan p = attn::plan(T, Hq, Hk, B, max_q, prefix_len, max_len);
    const size_t need = aweq_prefix_attention_ws(T, Hq, Hk, D, B, max_q, prefix_len, max_len);
    if (need && (!ws || ws_bytes < need)) return AWEQ_ERR_WORKSPACE;
    if (need && !aligned16(ws)) return AWEQ_ERR_ALIGN;
    attn::Args g = {};
    g.q = q; g.k_cache = k_cache; g.v_cache = v_cache; g.k_step = k_step; g.v_step = v_step;
    g.prefix_table = prefix_table; g.table = table; g.lens = lens; g.q_start = q_start;
    g.out = out; g.lse = lse; g.status = status;
    g.T = T; g.ldq = ldq; g.ldo = ldo; g.table_ld = table_ld; g.prefix_len = prefix_len; g.max_len = max_len;
    g.pages = (int)pages; g.page_size = (int)page_size; g.page_shift = __builtin_ctz((unsigned)page_size);
    g.Hq = (int)Hq; g.Hk = (int)Hk; g.G = (int)(Hq / Hk); g.B = (int)B; g.max_q = (int)max_q;
    g.q_bf16 = dt == AWEQ_BF16;
    g.parts = p.parts();
    g.scale_log2e = scale * attn::kLog2e;
    g.part_o = reinterpret_cast<float*>(ws);
    g.part_ml = reinterpret_cast<float2*>(g.part_o + (size_t)g.parts * (size_t)(T * Hq) * (size_t)D);
    hipStream_t st = as_stream(stream);
    if (cache_dt == AWEQ_I8) return attn::launch_head<int8_t>(g, p, D, st);
    if (dt == AWEQ_F16) return attn::launch_head<_Float16>(g, p, D, st);
    return attn::launch_head<__bf16>(g, p, D, st);
}
