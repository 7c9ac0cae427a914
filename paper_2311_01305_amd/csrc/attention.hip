// Attention of a batch over a shared prefix and over each sequence's own pages of the cache.
//
//   out = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q k_j - m),  m the running maximum: one pass over the keys, any range of them by itself.
//
// A range of keys belongs to all tokens (the prefix) or to one sequence's.  For a key head the rows that multiply it are its G = Hq / Hk query heads
// of each of those tokens, row r = token r / G, head r % G: the prefix is read once for all rows of the batch.
//
// A wavefront has 16 MT rows and takes the keys in tiles.  It forms S^T = K Q^T and O^T = V^T P^T with v_mfma_f32_16x16x32: the weights' side of
// both products comes from the cache, a lane has one row of Q in its column, so that a row's maximum and sum need two exchanges across the
// wavefront, and the four consecutive keys that a lane holds of a 16 x 16 tile of S^T are, two tiles at a time, the eight it has to supply of P^T: the order
// of the keys inside a product is free as long as V^T's is the same.  V^T's is made by the transposing LDS reads.
// The maximum is taken up lazily: any m gives the same quotient, so sum and O are only rescaled when a score is more than 2^8 above it.
//
// Two forms:
//  - tall (many rows: the prefix, prompts): four wavefronts with rows of their own share tiles of 64 keys (32 of 512 bytes), filled by LDS-DMA loads of 16 bytes a
//    lane, two tiles in turn; chunks of 16 bytes are XOR swizzled by choosing which one a lane fetches.  Codes go through registers instead, requested two tiles
//    ahead, and are binary16 in LDS: converted once for the workgroup's rows, not by each wavefront
//    (us: 2048 tokens behind 8192 keys 462 -> 373, 5 tokens of 16 sequences of up to 6000 48 -> 36, 64 tokens behind 8192 34.5 -> 31; with the steps as below 368, 37, 31).
//  - wide (up to 16 rows: one token's heads): four wavefronts have the same rows and tiles of 32 keys of their own, whose results meet in
//    LDS at the end.  K goes from memory to registers in the operand's order, V to registers and through the wavefront's own LDS; the next
//    tile is requested as soon as this one's registers are free.
// 16 neighbouring tokens lie in one page (its size is a multiple of 16), so a group of 16 rows has one base address.  A tile's rows past the range
// repeat its last token: what a page holds past the range is never read.
//
// A value that a row does not see has a probability of 0, which times an infinity or a NaN is not 0.  Where the workgroup's rows do not see all keys of its range
// and an output comes out not finite, the workgroup takes the range once more and counts what is not finite by rows that see it: up to twice the time, for
// such calls alone (the others: a look at the outputs, us, before -> now: 6 prompts behind 4111 keys 373.3 -> 376.2, 3 of 700 tokens 24.0 -> 25.1).
//
// An 8-bit cache is multiplied as binary16 codes.  The step of a key goes to its score.  The step of a value goes to the probability that multiplies
// its codes, p' = p step 2^e, with a power of two for each row that keeps p' in binary16's range and follows the largest step which the row has seen, as the
// maximum follows the scores; O is rescaled when it changes.  The exponential brings 2^e along, and the sum has it too: no operation more for a key.  (What
// is below 2^-60 or beyond 2^90, a power of two for the wavefront's rows together, goes to the steps first.)  Maximum and sum are of the scores alone: a value's
// step says nothing of its weight.
//
// What bounds it (heads of 128 values).  Wide: HBM, 4.9 - 5.5 TB/s of keys and values where they are many (24 sequences of 3000 - 15001 tokens and a prefix of
// 2000, 461 MB of codes, 100 us with the join; a copy of 1 GB reaches 5.2); for one sequence the launches and a round trip each (1900 tokens, 31 MB: 9 us and 3 for
// the join).  Tall: the clock under load: 950 - 980 TFLOP/s in binary16 (1024 new tokens of 2 sequences behind 8192), 80 % of what a product of 8192 x 8192 x 8192
// reaches here, the matrix cores busy for half of the cycles.  Products of one tile between the exponentials of another, 32 x 32 x 16 instructions, raised
// priority around the products and a third tile in flight left that as it was.  The prefix of a decode step, whose rows are few, is one round of
// workgroups that wait for their tiles (64 tokens behind 8192, 26 us, of which half the sequences' own keys; join 5).
#include "wide_unit.hpp"

#include <cmath>
#include <type_traits>

namespace aweq {
namespace attn {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kLazy = 8.0f;       // log2 of what a probability may be over 1
constexpr int kStepBits = 7;        // (codes) log2 of what a step 2^e may be, which multiplies that: together below binary16's 2^16
constexpr int kLeast = -60, kMost = 90;   // (codes) e that the exponential brings along: sums of 2^30 keys stay in range, and so do keys of 2^-60 of the largest
constexpr float kFar = 1 << 22;     // scores (log2) that binary32 holds to half or better
constexpr int kWaves = 4, kThreads = kWaves * kWave;
constexpr int kWideRows = 16, kWideKeys = 32, kTallKeys = 64;

// Workgroups of one kind in a launch: which rows, which keys
struct Work {
    int blocks;         // of the grid
    int tall;           // form
    int row_tiles;      // workgroups that cover a sequence's (the batch's) rows
    int splits;         // ranges of the keys
    int chunk;          // keys of a range; 0: an equal share of the tiles (tall, prefix and own keys in one list)
    int combos;         // (sequence, range, key head)
    int first_part;
};

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
    int prefix_len, max_len;
    int pages, page_size, page_shift;
    int Hq, Hk, G, max_q;
    int q_bf16;         // type of q and out (an 8-bit cache: either)
    int parts;          // of a row: 1: the result itself
    int fused;          // a sequence's rows take the prefix along
    float scale_log2e;
    Work shared, own;   // the prefix for all rows; a sequence's keys for its own
};

// Tables and lengths do not change during a launch and are read at uniform places: through the scalar cache, whose loads do not wait for
// the vector ones in flight
typedef const __attribute__((address_space(4))) int32_t* ConstInts;
__device__ __forceinline__ int scalar_at(const int32_t* p, int64_t i) { return ((ConstInts)(uintptr_t)p)[i]; }

template <int N>
__device__ __forceinline__ void wait_vm()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// lane i's 16 bytes land at lds_addr + 16 i; lds_addr and base wave-uniform
__device__ __forceinline__ void dma16(const char* base, uint32_t off, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds_addr), "v"(off), "s"(base) : "memory");
}

// over the four lanes that hold a row's keys: lanes l, l ^ 16, l ^ 32, l ^ 48
template <class Op>
__device__ __forceinline__ float row_reduce(float v, Op op)
{
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return op(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
struct Larger { __device__ float operator()(float a, float b) const { return fmaxf(a, b); } };

// E: type of the cache (int8_t: codes)
template <class E> struct Mfma;
template <> struct Mfma<_Float16> {
    typedef f16x8 V;
    typedef _Float16 S;
    static constexpr unsigned kExponent = 0x7c00;   // all ones
    static __device__ __forceinline__ f32x4 mul(V a, V b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <> struct Mfma<int8_t> : Mfma<_Float16> {};
template <> struct Mfma<__bf16> {
    typedef bf16x8 V;
    typedef __bf16 S;
    static constexpr unsigned kExponent = 0x7f80;
    static __device__ __forceinline__ f32x4 mul(V a, V b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};

// 8 codes to binary16: the byte u = code + 128 under the exponent of 1024 is 1024 + u
__device__ __forceinline__ f16x8 codes_to_f16(int w0, int w1)
{
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    union { uint32_t u[4]; h2 h[4]; f16x8 v; } r;
    const uint32_t u0 = (uint32_t)w0 ^ 0x80808080u, u1 = (uint32_t)w1 ^ 0x80808080u;
    r.u[0] = __builtin_amdgcn_perm(0x64646464u, u0, 0x04010400u);
    r.u[1] = __builtin_amdgcn_perm(0x64646464u, u0, 0x04030402u);
    r.u[2] = __builtin_amdgcn_perm(0x64646464u, u1, 0x04010400u);
    r.u[3] = __builtin_amdgcn_perm(0x64646464u, u1, 0x04030402u);
#pragma unroll
    for (int i = 0; i < 4; ++i) r.h[i] = r.h[i] - h2{(_Float16)1152.0f, (_Float16)1152.0f};
    return r.v;
}

template <class E, int D>
struct Shape {
    static constexpr bool kCodes = sizeof(E) == 1;
    static constexpr int kRow = D * (int)sizeof(E);            // bytes of a token's head
    static constexpr int kChunks = kRow / 16;
    static constexpr int kLoads = kRow * 16 / 1024;            // load instructions for 16 rows
    static constexpr int kRowsPerLoad = 1024 / kRow;
    // tall: K, V, in 16 bits, and (codes) for each group of 16 keys the steps of K and of V; tiles that leave room for two workgroups
    static constexpr int kTallRow = 2 * D;
    static constexpr int kTile = kTallRow == 512 ? 32 : kTallKeys, kGroups = kTile / 16;
    static constexpr int kHalf = kTile * kTallRow;
    static constexpr int kSlot = 2 * kHalf + (kCodes ? kGroups * 128 : 0);
    static constexpr int kTallLds = 2 * kSlot;
    // wide: V of a tile for each wavefront; at the end their O, maximum and sum
    static constexpr int kWideV = kWideKeys * kRow;
    static constexpr int kMerge = kWaves * (kWideRows * D * 4 + kWideRows * 8);
    static constexpr int kWideLds = kWaves * kWideV > kMerge ? kWaves * kWideV : kMerge;
    static constexpr int lds(bool tall) { return tall && kTallLds > kWideLds ? kTallLds : kWideLds; }
};

// Swizzles of the 16-byte chunks of a row (C of them): reads of one chunk of 16 rows (K), and the transposing reads of V (binary16: 8 rows x 2
// chunks, codes: rows 0 - 7 and 16 - 23 of one chunk) fall on different banks
template <int C>
__device__ __forceinline__ int swz_k(int row)
{
    if constexpr (C >= 16) return row & 15;
    else return (row / (16 / C)) & (C - 1);
}
template <int C, bool CODES>
__device__ __forceinline__ int swz_v(int row)
{
    constexpr int span = C >= 16 ? 1 : 16 / C;
    if constexpr (CODES) {
        constexpr int low = 8 / span;
        return ((row / span) & (low - 1)) + low * ((row >> 4) & 1);
    } else {
        return 2 * ((row / span) & (8 / span - 1));
    }
}

// What a workgroup has to do
struct Job {
    int64_t t0;         // first token of its rows
    int rows;           // rows in all: tokens times G
    int row0;           // the workgroup's first row
    int kvh;
    int pa, pb;         // keys of the prefix
    int oa, ob;         // keys of the sequence, up to what the workgroup's last row sees
    int sees0;          // row r sees sees0 + r / G of the sequence's keys
    const int32_t* table;
    int64_t part;
};

// PAIRS: K and V are multiplied as they lie in the cache, so that of codes 16 bytes are two operands
template <class E, int D, int MT, bool PAIRS>
struct Rows {
    using M = Mfma<E>;
    using V = typename M::V;
    static constexpr bool kCodes = Shape<E, D>::kCodes;
    static constexpr int kRow = PAIRS ? D : 2 * D, kChunks = kRow / 16;   // of V's tile

    int lane;
    V q[MT][D / 32];
    float scale[MT];        // to log2 (codes: the keys' steps bring that; the power of two that the queries have to lose)
    int sees[MT];           // own keys that the row sees
    f32x4 o[MT][D / 16];
    float m[MT], l[MT];     // (l: of this lane's keys)
    bool far;               // a maximum is so large that its last place is no small part of 1
    float most[MT];         // (codes) no value's step that the row has seen is larger; a power of two, or 0
    float use[MT];          // (codes) what the exponential takes off a score: the maximum less held(i)
    int base;               // (codes) the sum is 2^held(i) times what it stands for, O 2^(base + held(i)) times

    // Column lane % 16 of row tile i is row `row0` + 16 i + that; eight values of its head at a time, in the order that K is read in: 32 kk + 8 grp, or in
    // pairs 64 (kk / 2) + 16 grp + 8 (kk % 2)
    __device__ __forceinline__ void load(const Args& g, const Job& j, int row0, int of)
    {
        lane = of;
        const int col = lane & 15, grp = lane >> 4;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int r = min(row0 + 16 * i + col, j.rows - 1);
            sees[i] = j.sees0 + r / g.G;
            const char* src = reinterpret_cast<const char*>(g.q) + ((j.t0 + r / g.G) * g.ldq + (int64_t)(j.kvh * g.G + r % g.G) * D) * 2;
            auto at = [&](int kk) { return src + (PAIRS ? 64 * (kk / 2) + 16 * grp + 8 * (kk % 2) : 32 * kk + 8 * grp) * 2; };
            scale[i] = kCodes ? 1.0f : g.scale_log2e;
            if (kCodes && g.q_bf16) {
                // bfloat16 queries as binary16: scaled by a power of two, the largest value below 2^15
                float x[D / 32][8], big = 0.0f;
#pragma unroll
                for (int kk = 0; kk < D / 32; ++kk) {
                    widen<__bf16>(*reinterpret_cast<const bf16x8*>(at(kk)), x[kk]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) big = fmaxf(big, fabsf(x[kk][e]));
                }
                big = row_reduce(big, Larger());
                const int e2 = big > 0.0f ? 14 - ilogbf(big) : 0;
#pragma unroll
                for (int kk = 0; kk < D / 32; ++kk)
#pragma unroll
                    for (int e = 0; e < 8; ++e) q[i][kk][e] = (typename M::S)ldexpf(x[kk][e], e2);
                scale[i] = ldexpf(1.0f, -e2);
            } else {
#pragma unroll
                for (int kk = 0; kk < D / 32; ++kk) q[i][kk] = *reinterpret_cast<const V*>(at(kk));
            }
        }
        begin();
    }

    // no key yet
    __device__ __forceinline__ void begin()
    {
        far = false;
        base = 0;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            m[i] = -INFINITY;
            l[i] = 0.0f;
            most[i] = 0.0f;
            use[i] = 0.0f;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) o[i][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
    }

    // The queries have arrived: said before the loop over the keys, whose waits would be for them and, with them, for the keys in flight
    __device__ __forceinline__ void arrived()
    {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int kk = 0; kk < D / 32; ++kk) {
                i32x4 w = __builtin_bit_cast(i32x4, q[i][kk]);
                asm volatile("" : "+v"(w));
                q[i][kk] = __builtin_bit_cast(V, w);
            }
    }

    __device__ __forceinline__ int shift(int i) const { return kStepBits + 127 - (int)(__float_as_uint(most[i]) >> 23); }
    __device__ __forceinline__ int held(int i) const { return min(max(shift(i) - base, kLeast), kMost); }

    // of this lane's keys in a tile from key0 on, how far row i sees; end: of the range, own: the sequence's
    __device__ __forceinline__ int mine(int i, int key0, int end, bool own) const
    {
        return (own ? min(end, sees[i]) : end) - key0 - (lane >> 4) * 4;
    }

    // Scores s[i][n] of 16 keys each from key0 on: those that a row does not see to -inf, maxima and what hangs on them.  (codes) The steps of K are in the
    // scores, scaled and to log2; v_steps(n): those of V of this lane's four keys, asked for twice, since they are not kept across the branches between
    // (of keys past the range: anything); odd: one is not finite.
    template <int N, class VSteps>
    __device__ __forceinline__ void maxima(f32x4 (&s)[MT][N], int key0, int end, bool own, VSteps v_steps, bool& odd)
    {
        float top[MT], step[MT];   // (step: codes)
        bool high = false, loud = false;
        float widest = 0.0f;
        if constexpr (kCodes) {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const Float4 vs = v_steps(n);
#pragma unroll
                for (int v = 0; v < 4; ++v) widest = __builtin_elementwise_maximum(widest, vs.f[v]);   // (a NaN stays one)
            }
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            step[i] = widest;
            if (__builtin_amdgcn_ballot_w64(key0 + 16 * N > (own ? min(end, sees[i]) : end)) != 0) {
                const int in = mine(i, key0, end, own);
                if constexpr (kCodes) odd = __builtin_amdgcn_ballot_w64(!(widest < INFINITY)) != 0;
                step[i] = 0.0f;
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    Float4 vs;
                    if constexpr (kCodes) vs = v_steps(n);
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        s[i][n][v] = n * 16 + v < in ? s[i][n][v] : -INFINITY;
                        if constexpr (kCodes) step[i] = n * 16 + v < in ? __builtin_elementwise_maximum(step[i], vs.f[v]) : step[i];
                    }
                }
            }
            float t = -INFINITY;
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int v = 0; v < 4; ++v) t = fmaxf(t, s[i][n][v]);
            top[i] = t * scale[i];    // (scale > 0)
            high = high || top[i] > m[i] + kLazy;
            if constexpr (kCodes) loud = loud || !(step[i] <= most[i]);
        }
        if (__builtin_amdgcn_ballot_w64(high || loud) != 0) {
            float times[MT];
#pragma unroll
            for (int i = 0; i < MT; ++i) times[i] = 1.0f;
            if (!kCodes || __builtin_amdgcn_ballot_w64(high) != 0) {
                bool large = false;
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const float m_new = fmaxf(m[i], row_reduce(top[i], Larger()));
                    times[i] = __builtin_amdgcn_exp2f(m[i] - (m_new == -INFINITY ? 0.0f : m_new));
                    m[i] = m_new;
                    l[i] *= times[i];
                    large = large || (fabsf(m_new) > kFar && m_new != -INFINITY);
                }
                far = __builtin_amdgcn_ballot_w64(large) != 0;
            }
            if constexpr (kCodes) {
                if (__builtin_amdgcn_ballot_w64(loud) != 0) odd = rescale(step, times) || odd;
#pragma unroll
                for (int i = 0; i < MT; ++i) use[i] = (m[i] == -INFINITY || far ? 0.0f : m[i]) - (float)held(i);
            }
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int d = 0; d < D / 16; ++d) o[i][d] *= times[i];
        }
    }

    // Scores to probabilities for the second product
    template <int N, class VSteps>
    __device__ __forceinline__ void weights(f32x4 (&s)[MT][N], V (&p)[MT][N / 2], VSteps v_steps, bool odd)
    {
        float less[MT], times[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            less[i] = kCodes ? use[i] : m[i] == -INFINITY ? 0.0f : m[i];
            times[i] = scale[i];
        }
        if (far) {   // (what a maximum was rounded by would not cancel in the fused form: it may be more than any exponent)
#pragma unroll
            for (int i = 0; i < MT; ++i) {
#pragma unroll
                for (int n = 0; n < N; ++n)
#pragma unroll
                    for (int v = 0; v < 4; ++v) s[i][n][v] = s[i][n][v] * scale[i] - (m[i] == -INFINITY ? 0.0f : m[i]);
                if constexpr (!kCodes) less[i] = 0.0f;
                times[i] = 1.0f;
            }
        }
        float vs[N][4];
        if constexpr (kCodes) {
            asm volatile("" ::: "memory");
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const Float4 x = v_steps(n);
#pragma unroll
                for (int v = 0; v < 4; ++v) vs[n][v] = x.f[v];
            }
            if (base != 0 || odd) {   // (what is not finite, or too large for the power of two that suits what is seen, is for no row here)
#pragma unroll
                for (int n = 0; n < N; ++n)
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const float scaled = ldexpf(vs[n][v], base);
                        vs[n][v] = scaled < INFINITY ? scaled : 0.0f;
                    }
                asm volatile("" ::: "memory");
            }
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            float sum = 0.0f;
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][n][v], times[i], -less[i]));
                    sum += x;
                    p[i][n / 2][(n & 1) * 4 + v] = (typename M::S)(kCodes ? x * vs[n][v] : x);
                }
            l[i] += sum;
        }
    }

    // (codes) The powers of two after a step that is larger than those before; whether one is not finite.  step: of this lane's keys that a row sees; times: what
    // O is to be multiplied by
    __device__ __forceinline__ bool rescale(const float (&step)[MT], float (&times)[MT])
    {
        int before[MT];
        bool odd = false, outside = base != 0;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            before[i] = held(i);
            const float largest = row_reduce(step[i], OpMaximum());
            if (!(largest < INFINITY)) {
                odd = true;
                times[i] = NAN;
            } else if (largest > most[i]) {
                most[i] = __uint_as_float(((__float_as_uint(largest) >> 23) + 1) << 23);   // (the next power of two)
            }
            outside = outside || (most[i] > 0.0f && (shift(i) < kLeast || shift(i) > kMost));
        }
        const int old = base;
        if (__builtin_amdgcn_ballot_w64(outside) != 0) {
            int least = 1024, greatest = -1024;
#pragma unroll
            for (int i = 0; i < MT; ++i)
                if (most[i] > 0.0f) {
                    least = min(least, shift(i));
                    greatest = max(greatest, shift(i));
                }
            least = __builtin_amdgcn_readfirstlane(wave_allreduce(least, OpMin()));
            greatest = __builtin_amdgcn_readfirstlane(wave_allreduce(greatest, OpMax()));
            base = min(max(greatest - kMost, 0), least - kLeast);   // (rows whose steps are less than 2^-150 of another's of these have fewer digits)
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int up = held(i) - before[i];
            l[i] = ldexpf(l[i], up);
            times[i] = ldexpf(times[i], up + base - old);
        }
        return __builtin_amdgcn_ballot_w64(odd) != 0;
    }

    // After the last key.  (codes) The sum's power of two goes to the maximum, which it is as good as, and O's is the same; where it is a large one both lose it
    __device__ __forceinline__ void finish()
    {
        if constexpr (kCodes) {
            bool large = far || base != 0;
#pragma unroll
            for (int i = 0; i < MT; ++i) large = large || (m[i] != -INFINITY && (held(i) < -32 || held(i) > 32));
            if (__builtin_amdgcn_ballot_w64(large) == 0) {
#pragma unroll
                for (int i = 0; i < MT; ++i) m[i] = m[i] == -INFINITY ? m[i] : use[i];
            } else {
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    l[i] = ldexpf(l[i], -held(i));
#pragma unroll
                    for (int d = 0; d < D / 16; ++d)
#pragma unroll
                        for (int v = 0; v < 4; ++v) o[i][d][v] = ldexpf(o[i][d][v], -base - held(i));
                }
            }
        }
    }

    // Where a lane's transposing reads of V begin, for 16 values at d: keys 4 grp .. of the first 16 (codes: and of the second) of a tile
    __device__ __forceinline__ int value_offset(int d) const
    {
        constexpr int C = kChunks;
        const int col = lane & 15, grp = lane >> 4;
        if constexpr (PAIRS) {
            const int r = col >> 1, row = 16 * (r >> 2) + 4 * grp + (r & 3);
            return row * kRow + ((d ^ swz_v<C, true>(row)) * 16) + (col & 1) * 8;
        } else {
            const int row = 4 * grp + (col >> 2);
            return row * kRow + (((2 * d + ((col & 3) >> 1)) ^ swz_v<C, false>(row)) * 16) + (col & 1) * 8;
        }
    }

    // V^T of 16 values for keys 32 u .. 32 u + 31 of the tile at vt (the swizzles repeat every 16 rows, the codes' every 32)
    static __device__ __forceinline__ V value_operand(const char* vt, int u, int at)
    {
        const char* const from = vt + at + u * 32 * kRow;
        if constexpr (PAIRS) {
            const i32x2 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2*)from);
            return codes_to_f16(w[0], w[1]);
        } else {
            union { s16x4 h[2]; V v; } f;
#pragma unroll
            for (int half = 0; half < 2; ++half)
                f.h[half] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(from + half * 16 * kRow));
            return f.v;
        }
    }

    // O^T += V^T P^T for the tile at vt
    template <int N>
    __device__ __forceinline__ void values(const char* vt, const V (&p)[MT][N / 2], const int (&at)[D / 16])
    {
#pragma unroll
        for (int u = 0; u < N / 2; ++u)
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
                const V vf = value_operand(vt, u, at[d]);
#pragma unroll
                for (int i = 0; i < MT; ++i) o[i][d] = M::mul(vf, p[i][u], o[i][d]);
            }
    }

    // The same where some are not finite and rows do not see all keys: what is not finite is counted, with 1 in the place of what a row sees, and makes the outputs of
    // rows that see some NaN
    template <int N>
    __device__ __forceinline__ void values_seen(const char* vt, const V (&p)[MT][N / 2], const int (&at)[D / 16], int key0, int end, bool own)
    {
        typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
        constexpr unsigned short kBelow = M::kExponent - 1;
        const unsigned short one = __builtin_bit_cast(unsigned short, (typename M::S)1.0f);
#pragma unroll
        for (int u = 0; u < N / 2; ++u) {
            u16x8 sees_it[MT];
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) sees_it[i][e] = (2 * u + e / 4) * 16 + e % 4 < mine(i, key0, end, own) ? one : 0;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
                const u16x8 bits = __builtin_bit_cast(u16x8, value_operand(vt, u, at[d]));
                const u16x8 over = __builtin_elementwise_max((u16x8)(bits & (unsigned short)0x7fff), (u16x8)kBelow) - kBelow;
                const u16x8 mask = (u16x8)0 - __builtin_elementwise_min(over, (u16x8)1);    // all ones where it is not finite
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const f32x4 none = {0.0f, 0.0f, 0.0f, 0.0f};
                    const f32x4 bad = M::mul(__builtin_bit_cast(V, (u16x8)(mask & one)), __builtin_bit_cast(V, sees_it[i]), none);
                    o[i][d] = M::mul(__builtin_bit_cast(V, (u16x8)(bits & ~mask)), p[i][u], o[i][d]);
#pragma unroll
                    for (int v = 0; v < 4; ++v) o[i][d][v] = bad[v] > 0.0f ? NAN : o[i][d][v];
                }
                __builtin_amdgcn_sched_barrier(0);   // (few registers rather than few waits)
            }
        }
    }

    // All of it for a tile whose scores are s
    template <int N, bool SEEN, class VSteps>
    __device__ __forceinline__ void attend(f32x4 (&s)[MT][N], const char* vt, const int (&at)[D / 16], int key0, int end, bool own, VSteps v_steps)
    {
        bool odd = false;
        maxima<N>(s, key0, end, own, v_steps, odd);
        V p[MT][N / 2];
        weights<N>(s, p, v_steps, odd);
        if constexpr (SEEN) values_seen<N>(vt, p, at, key0, end, own);
        else values<N>(vt, p, at);
    }

    // Whether an output is not finite.  Where rows do not see all keys that may be another's doing: a probability of 0 times an infinity or a NaN is not 0.  Then
    // the workgroup does it all again with SEEN, which minds what a row sees.
    __device__ __forceinline__ bool not_finite() const
    {
        float z = 0.0f;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int d = 0; d < D / 16; ++d)
#pragma unroll
                for (int v = 0; v < 4; ++v) z = __builtin_elementwise_maximum(z, fabsf(o[i][d][v]));
        return __builtin_amdgcn_ballot_w64(!(z < INFINITY)) != 0;
    }
};

// four consecutive values of one row: the result, or a part's share of it
template <int D>
__device__ __forceinline__ void store_row(const Args& g, const Job& j, int r, int d, const f32x4& v, float m, float l)
{
    const int64_t t = j.t0 + r / g.G;
    const int h = j.kvh * g.G + r % g.G;
    if (g.parts == 1) {
        const float inv = l != 0.0f ? 1.0f / l : 0.0f;   // (0: no key; a NaN goes on)
        if (g.q_bf16) {
            typedef __bf16 b4 __attribute__((ext_vector_type(4)));
            *reinterpret_cast<b4*>(reinterpret_cast<__bf16*>(g.out) + t * g.ldo + (int64_t)h * D + d) =
                b4{(__bf16)(v[0] * inv), (__bf16)(v[1] * inv), (__bf16)(v[2] * inv), (__bf16)(v[3] * inv)};
        } else {
            *reinterpret_cast<f16x4*>(reinterpret_cast<_Float16*>(g.out) + t * g.ldo + (int64_t)h * D + d) =
                f16x4{(_Float16)(v[0] * inv), (_Float16)(v[1] * inv), (_Float16)(v[2] * inv), (_Float16)(v[3] * inv)};
        }
        if (d == 0 && g.lse) g.lse[t * g.Hq + h] = l != 0.0f ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
    } else {
        const int64_t at = j.part * (g.T * g.Hq) + t * g.Hq + h;
        if (l != 0.0f) *reinterpret_cast<f32x4*>(g.part_o + at * D + d) = v;   // (a part without keys is not read)
        if (d == 0) g.part_ml[at] = make_float2(m, l);
    }
}

// AGAIN: one that the compiler does not know to be the same, so that the second time keeps no registers through the first
template <bool AGAIN>
__device__ __forceinline__ int thread_index()
{
    int t = (int)threadIdx.x;
    if constexpr (AGAIN) asm volatile("" : "+v"(t));
    return t;
}

// SEEN: some value is not finite (both forms); true: it has to be done again with SEEN
template <class E, int D, int MT, bool SEEN>
__device__ __forceinline__ bool tall_block(const Args& g, const Job& j, char* lds)
{
    using SH = Shape<E, D>;
    using R = Rows<E, D, MT, false>;
    using V = typename R::V;
    constexpr int C = R::kChunks, kRow = R::kRow, N = SH::kGroups, kTile = SH::kTile;
    static_assert(N == kWaves || N == 2, "a wavefront fetches a group of K and of V, or one of the two");
    constexpr bool kCodes = SH::kCodes;
    const int thread = thread_index<SEEN>(), lane = thread & (kWave - 1), col = lane & 15, grp = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(thread / kWave);
    const int row0 = j.row0 + wave * 16 * MT;
    const int group = N == kWaves ? wave : wave & 1;   // of 16 keys of a tile, which this wavefront fetches

    // tiles: the prefix's, then the sequence's
    const int np = j.pb > j.pa ? (j.pb - j.pa + kTile - 1) / kTile : 0;
    const int tiles = np + (j.ob > j.oa ? (j.ob - j.oa + kTile - 1) / kTile : 0);
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds);
    uint32_t est = 0;
    auto first_key = [&](int tile) { return tile < np ? j.pa + tile * kTile : j.oa + (tile - np) * kTile; };
    auto page_of = [&](int tile) {    // of this wavefront's 16 keys
        const int key = min(first_key(tile) + group * 16, (tile < np ? j.pb : j.ob) - 1);
        return scalar_at(tile < np ? g.prefix_table : j.table, key >> g.page_shift);
    };
    int next_page = tiles > 0 ? page_of(0) : 0;
    const bool fetches_v = N < kWaves && wave >= 2;   // (short tiles: of V instead of K)
    // The group's first key of a tile is a multiple of 16, so that it lies in one page; past the end the last group that has a key.  Returns its row of the
    // cache; `last`: of the 16, the last that the range has.  Tiles are asked for in order: the next one's page is on its way by then.
    auto place = [&](int tile, int& last) {
        int page = next_page;
        if (tile + 1 < tiles) next_page = page_of(tile + 1);
        if ((unsigned)page >= (unsigned)g.pages) { est |= AWEQ_ST_INDEX; page = 0; }
        const int end = tile < np ? j.pb : j.ob, key0 = min(first_key(tile) + group * 16, (end - 1) & ~15);
        last = end - 1 - key0;
        return (((int64_t)page * g.Hk + j.kvh) << g.page_shift) + (key0 & (g.page_size - 1));
    };
    // 16 bits: LDS-DMA; this lane's 16 bytes of the load instructions of K and V, from the first of the 16 rows
    auto fetch_offset = [&](int q, bool v, int last) {
        const int sub = q * SH::kRowsPerLoad + lane / C, trow = group * 16 + sub;    // row of the 16, of the tile (the swizzle's)
        return (uint32_t)(min(sub, last) * kRow + ((lane % C) ^ (v ? swz_v<C, false>(trow) : swz_k<C>(trow))) * 16);
    };
    uint32_t from_k[SH::kLoads], from_v[SH::kLoads];
    if constexpr (!kCodes)
#pragma unroll
        for (int q = 0; q < SH::kLoads; ++q) { from_k[q] = fetch_offset(q, fetches_v, 15); from_v[q] = fetch_offset(q, true, 15); }
    auto fetch = [&](int tile, uint32_t slot) {
        int last;
        const int64_t row0 = place(tile, last);
        const char* const kb = reinterpret_cast<const char*>(g.k_cache) + row0 * kRow;
        const char* const vb = reinterpret_cast<const char*>(g.v_cache) + row0 * kRow;
        const uint32_t to = lds0 + slot + (uint32_t)(group * 16 * kRow);
        if constexpr (N < kWaves) {
            const char* const base = fetches_v ? vb : kb;
            const uint32_t half = to + (fetches_v ? SH::kHalf : 0);
            if (last >= 15) {
#pragma unroll
                for (int q = 0; q < SH::kLoads; ++q) dma16(base, from_k[q], half + q * 1024);
            } else {
#pragma unroll
                for (int q = 0; q < SH::kLoads; ++q) dma16(base, fetch_offset(q, fetches_v, last), half + q * 1024);
            }
        } else if (last >= 15) {
#pragma unroll
            for (int q = 0; q < SH::kLoads; ++q) { dma16(kb, from_k[q], to + q * 1024); dma16(vb, from_v[q], to + q * 1024 + SH::kHalf); }
        } else {
#pragma unroll
            for (int q = 0; q < SH::kLoads; ++q) { dma16(kb, fetch_offset(q, false, last), to + q * 1024); dma16(vb, fetch_offset(q, true, last), to + q * 1024 + SH::kHalf); }
        }
    };
    // Codes: to registers, and from there as binary16 to LDS, with what their steps enter: each is converted once for the workgroup's rows
    constexpr int kCodeChunks = D / 16;
    i32x4 code_k[SH::kLoads], code_v[SH::kLoads];
    float step_kv;
    auto request = [&](int tile) {
        int last;
        const int64_t row0 = place(tile, last);
        const char* const kb = reinterpret_cast<const char*>(fetches_v ? g.v_cache : g.k_cache) + row0 * D;
        const char* const vb = reinterpret_cast<const char*>(g.v_cache) + row0 * D;
#pragma unroll
        for (int q = 0; q < SH::kLoads; ++q) {
            const uint32_t from = (uint32_t)(min(q * SH::kRowsPerLoad + lane / kCodeChunks, last) * D + (lane % kCodeChunks) * 16);
            code_k[q] = *reinterpret_cast<const i32x4*>(kb + from);
            if constexpr (N == kWaves) code_v[q] = *reinterpret_cast<const i32x4*>(vb + from);
        }
        step_kv = ((grp & 1) ? g.v_step : g.k_step)[row0 + min(col, last)];
    };
    auto convert = [&](uint32_t slot) {
        char* const tile = lds + slot;
        auto put = [&](char* half, int row, int swz, const i32x4& w) {
            const int c = 2 * (lane % kCodeChunks);
            *reinterpret_cast<f16x8*>(half + row * kRow + ((c ^ swz) * 16)) = codes_to_f16(w[0], w[1]);
            *reinterpret_cast<f16x8*>(half + row * kRow + (((c + 1) ^ swz) * 16)) = codes_to_f16(w[2], w[3]);
        };
#pragma unroll
        for (int q = 0; q < SH::kLoads; ++q) {
            const int row = group * 16 + q * SH::kRowsPerLoad + lane / kCodeChunks;
            put(tile + (fetches_v ? SH::kHalf : 0), row, fetches_v ? swz_v<C, false>(row) : swz_k<C>(row), code_k[q]);
            if constexpr (N == kWaves) put(tile + SH::kHalf, row, swz_v<C, false>(row), code_v[q]);
        }
        if (!fetches_v && lane < 32) {
            float* const steps = reinterpret_cast<float*>(tile + 2 * SH::kHalf + group * 128) + col;
            if (grp == 0) steps[0] = step_kv * g.scale_log2e;
            else steps[16] = step_kv;
        }
    };

    __shared__ int s_again;
    const bool unseen = !kCodes && !SEEN && j.ob > max(j.oa, j.sees0 + j.row0 / g.G);   // (the workgroup's first row does not see all)
    if (unseen && threadIdx.x == 0) s_again = 0;   // (a barrier a tile before it is used)
    R rows;
    rows.load(g, j, row0, lane);
    if constexpr (kCodes) {
        if (tiles > 0) { request(0); convert(0); }
        if (tiles > 1) request(1);
    } else {
        if (tiles > 0) fetch(0, 0);
    }
    constexpr int kSteps = D / 32;
    int at_k[kSteps], at_v[D / 16];
#pragma unroll
    for (int kk = 0; kk < kSteps; ++kk) at_k[kk] = col * kRow + (((kk * 4 + grp) ^ swz_k<C>(col)) * 16);   // (repeats every 16 rows)
#pragma unroll
    for (int d = 0; d < D / 16; ++d) at_v[d] = rows.value_offset(d);
    rows.arrived();
    // Own keys that this wavefront's last row sees; tiles past them, and all where it has no rows, are left to the others (6 prompts of up to 1365 tokens behind
    // 4111: 389 us -> 373; as a branch inside the loop 380, and 4 - 7 % lost at heads of 64 and 256)
    const int seen = __builtin_amdgcn_readfirstlane(row0 < j.rows ? j.sees0 + (min(row0 + 16 * MT, j.rows) - 1) / g.G : 0);
    const int work_tiles = row0 >= j.rows ? 0 : np + (min(seen, j.ob) > j.oa ? (min(seen, j.ob) - j.oa + kTile - 1) / kTile : 0);
    auto landed = [&](int tile, uint32_t slot) {
        if constexpr (!kCodes) wait_vm<0>();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();     // the tile has landed for everyone, and everyone is done with the one before
        asm volatile("" ::: "memory");
        if constexpr (kCodes) {
            if (tile + 1 < tiles) convert(SH::kSlot - slot);
            if (tile + 2 < tiles) request(tile + 2);
        } else {
            if (tile + 1 < tiles) fetch(tile + 1, SH::kSlot - slot);
        }
    };
    auto step = [&](int tile, auto slot_c) {
        constexpr int slot = decltype(slot_c)::value * SH::kSlot;
        landed(tile, slot);
        const char* const kt = lds + slot;
        const char* const vt = kt + SH::kHalf;

        f32x4 s[MT][N];
#pragma unroll
        for (int n = 0; n < N; ++n) {
#pragma unroll
            for (int i = 0; i < MT; ++i) s[i][n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int kk = 0; kk < kSteps; ++kk) {
                const i32x4 w = *reinterpret_cast<const i32x4*>(kt + at_k[kk] + n * 16 * kRow);
#pragma unroll
                for (int i = 0; i < MT; ++i) s[i][n] = R::M::mul(__builtin_bit_cast(V, w), rows.q[i][kk], s[i][n]);
            }
        }
        const char* const steps = kt + 2 * SH::kHalf + grp * 16;
        if constexpr (kCodes) {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const Float4 ks = *reinterpret_cast<const Float4*>(steps + n * 128);
#pragma unroll
                for (int i = 0; i < MT; ++i) s[i][n] *= f32x4{ks.f[0], ks.f[1], ks.f[2], ks.f[3]};
            }
        }
        rows.template attend<N, SEEN>(s, vt, at_v, first_key(tile), tile < np ? j.pb : j.ob, tile >= np, [&](int n) { return *reinterpret_cast<const Float4*>(steps + n * 128 + 64); });
    };
    for (int tile = 0; tile < work_tiles; tile += 2) {
        step(tile, std::integral_constant<int, 0>{});
        if (tile + 1 < work_tiles) step(tile + 1, std::integral_constant<int, 1>{});
    }
    for (int tile = work_tiles; tile < tiles; ++tile) landed(tile, (tile & 1) * (uint32_t)SH::kSlot);
    if (est && lane == 0) raise_status(g.status, est);
    if (unseen) {
        if (rows.not_finite() && lane == 0) s_again = 1;
        __syncthreads();
        if (__builtin_amdgcn_readfirstlane(s_again) != 0) return true;
    }
    rows.finish();
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const float l = row_reduce(rows.l[i], OpAdd());
        const int r = row0 + 16 * i + col;
        if (r < j.rows) {
#pragma unroll
            for (int d = 0; d < D / 16; ++d) store_row<D>(g, j, r, d * 16 + grp * 4, rows.o[i][d], rows.m[i], l);
        }
    }
    return false;
}

// STREAM: past the caches
template <class E, int D, bool STREAM, bool SEEN>
__device__ __forceinline__ bool wide_block(const Args& g, const Job& j, char* lds)
{
    using SH = Shape<E, D>;
    using R = Rows<E, D, 1, SH::kCodes>;
    using V = typename R::V;
    constexpr int C = SH::kChunks, kRow = SH::kRow, N = kWideKeys / 16;
    constexpr bool kCodes = SH::kCodes;
    const int thread = thread_index<SEEN>(), lane = thread & (kWave - 1), col = lane & 15, grp = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(thread / kWave);

    // one range: the prefix's or the sequence's
    const bool own = j.ob > j.oa;
    const int begin = own ? j.oa : j.pa, end = own ? j.ob : j.pb;
    const int32_t* const table = own ? j.table : g.prefix_table;
    const int first = begin + wave * kWideKeys, step = kWaves * kWideKeys;
    const int tiles = end > first ? (end - first + step - 1) / step : 0;
    uint32_t est = 0;
    char* const vt = lds + wave * SH::kWideV;

    // a tile as it is in flight: K in the operand's order, V 16 bytes a lane, rows across the lanes
    constexpr int kK = N * D / (kCodes ? 64 : 32), kV = N * SH::kLoads;
    i32x4 kr[kK], vr[kV];
    Float4 kst[N], vst[N];
    int next_page[N];
    auto pages_of = [&](int tile) {
#pragma unroll
        for (int n = 0; n < N; ++n) next_page[n] = scalar_at(table, min(first + tile * step + n * 16, end - 1) >> g.page_shift);
    };
    auto value_at = [](const char* p) {
        const i32x4* const at = reinterpret_cast<const i32x4*>(p);
        if constexpr (STREAM) return __builtin_nontemporal_load(at);
        else return *at;
    };
    auto request = [&](int tile) {
        const int in_page = g.page_size - 1;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            int page = next_page[n];
            if ((unsigned)page >= (unsigned)g.pages) { est |= AWEQ_ST_INDEX; page = 0; }
            const int64_t head_row = ((int64_t)page * g.Hk + j.kvh) << g.page_shift;
            const int key0 = first + tile * step + n * 16;
            const char* const kb = reinterpret_cast<const char*>(g.k_cache) + head_row * kRow;
            const char* const vb = reinterpret_cast<const char*>(g.v_cache) + head_row * kRow;
            const int krow = min(key0 + col, end - 1) & in_page;
#pragma unroll
            for (int kk = 0; kk < kK / N; ++kk) kr[n * (kK / N) + kk] = value_at(kb + (uint32_t)(krow * kRow + (kk * 4 + grp) * 16));
#pragma unroll
            for (int q = 0; q < SH::kLoads; ++q) {
                const int row = min(key0 + q * SH::kRowsPerLoad + lane / C, end - 1) & in_page;
                vr[n * SH::kLoads + q] = value_at(vb + (uint32_t)(row * kRow + (lane % C) * 16));
            }
            if constexpr (kCodes) {   // (past the end: anything)
                const int row = ((key0 < end ? key0 : (end - 1) & ~15) & in_page) + grp * 4;
                kst[n] = *reinterpret_cast<const Float4*>(g.k_step + head_row + row);
                vst[n] = *reinterpret_cast<const Float4*>(g.v_step + head_row + row);
            }
        }
    };
    __shared__ int s_again;
    const bool unseen = !kCodes && !SEEN && own && end > j.sees0 + j.row0 / g.G;
    if (unseen) {
        if (threadIdx.x == 0) s_again = 0;
        __syncthreads();
    }
    R rows;
    if (tiles > 0) pages_of(0);
    rows.load(g, j, j.row0, lane);
    if (tiles > 0) {
        request(0);
        if (tiles > 1) pages_of(1);
    }
    int at_v[D / 16];
#pragma unroll
    for (int d = 0; d < D / 16; ++d) at_v[d] = rows.value_offset(d);
    rows.arrived();
    for (int tile = 0; tile < tiles; ++tile) {
        f32x4 s[1][N];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            s[0][n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int kk = 0; kk < kK / N; ++kk) {
                const i32x4 w = kr[n * (kK / N) + kk];
                if constexpr (kCodes) {
                    s[0][n] = R::M::mul(codes_to_f16(w[0], w[1]), rows.q[0][2 * kk], s[0][n]);
                    s[0][n] = R::M::mul(codes_to_f16(w[2], w[3]), rows.q[0][2 * kk + 1], s[0][n]);
                } else {
                    s[0][n] = R::M::mul(__builtin_bit_cast(V, w), rows.q[0][kk], s[0][n]);
                }
            }
        }
        wave_lds_fence();     // (the reads of the tile before are ahead of these writes)
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int q = 0; q < SH::kLoads; ++q) {
                const int row = n * 16 + q * SH::kRowsPerLoad + lane / C;
                *reinterpret_cast<i32x4*>(vt + row * kRow + (((lane % C) ^ swz_v<C, kCodes>(row)) * 16)) = vr[n * SH::kLoads + q];
            }
        wave_lds_fence();
        Float4 vs[N];
        if constexpr (kCodes) {
#pragma unroll
            for (int n = 0; n < N; ++n) {
#pragma unroll
                for (int v = 0; v < 4; ++v) s[0][n][v] *= kst[n].f[v] * g.scale_log2e;
                vs[n] = vst[n];
            }
        }
        if (tile + 1 < tiles) {
            request(tile + 1);
            if (tile + 2 < tiles) pages_of(tile + 2);
        }
        rows.template attend<N, SEEN>(s, vt, at_v, first + tile * step, end, own, [&](int n) { return vs[n]; });
    }
    if (est && lane == 0) raise_status(g.status, est);

    // the wavefronts' keys of the same 16 rows
    if (unseen && rows.not_finite() && lane == 0) s_again = 1;
    rows.finish();
    const float l = row_reduce(rows.l[0], OpAdd());
    __syncthreads();   // (every wavefront is done with its tiles)
    if (unseen && __builtin_amdgcn_readfirstlane(s_again) != 0) return true;
    float* const so = reinterpret_cast<float*>(lds);                         // [wave][row][D]
    float* const sm = so + kWaves * kWideRows * D;                           // [wave][row][2]
#pragma unroll
    for (int d = 0; d < D / 16; ++d) *reinterpret_cast<f32x4*>(so + (wave * 16 + col) * D + ((d * 4 + grp) ^ col) * 4) = rows.o[0][d];
    if (grp == 0) { sm[(wave * 16 + col) * 2] = rows.m[0]; sm[(wave * 16 + col) * 2 + 1] = l; }
    __syncthreads();
    for (int e = thread; e < kWideRows * D / 4; e += kThreads) {
        const int r = e / (D / 4), d = e % (D / 4);
        if (j.row0 + r >= j.rows) continue;
        float mm = -INFINITY, ll = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) mm = fmaxf(mm, sm[(w * 16 + r) * 2]);
        const float use = mm == -INFINITY ? 0.0f : mm;
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float a = __builtin_amdgcn_exp2f(sm[(w * 16 + r) * 2] - use);
            ll += a * sm[(w * 16 + r) * 2 + 1];
            v += a * *reinterpret_cast<const f32x4*>(so + (w * 16 + r) * D + (d ^ r) * 4);
        }
        store_row<D>(g, j, j.row0 + r, d * 4, v, mm, ll);
    }
    return false;
}

// Wavefronts a SIMD that the registers have to allow, and for which the compiler orders loads and products (with room for one more it waited for each load of a
// tile by itself: 8-bit codes, row tiles of 64, 5 tokens of 16 sequences of up to 6000 keys 42.0 us -> 36.6; binary16, 711 tokens x 8 heads 21.5 -> 20.0)
constexpr int waves_wanted(int D, int MT) { return D == 64 ? (MT == 2 ? 2 : 4) : D == 128 ? (MT == 0 ? 3 : 2) : MT == 1 ? 2 : 1; }

// MT: 16 MT rows for each wavefront of the tall form; 0: a launch without it.  STREAM (MT 0): keys and values past the caches (rule and figures at the launch)
template <class E, int D, int MT, bool STREAM, bool SEEN>
__device__ __forceinline__ bool attention_block(const Args& g, int block, char* lds)
{
    const bool shared = block < g.shared.blocks;
    const Work& w = shared ? g.shared : g.own;
    const int id = block - (shared ? 0 : g.shared.blocks);
    // Workgroup ids go round-robin over the XCDs: all row tiles of one range of a key head to the same one, whose L2 then has the range's K and V
    const int seq = id / kXcdCount, combo = seq / w.row_tiles * kXcdCount + id % kXcdCount;
    if (combo >= w.combos) return false;
    const int split = combo / g.Hk % w.splits, b = combo / g.Hk / w.splits;
    const int tile_rows = w.tall ? kWaves * 16 * MT : kWideRows;
    Job j;
    j.kvh = combo % g.Hk;
    j.row0 = (w.row_tiles - 1 - seq % w.row_tiles) * tile_rows;   // (a prompt's last rows, which see most keys, first)
    j.part = w.first_part + split;
    j.pa = j.pb = j.oa = j.ob = 0;
    j.sees0 = 0;
    j.table = g.table;
    uint32_t est = 0;
    if (shared) {
        j.t0 = 0;
        j.rows = (int)g.T * g.G;
        j.pa = split * w.chunk;
        j.pb = min(j.pa + w.chunk, g.prefix_len);
    } else {
        int64_t t0 = b, t1 = b + 1;
        if (g.q_start) {
            t0 = scalar_at(g.q_start, b);
            t1 = scalar_at(g.q_start, b + 1);
            if (t0 < 0 || t1 < t0 || t1 > g.T || t1 - t0 > g.max_q) est |= AWEQ_ST_INDEX;
            t0 = min(max(t0, (int64_t)0), g.T);
            t1 = min(max(t1, t0), min(g.T, t0 + g.max_q));
        }
        const int tokens = (int)(t1 - t0);
        int len = scalar_at(g.lens, b);
        const int most = (int)min((int64_t)g.max_len, g.table_ld << g.page_shift);
        if (len < 0 || len > most) est |= AWEQ_ST_INDEX;
        len = min(max(len, 0), most);
        if (est && threadIdx.x == 0) raise_status(g.status, est);
        j.t0 = t0;
        j.rows = tokens * g.G;
        if (j.row0 >= j.rows) return false;
        j.sees0 = len - tokens + 1;
        j.table = g.table + (int64_t)b * g.table_ld;
        const int seen = max(0, min(len, j.sees0 + min((j.row0 + tile_rows - 1) / g.G, tokens - 1)));   // by the workgroup's last row
        if (w.chunk) {
            j.oa = split * w.chunk;
            j.ob = min(j.oa + w.chunk, seen);
        } else {
            // a share of the tiles of the prefix and the sequence together
            const int np = g.fused ? (g.prefix_len + kTallKeys - 1) / kTallKeys : 0, all = np + (seen + kTallKeys - 1) / kTallKeys;
            const int lo = (int)((int64_t)all * split / w.splits), hi = (int)((int64_t)all * (split + 1) / w.splits);
            j.pa = min(lo, np) * kTallKeys;
            j.pb = min(min(hi, np) * kTallKeys, g.fused ? g.prefix_len : 0);
            j.oa = (max(lo, np) - np) * kTallKeys;
            j.ob = min((max(hi, np) - np) * kTallKeys, seen);
        }
    }
    if constexpr (MT > 0) return w.tall ? tall_block<E, D, MT, SEEN>(g, j, lds) : wide_block<E, D, false, SEEN>(g, j, lds);
    else return wide_block<E, D, STREAM, SEEN>(g, j, lds);
}

template <class E, int D, int MT, bool STREAM>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(waves_wanted(D, MT), waves_wanted(D, MT)))) void attention_kernel(Args g)
{
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    int block = (int)blockIdx.x;
    if (!attention_block<E, D, MT, STREAM, false>(g, block, lds) || Shape<E, D>::kCodes) return;
    // Once more, from the arguments on: nothing is kept in registers for it
    typedef const __attribute__((address_space(4))) Args* ConstArgs;
    ConstArgs from = (ConstArgs)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(from), "+s"(block)::"memory");
    __syncthreads();   // (of the tiles and the flag)
    const Args again = *(const Args*)from;
    attention_block<E, D, MT, STREAM, true>(again, block, lds);
}

constexpr int kJoinParts = 256;

// A row's parts joined by W wavefronts: a lane has the maximum and sum of the parts lane, lane + 64, .., wavefront v takes the values of the parts 64 c + W i
// + v, D / 4 lanes to a part, kFlight of them in flight
template <int D, int W>
__global__ __launch_bounds__(256) void join_kernel(Args g)
{
    constexpr int kRowsOf = 4 / W;   // rows of a workgroup
    __shared__ f32x4 s_part[W > 1 ? W : 1][W > 1 ? D / 4 : 1];
    const int wave = threadIdx.x / kWave, slice = wave % W, lane = threadIdx.x & (kWave - 1);
    const int64_t row = (int64_t)blockIdx.x * kRowsOf + wave / W, all_rows = g.T * g.Hq;
    if (row >= all_rows) return;     // (W > 1: all of the workgroup or nobody)
    constexpr int kLanes = D / 4, kAtOnce = kWave / kLanes, kOf = W > 1 ? kJoinParts / kWave : 1, kFlight = 8;
    const int sub = lane / kLanes, at = lane % kLanes * 4;
    float2 ml[kOf];
    float mm = -INFINITY;
#pragma unroll
    for (int c = 0; c < kOf; ++c) {
        ml[c] = make_float2(-INFINITY, 0.0f);
        if (c * kWave + lane < g.parts) ml[c] = g.part_ml[(int64_t)(c * kWave + lane) * all_rows + row];
        mm = fmaxf(mm, ml[c].x);
    }
    mm = wave_allreduce(mm, Larger());
    float w[kOf], ll = 0.0f;
    uint64_t there[kOf];             // parts that have keys: of no weight at all, they may still have a NaN or an infinity
#pragma unroll
    for (int c = 0; c < kOf; ++c) {
        const bool keys = ml[c].y != 0.0f;
        there[c] = __builtin_amdgcn_ballot_w64(keys);
        w[c] = keys ? __builtin_amdgcn_exp2f(ml[c].x - mm) : 0.0f;
        ll += w[c] * ml[c].y;
    }
    ll = wave_allreduce(ll, OpAdd());
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < kOf; ++c) {
        const int n = min(g.parts - c * kWave, kWave);
        for (int p0 = slice * kAtOnce; p0 < n; p0 += W * kAtOnce * kFlight) {
            f32x4 x[kFlight];
            float a[kFlight];
#pragma unroll
            for (int f = 0; f < kFlight; ++f) {
                const int p = p0 + f * W * kAtOnce + sub;
                a[f] = __shfl(w[c], p & (kWave - 1));
                x[f] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                if (p < n && (there[c] >> p & 1)) x[f] = *reinterpret_cast<const f32x4*>(g.part_o + ((int64_t)(c * kWave + p) * all_rows + row) * D + at);
            }
#pragma unroll
            for (int f = 0; f < kFlight; ++f) v += a[f] * x[f];
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (kAtOnce > 2) v[e] += __shfl_xor(v[e], 16);
        if constexpr (kAtOnce > 1) v[e] += __shfl_xor(v[e], 32);
    }
    if constexpr (W > 1) {
        if (sub == 0) s_part[slice][at / 4] = v;
        __syncthreads();
        if (slice != 0) return;
#pragma unroll
        for (int o = 1; o < W; ++o) v += s_part[o][at / 4];
    }
    const float inv = ll != 0.0f ? 1.0f / ll : 0.0f;
    if (sub == 0) {
        const int64_t to = row / g.Hq * g.ldo + row % g.Hq * D + at;
        if (g.q_bf16) {
            typedef __bf16 b4 __attribute__((ext_vector_type(4)));
            *reinterpret_cast<b4*>(reinterpret_cast<__bf16*>(g.out) + to) = b4{(__bf16)(v[0] * inv), (__bf16)(v[1] * inv), (__bf16)(v[2] * inv), (__bf16)(v[3] * inv)};
        } else {
            *reinterpret_cast<f16x4*>(reinterpret_cast<_Float16*>(g.out) + to) = f16x4{(_Float16)(v[0] * inv), (_Float16)(v[1] * inv), (_Float16)(v[2] * inv), (_Float16)(v[3] * inv)};
        }
    }
    if (lane == 0 && g.lse) g.lse[row] = ll != 0.0f ? (mm + __builtin_amdgcn_logf(ll)) * kLn2 : -INFINITY;
}

// How a call is cut up
struct Plan {
    int mt;             // row tiles of a wavefront of the tall form, 0: none
    int fused;
    Work shared, own;   // splits 0: no such work
    int parts() const { return shared.splits + own.splits; }
};

constexpr int kMostSplits = 128;
static_assert(2 * kMostSplits <= kJoinParts, "the join has room for them");

// ranges of `len` keys so that `items` of them each make up about `want` workgroups, of `least` keys or more
static int64_t split_count(int64_t items, int64_t len, int64_t want, int64_t least)
{
    const int64_t n = cdiv(want, items), most = cdiv(len, least);
    const int64_t k = n < most ? n : most;
    return k < 1 ? 1 : k > kMostSplits ? kMostSplits : k;
}
// Tall workgroups: one for each compute unit, of 512 keys or more, or two, which overlap one's products with the other's exponentials, where that leaves
// 1024 keys: a range's rows are written and read once more to be joined (us, one -> two: 1024 rows a key head against 16384 keys 95 -> 82, but 256 rows
// against 8192 23.1 -> 25.1, and with the batch's own keys in the same launch 38.2 -> 47.1).  Ranges of 256 keys where most compute units had none.
constexpr int64_t kTallWant = 512, kTallLeast = 256, kWideWant = 2048, kWideLeast = 128;
static int64_t tall_splits(int64_t items, int64_t len)
{
    const int64_t one = split_count(items, len, kTallWant / 2, 2 * kTallLeast), two = split_count(items, len, kTallWant, 4 * kTallLeast);
    if (items * one < 64) return split_count(items, len, kTallWant / 2, kTallLeast);
    return one > two ? one : two;
}
// Wide workgroups: eight for each compute unit (sequences differ in length; two for a single range), of 512 keys or more, or of less where most compute units had none (us, 256 ->
// 512: 64 sequences of up to 500 keys 20.4 -> 15.0, 128 of up to 400 40.4 -> 31.5, 8 of up to 4000 28.6 -> 25.3; but one of 1900 with 32 key heads 12.0 -> 13.0)
static int64_t wide_splits(int64_t items, int64_t len, bool one)
{
    int64_t n = 1;
    for (int64_t least = 4 * kWideLeast; least >= kWideLeast; least /= 2) {
        n = split_count(items, len, one ? kWideWant / 4 : kWideWant, least);
        if (items * n >= 256) break;
    }
    return n;
}
static void set_work(Work& w, int64_t rows, int mt, int64_t splits, int64_t len, int64_t items)
{
    const int tile = w.tall ? kWaves * 16 * mt : kWideRows, unit = w.tall ? kTallKeys : kWaves * kWideKeys;
    w.row_tiles = (int)cdiv(rows, tile);
    w.chunk = (int)(cdiv(cdiv(len, splits), unit) * unit);
    if (w.chunk < unit) w.chunk = unit;
    w.splits = len > 0 ? (int)cdiv(len, w.chunk) : 1;
    w.combos = (int)(items * w.splits);
}

static Plan plan(int64_t D, bool codes, int64_t T, int64_t Hq, int64_t Hk, int64_t B, int64_t max_q, int64_t prefix_len, int64_t max_len)
{
    const int64_t G = Hq / Hk, all_rows = T * G, most_rows = max_q * G;
    Plan p = {};
    const bool own_tall = most_rows > kWideRows, shared_tall = all_rows > kWideRows;
    // Where sequences have a tile's rows each, on average, they take the prefix along: every row tile reads it once either way, and nothing is
    // left to join
    p.fused = prefix_len > 0 && own_tall && all_rows >= B * 128;
    const bool has_shared = prefix_len > 0 && !p.fused, has_own = max_len > 0 || prefix_len == 0 || p.fused;
    // Row tiles of 16 a wavefront: one of 256 values, so that two workgroups share a compute unit (us, two -> one: 190-token chunks of 4 sequences of 4000 - 8000
    // keys 288 -> 209, 2048 tokens behind 4096 keys 271 -> 207); but where single tokens' workgroups have the launch in common, which hold 16-bit keys in the
    // registers of two (decode of 64 behind 8192 62 -> 84), not.  With shorter heads one where workgroups of two are no more than the compute units (us, two -> one: 300 tokens x 16
    // heads of codes 19.1 -> 12.9, 500 x 32 17.7 -> 15.3, 1000 x 32 heads of 64 20.1 -> 16.1, of 128 28.4 -> 25.5, two of 700 x 8 23.2 -> 21.7; but 2000 x 8 37.7 ->
    // 38.4, and where ranges of more keys fill the chip, 200 behind 6000, 44 -> 59)
    const int64_t own_keys = max_len + (p.fused ? prefix_len : 0), pairs = B * Hk * cdiv(most_rows, 2 * kWaves * 16);
    const bool fills = pairs * tall_splits(pairs, own_keys) > 256;
    p.mt = has_own && own_tall ? (most_rows > 64 && D < 256 && fills ? 2 : 1) : 0;
    if (has_shared && shared_tall && p.mt < 2) p.mt = D == 256 ? (has_own && !own_tall && !codes ? 2 : 1) : all_rows > 64 ? 2 : 1;
    if (has_shared) {
        p.shared.tall = shared_tall;
        const int64_t tile = shared_tall ? kWaves * 16 * p.mt : kWideRows;
        const int64_t items = Hk * cdiv(all_rows, tile);
        set_work(p.shared, all_rows, p.mt, shared_tall ? tall_splits(items, prefix_len) : wide_splits(items, prefix_len, true), prefix_len, Hk);
    }
    if (has_own) {
        p.own.tall = own_tall;
        const int64_t tile = own_tall ? kWaves * 16 * p.mt : kWideRows, items = B * Hk * cdiv(most_rows, tile);
        const int64_t keys = max_len + (p.fused ? prefix_len : 0);
        set_work(p.own, most_rows, p.mt, own_tall ? tall_splits(items, keys) : wide_splits(items, keys, B == 1), keys, B * Hk);
        if (own_tall) p.own.chunk = 0;
    }
    return p;
}

template <class E, int D, int MT, bool STREAM = false>
static int launch_one(const Args& g, int64_t blocks, hipStream_t st)
{
    constexpr int lds = Shape<E, D>::lds(MT > 0);
    const void* fn = reinterpret_cast<const void*>(attention_kernel<E, D, MT, STREAM>);
    int dev = 0, cus = 0;
    if (device_cus(dev, cus) != AWEQ_OK || raise_lds_limit(fn, dev, lds) != AWEQ_OK) return AWEQ_ERR_LAUNCH;
    void* args[] = {const_cast<Args*>(&g)};
    return hipLaunchKernel(fn, dim3((unsigned)blocks), dim3(kThreads), args, lds, st) == hipSuccess ? AWEQ_OK : AWEQ_ERR_LAUNCH;
}

template <class E, int D>
static int launch(Args& g, const Plan& p, hipStream_t st)
{
    int64_t blocks = 0;
    g.shared = p.shared;
    g.own = p.own;
    g.own.first_part = p.shared.splits;
    for (Work* w : {&g.shared, &g.own}) {
        const int64_t n = w->splits ? cdiv(w->combos, kXcdCount) * kXcdCount * w->row_tiles : 0;
        blocks += n;
        if (blocks > (1 << 24) - 1) return AWEQ_ERR_SHAPE;   // 2^32 threads
        w->blocks = (int)n;
    }
    // Past the caches where the sequences' own keys may not fit them (us, through -> past them: 368 MB of codes 100 -> 95, 737 MB 173 -> 162, 245 MB 51 -> 46, 209 MB
    // 31.6 -> 28.4, but 131 MB 14.9 -> 16.4)
    const bool stream = p.mt == 0 && (int64_t)p.own.combos / (p.own.splits ? p.own.splits : 1) * g.max_len * 2 * D * (int64_t)sizeof(E) > kCacheBytes / 4 * 3;
    const int rc = stream ? launch_one<E, D, 0, true>(g, blocks, st) : p.mt == 0 ? launch_one<E, D, 0>(g, blocks, st) : p.mt == 1 ? launch_one<E, D, 1>(g, blocks, st) : launch_one<E, D, D == 256 && Shape<E, D>::kCodes ? 1 : 2>(g, blocks, st);
    if (rc == AWEQ_OK && g.parts > 1) {
        const int64_t rows = g.T * g.Hq;
        // (up to 64 parts a wavefront is as fast as four or faster: 2048 rows of 18 parts 35.1 us with the attention, four each 44.7)
        if (g.parts > kWave) join_kernel<D, 4><<<(unsigned)rows, 256, 0, st>>>(g);
        else join_kernel<D, 1><<<(unsigned)cdiv(rows, 4), 256, 0, st>>>(g);
    }
    return rc != AWEQ_OK ? rc : launch_status();
}

template <class E>
static int launch_head(Args& g, const Plan& p, int64_t D, hipStream_t st)
{
    if (D == 64) return launch<E, 64>(g, p, st);
    if (D == 128) return launch<E, 128>(g, p, st);
    return launch<E, 256>(g, p, st);
}

// Rows (a token's query head) times ranges of one kind, at most, for up to `rows` of them and `len` keys.  The work items' tiles hold all rows, so that `want`
// workgroups of at most `tile` rows each, and one range more (rounding up), have no more; nor has a row more ranges than the keys allow.
static int64_t most_parts(int64_t rows, int64_t len)
{
    static_assert(kTallWant * kWaves * 32 >= kWideWant * kWideRows && kTallLeast >= kWideLeast, "the tall form has the larger product, the wide one the shorter ranges");
    const int64_t ranges = cdiv(len, kWideLeast), by_keys = rows * (ranges < kMostSplits ? ranges : kMostSplits), by_work = kTallWant * kWaves * 32 + rows;
    return by_keys < by_work ? by_keys : by_work;
}

static bool shapes_ok(int64_t T, int64_t Hq, int64_t Hk, int64_t D, int64_t B, int64_t max_q, int64_t prefix_len, int64_t max_len)
{
    if (T <= 0 || Hq <= 0 || Hk <= 0 || Hq % Hk != 0 || (D != 64 && D != 128 && D != 256) || B <= 0 || max_q <= 0) return false;
    if (prefix_len < 0 || max_len < 0 || prefix_len > (1 << 29) || max_len > (1 << 29)) return false;
    return T <= (1 << 24) && B <= (1 << 20) && Hq <= (1 << 16) && T * Hq < (1 << 24) && B * Hk <= (1 << 24);
}

}  // namespace attn
}  // namespace aweq

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
    if (!q || !out || !k_cache || !v_cache || !lens || (max_len > 0 && !table) || (prefix_len > 0 && !prefix_table)) return AWEQ_ERR_NULL;
    if ((dt != AWEQ_F16 && dt != AWEQ_BF16) || (cache_dt != dt && cache_dt != AWEQ_I8)) return AWEQ_ERR_DTYPE;
    if (cache_dt == AWEQ_I8 && (!k_step || !v_step)) return AWEQ_ERR_NULL;
    if (!attn::shapes_ok(T, Hq, Hk, D, B, max_q, prefix_len, max_len)) return AWEQ_ERR_SHAPE;
    max_q = max_q < T ? max_q : T;
    if (pages <= 0 || pages > 0x7fffffff || page_size < 16 || page_size > 256 || (page_size & (page_size - 1)) != 0) return AWEQ_ERR_SHAPE;
    if (!(scale > 0.0f) || !(scale < 0x1p127f)) return AWEQ_ERR_SHAPE;   // (to base 2 it has to be finite)
    if (ldq < Hq * D || ldo < Hq * D || (!q_start && (T != B || max_q != 1)) || (max_len > 0 && table_ld < 1)) return AWEQ_ERR_SHAPE;
    if (!aligned16(q) || !aligned16(out) || (ldq % 8) != 0 || (ldo % 8) != 0 || !aligned16(k_cache) || !aligned16(v_cache) ||
        (cache_dt == AWEQ_I8 && (!aligned16(k_step) || !aligned16(v_step))))
        return AWEQ_ERR_ALIGN;
    const attn::Plan p = attn::plan(D, cache_dt == AWEQ_I8, T, Hq, Hk, B, max_q, prefix_len, max_len);
    const size_t need = aweq_prefix_attention_ws(T, Hq, Hk, D, B, max_q, prefix_len, max_len);
    if (need && (!ws || ws_bytes < need)) return AWEQ_ERR_WORKSPACE;
    if (need && !aligned16(ws)) return AWEQ_ERR_ALIGN;
    attn::Args g = {};
    g.q = q; g.k_cache = k_cache; g.v_cache = v_cache; g.k_step = k_step; g.v_step = v_step;
    g.prefix_table = prefix_table; g.table = table; g.lens = lens; g.q_start = q_start;
    g.out = out; g.lse = lse; g.status = status;
    g.T = T; g.ldq = ldq; g.ldo = ldo; g.table_ld = table_ld; g.prefix_len = (int)prefix_len; g.max_len = (int)max_len;
    g.pages = (int)pages; g.page_size = (int)page_size; g.page_shift = __builtin_ctz((unsigned)page_size);
    g.Hq = (int)Hq; g.Hk = (int)Hk; g.G = (int)(Hq / Hk); g.max_q = (int)max_q;
    g.q_bf16 = dt == AWEQ_BF16;
    g.parts = p.parts();
    g.fused = p.fused;
    g.scale_log2e = scale * attn::kLog2e;
    g.part_o = reinterpret_cast<float*>(ws);
    g.part_ml = reinterpret_cast<float2*>(g.part_o + (size_t)g.parts * (size_t)(T * Hq) * (size_t)D);
    hipStream_t st = as_stream(stream);
    if (cache_dt == AWEQ_I8) return attn::launch_head<int8_t>(g, p, D, st);
    if (dt == AWEQ_F16) return attn::launch_head<_Float16>(g, p, D, st);
    return attn::launch_head<__bf16>(g, p, D, st);
}
