// Norm of every head of queries and keys, rotation by the token's position, and the way of keys and values into a paged cache, in one pass
// over a token's heads.
//
// HBM-bound: every value is read and written once.  Measured (us, TB/s of both): 4099 tokens x 128 heads of 128 binary16 values 48.4, 5.5; append of 7001
// tokens x 80 heads, normed, 55.5, 5.2, into 8-bit codes 61, 4.5; a copy of 1 GB reaches 5.2.  A decode step's call (48 tokens x 96 heads) is its launch, 4.8.
//
//   y = x w / sqrt(mean x^2 + eps);   the pair (a, b) of a head turns into (a cos - b sin, b cos + a sin), angle = pos freq[i]
//
// A lane holds two units of 8 values, chosen so that both values of its pairs are its own (units u and u + rot / 16 of the half layout; any of the
// interleaved one) and neighbouring lanes' units are neighbours in memory; nothing crosses lanes but the norm's sum.  2^G lanes have a head, and
// a workgroup walks over the heads of its tokens, the next ones requested while these are worked on.  Each of its tokens has rot / 2 angles, formed
// once, by a thread each, while the first values are on their way: the product pos freq in binary64, reduced to a part of a turn there (in binary32
// a position of 100000 has lost the angle's last three digits), then sine and cosine of that in binary32.
#include "wide_unit.hpp"

#include <cmath>

namespace aweq {
namespace rope {

constexpr int kThreads = 256;
constexpr int kMaxHead = 256;
constexpr int kMaxTokens = 8;   // of a workgroup

struct Args {
    const void *q, *k, *v;
    void *q_out, *k_out;        // (rows; k_out not with a cache)
    int64_t ldq, ldk, ldv, ldqo, ldko;
    const int32_t* pos;
    const double* freq;
    const float *q_norm, *k_norm;
    float eps, gain;
    int Hq, Hk, D, rot, interleaved;
    int rows;                   // heads of a token that the pass moves: queries, keys, then values
    int tokens;                 // of a workgroup
    int parts, part_rows;       // or (tokens = 1) workgroups to a token, and the heads of each
    int64_t T, first;           // all tokens; the launch's first one
    void *k_cache, *v_cache;
    float *k_step, *v_step;
    int64_t pages, page_size;
    const int64_t* slot;
    uint32_t* status;
};

enum { kRows, kCache, kCodes };   // where keys go: rows as queries do, a cache of the same type, a cache of 8-bit codes

// largest |x| of a head's values to a step, its codes and the step itself to the cache.  False where one is not finite: the step is NaN then, and what reads
// the head finds nothing but NaN, whatever the codes
template <int G>
__device__ __forceinline__ bool store_codes(int8_t* dst, float* step_at, const float a[8], const float b[8], int ua, int ub, int units, bool writes_step)
{
    float big = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) big = OpMaximum()(big, OpMaximum()(fabsf(a[i]), fabsf(b[i])));
    big = group_allreduce<G>(big, OpMaximum());
    const bool finite = big < INFINITY;
    float step = fmaxf(big / 127.0f, 1.17549435e-38f);   // (not subnormal: the quotients keep their digits)
    if (big == 0.0f) step = 1.0f;
    if (!finite) step = NAN;
    if (writes_step) *step_at = step;
    auto pack = [&](const float x[8]) {
        uint32_t w[2] = {0u, 0u};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = (int)rintf(__builtin_amdgcn_fmed3f(x[i] / step, -127.0f, 127.0f));
            w[i >> 2] |= (uint32_t)(c & 0xff) << (8 * (i & 3));
        }
        return make_uint2(w[0], w[1]);
    };
    if (ua < units) *reinterpret_cast<uint2*>(dst + ua * 8) = pack(a);
    if (ub < units) *reinterpret_cast<uint2*>(dst + ub * 8) = pack(b);
    return finite;
}

// STREAM: past the caches (the rule and figures at the launch)
template <class E, int G, int DEST, bool NORM, bool STREAM>
__global__ __launch_bounds__(kThreads) void rope_kernel(Args g)
{
    __shared__ __attribute__((aligned(16))) float s_cos[kMaxTokens][kMaxHead / 2], s_sin[kMaxTokens][kMaxHead / 2];
    __shared__ __attribute__((aligned(16))) float s_norm[NORM ? 2 : 1][NORM ? kMaxHead : 4];   // the norms' weights
    __shared__ int64_t s_row[kMaxTokens];   // row of the cache within a head's pages (page Hk page_size + row), negative: the token is left out
    static_assert(kThreads >= kMaxHead, "a thread each");
    constexpr int kLanes = 1 << G, kHeads = kThreads / kLanes;   // lanes of a head, heads of a round
    const int64_t t0 = g.first + (int64_t)(blockIdx.x / (unsigned)g.parts) * g.tokens;
    const int row0 = (int)(blockIdx.x % (unsigned)g.parts) * g.part_rows;
    const int tokens = (int)min((int64_t)g.tokens, g.T - t0);
    const int lane = threadIdx.x & (kLanes - 1), sub = threadIdx.x >> G;
    const int units = g.D / 8;

    // this lane's two units and whether they are rotated
    const int hh = g.interleaved ? 0 : g.rot / 16;      // pairs of units of the half layout, then the others, the first half of them and the second
    const int others = (units - 2 * hh + 1) / 2;
    const int ua = lane < hh ? lane : lane - hh < others ? hh + lane : units;
    const int ub = lane < hh ? lane + hh : lane - hh < others ? hh + others + lane : units;
    const bool ra = ua * 8 < g.rot, rb = ub * 8 < g.rot;

    // heads of the workgroup's tokens one after the other; a lane's next head moves on by a round
    struct Head {
        int t, h;               // token of the workgroup; head of its kind
        bool is_q, is_v, has_a, has_b;
        Unit<E> a, b;
    };
    const int last = min(row0 + g.part_rows, g.rows);   // (of each token)
    int at_t = 0, at_row = row0 + sub;
    while (at_row >= last && at_t < tokens) { at_row -= last - row0; ++at_t; }
    auto request = [&]() {
        Head x;
        const bool in = at_t < tokens;
        x.t = in ? at_t : 0;
        const int head = in ? at_row : row0;
        x.is_q = head < g.Hq;
        x.is_v = head >= g.Hq + g.Hk;
        x.h = x.is_q ? head : x.is_v ? head - g.Hq - g.Hk : head - g.Hq;
        const int64_t t = t0 + x.t;
        const E* const src = (x.is_q ? reinterpret_cast<const E*>(g.q) + t * g.ldq : x.is_v ? reinterpret_cast<const E*>(g.v) + t * g.ldv : reinterpret_cast<const E*>(g.k) + t * g.ldk) +
                             (int64_t)x.h * g.D;
        x.has_a = in && ua < units;
        x.has_b = in && ub < units;
        x.a = x.b = Unit<E>{};
        if (x.has_a) x.a = STREAM ? stream_unit(src + ua * 8) : load_unit(src + ua * 8);
        if (x.has_b) x.b = STREAM ? stream_unit(src + ub * 8) : load_unit(src + ub * 8);
        at_row += kHeads;
        while (at_row >= last && at_t < tokens) { at_row -= last - row0; ++at_t; }
        return x;
    };
    Head next = request();

    // angles, one thread each
    const int pairs = g.rot / 2;
    for (int i = threadIdx.x; i < pairs * tokens; i += kThreads) {
        const int t = i / pairs, p = i % pairs;
        double turns = (double)g.pos[t0 + t] * g.freq[p] * 0.15915494309189533577;
        turns -= rint(turns);
        float s, c;
        sincospif(2.0f * (float)turns, &s, &c);
        s_cos[t][p] = g.gain * c;
        s_sin[t][p] = g.gain * s;
    }
    if constexpr (NORM) {
        if ((int)threadIdx.x < g.D) {
            if (g.q_norm) s_norm[0][threadIdx.x] = g.q_norm[threadIdx.x];
            if (g.k_norm) s_norm[1][threadIdx.x] = g.k_norm[threadIdx.x];
        }
    }
    if constexpr (DEST != kRows) {
        if ((int)threadIdx.x < tokens) {
            const int64_t slot = g.slot[t0 + threadIdx.x], p = slot / g.page_size;
            const bool keep = slot >= 0 && p < g.pages;
            if (slot >= 0 && !keep && row0 == 0) raise_status(g.status, AWEQ_ST_INDEX);
            s_row[threadIdx.x] = keep ? p * g.Hk * g.page_size + (slot - p * g.page_size) : -1;
        }
    }
    __syncthreads();

    const int rounds = (tokens * (last - row0) + kHeads - 1) / kHeads;
    for (int round = 0; round < rounds; ++round) {
        const Head x = next;
        if (round + 1 < rounds) next = request();
        const bool is_q = x.is_q, is_v = x.is_v, has_a = x.has_a, has_b = x.has_b;
        const int h = x.h;
        const int64_t t = t0 + x.t;
        // interleaved: the angles of the first and the second unit; half: pairs 0 - 3 and 4 - 7
        float ca[4], sa[4], cb[4], sb[4];
        {
            const int fa = !ra ? 0 : g.interleaved ? ua * 4 : ua * 8, fb = g.interleaved ? (rb ? ub * 4 : 0) : fa + 4;
            const Float4 c0 = *reinterpret_cast<const Float4*>(&s_cos[x.t][fa]), s0 = *reinterpret_cast<const Float4*>(&s_sin[x.t][fa]);
            const Float4 c1 = *reinterpret_cast<const Float4*>(&s_cos[x.t][fb]), s1 = *reinterpret_cast<const Float4*>(&s_sin[x.t][fb]);
#pragma unroll
            for (int j = 0; j < 4; ++j) { ca[j] = c0.f[j]; sa[j] = s0.f[j]; cb[j] = c1.f[j]; sb[j] = s1.f[j]; }
        }
        float a[8], b[8];
        widen<E>(x.a, a);
        widen<E>(x.b, b);
        if constexpr (NORM) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += a[i] * a[i] + b[i] * b[i];
            sum = group_allreduce<G>(sum, OpAdd());
            if (!is_v && (is_q ? g.q_norm : g.k_norm)) {
                const float r = 1.0f / sqrtf(sum / (float)g.D + g.eps);
                const float* const w = s_norm[is_q ? 0 : 1];
                const f32x8 wa = load_unit(w + min(ua, units - 1) * 8), wb = load_unit(w + min(ub, units - 1) * 8);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    a[i] = a[i] * r * wa[i];
                    b[i] = b[i] * r * wb[i];
                }
            }
        }
        if (!is_v) {
            if (g.interleaved) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float v = a[2 * j], y = a[2 * j + 1], z = b[2 * j], u = b[2 * j + 1];
                    if (ra) { a[2 * j] = v * ca[j] - y * sa[j]; a[2 * j + 1] = y * ca[j] + v * sa[j]; }
                    if (rb) { b[2 * j] = z * cb[j] - u * sb[j]; b[2 * j + 1] = u * cb[j] + z * sb[j]; }
                }
            } else if (ra) {   // (both units or neither)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float c = j < 4 ? ca[j & 3] : cb[j & 3], s = j < 4 ? sa[j & 3] : sb[j & 3];
                    const float v = a[j], y = b[j];
                    a[j] = v * c - y * s;
                    b[j] = y * c + v * s;
                }
            }
        }
        auto put = [&](E* dst, bool pa, bool pb) {
            if constexpr (STREAM) {
                if (pa) stream_unit(dst + ua * 8, a);
                if (pb) stream_unit(dst + ub * 8, b);
            } else {
                if (pa) store_unit(dst + ua * 8, a);
                if (pb) store_unit(dst + ub * 8, b);
            }
        };
        if (DEST == kRows || is_q) {
            E* dst = (is_q ? reinterpret_cast<E*>(g.q_out) + t * g.ldqo : reinterpret_cast<E*>(g.k_out) + t * g.ldko) + (int64_t)h * g.D;
            put(dst, has_a, has_b);
        } else {
            const int64_t row = s_row[x.t], at = row + (int64_t)h * g.page_size;
            const bool keep = row >= 0;
            if constexpr (DEST == kCache) {
                E* dst = reinterpret_cast<E*>(is_v ? g.v_cache : g.k_cache) + at * g.D;
                put(dst, has_a && keep, has_b && keep);
            } else {
                const bool kept = (has_a || has_b) && keep;
                const bool finite = store_codes<G>(reinterpret_cast<int8_t*>(is_v ? g.v_cache : g.k_cache) + at * g.D, (is_v ? g.v_step : g.k_step) + at, a, b,
                                                   has_a && keep ? ua : units, has_b && keep ? ub : units, units, kept && lane == 0);
                if (!finite && kept && lane == 0) raise_status(g.status, AWEQ_ST_NONFINITE);
            }
        }
    }
}

template <class E, int DEST, bool NORM, bool STREAM>
static int launch_head(Args g, int64_t T, hipStream_t st)
{
    // 16 values a lane, lanes of a head a power of two
    int G = 0;
    while ((16 << G) < g.D) ++G;
    const int heads = kThreads >> G;
    g.T = T;
    // A workgroup costs some us (its angles, the norms' weights, a barrier) that others hide: a token each until there are 8192, a round of heads each
    // while they would not fill the chip (us: append of 16384 tokens with 48 heads, one token a workgroup -> two 83 -> 75.6, four 77.2; 7001 tokens with 80
    // heads, one -> three 55.6 -> 62.1; a round of 32 heads each 72.0)
    const int64_t share = T / 8192;
    g.tokens = (int)(share < 1 ? 1 : share > kMaxTokens ? kMaxTokens : share);
    g.parts = T < 1024 ? (g.rows + heads - 1) / heads : 1;
    g.part_rows = g.parts > 1 ? heads : g.rows;
    const int64_t most = ((1ll << 32) / kThreads - 1) / g.parts;   // token groups to a launch: fewer than 2^32 threads
    const int64_t groups = cdiv(T, g.tokens);
    for (int64_t b = 0; b < groups; b += most) {
        g.first = b * g.tokens;
        const unsigned grid = (unsigned)((groups - b < most ? groups - b : most) * g.parts);
        switch (G) {
        case 0: rope_kernel<E, 0, DEST, NORM, STREAM><<<grid, kThreads, 0, st>>>(g); break;
        case 1: rope_kernel<E, 1, DEST, NORM, STREAM><<<grid, kThreads, 0, st>>>(g); break;
        case 2: rope_kernel<E, 2, DEST, NORM, STREAM><<<grid, kThreads, 0, st>>>(g); break;
        case 3: rope_kernel<E, 3, DEST, NORM, STREAM><<<grid, kThreads, 0, st>>>(g); break;
        default: rope_kernel<E, 4, DEST, NORM, STREAM><<<grid, kThreads, 0, st>>>(g); break;
        }
        const int rc = launch_status();
        if (rc != AWEQ_OK) return rc;
    }
    return AWEQ_OK;
}

template <class E, int DEST>
static int launch(const Args& g, int64_t T, hipStream_t st)
{
    const bool norm = g.q_norm || g.k_norm;
    if constexpr (sizeof(E) == 2) {
        // Past the caches where the data does not fit them (us, through -> past them: 269 MB 53.8 -> 48.4, 287 MB 59.9 -> 55.5, 403 MB 79.2 -> 75.6; up to 100
        // MB no difference, and the attention that follows finds the data there)
        if (T * g.rows * g.D * 4 > kCacheBytes / 2) return norm ? launch_head<E, DEST, true, true>(g, T, st) : launch_head<E, DEST, false, true>(g, T, st);
    }
    return norm ? launch_head<E, DEST, true, false>(g, T, st) : launch_head<E, DEST, false, false>(g, T, st);
}

// what the two entry points check alike
static int check(const void* q, const void* k, aweq_dtype dt, bool f32, int64_t T, int64_t Hq, int64_t Hk, int64_t D, int64_t ldq, int64_t ldk,
                 const int32_t* pos, const double* freq, int64_t rot, int interleaved, const float* q_norm, const float* k_norm,
                 const void* q_out, int64_t ldqo)
{
    if (dt != AWEQ_F16 && dt != AWEQ_BF16 && !(f32 && dt == AWEQ_F32)) return AWEQ_ERR_DTYPE;
    if ((q != nullptr) != (q_out != nullptr) || (rot != 0 && (!pos || !freq))) return AWEQ_ERR_NULL;
    if (T <= 0 || D <= 0 || D > kMaxHead || (D % 8) != 0 || (q && Hq <= 0) || (k && Hk <= 0)) return AWEQ_ERR_SHAPE;
    if (Hq > (1 << 20) || Hk > (1 << 20)) return AWEQ_ERR_SHAPE;
    if (rot < 0 || rot > D || (rot % (interleaved ? 8 : 16)) != 0) return AWEQ_ERR_SHAPE;
    if ((q && (ldq < Hq * D || ldqo < Hq * D)) || (k && ldk < Hk * D)) return AWEQ_ERR_SHAPE;
    const int64_t unit = 16 / (int64_t)dtype_size(dt);
    if ((q && (!aligned16(q) || !aligned16(q_out) || (ldq % unit) != 0 || (ldqo % unit) != 0)) || (k && (!aligned16(k) || (ldk % unit) != 0)) ||
        (q_norm && !aligned16(q_norm)) || (k_norm && !aligned16(k_norm)) || (reinterpret_cast<uintptr_t>(pos) & 3u) ||
        (reinterpret_cast<uintptr_t>(freq) & 7u))
        return AWEQ_ERR_ALIGN;
    return AWEQ_OK;
}

}  // namespace rope
}  // namespace aweq

using namespace aweq;

extern "C" int aweq_rope_frequencies(int64_t rot, double base, int kind, double factor, double trained, double low, double high, double* freq)
{
    if (!freq) return AWEQ_ERR_NULL;
    if (rot <= 0 || (rot % 2) != 0 || !(base > 0.0) || std::isinf(base) || !(factor > 0.0) || std::isinf(factor)) return AWEQ_ERR_SHAPE;
    if (kind < AWEQ_ROPE_PLAIN || kind > AWEQ_ROPE_PARTS) return AWEQ_ERR_SHAPE;
    if (kind == AWEQ_ROPE_BASE && rot <= 2) return AWEQ_ERR_SHAPE;
    if (kind == AWEQ_ROPE_PARTS && !(trained > 0.0 && high > low)) return AWEQ_ERR_SHAPE;
    if (kind == AWEQ_ROPE_BASE) base *= std::pow(factor, (double)rot / (double)(rot - 2));
    for (int64_t i = 0; i < rot / 2; ++i) {
        const double f = std::pow(base, -2.0 * (double)i / (double)rot);
        if (kind == AWEQ_ROPE_LINEAR) freq[i] = f / factor;
        else if (kind == AWEQ_ROPE_PARTS) {
            const double turns = trained * f / 6.283185307179586477;
            const double kept = turns >= high ? 1.0 : turns <= low ? 0.0 : (turns - low) / (high - low);
            freq[i] = kept * f + (1.0 - kept) * f / factor;
        } else freq[i] = f;
    }
    return AWEQ_OK;
}

extern "C" int aweq_qk_rope(const void* q, const void* k, aweq_dtype dt, int64_t T, int64_t Hq, int64_t Hk, int64_t D, int64_t ldq, int64_t ldk,
                            const int32_t* pos, const double* freq, int64_t rot, int interleaved, float gain,
                            const float* q_norm, const float* k_norm, float eps, void* q_out, int64_t ldqo, void* k_out, int64_t ldko, void* stream)
{
    if (!q && !k) return AWEQ_ERR_NULL;
    int rc = rope::check(q, k, dt, true, T, Hq, Hk, D, ldq, ldk, pos, freq, rot, interleaved, q_norm, k_norm, q_out, ldqo);
    if (rc != AWEQ_OK) return rc;
    if ((k != nullptr) != (k_out != nullptr)) return AWEQ_ERR_NULL;
    if (k && ldko < Hk * D) return AWEQ_ERR_SHAPE;
    if (k && (!aligned16(k_out) || (ldko % (16 / (int64_t)dtype_size(dt))) != 0)) return AWEQ_ERR_ALIGN;
    rope::Args g = {};
    g.q = q; g.k = k; g.q_out = q_out; g.k_out = k_out; g.ldq = ldq; g.ldk = ldk; g.ldqo = ldqo; g.ldko = ldko;
    g.pos = pos; g.freq = freq; g.q_norm = q_norm; g.k_norm = k_norm; g.eps = eps; g.gain = gain;
    g.Hq = q ? (int)Hq : 0; g.Hk = k ? (int)Hk : 0; g.D = (int)D; g.rot = (int)rot; g.interleaved = interleaved != 0;
    g.rows = g.Hq + g.Hk;
    hipStream_t st = as_stream(stream);
    if (dt == AWEQ_F16) return rope::launch<_Float16, rope::kRows>(g, T, st);
    if (dt == AWEQ_BF16) return rope::launch<__bf16, rope::kRows>(g, T, st);
    return rope::launch<float, rope::kRows>(g, T, st);
}

extern "C" int aweq_kv_append(const void* q, const void* k, const void* v, aweq_dtype dt, int64_t T, int64_t Hq, int64_t Hk, int64_t D,
                              int64_t ldq, int64_t ldk, int64_t ldv, const int32_t* pos, const double* freq, int64_t rot, int interleaved, float gain,
                              const float* q_norm, const float* k_norm, float eps, void* q_out, int64_t ldqo,
                              void* k_cache, void* v_cache, float* k_step, float* v_step, aweq_dtype cache_dt, int64_t pages, int64_t page_size,
                              const int64_t* slot, uint32_t* status, void* stream)
{
    if (!k || !v || !k_cache || !v_cache || !slot) return AWEQ_ERR_NULL;
    const int rc = rope::check(q, k, dt, false, T, Hq, Hk, D, ldq, ldk, pos, freq, rot, interleaved, q_norm, k_norm, q_out, ldqo);
    if (rc != AWEQ_OK) return rc;
    if (cache_dt != dt && cache_dt != AWEQ_I8) return AWEQ_ERR_DTYPE;
    if (cache_dt == AWEQ_I8 && (!k_step || !v_step)) return AWEQ_ERR_NULL;
    if (ldv < Hk * D || pages <= 0 || page_size < 16 || page_size > 256 || (page_size & (page_size - 1)) != 0) return AWEQ_ERR_SHAPE;
    if (!aligned16(v) || (ldv % 8) != 0 || !aligned16(k_cache) || !aligned16(v_cache) || (reinterpret_cast<uintptr_t>(slot) & 7u) ||
        (cache_dt == AWEQ_I8 && (!aligned16(k_step) || !aligned16(v_step))))
        return AWEQ_ERR_ALIGN;
    rope::Args g = {};
    g.q = q; g.k = k; g.v = v; g.q_out = q_out; g.ldq = ldq; g.ldk = ldk; g.ldv = ldv; g.ldqo = ldqo;
    g.pos = pos; g.freq = freq; g.q_norm = q_norm; g.k_norm = k_norm; g.eps = eps; g.gain = gain;
    g.Hq = q ? (int)Hq : 0; g.Hk = (int)Hk; g.D = (int)D; g.rot = (int)rot; g.interleaved = interleaved != 0;
    g.rows = g.Hq + 2 * g.Hk;
    g.k_cache = k_cache; g.v_cache = v_cache; g.k_step = k_step; g.v_step = v_step;
    g.pages = pages; g.page_size = page_size; g.slot = slot; g.status = status;
    hipStream_t st = as_stream(stream);
    if (cache_dt == AWEQ_I8) {
        if (dt == AWEQ_F16) return rope::launch<_Float16, rope::kCodes>(g, T, st);
        return rope::launch<__bf16, rope::kCodes>(g, T, st);
    }
    if (dt == AWEQ_F16) return rope::launch<_Float16, rope::kCache>(g, T, st);
    return rope::launch<__bf16, rope::kCache>(g, T, st);
}
