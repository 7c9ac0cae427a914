// Norm of every head of queries and keys, rotation by the token's position, and the way of keys and values into a paged cache, in one pass
// over a token's heads.
//
//   y = x w / sqrt(mean x^2 + eps);   the pair (a, b) of a head turns into (a cos - b sin, b cos + a sin), angle = pos freq[i]
//
// A lane holds two units of 8 values, chosen so that both values of its pairs are its own: units u and u + rot / 16 of the half layout,
// 2 u and 2 u + 1 of the interleaved one, and nothing crosses lanes but the norm's sum.  2^G lanes have a head, a wavefront 2^(6 - G) heads of one
// token at a time.  A workgroup's token has rot / 2 angles, which some of its threads form once, while the first values are on their way: the
// product pos freq in binary64, reduced to a part of a turn there (in binary32 a position of 100000 has lost the angle's last three digits), then
// sine and cosine of that in binary32.
#include "wide_unit.hpp"

#include <cmath>

namespace aweq {
namespace rope {

constexpr int kThreads = 256;
constexpr int kMaxHead = 256;

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
    int per_block, blocks;      // rounds of a workgroup, workgroups to a token
    int64_t first;              // the launch's first token
    void *k_cache, *v_cache;
    float *k_step, *v_step;
    int64_t pages, page_size;
    const int64_t* slot;
    uint32_t* status;
};

enum { kRows, kCache, kCodes };   // where keys go: rows as queries do, a cache of the same type, a cache of 8-bit codes

// largest |x| of a head's values to a step, its codes and the step itself to the cache
template <int G>
__device__ __forceinline__ void store_codes(int8_t* dst, float* step_at, const float a[8], const float b[8], int ua, int ub, int units, bool writes_step)
{
    float big = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) big = fmaxf(big, fmaxf(fabsf(a[i]), fabsf(b[i])));
    big = group_allreduce<G>(big, OpMax());
    float step = big / 127.0f;
    if (!(step > 0.0f) || isinf(step)) step = 1.0f;
    if (writes_step) *step_at = step;
    auto pack = [&](const float x[8]) {
        uint32_t w[2] = {0u, 0u};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = (int)rintf(__builtin_amdgcn_fmed3f(x[i] / step, -127.0f, 127.0f));   // (a subnormal step can be off by half)
            w[i >> 2] |= (uint32_t)(c & 0xff) << (8 * (i & 3));
        }
        return make_uint2(w[0], w[1]);
    };
    if (ua < units) *reinterpret_cast<uint2*>(dst + ua * 8) = pack(a);
    if (ub < units) *reinterpret_cast<uint2*>(dst + ub * 8) = pack(b);
}

template <class E, int G, int DEST>
__global__ __launch_bounds__(kThreads) void rope_kernel(Args g)
{
    __shared__ float s_cos[kMaxHead / 2], s_sin[kMaxHead / 2];
    constexpr int kLanes = 1 << G, kHeads = kThreads / kLanes;   // lanes of a head, heads of a round
    const int64_t t = g.first + blockIdx.x / (unsigned)g.blocks;
    const int round0 = (int)(blockIdx.x % (unsigned)g.blocks) * g.per_block;
    const int lane = threadIdx.x & (kLanes - 1), sub = threadIdx.x >> G;
    const int units = g.D / 8;

    // this lane's two units, whether they are rotated, and the angles of their pairs (half: pair j has angle `first` + j; interleaved:
    // the four pairs of either unit)
    int ua, ub;
    if (g.interleaved) {
        ua = 2 * lane;
        ub = ua + 1;
    } else {
        const int h = g.rot / 16;
        ua = lane < h ? lane : 2 * h + 2 * (lane - h);
        ub = lane < h ? lane + h : ua + 1;
    }
    const bool ra = ua * 8 < g.rot, rb = ub * 8 < g.rot;

    // angles, one thread each
    const int pairs = g.rot / 2;
    const int32_t pos = pairs ? g.pos[t] : 0;
    const int64_t slot = DEST != kRows ? g.slot[t] : 0;
    for (int i = threadIdx.x; i < pairs; i += kThreads) {
        double turns = (double)pos * g.freq[i] * 0.15915494309189533577;
        turns -= rint(turns);
        float s, c;
        sincospif(2.0f * (float)turns, &s, &c);
        s_cos[i] = g.gain * c;
        s_sin[i] = g.gain * s;
    }
    bool keep = true;
    int64_t page = 0, row = 0;
    if constexpr (DEST != kRows) {
        const int64_t p = slot / g.page_size;
        keep = slot >= 0 && p < g.pages;
        if (slot >= 0 && !keep && threadIdx.x == 0 && round0 == 0) raise_status(g.status, AWEQ_ST_INDEX);
        page = keep ? p : 0;
        row = keep ? slot - p * g.page_size : 0;
    }
    __syncthreads();
    float ca[4], sa[4], cb[4], sb[4];   // interleaved: of the first and the second unit; half: pairs 0 - 3 and 4 - 7
    {
        const int fa = g.interleaved ? ua * 4 : ua * 8, fb = g.interleaved ? ub * 4 : ua * 8 + 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            ca[j] = ra ? s_cos[fa + j] : 1.0f;
            sa[j] = ra ? s_sin[fa + j] : 0.0f;
            const bool r = g.interleaved ? rb : ra;
            cb[j] = r ? s_cos[fb + j] : 1.0f;
            sb[j] = r ? s_sin[fb + j] : 0.0f;
        }
    }

    for (int round = round0; round < round0 + g.per_block; ++round) {
        const int head = round * kHeads + sub;
        if (head - sub >= g.rows) break;
        const bool in = head < g.rows;
        const bool is_q = head < g.Hq, is_v = head >= g.Hq + g.Hk;
        const int h = is_q ? head : is_v ? head - g.Hq - g.Hk : head - g.Hq;
        const E* src = is_q ? reinterpret_cast<const E*>(g.q) + t * g.ldq : is_v ? reinterpret_cast<const E*>(g.v) + t * g.ldv : reinterpret_cast<const E*>(g.k) + t * g.ldk;
        src += (int64_t)h * g.D;
        const bool has_a = in && ua < units, has_b = in && ub < units;
        float a[8] = {}, b[8] = {};
        if (has_a) widen<E>(load_unit(src + ua * 8), a);
        if (has_b) widen<E>(load_unit(src + ub * 8), b);
        const float* w = is_q ? g.q_norm : is_v ? nullptr : g.k_norm;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += a[i] * a[i] + b[i] * b[i];
        sum = group_allreduce<G>(sum, OpAdd());
        if (w) {
            const float r = 1.0f / sqrtf(sum / (float)g.D + g.eps);
            if (has_a) {
                const f32x8 u = load_unit(w + ua * 8);
#pragma unroll
                for (int i = 0; i < 8; ++i) a[i] = a[i] * r * u[i];
            }
            if (has_b) {
                const f32x8 u = load_unit(w + ub * 8);
#pragma unroll
                for (int i = 0; i < 8; ++i) b[i] = b[i] * r * u[i];
            }
        }
        if (!is_v) {
            if (g.interleaved) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float x = a[2 * j], y = a[2 * j + 1], z = b[2 * j], u = b[2 * j + 1];
                    if (ra) { a[2 * j] = x * ca[j] - y * sa[j]; a[2 * j + 1] = y * ca[j] + x * sa[j]; }
                    if (rb) { b[2 * j] = z * cb[j] - u * sb[j]; b[2 * j + 1] = u * cb[j] + z * sb[j]; }
                }
            } else if (ra) {   // (both units or neither)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float c = j < 4 ? ca[j & 3] : cb[j & 3], s = j < 4 ? sa[j & 3] : sb[j & 3];
                    const float x = a[j], y = b[j];
                    a[j] = x * c - y * s;
                    b[j] = y * c + x * s;
                }
            }
        }
        if (DEST == kRows || is_q) {
            E* dst = (is_q ? reinterpret_cast<E*>(g.q_out) + t * g.ldqo : reinterpret_cast<E*>(g.k_out) + t * g.ldko) + (int64_t)h * g.D;
            if (has_a) store_unit(dst + ua * 8, a);
            if (has_b) store_unit(dst + ub * 8, b);
        } else {
            const int64_t at = (page * g.Hk + h) * g.page_size + row;
            if constexpr (DEST == kCache) {
                E* dst = reinterpret_cast<E*>(is_v ? g.v_cache : g.k_cache) + at * g.D;
                if (has_a && keep) store_unit(dst + ua * 8, a);
                if (has_b && keep) store_unit(dst + ub * 8, b);
            } else {
                const bool put = in && keep;
                store_codes<G>(reinterpret_cast<int8_t*>(is_v ? g.v_cache : g.k_cache) + at * g.D, (is_v ? g.v_step : g.k_step) + at, a, b,
                               put ? ua : units, put ? ub : units, units, put && lane == 0);
            }
        }
    }
}

template <class E, int DEST>
static int launch_head(Args g, int64_t T, hipStream_t st)
{
    // 16 values a lane, lanes of a head a power of two
    int G = 0;
    while ((16 << G) < g.D) ++G;
    const int heads = kThreads >> G, rounds = (g.rows + heads - 1) / heads;
    g.per_block = T * rounds > 8192 ? rounds : 1;
    g.blocks = (rounds + g.per_block - 1) / g.per_block;
    const int64_t most = ((1ll << 32) / kThreads - 1) / g.blocks;   // tokens to a launch: fewer than 2^32 threads
    for (int64_t first = 0; first < T; first += most) {
        g.first = first;
        const unsigned grid = (unsigned)((T - first < most ? T - first : most) * g.blocks);
        switch (G) {
        case 0: rope_kernel<E, 0, DEST><<<grid, kThreads, 0, st>>>(g); break;
        case 1: rope_kernel<E, 1, DEST><<<grid, kThreads, 0, st>>>(g); break;
        case 2: rope_kernel<E, 2, DEST><<<grid, kThreads, 0, st>>>(g); break;
        case 3: rope_kernel<E, 3, DEST><<<grid, kThreads, 0, st>>>(g); break;
        default: rope_kernel<E, 4, DEST><<<grid, kThreads, 0, st>>>(g); break;
        }
        const int rc = launch_status();
        if (rc != AWEQ_OK) return rc;
    }
    return AWEQ_OK;
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
    if (dt == AWEQ_F16) return rope::launch_head<_Float16, rope::kRows>(g, T, st);
    if (dt == AWEQ_BF16) return rope::launch_head<__bf16, rope::kRows>(g, T, st);
    return rope::launch_head<float, rope::kRows>(g, T, st);
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
        if (dt == AWEQ_F16) return rope::launch_head<_Float16, rope::kCodes>(g, T, st);
        return rope::launch_head<__bf16, rope::kCodes>(g, T, st);
    }
    if (dt == AWEQ_F16) return rope::launch_head<_Float16, rope::kCache>(g, T, st);
    return rope::launch_head<__bf16, rope::kCache>(g, T, st);
}
