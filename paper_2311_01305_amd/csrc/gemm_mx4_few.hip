// Product in microscaled 4-bit floating point for few tokens, when one read of the weight's codes is nearly all there is to do.
//
// A workgroup of 8 wavefronts owns 16 NT output channels x 16 TT tokens and splits K between its wavefronts, whose fp32 sums meet in LDS in a fixed
// order.  Both operands come straight from their panels (16 rows of one are 1 KiB contiguous) in the operand order of v_mfma_scale_f32_16x16x128_f8f6f4: lane l
// holds row l % 16, the 32 values of block l / 16 of the panel.  The scales of that block in four panels are one register, of which each instruction names
// the byte; so a wavefront takes the panels in groups of four.
//
// Bound by the launch and a round trip or two for small weights, by HBM for large ones (us, weights that are in no cache, tokens quantised by the launch: one
// token 4096 x 4096 4.5, 11008 x 4096 7.4, 22016 x 8192 20.3; codes given 4.2, 6.9, 18.9: 96 MB at 5.1 TB/s).
#include "gemm_mx4.hpp"

#include <type_traits>

namespace aweq {
namespace mxfew {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / kWave;

template <int J>
__device__ __forceinline__ f32x4 mul(const v4i& w, const v4i& x, const f32x4& c, int w_scale, int x_scale)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx_operand(w), mx_operand(x), c, 4, 4, J, w_scale, J, x_scale);
}

// E: void: the tokens' codes are in memory.  Otherwise every workgroup quantises the few tokens, of that type, for itself while its first weights are on their way, the
// first one also for the caller; ROUNDS: units of eight values of a thread, at most.
// ONCE: the tokens are one tile, so that nobody else reads these weights: past the caches, which the other layers' weights have gone through since (us, through ->
// past them: one token 22016 x 8192 20.0 -> 18.9, 16 tokens 21.8 -> 19.6, 8192 x 8192 8.5 -> 8.1; of the caches, a layer again and again, 7.2 -> 7.8; but 200
// tokens 5120 x 1536, 13 tiles, 8.9 -> 9.5).
template <int TT, int NT, bool ONCE, class E, int ROUNDS>
__global__ __launch_bounds__(kThreads) void gemm_mx4_few(MxArgs g, MxIn in, int first_tile)
{
    constexpr bool QX = !std::is_same<E, void>::value;
    extern __shared__ __attribute__((aligned(16))) float red[];   // [wave][TT NT][lane][4], then (QX) the tokens' codes and their scales
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
    const int r = lane & 15, q = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * (16 * NT), t0 = (int64_t)(first_tile + (int)blockIdx.y) * (16 * TT);
    const int np = (int)mx_panels(g.K), ng = (int)mx_groups(g.K);
    const int rows_left = (int)min(g.N - n0, (int64_t)(16 * NT)) - 1, tokens_left = (int)min(g.T - t0, (int64_t)(16 * TT)) - 1;

    // rows past the edge re-read the last valid row; their results are never stored
    uint32_t wo[NT], xo[TT];
    const int place = mx_scale_place(q);
#pragma unroll
    for (int j = 0; j < NT; ++j) wo[j] = (uint32_t)min(16 * j + r, rows_left);
#pragma unroll
    for (int i = 0; i < TT; ++i) xo[i] = (uint32_t)min(16 * i + r, tokens_left);
    const uint8_t* const wbase = g.b + n0 * 64 + q * 16;
    const uint8_t* const xbase = g.a + t0 * 64 + q * 16;
    const uint8_t* const wsbase = g.b_scale + n0 * 16 + place;
    const uint8_t* const xsbase = g.a_scale + t0 * 16 + place;
    const int64_t wp = g.N * 64, xp = g.T * 64;

    f32x4 acc[TT][NT];
#pragma unroll
    for (int i = 0; i < TT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    // Groups wave, wave + 8, ...: each panel's registers are refilled with the next group's as soon as it has been multiplied
    v4i w[kMxGroup][NT], x[kMxGroup][TT];
    int ws[NT], xs[TT], ws_next[NT], xs_next[TT];
    auto load = [&](int j, int group) {
        const int64_t p = min(group * kMxGroup + j, np - 1);   // (panels past the last one re-read it: they are not multiplied)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const v4i* const at = reinterpret_cast<const v4i*>(wbase + p * wp + wo[n] * 64);
            w[j][n] = ONCE ? __builtin_nontemporal_load(at) : *at;
        }
        if constexpr (!QX) {
#pragma unroll
            for (int t = 0; t < TT; ++t) x[j][t] = *reinterpret_cast<const v4i*>(xbase + p * xp + xo[t] * 64);
        }
    };
    auto load_scales = [&](int group, int (&a)[NT], int (&b)[TT]) {
#pragma unroll
        for (int n = 0; n < NT; ++n) a[n] = *reinterpret_cast<const int*>(wsbase + (int64_t)group * g.N * 16 + wo[n] * 16);
        if constexpr (!QX) {
#pragma unroll
            for (int t = 0; t < TT; ++t) b[t] = *reinterpret_cast<const int*>(xsbase + (int64_t)group * g.T * 16 + xo[t] * 16);
        }
    };
    // (QX) the tokens ahead of the weights: loads return in order
    using U = typename std::conditional<QX, E, float>::type;
    Unit<U> raw[QX ? ROUNDS : 1];
    float factor[QX ? ROUNDS : 1][8];
    const int units = (int)(g.K / 8), padded = np * 16;                            // of a token
    if constexpr (QX) {
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i) {
            const int at = i * kThreads + (int)threadIdx.x;
            if (i * kThreads >= padded * (int)g.T) break;
            const int t = min(at / padded, (int)g.T - 1), u = min(at % padded, units - 1);   // (past the end: not kept)
            raw[i] = load_unit(reinterpret_cast<const U*>(in.X) + t * in.ldx + u * 8);
#pragma unroll
            for (int e = 0; e < 8; ++e) factor[i][e] = 1.0f;
            if (in.factor) {
                const f32x8 f = load_unit(in.factor + u * 8);
#pragma unroll
                for (int e = 0; e < 8; ++e) factor[i][e] = f[e];
            }
        }
    }
    // what the epilogue needs of a channel waits in LDS
    __shared__ float s_bias[16 * NT];
    float bias = 0.0f;
    if (g.bias && (int)threadIdx.x <= rows_left) bias = g.bias[n0 + threadIdx.x];
    if (wave < ng) {
#pragma unroll
        for (int j = 0; j < kMxGroup; ++j) load(j, wave);
        load_scales(wave, ws, xs);
    }
    uint8_t* const codes = reinterpret_cast<uint8_t*>(red + kWaves * TT * NT * kWave * 4);
    uint8_t* const scales = codes + (QX ? (int)g.T * np * 64 : 0);
    if constexpr (QX) {
        uint32_t st = 0;
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i) {
            const int at = i * kThreads + (int)threadIdx.x;
            if (i * kThreads >= padded * (int)g.T) break;
            const int t = at / padded, u = at % padded, p = u / 16, b = u / 4 % 4;
            uint32_t scale;
            uint32_t c = mx_unit<true, U>(raw[i], factor[i], scale);
            if (u >= units) { c = 0u; scale = 127u; }     // (the zero fill of the last panel)
            if (t >= (int)g.T) continue;
            if (scale == 255u) st = AWEQ_ST_NONFINITE;
            const int to = p / kMxGroup * 16 + mx_scale_place(b) + p % kMxGroup;
            *reinterpret_cast<uint32_t*>(codes + (t * padded + u) * 4) = c;
            if ((u & 3) == 0) scales[t * ng * 16 + to] = (uint8_t)scale;
            if (blockIdx.x == 0) {
                *reinterpret_cast<uint32_t*>(in.xq + ((int64_t)p * g.T + t) * 64 + u % 16 * 4) = c;
                if ((u & 3) == 0) in.x_scale[((int64_t)(p / kMxGroup) * g.T + t) * 16 + to % 16] = (uint8_t)scale;
            }
        }
        if (blockIdx.x == 0) raise_status(g.status, st);
        __syncthreads();
    }
    const int own = min(r, (int)g.T - 1);                   // (QX: one row of 16 tokens)
    auto token = [&](int j, int group) {
        if constexpr (QX) {
            x[j][0] = *reinterpret_cast<const v4i*>(codes + (own * np + min(group * kMxGroup + j, np - 1)) * 64 + q * 16);
            if (j == 0) xs[0] = *reinterpret_cast<const int*>(scales + (own * ng + group) * 16 + place);
        }
    };
    auto panel = [&](auto jc, int group) {
        constexpr int j = decltype(jc)::value;
        token(j, group);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int t = 0; t < TT; ++t) acc[t][n] = mul<j>(w[j][n], x[j][t], acc[t][n], ws[n], xs[t]);
    };
    using std::integral_constant;
    int group = wave;
    for (; group + kWaves < ng; group += kWaves) {
        const int next = group + kWaves;
        load_scales(next, ws_next, xs_next);
        panel(integral_constant<int, 0>{}, group); load(0, next);
        panel(integral_constant<int, 1>{}, group); load(1, next);
        panel(integral_constant<int, 2>{}, group); load(2, next);
        panel(integral_constant<int, 3>{}, group); load(3, next);
#pragma unroll
        for (int n = 0; n < NT; ++n) ws[n] = ws_next[n];
        if constexpr (!QX) {
#pragma unroll
            for (int t = 0; t < TT; ++t) xs[t] = xs_next[t];
        }
    }
    if (group < ng) {
        const int left = np - group * kMxGroup;
        panel(integral_constant<int, 0>{}, group);
        if (left > 1) panel(integral_constant<int, 1>{}, group);
        if (left > 2) panel(integral_constant<int, 2>{}, group);
        if (left > 3) panel(integral_constant<int, 3>{}, group);
    }

    // register v of lane l is output channel 4 (l / 16) + v of the 16, token l % 16
    constexpr int kTiles = TT * NT;
#pragma unroll
    for (int i = 0; i < TT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) *reinterpret_cast<f32x4*>(red + ((wave * kTiles + i * NT + j) * kWave + lane) * 4) = acc[i][j];
    if ((int)threadIdx.x < 16 * NT) s_bias[threadIdx.x] = bias;
    __syncthreads();
    for (int e = threadIdx.x; e < kTiles * kWave; e += kThreads) {
        const int tile = e / kWave, l = e & (kWave - 1);
        const int nl = 16 * (tile % NT) + 4 * (l >> 4);
        const int64_t t = t0 + 16 * (tile / NT) + (l & 15), n = n0 + nl;
        if (t >= g.T || n >= g.N) continue;     // N % 4 == 0: all four channels or none
        f32x4 o = *reinterpret_cast<const f32x4*>(red + (tile * kWave + l) * 4);
#pragma unroll
        for (int wv = 1; wv < kWaves; ++wv) o += *reinterpret_cast<const f32x4*>(red + ((wv * kTiles + tile) * kWave + l) * 4);
        const float y[4] = {o[0] + s_bias[nl], o[1] + s_bias[nl + 1], o[2] + s_bias[nl + 2], o[3] + s_bias[nl + 3]};
        mx_store(g, t, n, y);
    }
}

// Token tiles ride on the grid's y dimension: at most 65535 of them to a launch, and fewer than 2^32 threads
template <int TT, int NT, bool ONCE, class E = void, int ROUNDS = 0>
static int launch_tile(MxArgs g, hipStream_t st, MxIn in = {})
{
    constexpr bool QX = !std::is_same<E, void>::value;
    constexpr int kSums = kWaves * TT * NT * kWave * 16;
    static_assert(!QX || TT == 1, "one row of tokens");
    const int lds = kSums + (QX ? (int)(g.T * (mx_panels(g.K) * 64 + mx_groups(g.K) * 16)) : 0);
    const void* fn = reinterpret_cast<const void*>(gemm_mx4_few<TT, NT, ONCE, E, ROUNDS>);
    int dev = 0, cus = 0;
    if (lds > 32768 && (device_cus(dev, cus) != AWEQ_OK || raise_lds_limit(fn, dev, lds > 65536 ? 131072 : 65536) != AWEQ_OK)) return AWEQ_ERR_LAUNCH;
    const int64_t tiles = cdiv(g.T, 16 * TT), blocks = cdiv(g.N, 16 * NT), by_threads = ((1ll << 32) - 1) / (blocks * kThreads);
    const int64_t most = by_threads < 65535 ? by_threads : 65535;
    if (most < 1) return AWEQ_ERR_SHAPE;
    for (int64_t t = 0; t < tiles; t += most) {
        int first = (int)t;
        void* args[] = {&g, &in, &first};
        if (hipLaunchKernel(fn, dim3((unsigned)blocks, (unsigned)(tiles - t < most ? tiles - t : most)), dim3(kThreads), args, lds, st) != hipSuccess)
            return AWEQ_ERR_LAUNCH;
    }
    return launch_status();
}

template <int TT, int NT>
static int launch_given(const MxArgs& g, hipStream_t st)
{
    return g.T <= 16 * TT ? launch_tile<TT, NT, true>(g, st) : launch_tile<TT, NT, false>(g, st);
}

// Units of eight values that a workgroup quantises, and how many of them a thread has at most: all are asked for ahead of the first weights, so that a thread keeps
// them in registers (us, 8 of them for every call -> as many as there are: one token 11008 x 4096 10.9 -> 7.8, 22016 x 8192 24.6 -> 21.5)
static int64_t units_of(int64_t T, int64_t K) { return T * mx_panels(K) * 16; }
constexpr int kMostRounds = 4;

template <int NT, class E>
static int launch_rounds(const MxArgs& g, const MxIn& in, hipStream_t st)
{
    const int64_t units = units_of(g.T, g.K);
    if (units <= kThreads) return launch_tile<1, NT, true, E, 1>(g, st, in);
    if (units <= 2 * kThreads) return launch_tile<1, NT, true, E, 2>(g, st, in);
    return launch_tile<1, NT, true, E, kMostRounds>(g, st, in);
}

template <class E>
static int launch_quant(const MxArgs& g, const MxIn& in, int nt, hipStream_t st)
{
    return nt == 2 ? launch_rounds<2, E>(g, in, st) : launch_rounds<1, E>(g, in, st);
}

}  // namespace mxfew

int launch_mx4_few(const MxArgs& g, int tt, int nt, hipStream_t st)
{
    if (tt == 1) return nt == 1 ? mxfew::launch_given<1, 1>(g, st) : mxfew::launch_given<1, 2>(g, st);
    if (tt == 2) return nt == 1 ? mxfew::launch_given<2, 1>(g, st) : mxfew::launch_given<2, 2>(g, st);
    return nt == 2 ? mxfew::launch_given<4, 2>(g, st) : mxfew::launch_given<4, 4>(g, st);
}

// Every workgroup repeats the work.  That is less than a launch of the quantizer's own (2.7 us) up to two units a thread, or up to four where each compute unit has a
// workgroup (us, in the launch / before it: 4096 x 4096 one token 4.5 / 7.0, four tokens 6.3 / 7.0; 11008 x 4096 two 8.6 / 9.9, four 11.8 / 10.6;
// 8192 x 8192 two 10.4 / 11.0)
bool mx4_few_quantises(int64_t T, int64_t N, int64_t K, int nt)
{
    const int64_t units = mxfew::units_of(T, K);
    return T <= 16 && (units <= 2 * mxfew::kThreads || (units <= mxfew::kMostRounds * mxfew::kThreads && cdiv(N, 16 * nt) <= 256));
}

int launch_mx4_few_quant(const MxArgs& g, const MxIn& in, aweq_dtype dt, int nt, hipStream_t st)
{
    if (dt == AWEQ_F16) return mxfew::launch_quant<_Float16>(g, in, nt, st);
    if (dt == AWEQ_BF16) return mxfew::launch_quant<__bf16>(g, in, nt, st);
    return mxfew::launch_quant<float>(g, in, nt, st);
}

}  // namespace aweq
