// Quantizer of Eq. 1-2 with b = 8 whose slice is a token: Step and Z from the token's own range, widened to contain 0.
//
// HBM-bound: 2 bytes in (binary16 / bfloat16), 1 byte out per value, and 7 vector operations a value beside that (11 with scales).  The range
// has to be known before the first code, so a workgroup keeps the values of its tokens in registers between the two: every value is read once.
// Measured: 8192 tokens of 22016 bfloat16 values 112 - 122 us, 4.4 - 4.8 TB/s of both; 1777 of 11008 binary16 values with scales 18.8, 3.1 (889 workgroups
// of two tokens each are one round, which loads, computes and stores at the same time everywhere); 29 of 8192 5, a launch and two exchanges.
#include "gemm_tokens.hpp"
#include "token_range.hpp"

namespace aweq {
namespace tok {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;

struct Args {
    const void* X;
    int64_t T, K, ldx;
    const float* inv_s;
    int8_t* xq;
    float* step;
    int32_t* zero;
    int32_t* rowsum;
    uint32_t* status;
    int64_t first;
};

// R tokens a workgroup, U units of 8 values of each a thread (unit threadIdx + 256 i)
template <class E, int U, int R, bool FOLD>
__global__ __launch_bounds__(kThreads) void quant_token_kernel(Args g)
{
    __shared__ float s_lo[kWaves][R], s_hi[kWaves][R];
    __shared__ int s_sum[kWaves][R];
    const int64_t t0 = g.first + (int64_t)blockIdx.x * R;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int units = (int)(g.K / 8), padded = (int)panel_count(g.K) * (kPanel / 8);
    const int tokens = (int)min((int64_t)R, g.T - t0);
    const E* const X = reinterpret_cast<const E*>(g.X) + t0 * g.ldx;

    Unit<E> raw[R][U];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int u = i * kThreads + (int)threadIdx.x;
            if (u < units && r < tokens) raw[r][i] = load_unit(X + r * g.ldx + u * 8);
        }
    float lo[R], hi[R];
#pragma unroll
    for (int r = 0; r < R; ++r) lo[r] = hi[r] = 0.0f;
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int u = i * kThreads + (int)threadIdx.x;
        if (u >= units) break;
        float is[8];
        load_scales<FOLD>(g.inv_s, u, is);
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (r < tokens) token_extremes<FOLD, E>(raw[r][i], is, lo[r], hi[r]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        lo[r] = wave_allreduce(lo[r], OpMinimum());
        hi[r] = wave_allreduce(hi[r], OpMaximum());
        if (lane == 0) { s_lo[wave][r] = lo[r]; s_hi[wave][r] = hi[r]; }
    }
    __syncthreads();
    ActParams p[R];
    uint32_t st = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int w = 0; w < kWaves; ++w) { lo[r] = OpMinimum()(lo[r], s_lo[w][r]); hi[r] = OpMaximum()(hi[r], s_hi[w][r]); }
        float step;
        int zero;
        token_params(lo[r], hi[r], step, zero, st);
        p[r] = quot_params(step, zero);
        if (threadIdx.x == 0 && r < tokens) { g.step[t0 + r] = step; g.zero[t0 + r] = zero; }
    }
    int sum[R];
#pragma unroll
    for (int r = 0; r < R; ++r) sum[r] = 0;
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int u = i * kThreads + (int)threadIdx.x;
        if (u >= padded) break;
        float is[8];
        load_scales<FOLD>(g.inv_s, u < units ? u : 0, is);
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (r < tokens) {
                uint2 c = make_uint2(0u, 0u);
                if (u < units) c = token_unit<FOLD, E>(raw[r][i], is, p[r], sum[r]);
                *reinterpret_cast<uint2*>(g.xq + ((int64_t)(u >> 3) * g.T + t0 + r) * kPanel + (u & 7) * 8) = c;
            }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        sum[r] = wave_allreduce(sum[r], OpAdd());
        if (lane == 0) s_sum[wave][r] = sum[r];
    }
    __syncthreads();
    if ((int)threadIdx.x < tokens) {
        int s = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) s += s_sum[w][threadIdx.x];
        g.rowsum[t0 + threadIdx.x] = s;
    }
    if (threadIdx.x == 0) raise_status(g.status, st);
}

template <class E, int U, int R, bool FOLD>
static int launch_rows(Args g, hipStream_t st)
{
    const int64_t blocks = cdiv(g.T, R), most = (1ll << 32) / kThreads - 1;   // fewer than 2^32 threads to a launch
    for (int64_t b = 0; b < blocks; b += most) {
        g.first = b * R;
        quant_token_kernel<E, U, R, FOLD><<<(unsigned)(blocks - b < most ? blocks - b : most), kThreads, 0, st>>>(g);
    }
    return launch_status();
}

template <class E, int U, int R>
static int launch_units(const Args& g, hipStream_t st)
{
    return g.inv_s ? launch_rows<E, U, R, true>(g, st) : launch_rows<E, U, R, false>(g, st);
}

// Two tokens a workgroup from 1024 on: a panel's rows of two tokens are a whole line, and the scales are read once for both (us, one token -> two, four:
// 1777 x 11008 with scales 23.4 -> 18.3, 20.2; 8192 x 4096 30.1 -> 21.7, 24.9; 8192 x 8192 55.7 -> 42.3 (4.8 TB/s), 43.3; 8192 x 22016 130 -> 122, 127; but
// 256 x 4096 4.1 -> 4.5, 29 x 8192 4.6 -> 5.6).  Values of binary32 take twice the registers: one token in the longest rows.
template <class E, int U>
static int launch_tokens(const Args& g, hipStream_t st)
{
    if constexpr (U * sizeof(E) <= 32) {
        if (g.T >= 1024) return launch_units<E, U, 2>(g, st);
    }
    return launch_units<E, U, 1>(g, st);
}

template <class E>
static int launch(const Args& g, hipStream_t st)
{
    const int64_t units = panel_count(g.K) * (kPanel / 8);
    if (units <= 2 * kThreads) return launch_tokens<E, 2>(g, st);
    if (units <= 4 * kThreads) return launch_tokens<E, 4>(g, st);
    if (units <= 6 * kThreads) return launch_tokens<E, 6>(g, st);
    if (units <= 8 * kThreads) return launch_tokens<E, 8>(g, st);
    if (units <= 11 * kThreads) return launch_tokens<E, 11>(g, st);
    return launch_tokens<E, 16>(g, st);
}

}  // namespace tok

int check_quant_tokens(const void* X, aweq_dtype dt, int64_t T, int64_t K, int64_t ldx, const float* inv_s, const int8_t* xq, const float* step,
                       const int32_t* zero, const int32_t* rowsum)
{
    if (!X || !xq || !step || !zero || !rowsum) return AWEQ_ERR_NULL;
    if (dt != AWEQ_F32 && dt != AWEQ_F16 && dt != AWEQ_BF16) return AWEQ_ERR_DTYPE;
    if (T <= 0 || K <= 0 || (K % 8) != 0 || K > 32768 || ldx < K) return AWEQ_ERR_SHAPE;
    if (!aligned16(X) || (ldx * (int64_t)dtype_size(dt)) % 16 != 0 || !aligned16(xq) || (inv_s && !aligned16(inv_s))) return AWEQ_ERR_ALIGN;
    return AWEQ_OK;
}

int launch_quant_tokens(const void* X, aweq_dtype dt, int64_t T, int64_t K, int64_t ldx, const float* inv_s, int8_t* xq, float* step, int32_t* zero,
                        int32_t* rowsum, uint32_t* status, hipStream_t st)
{
    const tok::Args g = {X, T, K, ldx, inv_s, xq, step, zero, rowsum, status, 0};
    if (dt == AWEQ_F16) return tok::launch<_Float16>(g, st);
    if (dt == AWEQ_BF16) return tok::launch<__bf16>(g, st);
    return tok::launch<float>(g, st);
}

}  // namespace aweq

using namespace aweq;

extern "C" int aweq_quant_tokens(const void* X, aweq_dtype dt, int64_t T, int64_t K, int64_t ldx, const float* inv_s,
                                 int8_t* xq, float* step_x, int32_t* zero_x, int32_t* rowsum_x, uint32_t* status, void* stream)
{
    const int rc = check_quant_tokens(X, dt, T, K, ldx, inv_s, xq, step_x, zero_x, rowsum_x);
    return rc != AWEQ_OK ? rc : launch_quant_tokens(X, dt, T, K, ldx, inv_s, xq, step_x, zero_x, rowsum_x, status, as_stream(stream));
}
