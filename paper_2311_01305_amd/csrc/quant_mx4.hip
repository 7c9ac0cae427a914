// Quantizer to microscaled 4-bit floating point, and the values that its codes stand for.
//
// HBM-bound: 2 bytes in and 17/32 out a value (16-bit types), and about five vector operations.  A block's 32 values are four lanes' units of eight; 16 lanes
// have a row's panel and a wavefront four rows of it, four panels one after the other, so that the four scales that a lane's block has in them are the four bytes
// which belong together, and the codes of four rows are 256 bytes in one piece.
// Measured, 16-bit types: 22016 x 8192 76 - 81 us (5.6 - 6 TB/s; a copy of 1 GiB reaches 5.1), the values back 70 (6.5); 777 x 11008 7.8 and 6.4, one round of
// workgroups of which the launch is 2.2.
#include "mx4.hpp"

namespace aweq {
namespace mx {

constexpr int kThreads = 256;
constexpr int kRows = 16;      // of a workgroup

struct QuantArgs {
    const void* X;
    int64_t rows, K, ldx;
    const float* factor;
    uint8_t *codes, *scales;
    uint32_t* status;
    int groups;
    int64_t first;     // row of the launch
};

template <class E, bool FACTOR, bool STREAM>
__global__ __launch_bounds__(kThreads) void quant_kernel(QuantArgs g)
{
    const int group = (int)(blockIdx.x % (unsigned)g.groups);
    const int64_t r = g.first + (int64_t)(blockIdx.x / (unsigned)g.groups) * kRows + threadIdx.x / 16;
    const int c = threadIdx.x & 15;
    const int64_t row = min(r, g.rows - 1);                                      // (rows past the last one: nothing is written)
    const int64_t k0 = (int64_t)group * (kMxPanel * kMxGroup) + c * 8;
    const E* const from = reinterpret_cast<const E*>(g.X) + row * g.ldx;
    Unit<E> raw[kMxGroup];
    float factor[kMxGroup][8];
#pragma unroll
    for (int p = 0; p < kMxGroup; ++p) {
        const int64_t k = k0 + p * kMxPanel;
#pragma unroll
        for (int e = 0; e < 8; ++e) { raw[p][e] = (E)0.0f; factor[p][e] = 1.0f; }
        if (k < g.K) {
            raw[p] = STREAM ? stream_unit(from + k) : load_unit(from + k);
            if constexpr (FACTOR) {
                const f32x8 f = load_unit(g.factor + k);
#pragma unroll
                for (int e = 0; e < 8; ++e) factor[p][e] = f[e];
            }
        }
    }
    uint32_t scales = 0, st = 0;
#pragma unroll
    for (int p = 0; p < kMxGroup; ++p) {
        const int64_t k = k0 + p * kMxPanel;
        uint32_t scale;
        const uint32_t w = mx_unit<FACTOR, E>(raw[p], factor[p], scale);
        if (scale == 255u) st = AWEQ_ST_NONFINITE;
        scales |= (k < g.K ? scale : 127u) << (8 * p);
        const int64_t panel = (int64_t)group * kMxGroup + p;
        if (r < g.rows && panel * kMxPanel < g.K) *reinterpret_cast<uint32_t*>(g.codes + (panel * g.rows + r) * 64 + c * 4) = w;
    }
    if (r < g.rows && (c & 3) == 0) *reinterpret_cast<uint32_t*>(g.scales + ((int64_t)group * g.rows + r) * 16 + mx_scale_place(c >> 2)) = scales;
    raise_status(g.status, st);
}

typedef float f32x2 __attribute__((ext_vector_type(2)));

struct ValueArgs {
    const uint8_t *codes, *scales;
    int64_t rows, K, ldo;
    void* out;
    int groups;
    int64_t first;     // row of the launch
};

// STREAM: what is written goes past the caches
template <class E, bool STREAM>
__global__ __launch_bounds__(kThreads) void value_kernel(ValueArgs g)
{
    const int group = (int)(blockIdx.x % (unsigned)g.groups);
    const int64_t r = g.first + (int64_t)(blockIdx.x / (unsigned)g.groups) * kRows + threadIdx.x / 16;
    const int c = threadIdx.x & 15;
    if (r >= g.rows) return;
    const uint32_t scales = *reinterpret_cast<const uint32_t*>(g.scales + ((int64_t)group * g.rows + r) * 16 + mx_scale_place(c >> 2));
    const int64_t first = (int64_t)group * kMxGroup, last = mx_panels(g.K) - 1;
    uint32_t codes[kMxGroup];       // (all ahead of the first store)
#pragma unroll
    for (int p = 0; p < kMxGroup; ++p) codes[p] = *reinterpret_cast<const uint32_t*>(g.codes + (min(first + p, last) * g.rows + r) * 64 + c * 4);
#pragma unroll
    for (int p = 0; p < kMxGroup; ++p) {
        const int64_t k = (first + p) * kMxPanel + c * 8;
        if (k >= g.K) continue;
        const uint32_t w = codes[p];
        const uint32_t s = scales >> (8 * p) & 255u;
        const float step = s == 255u ? NAN : s == 0u ? 0x1p-127f : __uint_as_float(s << 23);
        // v_cvt_scalef32_pk_f32_fp4: a byte's two values, exact; the step is a factor of its own, since it may be subnormal or NaN
        const f32x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1),
                            __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3)};
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = v[e / 2][e % 2] * step;
        if constexpr (STREAM) stream_unit(reinterpret_cast<E*>(g.out) + r * g.ldo + k, x);
        else store_unit(reinterpret_cast<E*>(g.out) + r * g.ldo + k, x);
    }
}

// blocks of 16 rows and 512 values; fewer than 2^32 threads to a launch
template <class A, class F>
static int launch_blocks(A g, F kernel, hipStream_t st)
{
    g.groups = (int)mx_groups(g.K);
    const int64_t most = ((1ll << 32) / kThreads - 1) / g.groups;     // blocks of rows of a launch
    for (int64_t b = 0; b < cdiv(g.rows, kRows); b += most) {
        g.first = b * kRows;
        const int64_t left = cdiv(g.rows, kRows) - b;
        kernel<<<(unsigned)((left < most ? left : most) * g.groups), kThreads, 0, st>>>(g);
    }
    return launch_status();
}

// past: what is read goes past the caches, where it does not fit them (us, bfloat16, through -> past them, the same tokens again / others: 16384 x 8192 60.8 -> 54.9 /
// 64.9 -> 57.5, but 8192 x 8192 27.2 -> 30.8 / 35.2 -> 31.3, 777 x 11008 5.8 -> 6.1 / 7.6 -> 6.9; binary32 gains nothing)
template <class E>
static int launch_type(const QuantArgs& g, bool past, hipStream_t st)
{
    if constexpr (sizeof(E) == 2)
        if (past) return g.factor ? launch_blocks(g, quant_kernel<E, true, true>, st) : launch_blocks(g, quant_kernel<E, false, true>, st);
    return g.factor ? launch_blocks(g, quant_kernel<E, true, false>, st) : launch_blocks(g, quant_kernel<E, false, false>, st);
}

// Past the caches what they would not hold until somebody reads it (us, through -> past them, by itself / with a kernel that reads it: 22016 x 8192 98 -> 71 / 210 ->
// 207, 8192 x 8192 40.5 -> 27.1 / 83.1 -> 82.8, but 777 x 11008 6.3 -> 5.1 / 12.9 -> 13.8)
template <class E>
static int launch_values(const ValueArgs& g, hipStream_t st)
{
    if constexpr (sizeof(E) == 2)
        if (g.rows * g.K * 2 >= kCacheBytes / 2) return launch_blocks(g, value_kernel<E, true>, st);
    return launch_blocks(g, value_kernel<E, false>, st);
}

}  // namespace mx

int check_quant_mx4(const void* X, aweq_dtype dt, int64_t rows, int64_t K, int64_t ldx, const float* factor, const uint8_t* codes, const uint8_t* scales)
{
    if (!X || !codes || !scales) return AWEQ_ERR_NULL;
    if (dt != AWEQ_F32 && dt != AWEQ_F16 && dt != AWEQ_BF16) return AWEQ_ERR_DTYPE;
    if (!mx_shape_ok(rows, K) || ldx < K) return AWEQ_ERR_SHAPE;
    if (!aligned16(X) || (ldx * (int64_t)dtype_size(dt)) % 16 != 0 || (factor && !aligned16(factor)) || !aligned16(codes) || !aligned16(scales)) return AWEQ_ERR_ALIGN;
    return AWEQ_OK;
}

int launch_quant_mx4(const void* X, aweq_dtype dt, int64_t rows, int64_t K, int64_t ldx, const float* factor, uint8_t* codes, uint8_t* scales,
                     uint32_t* status, hipStream_t st)
{
    const mx::QuantArgs g = {X, rows, K, ldx, factor, codes, scales, status, 0, 0};
    const bool past = rows * K * (int64_t)dtype_size(dt) > kCacheBytes / 4 * 3;
    if (dt == AWEQ_F16) return mx::launch_type<_Float16>(g, past, st);
    if (dt == AWEQ_BF16) return mx::launch_type<__bf16>(g, past, st);
    return mx::launch_type<float>(g, past, st);
}

}  // namespace aweq

using namespace aweq;

extern "C" size_t aweq_mx4_code_bytes(int64_t rows, int64_t K) { return mx_shape_ok(rows, K) ? (size_t)(mx_panels(K) * rows * 64) : 0; }

extern "C" size_t aweq_mx4_scale_bytes(int64_t rows, int64_t K) { return mx_shape_ok(rows, K) ? (size_t)(mx_groups(K) * rows * 16) : 0; }

extern "C" int aweq_quant_mx4(const void* X, aweq_dtype dt, int64_t rows, int64_t K, int64_t ldx, const float* factor, uint8_t* codes, uint8_t* scales,
                              uint32_t* status, void* stream)
{
    const int rc = check_quant_mx4(X, dt, rows, K, ldx, factor, codes, scales);
    return rc != AWEQ_OK ? rc : launch_quant_mx4(X, dt, rows, K, ldx, factor, codes, scales, status, as_stream(stream));
}

extern "C" int aweq_mx4_values(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t K, void* out, aweq_dtype out_dt, int64_t ldo, void* stream)
{
    if (!codes || !scales || !out) return AWEQ_ERR_NULL;
    if (out_dt != AWEQ_F32 && out_dt != AWEQ_F16 && out_dt != AWEQ_BF16) return AWEQ_ERR_DTYPE;
    if (!mx_shape_ok(rows, K) || ldo < K) return AWEQ_ERR_SHAPE;
    if (!aligned16(codes) || !aligned16(scales) || !aligned16(out) || (ldo * (int64_t)dtype_size(out_dt)) % 16 != 0) return AWEQ_ERR_ALIGN;
    const mx::ValueArgs g = {codes, scales, rows, K, ldo, out, 0, 0};
    if (out_dt == AWEQ_F16) return mx::launch_values<_Float16>(g, as_stream(stream));
    if (out_dt == AWEQ_BF16) return mx::launch_values<__bf16>(g, as_stream(stream));
    return mx::launch_values<float>(g, as_stream(stream));
}
