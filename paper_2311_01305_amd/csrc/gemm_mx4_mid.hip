// Product in microscaled 4-bit floating point for some hundred tokens, when the tiles of the kernel for many leave most compute units without one.
//
// A workgroup of 8 wavefronts owns 64 WM tokens x 64 WN channels.  A stage is WK panels of K (64 bytes a row each): wavefront (k, m, n) multiplies panel k of it
// for its 64 x 64 corner as 2 x 2 v_mfma_scale_f32_32x32x64_f8f6f4 tiles, and the WK partial sums meet in LDS at the end, in a fixed order.  Stages go through a
// ring of LDS slots filled by LDS-DMA loads, one barrier a stage; a stage brings the scales of its group of four panels along, and a wavefront shifts its panel's
// to the lowest byte.
//
// Bound by the loads of the one workgroup that a compute unit has room for, 40 - 60 GB/s with a barrier a stage: 64 tokens 22016 x 8192 23.5 us (4.1 TB/s of
// weights), 512 tokens 4096 x 4096 12.6 (1.4 PFLOP/s), 8192 x 8192 27.4 (2.5).
#include "gemm_mx4.hpp"

namespace aweq {
namespace mxmid {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef int v2i __attribute__((ext_vector_type(2)));

constexpr int kThreads = 512;

struct Args : MxArgs {
    int tiles_m, tiles_n, run;
};

template <int WM, int WN, int WK>
struct Tile {
    static_assert(WM * WN * WK == 8 && (WK == 2 || WK == 4), "eight wavefronts, stages that do not cross a group of panels");
    static constexpr int kM = 64 * WM, kN = 64 * WN;
    static constexpr int kPanelBytes = (kM + kN) * 64;                  // one panel: the token rows, then the weight rows
    static constexpr int kScales = WK * kPanelBytes;                    // then the scales of both, 16 bytes a row
    static constexpr int kSlot = kScales + (kM + kN) * 16;
    static constexpr int kSlots = 160 * 1024 / kSlot >= 4 ? 4 : 160 * 1024 / kSlot;
    static constexpr int kUnits = WK * kPanelBytes / 1024 / 8;          // load instructions per wavefront and stage, and one of scales
    static constexpr int kLoads = kUnits + 1;
    static constexpr int kSums = 128 * 1024;                            // partial sums: 16 KiB per wavefront
    static constexpr int kLds = kSlots * kSlot > kSums ? kSlots * kSlot : kSums;
    static_assert((kM + kN) / 64 <= 8, "a load of scales each is enough");
};

__device__ __forceinline__ int f4(int r) { return (r >> 2) & 3; }

__device__ __forceinline__ void dma16(const uint8_t* sbase, uint32_t voff, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds_addr), "v"(voff), "s"(sbase) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_vm()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

template <int WM, int WN, int WK>
__global__ __launch_bounds__(kThreads) void gemm_mx4_mid(Args g)
{
    using TL = Tile<WM, WN, WK>;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int wk = wave / (WM * WN), wm = wave / WN % WM, wn = wave % WN;

    // ids are dealt round-robin to the XCDs: each XCD takes an equal run of the tiles, token tiles fastest, so that a weight
    // row is read by one or two XCDs only
    const int l = (int)(blockIdx.x % kXcdCount) * g.run + (int)(blockIdx.x / kXcdCount);
    if (l >= g.tiles_m * g.tiles_n) return;
    const int64_t m0 = (int64_t)(l % g.tiles_m) * TL::kM, n0 = (int64_t)(l / g.tiles_m) * TL::kN;

    const int np = (int)mx_panels(g.K), ns = (np + WK - 1) / WK;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;

    // this thread's share of the epilogue: four channels, every kRowStep-th token
    constexpr int kRowThreads = TL::kN / 4, kRowStep = kThreads / kRowThreads, kRows = TL::kM / kRowStep;
    const int ec = tid % kRowThreads, er = tid / kRowThreads;
    const int64_t n = n0 + ec * 4;
    const bool n_ok = n < g.N;     // N % 4 == 0: all four channels or none
    Float4 bias = {{0.0f, 0.0f, 0.0f, 0.0f}};
    if (g.bias && n_ok) bias = *reinterpret_cast<const Float4*>(g.bias + n);
#pragma unroll
    for (int c = 0; c < 4; ++c) asm volatile("" : "+v"(bias.f[c]));   // (waited for here, ahead of the loads that the compiler does not see)

    // load q of this wavefront brings 16 rows of one panel of the stage: unit wave kUnits + q of (panel, 16-row group)
    constexpr int kGroups = 4 * (WM + WN);
    uint32_t voff[TL::kUnits];
    const int last_m = (int)min((int64_t)TL::kM, g.T - m0) - 1, last_n = (int)min((int64_t)TL::kN, g.N - n0) - 1;
#pragma unroll
    for (int q = 0; q < TL::kUnits; ++q) {
        const int grp = (wave * TL::kUnits + q) % kGroups, sub = lane >> 2;
        // rows past the edge re-read the last valid row; their results are never stored
        const int row = grp < 4 * WM ? min(grp * 16 + sub, last_m) : min((grp - 4 * WM) * 16 + sub, last_n);
        voff[q] = (uint32_t)(row * 64 + ((lane & 3) ^ f4(sub)) * 16);
    }
    const uint8_t* const baseA = g.a + m0 * 64;
    const uint8_t* const baseB = g.b + n0 * 64;
    // scales: 64 rows a wavefront, some of them twice
    const int srow = wave % (WM + WN);
    const bool sb_ = srow >= WM;
    const uint32_t soff = (uint32_t)((sb_ ? min((srow - WM) * 64 + lane, last_n) : min(srow * 64 + lane, last_m)) * 16);
    const uint8_t* const baseS = sb_ ? g.b_scale + n0 * 16 : g.a_scale + m0 * 16;
    const int64_t stepS = (sb_ ? g.N : g.T) * 16;
    auto issue = [&](int s) {
        const uint32_t slot = lds0 + (uint32_t)(s % TL::kSlots) * TL::kSlot;
        dma16(baseS + (s * WK / kMxGroup) * stepS, soff, slot + TL::kScales + (uint32_t)srow * 1024);
#pragma unroll
        for (int q = 0; q < TL::kUnits; ++q) {
            const int unit = wave * TL::kUnits + q;
            const int64_t p = min(s * WK + unit / kGroups, np - 1);   // (panels past the last one re-read it: they are not multiplied)
            const bool a = unit % kGroups < 4 * WM;
            dma16((a ? baseA : baseB) + p * ((a ? g.T : g.N) * 64), voff[q], slot + (uint32_t)unit * 1024);
        }
    };

    const int fr_row = lane & 31, fr_half = lane >> 5;
    int offA[2], offB[2];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
        const int chunk = ((ks * 2 + fr_half) ^ f4(fr_row)) * 16;
        offA[ks] = wk * TL::kPanelBytes + (wm * 64 + fr_row) * 64 + chunk;
        offB[ks] = wk * TL::kPanelBytes + (TL::kM + wn * 64 + fr_row) * 64 + chunk;
    }
    const int offSA = TL::kScales + (wm * 64 + fr_row) * 16 + fr_half * 8, offSB = TL::kScales + (TL::kM + wn * 64 + fr_row) * 16 + fr_half * 8;

    v16f acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;

    for (int s = 0; s < TL::kSlots - 1 && s < ns; ++s) issue(s);
    for (int s = 0; s < ns; ++s) {
        // stage s has landed for this wavefront (stages after it may be out), its reads of stage s - 1 are done; after the
        // barrier that holds for every wavefront, and stage s + kSlots - 1 can take the slot of stage s - 1
        const int newer = min(TL::kSlots - 2, ns - 1 - s);
        if (newer == 0) wait_vm<0>();
        else if (newer == 1) wait_vm<TL::kLoads>();
        else wait_vm<2 * TL::kLoads>();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        if (s + TL::kSlots - 1 < ns) issue(s + TL::kSlots - 1);
        const int p = s * WK + wk;
        if (p < np) {
            const char* const st = lds + (s % TL::kSlots) * TL::kSlot;
            const int by = (p & 3) * 8;
            v4i a[2][2], b[2][2];
            v2i sa[2], sb[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                sa[i] = *reinterpret_cast<const v2i*>(st + offSA + i * 32 * 16);
                sb[i] = *reinterpret_cast<const v2i*>(st + offSB + i * 32 * 16);
            }
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    a[ks][i] = *reinterpret_cast<const v4i*>(st + offA[ks] + i * 32 * 64);
                    b[ks][i] = *reinterpret_cast<const v4i*>(st + offB[ks] + i * 32 * 64);
                }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) {
                    sa[i][ks] = (int)((uint32_t)sa[i][ks] >> by);
                    sb[i][ks] = (int)((uint32_t)sb[i][ks] >> by);
                }
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx_operand(b[ks][j]), mx_operand(a[ks][i]), acc[i][j], 4, 4, 0, sb[j][ks], 0, sa[i][ks]);
        }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();   // every wavefront is done with the ring

    // register v of lane l in sub-tile (i, j) is token 32 i + l % 32 and channel 32 j + 8 (v / 4) + 4 (l / 32) + v % 4 of the
    // wavefront's corner: rows of 256 bytes, 16-byte chunks XOR swizzled
    {
        char* const mine = lds + wave * 16384;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int t = 32 * i + fr_row;
                    *reinterpret_cast<f32x4*>(mine + t * 256 + (((8 * j + 2 * q + fr_half) ^ (t & 15)) * 16)) =
                        f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const int r = er + i * kRowStep;
        const int64_t t = m0 + r;
        if (t >= g.T || !n_ok) continue;
        f32x4 o = {bias.f[0], bias.f[1], bias.f[2], bias.f[3]};
#pragma unroll
        for (int k = 0; k < WK; ++k) {
            const char* const part = lds + ((k * WM + r / 64) * WN + ec / 16) * 16384;
            o += *reinterpret_cast<const f32x4*>(part + (r & 63) * 256 + (((ec & 15) ^ (r & 15)) * 16));
        }
        const float y[4] = {o[0], o[1], o[2], o[3]};
        mx_store(g, t, n, y);
    }
}

template <int WM, int WN, int WK>
static int launch_tile(const MxArgs& m, hipStream_t st)
{
    using TL = Tile<WM, WN, WK>;
    Args g = {};
    static_cast<MxArgs&>(g) = m;
    const int64_t tiles_m = cdiv(g.T, TL::kM), tiles_n = cdiv(g.N, TL::kN);
    if (tiles_m * tiles_n > (1 << 22)) return AWEQ_ERR_SHAPE;
    g.tiles_m = (int)tiles_m;
    g.tiles_n = (int)tiles_n;
    g.run = (int)cdiv(tiles_m * tiles_n, kXcdCount);
    const void* fn = reinterpret_cast<const void*>(gemm_mx4_mid<WM, WN, WK>);
    int dev = 0, cus = 0;
    if (device_cus(dev, cus) != AWEQ_OK || raise_lds_limit(fn, dev, TL::kLds) != AWEQ_OK) return AWEQ_ERR_LAUNCH;
    void* args[] = {&g};
    if (hipLaunchKernel(fn, dim3((unsigned)(g.run * kXcdCount)), dim3(kThreads), args, TL::kLds, st) != hipSuccess) return AWEQ_ERR_LAUNCH;
    return launch_status();
}

}  // namespace mxmid

int launch_mx4_mid(const MxArgs& g, bool square, hipStream_t st) { return square ? mxmid::launch_tile<2, 2, 2>(g, st) : mxmid::launch_tile<1, 2, 4>(g, st); }

}  // namespace aweq
