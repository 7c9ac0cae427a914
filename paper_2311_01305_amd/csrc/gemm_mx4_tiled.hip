// Product in microscaled 4-bit floating point for many tokens.
//
// One workgroup of 8 wavefronts (two per SIMD) owns a tile of 64 MI tokens x 256 channels, each wavefront 32 MI x 64 of it as MI x 2
// v_mfma_scale_f32_32x32x64_f8f6f4 tiles; a lane's operand is 16 consecutive bytes of one row, a block of 32 values.  Panels (64 bytes a row of both operands) go
// through a ring of LDS slots filled by LDS-DMA loads, three or four panels ahead of the one being multiplied, since a load's round trip is longer than
// a panel's instructions last; the slots are XOR swizzled by choosing which 16-byte chunk a lane fetches.  The scales of four panels are 16 bytes a row:
// two more LDS slots in turn, and per sub-tile two registers for four panels, of which the instruction names the byte; so the loop is unrolled by four panels.
// The weight is the instruction's first operand: a lane ends up with four consecutive channels of one token.  The bias is what the sums begin with.
// Persistent: the first panels of a workgroup's next tile are requested before it stores the current one.
//
// Several rounds are bound by the clock under load: 8192 x 8192 x 22016 585 - 610 us, 4.9 - 5.05 PFLOP/s, where the matrix unit alone sustains 6.7 on random codes
// (9.8 on zeros).  A single round of 172 workgroups, 333 tokens 22016 x 8192, takes 44 us: products and LDS reads with nothing loaded 37 (on zeros 30), loads with
// nothing multiplied 41 (33 where the weights are in the caches), and a barrier a panel lets them overlap in part.  A fifth slot for tiles of 192 tokens
// changed nothing.
#include "gemm_mx4.hpp"

#include <type_traits>

namespace aweq {
namespace mxtiled {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef int v2i __attribute__((ext_vector_type(2)));

constexpr int BN = 256;

struct Args : MxArgs, TileWalk {
    int wide;      // rows of a 16-bit output begin at multiples of 16 bytes: eight channels a store (us, against four: 4096 x 4096 x 4096 40.3 -> 38.8)
};

constexpr int kThreads = 512, kWaves = 8, kWn = 4;   // wavefronts: 2 x 4
constexpr int NJ = 2;                                // MI x 2 instruction tiles each (MI x 4, with half as many wavefronts, reads a third less of LDS and is slower:
                                                     // us, 8192 x 8192 x 22016 615 -> 652, 4096 x 4096 x 4096 37.4 -> 41.1)
template <int MI>
struct Tile {
    static constexpr int kRows = 64 * MI;
    static constexpr int kHalfA = kRows * 64;                     // token rows of a slot, then 16 KiB of weight rows
    static constexpr int kSlot = kHalfA + BN * 64;                // 16 KiB + 4 MI KiB
    static constexpr int kSlots = MI >= 3 ? 4 : 5;
    static constexpr int kAhead = kSlots - 1;                     // panels requested ahead of the one being multiplied
    static constexpr int kLoadsA = (4 * MI + kWaves - 1) / kWaves;   // load instructions per wavefront and panel, 16 rows each (MI odd: some rows twice)
    static constexpr int kLoadsB = 16 / kWaves, kLoadsS = 8 / kWaves;   // of the weight, and of a group's scales
    static constexpr int kLoads = kLoadsA + kLoadsB;
    static constexpr int kSlabs = kAhead * kSlot;                 // 4 KiB per wavefront for the outputs: the last slot and what is behind it
    static constexpr int kScales = 128 * 1024;                    // two slots of (kRows + 256) * 16 bytes
    static constexpr int kScaleSlot = (kRows + BN) * 16;
    static constexpr int kBias = kScales + 2 * kScaleSlot;        // 1 KiB
    static constexpr int kLds = kBias + 1024;
    static_assert(kSlabs + 8 * 4096 <= kScales && kSlots * kSlot <= kScales, "the ring, then the scales");
};

// chunk swizzle for 64-byte slot rows: 16 consecutive rows read at one chunk index land on distinct banks
__device__ __forceinline__ int f4(int r) { return (r >> 2) & 3; }

// LDS-DMA load the compiler does not track: lane i's 16 bytes land at lds_addr + 16 i, lds_addr wave-uniform
__device__ __forceinline__ void dma16(const uint8_t* sbase, uint32_t voff, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds_addr), "v"(voff), "s"(sbase) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_vm()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// The same unless skip is not 0: a branch that the compiler does not see, since it would move products of the loop past one of its own
template <int N>
__device__ __forceinline__ void wait_vm_unless(uint32_t skip)
{
    asm volatile("s_cmp_lg_u32 %1, 0\n\ts_cbranch_scc1 1f\n\ts_waitcnt vmcnt(%0)\n1:" ::"n"(N), "s"(skip) : "memory", "scc");
}

#define SB() __builtin_amdgcn_sched_barrier(0)
#define MF(A_, B_, S, i, j)                                                                                                                    \
    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx_operand(B_[j]), mx_operand(A_[i]), acc[i][j], 4, 4, J, sb[j][S], J, sa[i][S])

// OUT: kMx*
template <int MI, int OUT>
__global__ __launch_bounds__(kThreads) void gemm_mx4_tiled(Args g)
{
    using TL = Tile<MI>;
    constexpr int kFirstRow = 32 * MI, kFirstCol = 32 * NJ;
    constexpr int kSlot = TL::kSlot, kHalfA = TL::kHalfA, kAhead = TL::kAhead, kLoads = TL::kLoads;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / kWn, wn = wave % kWn;
    const int stride = gridDim.x;

    int vb = blockIdx.x, tile_m = 0, tile_n = 0;
    while (vb < g.n_ids && !tile_of(g, vb, tile_m, tile_n)) vb += stride;
    if (vb >= g.n_ids) return;

    const int64_t panelA = g.T * 64, panelB = g.N * 64;
    const int nh = (int)mx_panels(g.K);
    const int pre = nh < kAhead ? nh : kAhead;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
    // load q of this wavefront: rows of group (16 of them) wave + kWaves q, of the tokens around again where their groups are not a multiple
    uint32_t oa[TL::kLoadsA], ob[TL::kLoadsB], os[TL::kLoadsS];   // byte offsets from the tile's first row inside a panel, of scales
    auto groupA = [&](int q) { return (wave + kWaves * q) % (4 * MI); };
    const uint8_t *srcA, *srcB;       // the tile's rows in the panel being fetched
    int64_t panel_group;              // the group of scales being fetched
    int64_t m0, n0;
    // scales: a load is 64 rows of the tokens, then of the weight (with fewer tokens some of them once more, so that every wavefront has as many)
    auto scale_of_b = [&](int q) { return (wave + kWaves * q) % (MI + 4) >= MI; };
    auto scale_row = [&](int q) { const int u = (wave + kWaves * q) % (MI + 4); return (u >= MI ? u - MI : u) * 64; };

#define DMA_A(q) dma16(srcA, oa[q], dst_slot + (uint32_t)groupA(q) * 1024)
#define DMA_B(q) dma16(srcB, ob[q], dst_slot + kHalfA + (uint32_t)(wave + kWaves * (q)) * 1024)
    uint32_t scale_slot = 0;         // where the next group's scales go
    auto fetch_scales = [&]() {
#pragma unroll
        for (int q = 0; q < TL::kLoadsS; ++q) {
            const bool of_b = scale_of_b(q);
            const uint8_t* const from = of_b ? g.b_scale + (panel_group * g.N + n0) * 16 : g.a_scale + (panel_group * g.T + m0) * 16;
            dma16(from, os[q], lds0 + TL::kScales + scale_slot + (uint32_t)((of_b ? TL::kRows : 0) + scale_row(q)) * 16);
        }
        ++panel_group;
        scale_slot = TL::kScaleSlot - scale_slot;
    };
    // addresses of tile (tm, tn) and its bias, first scales and first `pre` panels on their way
    auto start_tile = [&](int tm, int tn) {
        m0 = (int64_t)__builtin_amdgcn_readfirstlane(tm) * TL::kRows;
        n0 = (int64_t)__builtin_amdgcn_readfirstlane(tn) * BN;
        // rows past the edge re-read the last valid row; their results are never stored
        int lane_ = lane;
        asm volatile("" : "+v"(lane_));   // (hidden: formed again for every tile instead of living through the multiplications)
        const int last_m = (int)min((int64_t)TL::kRows, g.T - m0) - 1, last_n = (int)min((int64_t)BN, g.N - n0) - 1;
        const int sub = lane_ >> 2, chunk = (lane_ & 3) ^ f4(sub);   // (loads start at multiples of 16 rows)
#pragma unroll
        for (int q = 0; q < TL::kLoadsA; ++q) oa[q] = (uint32_t)(min(groupA(q) * 16 + sub, last_m) * 64 + chunk * 16);
#pragma unroll
        for (int q = 0; q < TL::kLoadsB; ++q) ob[q] = (uint32_t)(min((wave + kWaves * q) * 16 + sub, last_n) * 64 + chunk * 16);
#pragma unroll
        for (int q = 0; q < TL::kLoadsS; ++q) os[q] = (uint32_t)(min(scale_row(q) + lane_, scale_of_b(q) ? last_n : last_m) * 16);
        srcA = g.a + m0 * 64;
        srcB = g.b + n0 * 64;
        panel_group = 0;
        scale_slot = 0;
        if (g.bias && wave == 0) dma16(reinterpret_cast<const uint8_t*>(g.bias + n0), (uint32_t)(min(lane_ * 4, last_n - 3) * 4), lds0 + TL::kBias);
        fetch_scales();
        for (int p = 0; p < pre; ++p) {
            const uint32_t dst_slot = lds0 + p * kSlot;
#pragma unroll
            for (int q = 0; q < TL::kLoadsA; ++q) DMA_A(q);
#pragma unroll
            for (int q = 0; q < TL::kLoadsB; ++q) DMA_B(q);
            srcA += panelA; srcB += panelB;
        }
    };

    start_tile(tile_m, tile_n);
    if (pre == kAhead) wait_vm<(kAhead - 1) * kLoads>(); else wait_vm<0>();

    // Vector memory operations of a wave complete in the order issued.  A tile that lies inside the output issues kStores stores per wave or more after
    // requesting the next tile's first panels, so "at most kStores operations pending" means those panels have landed while the stores may
    // still be on their way (relaxed: set for the tile that follows).
    constexpr int kStores = OUT == kMxF32 ? 8 * MI : 4 * MI;
    bool relaxed = false;

    for (;;) {
        const int64_t cm0 = m0, cn0 = n0;   // the tile being multiplied
        // fragment of K-step ks of a panel: lane reads row lane % 32 of a 32-row sub-tile, chunk 2 ks + lane / 32 (block 2 ks + lane / 32 of the panel)
        int fl_ = lane;
        asm volatile("" : "+v"(fl_));
        const int fr_row = fl_ & 31, fr_half = fl_ >> 5;
        int offA[2], offB[2];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            offA[ks] = (wm * kFirstRow + fr_row) * 64 + ((ks * 2 + fr_half) ^ f4(fr_row)) * 16;
            offB[ks] = kHalfA + (wn * kFirstCol + fr_row) * 64 + ((ks * 2 + fr_half) ^ f4(fr_row)) * 16;
        }
        const int offSA = TL::kScales + (wm * kFirstRow + fr_row) * 16 + fr_half * 8;
        const int offSB = TL::kScales + (TL::kRows + wn * kFirstCol + fr_row) * 16 + fr_half * 8;
        v4i a0[MI], b0[NJ], a1[MI], b1[NJ];
        v2i sa[MI], sb[NJ];
        v16f acc[MI][NJ];

#define RDA(dst, ks, i) dst[i] = *reinterpret_cast<const v4i*>(st + offA[ks] + (i) * 32 * 64)
#define RDB(dst, ks, j) dst[j] = *reinterpret_cast<const v4i*>(st + offB[ks] + (j) * 32 * 64)
#define RDSA(dst, i) dst[i] = *reinterpret_cast<const v2i*>(lds + offSA + read_scale + (i) * 32 * 16)
#define RDSB(dst, j) dst[j] = *reinterpret_cast<const v2i*>(lds + offSB + read_scale + (j) * 32 * 16)
        uint32_t read_scale = 0;
        __builtin_amdgcn_s_barrier();  // panel 0, its scales and the bias have landed for every wave
        {
            const char* st = lds;
#pragma unroll
            for (int i = 0; i < MI; ++i) { RDA(a0, 0, i); RDSA(sa, i); }
#pragma unroll
            for (int j = 0; j < NJ; ++j) { RDB(b0, 0, j); RDSB(sb, j); }
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    Float4 b = {{0.0f, 0.0f, 0.0f, 0.0f}};
                    if (g.bias) b = *reinterpret_cast<const Float4*>(lds + TL::kBias + (wn * kFirstCol + 32 * j + 8 * q + 4 * fr_half) * 4);
#pragma unroll
                    for (int i = 0; i < MI; ++i)
#pragma unroll
                        for (int v = 0; v < 4; ++v) acc[i][j][4 * q + v] = b.f[v];
                }
        }

        // one panel = two K-steps of 2 MI instructions per wave.  a0, b0 / a1, b1: fragments of the two; each K-step multiplies one set and fetches the
        // other.  ISSUE: panel h + kAhead is fetched into the slot panel h - 1 occupied (every wave finished reading it before the
        // barrier of panel h - 1), before a group's first one the group's scales.  wait: until panel h + 1 is complete.  J: which byte the scales are in; GROUP: whether
        // h is a group's last panel (1), or not (0), or may be (2).
        constexpr int kReads = (MI + NJ + MI * NJ / 2 - 1) / (MI * NJ / 2);        // fragments an instruction, so that half of them are enough
        constexpr int kIssues = (kLoads + MI * NJ - 2) / (MI * NJ - 1);
        uint32_t slot = 0;   // byte offset of panel h's slot
        int h = 0;
        auto half = [&](auto j_c, auto group_c, auto issue_c, auto next_c, auto scales_c, auto wait) {
            constexpr int J = decltype(j_c)::value, GROUP = decltype(group_c)::value, SCALES = decltype(scales_c)::value;
            constexpr bool ISSUE = decltype(issue_c)::value, NEXT = decltype(next_c)::value;
            const uint32_t next_slot = slot == kAhead * kSlot ? 0 : slot + kSlot;
            const uint32_t dst_slot = lds0 + (slot == 0 ? kAhead * kSlot : slot - kSlot);
            const char* st = lds + slot;
            // the second K-step's fragments and the loads one by one between the instructions
#pragma unroll
            for (int u = 0; u < MI * NJ; ++u) {
                const int i = u / NJ, j = u % NJ;
                SB();
#pragma unroll
                for (int r = 0; r < kReads; ++r) {
                    const int f = u * kReads + r;
                    if (f == 0) RDA(a1, 1, 0);
                    else if (f <= NJ) RDB(b1, 1, f - 1);
                    else if (f < MI + NJ) RDA(a1, 1, f - NJ);
                }
                if constexpr (ISSUE) {
                    if (u == 0 && (SCALES == 1 || (SCALES == 2 && ((h + kAhead) & 3) == 0))) fetch_scales();
#pragma unroll
                    for (int r = 0; r < kIssues; ++r) {
                        const int f = u * kIssues + r;
                        if (f < TL::kLoadsA) DMA_A(f);
                        else if (f < kLoads) DMA_B(f - TL::kLoadsA);
                    }
                }
                MF(a0, b0, 0, i, j);
            }
            SB();
            if constexpr (ISSUE) { srcA += panelA; srcB += panelB; }
            if constexpr (NEXT) {
                // my loads of the next panel have landed, my reads of this one are done; after the barrier that holds for every wave
                wait();
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                __builtin_amdgcn_s_barrier();
                SB();
                st = lds + next_slot;
                v2i na[MI], nb[NJ];
                if constexpr (GROUP == 1) {
                    read_scale = TL::kScaleSlot - read_scale;
#pragma unroll
                    for (int i = 0; i < MI; ++i) RDSA(na, i);
#pragma unroll
                    for (int j = 0; j < NJ; ++j) RDSB(nb, j);
                }
#pragma unroll
                for (int u = 0; u < MI * NJ; ++u) {
                    const int i = u / NJ, j = u % NJ;
                    SB();
#pragma unroll
                    for (int r = 0; r < kReads; ++r) {
                        const int f = u * kReads + r;
                        if (f == 0) RDA(a0, 0, 0);
                        else if (f <= NJ) RDB(b0, 0, f - 1);
                        else if (f < MI + NJ) RDA(a0, 0, f - NJ);
                    }
                    MF(a1, b1, 1, i, j);
                }
                SB();
                if constexpr (GROUP == 1) {
#pragma unroll
                    for (int i = 0; i < MI; ++i) sa[i] = na[i];
#pragma unroll
                    for (int j = 0; j < NJ; ++j) sb[j] = nb[j];
                } else if constexpr (GROUP == 2) {
                    if ((h & 3) == 3) {
                        read_scale = TL::kScaleSlot - read_scale;
#pragma unroll
                        for (int i = 0; i < MI; ++i) RDSA(sa, i);
#pragma unroll
                        for (int j = 0; j < NJ; ++j) RDSB(sb, j);
                    } else {
#pragma unroll
                        for (int i = 0; i < MI; ++i) sa[i] = v2i{(int)((uint32_t)sa[i][0] >> 8), (int)((uint32_t)sa[i][1] >> 8)};
#pragma unroll
                        for (int j = 0; j < NJ; ++j) sb[j] = v2i{(int)((uint32_t)sb[j][0] >> 8), (int)((uint32_t)sb[j][1] >> 8)};
                    }
                }
            } else {
#pragma unroll
                for (int u = 0; u < MI * NJ; ++u) MF(a1, b1, 1, u / NJ, u % NJ);
            }
            slot = next_slot;
            ++h;
        };
        using std::integral_constant;
        using std::true_type;
        using std::false_type;
        // Four panels at a time while all of them have one to request.  In flight when panel h + 1 has to be complete: kAhead - 1 panels, and scales where
        // one of them begins a group.  relaxed: the panels requested before the stores landed together with panel 0: nothing to wait for, and a count would
        // wait for the stores.
        uint32_t landed = relaxed ? 1u : 0u;      // (in the first four)
        auto steady = [&](auto j_c) {
            constexpr int J = decltype(j_c)::value;
            constexpr bool scales = (J + 2) % 4 == 0 || (J + 3) % 4 == 0 || (kAhead > 3 && (J + 4) % 4 == 0);
            half(j_c, integral_constant<int, J == 3 ? 1 : 0>{}, true_type{}, true_type{}, integral_constant<int, (J + kAhead) % 4 == 0 ? 1 : 0>{}, [&]() {
                constexpr int left = (kAhead - 1) * kLoads + (scales ? TL::kLoadsS : 0);
                if constexpr (J >= kAhead - 1) wait_vm<left>();
                else wait_vm_unless<left>(landed);
            });
        };
        while (h + kAhead + 3 < nh) {
            steady(integral_constant<int, 0>{});
            steady(integral_constant<int, 1>{});
            steady(integral_constant<int, 2>{});
            steady(integral_constant<int, 3>{});
            landed = 0;
        }
        // The rest, at most kAhead + 3: the scales of the panel in the lowest byte
        const integral_constant<int, 0> low;
        const integral_constant<int, 2> may_be;
        while (h + kAhead < nh) half(low, may_be, true_type{}, true_type{}, may_be, [&]() { wait_vm<(kAhead - 1) * kLoads>(); });
        if constexpr (kAhead > 3) {
            if (h + 3 < nh) half(low, may_be, false_type{}, true_type{}, low, [&]() { wait_vm<2 * kLoads>(); });
        }
        if (h + 2 < nh) half(low, may_be, false_type{}, true_type{}, low, [&]() { wait_vm<kLoads>(); });
        if (h + 1 < nh) half(low, may_be, false_type{}, true_type{}, low, [&]() { wait_vm<0>(); });
        half(low, low, false_type{}, false_type{}, low, [&]() {});
#undef RDA
#undef RDB
#undef RDSA
#undef RDSB

        // ---- the next tile of this workgroup, then this one's outputs.  Register v of lane l in sub-tile (i, j) is token t = m0 + 32 MI wm + 32 i + l % 32 and
        // channel n = n0 + 64 wn + 32 j + 8 (v / 4) + 4 (l / 32) + v % 4.  Each wave turns 32 tokens around in 4 KiB of LDS of its own (chunks XOR swizzled), so
        // that neighbouring lanes store neighbouring channels.
        int nvb = vb + stride, ntm = 0, ntn = 0;
        while (nvb < g.n_ids && !tile_of(g, nvb, ntm, ntn)) nvb += stride;
        const bool more = nvb < g.n_ids;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();  // every wave is done reading the ring
        if (more) start_tile(ntm, ntn);
        int lane_ = lane;
        asm volatile("" : "+v"(lane_));
        char* const slab = lds + TL::kSlabs + wave * 4096;
        const int tok = lane_ & 31, part = lane_ >> 5;
        const int64_t wave_t = cm0 + wm * kFirstRow, wave_n = cn0 + wn * kFirstCol;
        const bool inside = cm0 + TL::kRows <= g.T && cn0 + BN <= g.N;
        if constexpr (OUT == kMxF32) {
            // 32 channels at a time: rows of 128 bytes, 8 lanes each
            const int rd_r = lane_ >> 3, rd_c = lane_ & 7;
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    wave_lds_fence();
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *reinterpret_cast<Float4*>(slab + tok * 128 + ((2 * q + part) ^ (tok & 7)) * 16) =
                            Float4{{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]}};
                    wave_lds_fence();
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        const int r = 8 * p + rd_r;
                        const int64_t t = wave_t + 32 * i + r, n = wave_n + 32 * j + rd_c * 4;
                        const Float4 v = *reinterpret_cast<const Float4*>(slab + r * 128 + (rd_c ^ (r & 7)) * 16);
                        if (inside || (t < g.T && n < g.N)) *reinterpret_cast<Float4*>(reinterpret_cast<float*>(g.out) + t * g.ldo + n) = v;
                    }
                }
        } else {
            using E = typename std::conditional<OUT == kMxF16, _Float16, __bf16>::type;
            typedef E e4 __attribute__((ext_vector_type(4)));
            const int rd_r = lane_ >> 4, rd_c = lane_ & 15;
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                wave_lds_fence();
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const v16f& a = acc[i][j];
                        *reinterpret_cast<e4*>(slab + tok * 128 + ((8 * j + 2 * q + part) ^ (tok & 15)) * 8) =
                            e4{(E)a[4 * q], (E)a[4 * q + 1], (E)a[4 * q + 2], (E)a[4 * q + 3]};
                    }
                wave_lds_fence();
                if (g.wide && inside) {
                    const int r0 = lane_ >> 3, c = (lane_ & 7) * 2;
                    E* const row = reinterpret_cast<E*>(g.out) + (wave_t + 32 * i + r0) * g.ldo + wave_n + c * 4;
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        const int r = 8 * p + r0;
                        union { e4 h[2]; v4i v; } u;
                        u.h[0] = *reinterpret_cast<const e4*>(slab + r * 128 + (c ^ (r & 15)) * 8);
                        u.h[1] = *reinterpret_cast<const e4*>(slab + r * 128 + ((c + 1) ^ (r & 15)) * 8);
                        *reinterpret_cast<v4i*>(row + (int64_t)(8 * p) * g.ldo) = u.v;
                    }
                    continue;
                }
#pragma unroll
                for (int p = 0; p < 8; ++p) {
                    const int r = 4 * p + rd_r;
                    const int64_t t = wave_t + 32 * i + r, n = wave_n + rd_c * 4;
                    const e4 v = *reinterpret_cast<const e4*>(slab + r * 128 + (rd_c ^ (r & 15)) * 8);
                    if (inside || (t < g.T && n < g.N)) *reinterpret_cast<e4*>(reinterpret_cast<E*>(g.out) + t * g.ldo + n) = v;
                }
            }
        }
        if (!more) break;
        relaxed = nh > kAhead + 3 && inside;
        if (relaxed) wait_vm<kStores>();
        else wait_vm<0>();
        vb = nvb;
    }
#undef DMA_A
#undef DMA_B
}
#undef MF
#undef SB

}  // namespace mxtiled

bool plan_mx4_tiled(int64_t T, int64_t N, int64_t K, int mi, int64_t& tiles, int64_t& rounds)
{
    mxtiled::Args g = {};
    int64_t blocks = 0;
    if (plan_walk(g, T, N, K / 2, 64 * mi, blocks) != AWEQ_OK) return false;
    tiles = (int64_t)g.tiles_m * g.tiles_n;
    rounds = rounds_of(g);
    return true;
}

template <int MI>
static int launch_tile(mxtiled::Args& g, hipStream_t st)
{
    const void* fn = g.out_kind == kMxF32   ? reinterpret_cast<const void*>(mxtiled::gemm_mx4_tiled<MI, kMxF32>)
                     : g.out_kind == kMxF16 ? reinterpret_cast<const void*>(mxtiled::gemm_mx4_tiled<MI, kMxF16>)
                                            : reinterpret_cast<const void*>(mxtiled::gemm_mx4_tiled<MI, kMxBf16>);
    return launch_persistent(fn, mxtiled::kThreads, mxtiled::Tile<MI>::kLds, &g, g.n_ids, st);
}

int launch_mx4_tiled(const MxArgs& m, int mi, hipStream_t st)
{
    mxtiled::Args g = {};
    static_cast<MxArgs&>(g) = m;
    g.wide = g.ldo % 8 == 0;     // (out is 16-byte aligned)
    int64_t blocks = 0;
    const int rc = plan_walk(g, g.T, g.N, g.K / 2, 64 * mi, blocks);
    if (rc != AWEQ_OK) return rc;
    return mi == 4 ? launch_tile<4>(g, st) : mi == 3 ? launch_tile<3>(g, st) : mi == 2 ? launch_tile<2>(g, st) : launch_tile<1>(g, st);
}

}  // namespace aweq
