// Around the attention of drafted tokens: the plan of a step (pages, slots, rows), the masks of the trees, the move of an accepted path.
// All three are a launch and a few dependent reads: what bounds them is latency.
#include "common.hpp"

namespace aweq {
namespace drafts {

// ---------------------------------------------------------------- the step's plan
// Every workgroup reads all lengths and adds them up for itself (three running sums: new tokens, pages taken, pages given back), so that one launch does it; then the
// threads of all of them share tokens, pages and sequences.  Nothing that is read is written: pages taken go behind a sequence's own in its row, pages
// given back are read from the end of theirs, the stack is read below its top and written above.
// (us, a launch being 2.2: 7 sequences of a token each 4.3, 600 with 19544 new tokens, of which 112 give back, 7.7: lengths, running sums, pages)
constexpr int kPlanThreads = 512, kPlanWaves = kPlanThreads / kWave;
constexpr int kPlanMost = 8192;     // sequences

struct PlanArgs {
    const int32_t *lens, *change;
    int32_t* table;
    int32_t* free_pages;
    const int32_t* free_count;
    int32_t *lens_out, *count_out, *q_start, *pos;
    int64_t* slot;
    uint32_t* status;
    int64_t table_ld, T;
    int B, page_size, page_shift, pages, table_pages, prefix_len;
};

__device__ __forceinline__ long long wave_scan(long long v, int lane)
{
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const long long o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}

// the last sequence whose running sum is at most i (sums[0] = 0, rising; i below the last)
__device__ __forceinline__ int sequence_of(const int* sums, int B, int i)
{
    int lo = 0, hi = B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (sums[mid] <= i) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// EACH: sequences of a thread, at most
template <int EACH>
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(PlanArgs g)
{
    extern __shared__ int sums[];    // [3][B + 1]: tokens, pages taken, pages given back ahead of each sequence; [B]: what it had
    int* const s_new = sums;
    int* const s_take = sums + g.B + 1;
    int* const s_give = s_take + g.B + 1;
    int* const s_len = s_give + g.B + 1;
    __shared__ long long s_part[3][kPlanWaves];
    __shared__ unsigned s_bad;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    if (tid == 0) s_bad = 0;
    // a thread has some sequences in a row, whose numbers it asks for at once
    const int per = (g.B + kPlanThreads - 1) / kPlanThreads, from = min(tid * per, g.B), mine = min(per, g.B - from);
    int len[EACH], change[EACH];
#pragma unroll
    for (int k = 0; k < EACH; ++k)
        if (k < mine) { len[k] = g.lens[from + k]; change[k] = g.change[from + k]; }
    const int count = *g.free_count;
    const long long room = (long long)g.table_pages << g.page_shift;
    auto pages_of = [&](int tokens) { return (tokens + g.page_size - 1) >> g.page_shift; };
    long long add[3] = {0, 0, 0};
    bool bad = count < 0 || count > g.pages;
#pragma unroll
    for (int k = 0; k < EACH; ++k)
        if (k < mine) {
            const long long after = (long long)len[k] + change[k];
            if (len[k] < 0 || len[k] > room || after < 0 || after > room) {
                bad = true;
            } else {
                const int had = pages_of(len[k]), has = pages_of((int)after);
                add[0] += max(change[k], 0);
                add[1] += max(has - had, 0);
                add[2] += max(had - has, 0);
            }
        }
    __syncthreads();
    if (bad) atomicOr(&s_bad, (unsigned)AWEQ_ST_INDEX);
    long long sum[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        sum[k] = wave_scan(add[k], lane);
        if (lane == kWave - 1) s_part[k][wave] = sum[k];
    }
    __syncthreads();
    long long total[3] = {0, 0, 0};
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        sum[k] -= add[k];
        for (int w = 0; w < kPlanWaves; ++w) {
            if (w < wave) sum[k] += s_part[k][w];
            total[k] += s_part[k][w];
        }
    }
    uint32_t st = s_bad;
    if (total[0] > g.T || count + total[2] > g.pages) st |= AWEQ_ST_INDEX;
    if (total[1] > count + total[2]) st |= AWEQ_ST_PAGES;
    if (st & AWEQ_ST_INDEX) st = AWEQ_ST_INDEX;
    const int64_t first = (int64_t)blockIdx.x * kPlanThreads + tid, step = (int64_t)gridDim.x * kPlanThreads;
    if (st) {
        // nothing changes
        if (blockIdx.x == 0 && tid == 0) raise_status(g.status, st);
        for (int64_t b = first; b <= g.B; b += step) {
            g.q_start[b] = 0;
            if (b < g.B) g.lens_out[b] = g.lens[b];
        }
        for (int64_t t = first; t < g.T; t += step) { g.pos[t] = 0; g.slot[t] = -1; }
        if (first == 0) *g.count_out = count;
        return;
    }
    // (the totals fit 32 bits: tokens are no more than T, pages given back, and with the stack those taken, no more than there are)
#pragma unroll
    for (int k = 0; k < EACH; ++k)
        if (k < mine) {
            const int had = pages_of(len[k]), has = pages_of(len[k] + change[k]);
            s_new[from + k] = (int)sum[0]; s_take[from + k] = (int)sum[1]; s_give[from + k] = (int)sum[2];
            s_len[from + k] = len[k];
            sum[0] += max(change[k], 0); sum[1] += max(has - had, 0); sum[2] += max(had - has, 0);
        }
    const int tokens = (int)total[0], taken = (int)total[1], given = (int)total[2];
    if (tid == 0) { s_new[g.B] = tokens; s_take[g.B] = taken; s_give[g.B] = given; }
    __syncthreads();
    auto returned = [&](int i) {         // the i-th page that is given back
        const int b = sequence_of(s_give, g.B, i);
        return g.table[b * g.table_ld + pages_of(s_len[b]) - s_give[b + 1] + i];   // (it keeps its pages less those that it gives)
    };
    auto page_at = [&](int i) { return i < given ? returned(i) : g.free_pages[count - 1 - (i - given)]; };
    for (int64_t b = first; b <= g.B; b += step) {
        g.q_start[b] = s_new[b];
        if (b < g.B) g.lens_out[b] = s_len[b] + g.change[b];
    }
    for (int64_t t = first; t < g.T; t += step) {
        int pos = 0;
        int64_t slot = -1;
        if (t < tokens) {
            const int b = sequence_of(s_new, g.B, (int)t), had_tokens = s_len[b], p = had_tokens + ((int)t - s_new[b]), j = p >> g.page_shift, had = pages_of(had_tokens);
            const int page = j < had ? g.table[b * g.table_ld + j] : page_at(s_take[b] + j - had);
            pos = g.prefix_len + p;
            slot = ((int64_t)page << g.page_shift) + (p & (g.page_size - 1));
        }
        g.pos[t] = pos;
        g.slot[t] = slot;
    }
    for (int64_t i = first; i < taken; i += step) {
        const int b = sequence_of(s_take, g.B, (int)i);
        g.table[b * g.table_ld + pages_of(s_len[b]) + ((int)i - s_take[b])] = page_at((int)i);
    }
    for (int64_t i = first; i < given - taken; i += step) g.free_pages[count + i] = returned(taken + (int)i);
    if (first == 0) *g.count_out = count + given - taken;
}

// ---------------------------------------------------------------- masks of trees
constexpr int kMaskThreads = 256;
constexpr int kMaskMost = 4096;     // new tokens of a sequence

struct MaskArgs {
    const int32_t *parent, *q_start, *lens;
    uint64_t* mask;
    int32_t* pos;
    uint32_t* status;
    int64_t T, mask_ld;
    int max_q, words, prefix_len;
};

// A workgroup has a sequence, a thread a token and its path: the places on it fall, so that a word of the mask is complete when the next one begins (a tree of 12
// tokens 2.5 us, five of up to 211 5.4: the longest path, a read of LDS after the other)
__global__ __launch_bounds__(kMaskThreads) void mask_kernel(MaskArgs g)
{
    extern __shared__ int s_parent[];
    const int b = blockIdx.x;
    uint32_t st = 0;
    int64_t t0 = g.q_start[b], t1 = g.q_start[b + 1];
    const int len = g.pos ? g.lens[b] : 0;
    if (t0 < 0 || t1 < t0 || t1 > g.T || t1 - t0 > g.max_q) st |= AWEQ_ST_INDEX;
    t0 = min(max(t0, (int64_t)0), g.T);
    t1 = min(max(t1, t0), min(g.T, t0 + g.max_q));
    const int m = (int)(t1 - t0);
    for (int i = threadIdx.x; i < m; i += kMaskThreads) {
        int p = g.parent[t0 + i];
        if (p < -1 || p >= i) { st |= AWEQ_ST_INDEX; p = -1; }
        s_parent[i] = p;
    }
    __syncthreads();
    const int base = g.prefix_len + len - m;
    for (int i = threadIdx.x; i < m; i += kMaskThreads) {
        uint64_t* const row = g.mask + (t0 + i) * g.mask_ld;
        int word = g.words - 1, depth = -1;
        uint64_t bits = 0;
        for (int at = i; at >= 0; at = s_parent[at]) {
            for (; word > at >> 6; --word) { row[word] = bits; bits = 0; }
            bits |= 1ull << (at & 63);
            ++depth;
        }
        for (; word >= 0; --word) { row[word] = bits; bits = 0; }
        if (g.pos) g.pos[t0 + i] = base + depth;
    }
    raise_status(g.status, st);
}

// ---------------------------------------------------------------- an accepted path to the front
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct KeepArgs {
    char *k_cache, *v_cache;
    float *k_step, *v_step;
    const int32_t *table, *lens, *q_start, *kept, *count;
    int32_t* change;
    uint32_t* status;
    int64_t table_ld, kept_ld, T;
    int B, Hk, pages, page_size, page_shift;
    int chunk, chunks;      // bytes a lane moves of a row, and how many of them it has
};

// A wavefront has a sequence's head in one of the caches.  Place j goes from kept[j] >= j to j, and the places rise: rows that have been written are none that is
// still to be read, so that as many as lanes and registers hold go at a time, reads ahead of writes.  A lane has the rows of one place of 64, found with few
// reads that wait for one another: the counts, then the places (no more of a row than its count need be there), the pages, the rows (us: one path of 5 of 12 tokens and 32 heads
// 3.6, 256 of 9 of 64 with 8 heads of codes 5.2, a launch being 2.2).
// V: a vector type of the compiler's (of a structure the rows in flight went to LDS: one path 8.0 us, 32 of them 17)
template <class V>
__global__ __launch_bounds__(kWave) void keep_kernel(KeepArgs g)
{
    const int b = blockIdx.x, head = blockIdx.y, lane = threadIdx.x;
    const bool values = blockIdx.z != 0;
    const int32_t* const kept = g.kept + b * g.kept_ld;
    const int64_t t0 = g.q_start[b], t1 = g.q_start[b + 1];
    const int len = g.lens[b], n = g.count[b];
    bool ok = t0 >= 0 && t1 >= t0 && t1 <= g.T && len >= t1 - t0 && len <= (g.table_ld << g.page_shift);
    const int m = ok ? (int)(t1 - t0) : 0, base = len - m;
    ok = ok && n >= 0 && n <= m && n <= g.kept_ld;
    int place = 0;          // kept[b][lane]
    if (ok) {
        if (lane < n) place = kept[lane];
        bool order = true;
        const int before = __shfl_up(place, 1);
        if (lane < n) order = place > (lane ? before : -1) && place < m;
        for (int j = lane + kWave; j < n; j += kWave) order = order && kept[j] > kept[j - 1] && kept[j] < m;
        ok = __builtin_amdgcn_ballot_w64(!order) == 0;
    }
    uint32_t st = ok ? 0u : (uint32_t)AWEQ_ST_INDEX;
    if (head == 0 && !values && lane == 0) g.change[b] = ok ? n - m : 0;
    if (ok) {
        char* const cache = values ? g.v_cache : g.k_cache;
        float* const step = values ? g.v_step : g.k_step;
        const int32_t* const table = g.table + b * g.table_ld;
        const int rows = kWave / g.chunks, sub = lane / g.chunks, part = lane % g.chunks;
        const int64_t bytes = (int64_t)g.chunk * g.chunks;
        constexpr int kAtOnce = 4;
        for (int from = 0; from < n; from += kWave) {
            // rows of place from + lane: where they are, and where they go; -1: they stay
            const int j = from + lane;
            if (from && j < n) place = kept[j];
            int64_t source = -1, dest = -1;
            if (j < n && place != j) {
                const int ks = base + place, kd = base + j;
                const int ps = table[ks >> g.page_shift], pd = table[kd >> g.page_shift];
                if ((unsigned)ps >= (unsigned)g.pages || (unsigned)pd >= (unsigned)g.pages) {
                    st |= AWEQ_ST_INDEX;
                } else {
                    source = (((int64_t)ps * g.Hk + head) << g.page_shift) + (ks & (g.page_size - 1));
                    dest = (((int64_t)pd * g.Hk + head) << g.page_shift) + (kd & (g.page_size - 1));
                }
            }
            const int here = min(n - from, kWave);
            for (int j0 = 0; j0 < here; j0 += rows * kAtOnce) {
                V v[kAtOnce];
                float s[kAtOnce];
                int64_t to[kAtOnce];
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    const int at = j0 + u * rows + sub;
                    const int64_t row = __shfl(source, at & (kWave - 1));
                    to[u] = __shfl(dest, at & (kWave - 1));
                    if (sub >= rows || at >= here) to[u] = -1;
                    if (to[u] >= 0) {
                        v[u] = *reinterpret_cast<const V*>(cache + row * bytes + part * g.chunk);
                        s[u] = step ? step[row] : 0.0f;
                    }
                }
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // (a row read by one lane may be another's to write)
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u)
                    if (to[u] >= 0) {
                        *reinterpret_cast<V*>(cache + to[u] * bytes + part * g.chunk) = v[u];
                        if (step && part == 0) step[to[u]] = s[u];
                    }
            }
        }
    }
    raise_status(g.status, st);
}

static bool page_ok(int64_t page_size) { return page_size >= 16 && page_size <= 256 && (page_size & (page_size - 1)) == 0; }
static bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

}  // namespace drafts
}  // namespace aweq

using namespace aweq;

extern "C" int aweq_step_plan(const int32_t* lens, const int32_t* change, int64_t B, int64_t page_size, int64_t pages, int32_t* table, int64_t table_ld,
                              int64_t table_pages, int32_t* free_pages, const int32_t* free_count, int64_t prefix_len, int64_t T,
                              int32_t* lens_out, int32_t* count_out, int32_t* q_start, int32_t* pos, int64_t* slot, uint32_t* status, void* stream)
{
    if (!lens || !change || !table || !free_pages || !free_count || !lens_out || !count_out || !q_start || !pos || !slot) return AWEQ_ERR_NULL;
    if (B <= 0 || B > drafts::kPlanMost || T <= 0 || T > (1 << 24) || !drafts::page_ok(page_size) || pages <= 0 || pages > 0x7fffffff || table_pages <= 0 ||
        table_pages > (1 << 24) || table_ld < table_pages || table_pages * page_size > (1 << 29) || prefix_len < 0 || prefix_len > (1 << 29))
        return AWEQ_ERR_SHAPE;
    for (const void* p : {(const void*)lens, (const void*)change, (const void*)table, (const void*)free_pages, (const void*)free_count, (const void*)lens_out,
                          (const void*)count_out, (const void*)q_start, (const void*)pos})
        if (!drafts::aligned(p, 4)) return AWEQ_ERR_ALIGN;
    if (!drafts::aligned(slot, 8)) return AWEQ_ERR_ALIGN;
    // in place a workgroup would read what another one has written
    const Span in[] = {{lens, B * 4}, {change, B * 4}, {free_count, 4}}, state[] = {matrix_span(table, B, table_pages, table_ld, 4), {free_pages, pages * 4}};
    const Span out[] = {{lens_out, B * 4}, {count_out, 4}, {q_start, (B + 1) * 4}, {pos, T * 4}, {slot, T * 8}};
    for (const Span& o : out)
        if (overlap({o}, {in[0], in[1], in[2], state[0], state[1]})) return AWEQ_ERR_ALIGN;
    drafts::PlanArgs g = {};
    g.lens = lens; g.change = change; g.table = table; g.free_pages = free_pages; g.free_count = free_count;
    g.lens_out = lens_out; g.count_out = count_out; g.q_start = q_start; g.pos = pos; g.slot = slot; g.status = status;
    g.table_ld = table_ld; g.T = T; g.B = (int)B; g.page_size = (int)page_size; g.page_shift = __builtin_ctz((unsigned)page_size);
    g.pages = (int)pages; g.table_pages = (int)table_pages; g.prefix_len = (int)prefix_len;
    const int lds = (3 * ((int)B + 1) + (int)B) * 4;
    const int64_t each = cdiv(B, drafts::kPlanThreads), want = cdiv(T > B ? T : B, drafts::kPlanThreads);
    const void* fn = each == 1   ? reinterpret_cast<const void*>(drafts::plan_kernel<1>)
                     : each == 2 ? reinterpret_cast<const void*>(drafts::plan_kernel<2>)
                                 : reinterpret_cast<const void*>(drafts::plan_kernel<drafts::kPlanMost / drafts::kPlanThreads>);
    int dev = 0, cus = 0;
    if (lds > 32768 && (device_cus(dev, cus) != AWEQ_OK || raise_lds_limit(fn, dev, (4 * drafts::kPlanMost + 3) * 4) != AWEQ_OK)) return AWEQ_ERR_LAUNCH;
    void* args[] = {&g};
    if (hipLaunchKernel(fn, dim3((unsigned)(want < 256 ? want : 256)), dim3(drafts::kPlanThreads), args, lds, as_stream(stream)) != hipSuccess) return AWEQ_ERR_LAUNCH;
    return launch_status();
}

extern "C" int aweq_tree_mask(const int32_t* parent, int64_t T, const int32_t* q_start, int64_t B, int64_t max_q, const int32_t* lens, int64_t prefix_len,
                              uint64_t* mask, int64_t mask_ld, int32_t* pos, uint32_t* status, void* stream)
{
    if (!parent || !q_start || !mask || (pos && !lens)) return AWEQ_ERR_NULL;
    if (T <= 0 || T > (1 << 24) || B <= 0 || B > (1 << 20) || max_q <= 0 || max_q > drafts::kMaskMost || prefix_len < 0 || prefix_len > (1 << 29) || mask_ld < cdiv(max_q, 64))
        return AWEQ_ERR_SHAPE;
    if (!drafts::aligned(parent, 4) || !drafts::aligned(q_start, 4) || !drafts::aligned(lens, 4) || !drafts::aligned(mask, 8) || !drafts::aligned(pos, 4)) return AWEQ_ERR_ALIGN;
    if (overlap({matrix_span(mask, T, cdiv(max_q, 64), mask_ld, 8), {pos, T * 4}}, {{parent, T * 4}, {q_start, (B + 1) * 4}, {pos ? lens : nullptr, B * 4}}))
        return AWEQ_ERR_ALIGN;
    const drafts::MaskArgs g = {parent, q_start, lens, mask, pos, status, T, mask_ld, (int)max_q, (int)cdiv(max_q, 64), (int)prefix_len};
    drafts::mask_kernel<<<(unsigned)B, drafts::kMaskThreads, (size_t)max_q * 4, as_stream(stream)>>>(g);
    return launch_status();
}

extern "C" int aweq_kv_keep(void* k_cache, void* v_cache, float* k_step, float* v_step, aweq_dtype cache_dt, int64_t pages, int64_t page_size, int64_t Hk, int64_t D,
                            const int32_t* table, int64_t table_ld, const int32_t* lens, const int32_t* q_start, int64_t B, int64_t T,
                            const int32_t* kept, int64_t kept_ld, const int32_t* count, int32_t* change, uint32_t* status, void* stream)
{
    if (!k_cache || !v_cache || !table || !lens || !q_start || !kept || !count || !change) return AWEQ_ERR_NULL;
    if (cache_dt != AWEQ_F16 && cache_dt != AWEQ_BF16 && cache_dt != AWEQ_I8) return AWEQ_ERR_DTYPE;
    const bool codes = cache_dt == AWEQ_I8;
    if (codes && (!k_step || !v_step)) return AWEQ_ERR_NULL;
    if (pages <= 0 || pages > 0x7fffffff || !drafts::page_ok(page_size) || Hk <= 0 || Hk > (1 << 16) - 1 || D <= 0 || D > 256 || D % 8 != 0 || B <= 0 || B > (1 << 20) ||
        T <= 0 || T > (1 << 24) || table_ld < 1 || kept_ld < 1 || B * Hk > (1 << 24))
        return AWEQ_ERR_SHAPE;
    if (!aligned16(k_cache) || !aligned16(v_cache) || (codes && (!aligned16(k_step) || !aligned16(v_step)))) return AWEQ_ERR_ALIGN;
    for (const void* p : {(const void*)table, (const void*)lens, (const void*)q_start, (const void*)kept, (const void*)count, (const void*)change})
        if (!drafts::aligned(p, 4)) return AWEQ_ERR_ALIGN;
    // (a workgroup would read what another one has written)
    if (overlap({{change, B * 4}}, {{lens, B * 4}, {count, B * 4}, {q_start, (B + 1) * 4}, matrix_span(kept, B, kept_ld < T ? kept_ld : T, kept_ld, 4), matrix_span(table, B, 1, table_ld, 4)}))
        return AWEQ_ERR_ALIGN;
    drafts::KeepArgs g = {};
    g.k_cache = reinterpret_cast<char*>(k_cache); g.v_cache = reinterpret_cast<char*>(v_cache);
    g.k_step = codes ? k_step : nullptr; g.v_step = codes ? v_step : nullptr;
    g.table = table; g.lens = lens; g.q_start = q_start; g.kept = kept; g.count = count; g.change = change; g.status = status;
    g.table_ld = table_ld; g.kept_ld = kept_ld; g.T = T;
    g.B = (int)B; g.Hk = (int)Hk; g.pages = (int)pages; g.page_size = (int)page_size; g.page_shift = __builtin_ctz((unsigned)page_size);
    g.chunk = codes ? 8 : 16;
    g.chunks = (int)(D / 8);
    const dim3 grid((unsigned)B, (unsigned)Hk, 2);
    if (codes) drafts::keep_kernel<drafts::u32x2><<<grid, kWave, 0, as_stream(stream)>>>(g);
    else drafts::keep_kernel<drafts::u32x4><<<grid, kWave, 0, as_stream(stream)>>>(g);
    return launch_status();
}
