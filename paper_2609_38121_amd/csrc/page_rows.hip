// wushkv_shared_prefixes and wushkv_evict_pages: what the rows of the page table
// have in common, and the pages that leave them.  Whole numbers; the results depend
// on the arguments alone.
//
// shared_prefixes: one workgroup per sequence goes over the others whose first entry
// is its own, a wave each, 256 entries at a time.
//
// evict: one workgroup per sequence.  The scores (a page's weights over the kv heads,
// summed in fp64) become 32-bit keys in the order of their values; four rounds of
// 256-bin histograms find the key of the last page to leave, prefix sums over the
// pages settle the ties and write the list.  Where the references go to another
// array, a launch before it copies them.
//
// Both are a launch and chains of dependent reads: 64 sequences that share 8-32K tokens
// with 15 others 6.4 us, of 8 forks 3.6; eviction from 64 sequences of 16-32K tokens, 8 kv
// heads, 14.3 us (1 MB of weights; a workgroup of 1024 a sequence, so that a row's keys stay
// in LDS and no launch lies between its rounds) and the copy 1.9.
#include "common.h"
#include "merge.h"

namespace wushkv {

struct PageRows {
    const int32_t *page_table, *seq_len, *quant_end;
    int32_t batch, n_kv, s_sink, max_pages, n_pages;
};

// Quantised positions of sequence b behind the sink.
__device__ __forceinline__ int32_t quantised(const PageRows &a, int32_t b)
{
    return max(min(a.quant_end[b], a.seq_len[b]) - a.s_sink, 0);
}

// ------------------------------------------------------------------ prefixes

constexpr int kPrefixThreads = 1024;

__global__ void __launch_bounds__(kPrefixThreads) shared_prefixes_kernel(PageRows a, int32_t min_pages, int32_t *leader,
                                                                         int32_t *shared)
{
    constexpr int kWaves = kPrefixThreads / 64, kAhead = 4;
    __shared__ int32_t s_best[kWaves], s_who[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int32_t b = blockIdx.x;
    const int32_t *row = a.page_table + (int64_t)b * a.max_pages;
    const int32_t full = min(quantised(a, b) / kPage, a.max_pages);
    const int32_t first = full > 0 ? row[0] : -1;
    int32_t best = 0, who = b;
    // sequences base + 16 lane + wave, so that a small batch falls to all the waves
    for (int32_t base = 0; base < a.batch && full > 0; base += kPrefixThreads) {
        const int32_t c = base + kWaves * lane + wave;
        int32_t most = 0;
        if (c < a.batch && c != b && a.page_table[(int64_t)c * a.max_pages] == first)
            most = min(full, min(quantised(a, c) / kPage, a.max_pages));
        for (uint64_t todo = __ballot(most > 0); todo != 0; todo &= todo - 1) {
            const int i = __builtin_ctzll(todo);
            const int32_t lim = __builtin_amdgcn_readlane(most, i), other = __builtin_amdgcn_readlane(c, i);
            const int32_t *theirs = a.page_table + (int64_t)other * a.max_pages;
            int32_t common = 0;
            bool same = true;
            for (int32_t p0 = 0; same && p0 < lim; p0 += 64 * kAhead) {
                int32_t x[kAhead], y[kAhead];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    const int32_t p = min(p0 + 64 * k + lane, lim - 1);
                    x[k] = row[p];
                    y[k] = theirs[p];
                }
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    const uint64_t eq = __ballot(p0 + 64 * k + lane < lim && x[k] == y[k]);
                    uint64_t held = __ballot(x[k] >= 0 && x[k] < a.n_pages);
                    const int n = ~eq != 0 ? __builtin_ctzll(~eq) : 64;
                    held &= n < 64 ? (1ull << n) - 1 : ~0ull;
                    if (same && held != 0) common = p0 + 64 * k + 64 - __builtin_clzll(held);
                    same &= n == 64;
                }
            }
            if (common > best || (common == best && common > 0 && other < who)) {
                best = common;
                who = other;
            }
        }
    }
    if (lane == 0) {
        s_best[wave] = best;
        s_who[wave] = who;
    }
    __syncthreads();
    if (tid != 0) return;
    for (int w = 0; w < kWaves; ++w) best = max(best, s_best[w]);
    who = b;
    for (int w = 0; w < kWaves; ++w)
        if (s_best[w] == best) who = min(who, s_who[w]);
    const bool with = best >= min_pages && who != b;
    leader[b] = with ? who : b;
    shared[b] = with ? best : 0;
}

// ------------------------------------------------------------------ eviction

constexpr int kEvictThreads = 1024;
// Pages whose keys stay in LDS; those of longer rows are formed again each round.
constexpr int kEvictKeys = 8192;

struct EvictArgs {
    PageRows r;
    int32_t *refs_out;
    const int32_t *held;
    int32_t *low;
    const float *weights;   // [batch][n_kv][max_pages]
    const int32_t *budget;  // [batch]
    int32_t recent, max_sel;
    int32_t *table_out, *sel, *n_sel, *evicted;
};

__global__ void __launch_bounds__(256) evict_refs_kernel(const int32_t *refs, int32_t *refs_out, int32_t n)
{
    const int32_t i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) refs_out[i] = refs[i];
}

// Exclusive prefix sum over the workgroup's threads, and the total.
__device__ __forceinline__ int32_t evict_scan(int32_t x, int32_t *sums, int32_t &total)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int32_t in = wave_scan(x);
    __syncthreads();  // the last call's sums are read
    if (lane == 63) sums[wave] = in;
    __syncthreads();
    int32_t before = 0, all = 0;
    for (int w = 0; w < kEvictThreads / 64; ++w) {
        const int32_t v = sums[w];
        if (w < wave) before += v;
        all += v;
    }
    total = all;
    return before + in - x;
}

__global__ void __launch_bounds__(kEvictThreads) evict_kernel(EvictArgs a)
{
    __shared__ uint32_t keys[kEvictKeys];
    __shared__ int32_t bins[256], sums[kEvictThreads / 64], s_digit, s_left;
    const int tid = threadIdx.x;
    const int32_t b = blockIdx.x, mp = a.r.max_pages, hk = a.r.n_kv;
    const int32_t *row = a.r.page_table + (int64_t)b * mp;
    const int32_t q = quantised(a.r, b), full = q / kPage;
    const int32_t held = min(max(a.held[b], 0), mp);
    const int32_t n = min(full, held);                    // complete pages there may be
    const int32_t open = full - max(a.recent, 0);         // candidates lie below
    const int32_t budget = a.budget[b];
    auto lives = [&](int32_t p) -> bool { return p >= 0 && p < a.r.n_pages; };
    // a page's weight as a key in the order of the values (equal weights, equal
    // keys; no number counts as the largest)
    auto key_of = [&](int32_t i) -> uint32_t {
        double w = 0.0;
        for (int32_t h = 0; h < hk; ++h) w += (double)a.weights[((int64_t)b * hk + h) * mp + i];
        const float f = (float)w + 0.0f;
        const uint32_t u = __float_as_uint(f);
        return f != f ? 0xFFFFFFFFu : (u & 0x80000000u) ? ~u : u | 0x80000000u;
    };
    int32_t live = 0, free_ = 0;
    for (int32_t i = tid; i < n; i += kEvictThreads) {
        const bool here = lives(row[i]);
        live += here;
        free_ += here && i < open;
    }
    int32_t all_live, all_free;
    evict_scan(live, sums, all_live);
    evict_scan(free_, sums, all_free);
    const int32_t over = budget < 0 ? 0 : min(max(all_live - budget, 0), all_free);
    uint32_t last = 0u;   // the key of the last page to leave,
    int32_t ties = 0;     // and how many of that key leave
    const bool kept = n <= kEvictKeys;
    if (over > 0) {
        if (kept)
            for (int32_t i = tid; i < n; i += kEvictThreads) keys[i] = key_of(i);
        ties = over;
        for (int shift = 24; shift >= 0; shift -= 8) {
            __syncthreads();
            if (tid < 256) bins[tid] = 0;
            __syncthreads();
            for (int32_t i = tid; i < n; i += kEvictThreads) {
                if (i >= open || !lives(row[i])) continue;
                const uint32_t k = kept ? keys[i] : key_of(i);
                if (shift == 24 || (k >> (shift + 8)) == (last >> (shift + 8))) atomicAdd(&bins[(k >> shift) & 255u], 1);
            }
            __syncthreads();
            int32_t total;
            const int32_t mine = tid < 256 ? bins[tid] : 0;
            const int32_t before = evict_scan(mine, sums, total);
            if (tid < 256 && before < ties && ties <= before + mine) {
                s_digit = tid;
                s_left = ties - before;
            }
            __syncthreads();
            last |= (uint32_t)s_digit << shift;
            ties = s_left;
        }
    }
    // in the order of the pages: ties, the list, the table and the references
    int32_t ties_before = 0, kept_before = 0;
    const int32_t every = min((q + kPage - 1) / kPage, held);
    // (pages left, so that a list that is too short begins later)
    int32_t left = all_live - over;
    if (every > full && lives(row[full])) left += 1;
    const int32_t skip = max(left - a.max_sel, 0);  // (all of them where the list has no entries)
    for (int32_t i0 = 0; i0 < mp; i0 += kEvictThreads) {
        const int32_t i = i0 + tid;
        const int32_t phys = i < mp ? row[i] : -1;
        const bool here = i < every && lives(phys);
        bool gone = false;
        if (over > 0 && i0 < n) {
            const bool could = here && i < n && i < open;
            const uint32_t k = could ? (kept ? keys[i] : key_of(i)) : 0u;
            int32_t total;
            const int32_t rank = ties_before + evict_scan(could && k == last, sums, total);
            ties_before += total;
            gone = could && (k < last || (k == last && rank < ties));
        }
        if (i < mp && (gone || a.table_out != a.r.page_table)) a.table_out[(int64_t)b * mp + i] = gone ? -1 : phys;
        if (gone && atomicSub(a.refs_out + phys, 1) <= 1) atomicMin(a.low, phys);
        if (a.n_sel != nullptr && i0 < every) {
            const bool stays = here && !gone;
            int32_t total;
            const int32_t at = kept_before + evict_scan(stays, sums, total) - skip;
            kept_before += total;
            if (stays && at >= 0)
                for (int32_t h = 0; h < hk; ++h) a.sel[((int64_t)b * hk + h) * a.max_sel + at] = i;
        }
    }
    const int32_t listed = min(left, a.max_sel);
    if (a.n_sel != nullptr) {
        const int32_t behind = a.max_sel - listed;
        for (int64_t x = tid; x < (int64_t)behind * hk; x += kEvictThreads)
            a.sel[((int64_t)b * hk + x / behind) * a.max_sel + listed + x % behind] = -1;
        for (int32_t h = tid; h < hk; h += kEvictThreads) a.n_sel[(int64_t)b * hk + h] = listed;
    }
    if (tid == 0) a.evicted[b] = over;
}

}  // namespace wushkv

using namespace wushkv;

int wushkv_validate_cache(const wushkv_cache *c);

static PageRows rows_of(const wushkv_cache *c)
{
    // (a pool of no pages needs no table; one that is there is copied all the same)
    return PageRows{c->page_table, c->seq_len, c->quant_end, c->batch, c->n_kv_heads, c->s_sink,
                    c->page_table != nullptr ? c->max_pages_per_seq : 0, c->n_pages};
}

extern "C" int wushkv_shared_prefixes(const wushkv_cache *c, int32_t min_pages, int32_t *leader, int32_t *shared,
                                      wushkv_stream_t stream)
{
    const int st = wushkv_validate_cache(c);
    if (st != WUSHKV_OK) return st;
    if (min_pages < 1 || !leader || !shared || ((uintptr_t)leader | (uintptr_t)shared) & 15u) return WUSHKV_EINVAL;
    launch("shared_prefixes_kernel", shared_prefixes_kernel, dim3(c->batch), dim3(kPrefixThreads),
           reinterpret_cast<hipStream_t>(stream), rows_of(c), min_pages, leader, shared);
    return hipGetLastError() != hipSuccess ? WUSHKV_ELAUNCH : WUSHKV_OK;
}

extern "C" int wushkv_evict_pages(const wushkv_cache *c, const wushkv_pool *pool, const float *weights,
                                  const int32_t *budget, int32_t recent, int32_t *table_out, int32_t *refs_out,
                                  int32_t *sel, int32_t *n_sel, int32_t max_sel, int32_t *evicted, wushkv_stream_t stream)
{
    const int st = wushkv_validate_cache(c);
    if (st != WUSHKV_OK) return st;
    if (!pool || !pool->refs || !pool->held || !pool->low || !weights || !budget || !table_out || !refs_out || !evicted ||
        recent < 0 || max_sel < 0 || (sel != nullptr && !n_sel) || (!sel && n_sel && max_sel > 0))
        return WUSHKV_EINVAL;
    if (((uintptr_t)pool->refs | (uintptr_t)pool->held | (uintptr_t)pool->low | (uintptr_t)weights | (uintptr_t)budget |
         (uintptr_t)table_out | (uintptr_t)refs_out | (uintptr_t)sel | (uintptr_t)n_sel | (uintptr_t)evicted) & 15u)
        return WUSHKV_EINVAL;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (refs_out != pool->refs && c->n_pages > 0)
        launch("evict_refs_kernel", evict_refs_kernel, dim3((unsigned)(((int64_t)c->n_pages + 255) / 256)), dim3(256), s,
               (const int32_t *)pool->refs, refs_out, c->n_pages);
    const EvictArgs a{rows_of(c), refs_out, pool->held, pool->low, weights, budget, recent, max_sel, table_out, sel, n_sel, evicted};
    launch("evict_kernel", evict_kernel, dim3(c->batch), dim3(kEvictThreads), s, a);
    return hipGetLastError() != hipSuccess ? WUSHKV_ELAUNCH : WUSHKV_OK;
}
