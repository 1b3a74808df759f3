// wushkv_assign_pages and wushkv_compact_pages: which sequence holds which
// physical page of a shared pool.  Whole numbers and copies only; every page
// goes by a rank that a prefix sum gives, never by the order of atomics, so
// the result depends on the arguments alone.
//
// assign, up to three launches:
//   assign_rows_kernel   (a source map over more than a few entries) one thread
//                        per (sequence, logical page): drops the references of
//                        freed and forked rows, writes the forks' shared entries
//                        and counts them.
//   assign_pages_kernel  one workgroup: what every sequence needs, a prefix sum
//                        over the sequences, then the free pages in order from
//                        pool->low on, each to the sequence its rank falls to; the
//                        others copy the forks' windows.
//   assign_copy_kernel   (with a source map) the forks' pages being filled.
// compact, two launches, three for large pools:
//   compact_count_kernel (large pools) used pages per block of kBlock references.
//   compact_plan_kernel  ranks: free pages below n and used ones from n on.
//   compact_move_kernel  the pages, the boxes, references and table entries.
// What bounds them: small calls are launches (about 4 us each) and the one
// workgroup's dependent reads; large ones are copies, 64 sequences with 56 forks
// 16 us a call for 44 MB written (their sources are read from the caches), 1950
// moved pages of 36 KB with their boxes 28 us, 5.3 TB/s read and written.
#include "common.h"
#include "merge.h"

namespace wushkv {

constexpr int kMaxAssignBatch = 16384;  // the sequences' starts and bases stay in LDS
constexpr int kAssignThreads = 1024;
constexpr int kFewSequences = 1024;     // the same, in less LDS
// Table entries up to which the one workgroup goes through them itself (slots
// taken again, replayed from a graph): 248 entries 9.2 us a call, with a launch for
// them 10.1; 1024, 10.9 and 11.1; 1536, 13.3 and 11.4; 8064, 41.8 and 16.6.
constexpr int kOneAssign = 1024;

struct AssignArgs {
    uint8_t *pages;
    int32_t *page_table;
    uint16_t *win_k, *win_v;
    int32_t *seq_len, *quant_end;
    int32_t *refs, *held, *low;
    const int32_t *source, *reach;
    int32_t *status;
    int32_t batch, n_kv, s_sink, max_pages, n_pages;
    int64_t page_units, win_units;  // 16-byte units of a page (all heads) and of one window of a sequence
    int32_t row_blocks, win_blocks, copy_blocks;  // of a row, a window, a page
};

enum { kKeep = 0, kFree = 1, kFork = 2, kRefused = 3 };

// What source[b] asks for, and the sequence it names.
__device__ __forceinline__ int source_kind(const AssignArgs &a, int32_t b, int32_t &s)
{
    s = b;
    if (a.source == nullptr) return kKeep;
    const int32_t v = a.source[b];
    if (v == b) return kKeep;
    if (v == -1) return kFree;
    if (v < 0 || v >= a.batch || a.source[v] != v) return kRefused;
    s = v;
    return kFork;
}

// Quantised positions of sequence b (from s_sink on).
__device__ __forceinline__ int32_t quantised(const AssignArgs &a, int32_t b)
{
    const int32_t q = min(a.quant_end[b], a.seq_len[b]);
    return q > a.s_sink ? q - a.s_sink : 0;
}

__device__ __forceinline__ int32_t held_pages(const AssignArgs &a, int32_t b)
{
    return min(max(a.held[b], 0), a.max_pages);
}

// Entry lp of sequence b's row, if that is freed or forked.
__device__ __forceinline__ void assign_entry(const AssignArgs &a, int32_t b, int32_t lp)
{
    int32_t s;
    const int kind = source_kind(a, b, s);
    if (kind != kFree && kind != kFork) return;
    int32_t *row = a.page_table + (int64_t)b * a.max_pages;
    const int32_t old = row[lp];
    int32_t now = -1;
    // (the source is kept: nobody writes its row in this launch)
    if (kind == kFork && lp < min(quantised(a, s) / kPage, held_pages(a, s)))
        now = a.page_table[(int64_t)s * a.max_pages + lp];
    if (lp < held_pages(a, b) && old >= 0 && old < a.n_pages) {
        if (atomicSub(a.refs + old, 1) <= 1) atomicMin(a.low, old);
    }
    if (now >= 0 && now < a.n_pages) atomicAdd(a.refs + now, 1);
    row[lp] = now;
}

__global__ void __launch_bounds__(256) assign_rows_kernel(AssignArgs a)
{
    const int32_t lp = (blockIdx.x % a.row_blocks) * 256 + threadIdx.x;
    if (lp < a.max_pages) assign_entry(a, blockIdx.x / a.row_blocks, lp);
}

__device__ __forceinline__ int32_t load_agent(const int32_t *p)
{
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Exclusive prefix sum over the workgroup's threads, and the total.
__device__ __forceinline__ int32_t block_scan(int32_t x, int32_t *sums, int32_t &total)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = blockDim.x >> 6;
    const int32_t in = wave_scan(x);
    __syncthreads();  // the last call's sums are read
    if (lane == 63) sums[wave] = in;
    __syncthreads();
    int32_t before = 0, all = 0;
    for (int w = 0; w < waves; ++w) {
        const int32_t v = sums[w];
        if (w < wave) before += v;
        all += v;
    }
    total = all;
    return before + in - x;
}

// Up to 2 NT 16-byte units, by NT threads.  The stores are nontemporal: lines
// that nothing reads soon, kept, cost the caches twice the time (112 windows and
// 56 pages of 56 forks 29.3 us, so 14.6; 1950 moved pages 56.7, so 28.3), and two
// units a thread are the best of 1 to 16 (30.3, 28.3, 38.4, 46.6, 33.2).
template <int NT>
__device__ __forceinline__ void copy_units(const u32x4 *src, u32x4 *dst, int64_t n)
{
    u32x4 v[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (NT * i + threadIdx.x < n) v[i] = src[NT * i + threadIdx.x];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (NT * i + threadIdx.x < n) __builtin_nontemporal_store(v[i], dst + NT * i + threadIdx.x);
}
constexpr int kCopyUnits = 512;  // of 256 threads

// The first workgroup hands out pages; the others, if any, copy the forks'
// windows meanwhile (nothing that the first one writes is read for that).
// ROWS: the first one goes through the table's entries too, before anything else.
template <bool ROWS, int MAX_BATCH>
__global__ void __launch_bounds__(kAssignThreads) assign_pages_kernel(AssignArgs a)
{
    __shared__ int32_t start[MAX_BATCH + 1], base[MAX_BATCH];
    __shared__ int32_t sums[kAssignThreads / 64];
    const int tid = threadIdx.x;
    if (blockIdx.x > 0) {
        for (int64_t w = blockIdx.x - 1; w < (int64_t)a.batch * 2 * a.win_blocks; w += gridDim.x - 1) {
            const int32_t b = (int32_t)(w / (2 * a.win_blocks)), part = (int32_t)(w % (2 * a.win_blocks));
            int32_t s;
            if (source_kind(a, b, s) != kFork) continue;
            const int64_t at = (int64_t)(part % a.win_blocks) * 2 * kAssignThreads;
            uint16_t *win = part < a.win_blocks ? a.win_k : a.win_v;
            copy_units<kAssignThreads>(reinterpret_cast<const u32x4 *>(win) + s * a.win_units + at,
                                       reinterpret_cast<u32x4 *>(win) + b * a.win_units + at, a.win_units - at);
        }
        return;
    }
    if constexpr (ROWS) {
        for (int32_t i = tid; i < a.batch * a.max_pages; i += kAssignThreads) assign_entry(a, i / a.max_pages, i % a.max_pages);
        __syncthreads();  // (the references are read below, at the scope of their atomics)
    }
    // what each sequence needs: pages base .. base + need - 1 of its row
    int32_t total = 0;
    for (int32_t b0 = 0; b0 < a.batch; b0 += kAssignThreads) {
        const int32_t b = b0 + tid;
        int32_t need = 0;
        if (b < a.batch) {
            int32_t s;
            const int kind = source_kind(a, b, s);
            int32_t from = held_pages(a, b), part = 0;
            if (kind == kFree) from = 0;
            if (kind == kFork) {
                const int32_t q = quantised(a, s);
                from = min(q / kPage, held_pages(a, s));
                part = q % kPage != 0;
            }
            const int64_t span = a.reach != nullptr ? (int64_t)a.reach[b] - a.s_sink : 0;
            const int32_t target = span > 0 ? (int32_t)min((span + kPage - 1) / kPage, (int64_t)a.max_pages) : 0;
            need = min(max(part, target - from), a.max_pages - from);
            base[b] = from;
        }
        int32_t sum;
        const int32_t at = block_scan(need, sums, sum);
        if (b < a.batch) start[b] = total + at;
        total += sum;
    }
    if (tid == 0) start[a.batch] = total;
    // the free pages in order: the i-th goes to the sequence whose needs span i
    const int32_t first = total > 0 ? max(load_agent(a.low), 0) : 0;
    __syncthreads();  // (and the starts)
    int32_t found = 0;
    for (int64_t p0 = first & ~3; p0 < a.n_pages && found < total; p0 += 4 * kAssignThreads) {
        const int64_t p = p0 + 4 * tid;
        int4 r = make_int4(1, 1, 1, 1);
        if (ROWS) {
            if (p < a.n_pages) r.x = load_agent(a.refs + p);
            if (p + 1 < a.n_pages) r.y = load_agent(a.refs + p + 1);
            if (p + 2 < a.n_pages) r.z = load_agent(a.refs + p + 2);
            if (p + 3 < a.n_pages) r.w = load_agent(a.refs + p + 3);
        } else if (p + 3 < a.n_pages) {
            r = *reinterpret_cast<const int4 *>(a.refs + p);
        } else {
            if (p < a.n_pages) r.x = a.refs[p];
            if (p + 1 < a.n_pages) r.y = a.refs[p + 1];
            if (p + 2 < a.n_pages) r.z = a.refs[p + 2];
        }
        const int32_t v[4] = {r.x, r.y, r.z, r.w};
        int32_t n = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) n += v[e] <= 0;
        int32_t sum;
        int32_t i = found + block_scan(n, sums, sum);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (v[e] > 0) continue;
            if (i < total) {
                int32_t lo = 0, hi = a.batch;  // the last sequence with start <= i
                while (hi - lo > 1) {
                    const int32_t mid = (lo + hi) / 2;
                    if (start[mid] <= i) lo = mid;
                    else hi = mid;
                }
                a.page_table[(int64_t)lo * a.max_pages + base[lo] + (i - start[lo])] = (int32_t)p + e;
                a.refs[p + e] = 1;
                if (i == total - 1) a.low[0] = (int32_t)p + e + 1;
            }
            ++i;
        }
        found += sum;
    }
    if (tid == 0 && found < total) a.low[0] = a.n_pages;
    for (int32_t b = tid; b < a.batch; b += kAssignThreads) {
        int32_t s;
        const int kind = source_kind(a, b, s);
        const int32_t need = start[b + 1] - start[b];
        const int32_t got = min(max(found - start[b], 0), need);
        a.held[b] = base[b] + got;
        for (int32_t i = got; i < need; ++i) a.page_table[(int64_t)b * a.max_pages + base[b] + i] = -1;
        a.status[b] = kind == kRefused ? got - need - 1 : need - got;
        if (kind == kFree) a.seq_len[b] = a.quant_end[b] = 0;
        if (kind == kFork) {
            a.seq_len[b] = a.seq_len[s];
            a.quant_end[b] = a.quant_end[s];
        }
    }
}

__global__ void __launch_bounds__(256) assign_copy_kernel(AssignArgs a)
{
    const int32_t b = blockIdx.x / a.copy_blocks;
    int32_t s;
    if (source_kind(a, b, s) != kFork) return;
    const int64_t at = (int64_t)(blockIdx.x % a.copy_blocks) * kCopyUnits;
    const int32_t q = quantised(a, s), lp = q / kPage;
    // (neither row is read beyond what its sequence holds)
    if (q % kPage == 0 || lp >= a.max_pages || lp >= a.held[b] || lp >= a.held[s]) return;
    const int32_t from = a.page_table[(int64_t)s * a.max_pages + lp], to = a.page_table[(int64_t)b * a.max_pages + lp];
    if (from < 0 || from >= a.n_pages || to < 0 || to >= a.n_pages) return;
    u32x4 *pool = reinterpret_cast<u32x4 *>(a.pages);
    copy_units<256>(pool + from * a.page_units + at, pool + to * a.page_units + at, a.page_units - at);
}

// ------------------------------------------------------------------ compact

constexpr int kBlock = 4096;  // references per workgroup of the count and the plan
// Blocks up to which the plan counts them itself (a pool with nothing to move,
// replayed from a graph): 2 blocks 7.6 us a call, with a launch for them 8.8; 4, 8.8
// both; 6, 10.1 and 8.9; 8, 11.4 and 8.9.
constexpr int kOwnCount = 4;

struct CompactArgs {
    uint8_t *pages;
    int8_t *codes;      // null: no boxes
    float *scales;
    const int32_t *table, *held, *refs;
    int32_t *table_out, *refs_out, *live_out;
    int32_t batch, n_kv, head_dim, max_pages, n_pages;
    int64_t page_units, code_units;
    int32_t n_blocks, table_blocks;
    // workspace
    int32_t *head;      // n (pages in use), moves
    int32_t *counts;    // [n_blocks]
    int32_t *hole, *mover, *mover_refs;  // [n_pages / 2 + 1]
    int32_t *rank;      // [n_pages]: a mover's place in the lists
};

__device__ __forceinline__ int32_t block_sum(int32_t x, int32_t *sums)
{
    int32_t total;
    (void)block_scan(x, sums, total);
    return total;
}

// References p .. p + 3, 0 behind the last page.
__device__ __forceinline__ int4 four_refs(const CompactArgs &a, int64_t p)
{
    int4 r = make_int4(0, 0, 0, 0);
    if (p + 3 < a.n_pages) return *reinterpret_cast<const int4 *>(a.refs + p);
    if (p < a.n_pages) r.x = a.refs[p];
    if (p + 1 < a.n_pages) r.y = a.refs[p + 1];
    if (p + 2 < a.n_pages) r.z = a.refs[p + 2];
    return r;
}
__device__ __forceinline__ int32_t in_use(const int4 &r) { return (r.x > 0) + (r.y > 0) + (r.z > 0) + (r.w > 0); }

__global__ void __launch_bounds__(kBlock / 4) compact_count_kernel(CompactArgs a)
{
    __shared__ int32_t sums[kBlock / 256];
    const int32_t n = block_sum(in_use(four_refs(a, (int64_t)blockIdx.x * kBlock + 4 * threadIdx.x)), sums);
    if (threadIdx.x == 0) a.counts[blockIdx.x] = n;
}

// COUNTED: the blocks' counts are there; otherwise every workgroup counts the
// (few) blocks itself.  Workgroups start in any order, and each reads references
// of other blocks: in place, this launch therefore writes none of them.
template <bool COUNTED>
__global__ void __launch_bounds__(kBlock / 4) compact_plan_kernel(CompactArgs a)
{
    __shared__ int32_t sums[kBlock / 256];
    const int tid = threadIdx.x;
    const int32_t mine = blockIdx.x;
    // pages in use: in all, before this block, and below n
    int32_t all = 0, before = 0;
    if constexpr (COUNTED) {
        for (int32_t i = tid; i < a.n_blocks; i += kBlock / 4) {
            const int32_t v = a.counts[i];
            all += v;
            if (i < mine) before += v;
        }
    } else {
        for (int32_t i = 0; i < a.n_blocks; ++i) {
            const int32_t v = in_use(four_refs(a, (int64_t)i * kBlock + 4 * tid));
            all += v;
            if (i < mine) before += v;
        }
    }
    const int32_t live = block_sum(all, sums);
    before = block_sum(before, sums);
    int32_t below = 0;
    const int32_t whole = live / kBlock;
    if constexpr (COUNTED) {
        for (int32_t i = tid; i < whole; i += kBlock / 4) below += a.counts[i];
    }
    for (int64_t p = (COUNTED ? (int64_t)whole * kBlock : 0) + tid; p < live; p += kBlock / 4) below += a.refs[p] > 0;
    below = block_sum(below, sums);
    if (mine == 0 && tid == 0) {
        a.head[0] = live;
        a.head[1] = live - below;
        if (a.live_out != nullptr) a.live_out[0] = live;
    }
    const int64_t p0 = (int64_t)mine * kBlock + 4 * tid;
    const int4 r = four_refs(a, p0);
    int32_t sum;
    int32_t at = before + block_scan(in_use(r), sums, sum);  // pages in use before p
    const int32_t v[4] = {r.x, r.y, r.z, r.w};
    const bool in_place = a.refs_out == a.refs;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int64_t p = p0 + e;
        if (p >= a.n_pages) break;
        if (p < live) {
            if (v[e] <= 0) a.hole[p - at] = (int32_t)p;
            else if (!in_place) a.refs_out[p] = v[e];
        } else {
            if (v[e] > 0) {
                a.mover[at - below] = (int32_t)p;
                a.mover_refs[at - below] = v[e];
            }
            a.rank[p] = v[e] > 0 ? at - below : -1;
            if (!in_place) a.refs_out[p] = 0;
        }
        at += v[e] > 0;
    }
}

__global__ void __launch_bounds__(256) compact_move_kernel(CompactArgs a)
{
    const int tid = threadIdx.x;
    const int32_t live = a.head[0], moves = a.head[1];
    // (the plan wrote no reference; the moves write those below n only)
    if (a.refs_out == a.refs)
        for (int64_t p = (int64_t)live + blockIdx.x * 256 + tid; p < a.n_pages; p += (int64_t)gridDim.x * 256) a.refs_out[p] = 0;
    if ((int32_t)blockIdx.x < a.table_blocks) {
        const int64_t n = (int64_t)a.batch * a.max_pages;
        for (int64_t i = (int64_t)blockIdx.x * 256 + tid; i < n; i += (int64_t)a.table_blocks * 256) {
            const int32_t p = a.table[i];
            int32_t to = -1;
            if (i % a.max_pages < a.held[i / a.max_pages] && p >= 0 && p < a.n_pages)
                to = p >= live && a.rank[p] >= 0 ? a.hole[a.rank[p]] : p;
            a.table_out[i] = to;
        }
        return;
    }
    // the moves, in blocks of kCopyUnits; a block more of each for the rest
    const int32_t per = (int32_t)((a.page_units + kCopyUnits - 1) / kCopyUnits);
    const int32_t each = per + 1;
    const int64_t step = gridDim.x - a.table_blocks;
    for (int64_t w = blockIdx.x - a.table_blocks; w < (int64_t)moves * each; w += step) {
        const int32_t i = (int32_t)(w / each), part = (int32_t)(w % each);
        const int64_t from = a.mover[i], to = a.hole[i];
        if (part < per) {
            u32x4 *pool = reinterpret_cast<u32x4 *>(a.pages);
            const int64_t at = (int64_t)part * kCopyUnits;
            copy_units<256>(pool + from * a.page_units + at, pool + to * a.page_units + at, a.page_units - at);
            continue;
        }
        if (tid == 0) a.refs_out[to] = a.mover_refs[i];
        if (a.codes == nullptr) continue;
        u32x4 *codes = reinterpret_cast<u32x4 *>(a.codes);
        for (int64_t u = tid; u < a.code_units; u += 256) codes[to * a.code_units + u] = codes[from * a.code_units + u];
        for (int32_t h = tid; h < a.n_kv; h += 256) a.scales[(int64_t)h * a.n_pages + to] = a.scales[(int64_t)h * a.n_pages + from];
    }
}

}  // namespace wushkv

using namespace wushkv;

int wushkv_validate_cache(const wushkv_cache *c);  // api.hip

static bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }

static int check_pool(const wushkv_cache *c, const wushkv_pool *pool)
{
    const int st = wushkv_validate_cache(c);
    if (st != WUSHKV_OK) return st;
    if (!pool || !pool->refs || !pool->held || !pool->low) return WUSHKV_EINVAL;
    if (!aligned16(pool->refs) || !aligned16(pool->held) || !aligned16(pool->low)) return WUSHKV_EINVAL;
    return WUSHKV_OK;
}

extern "C" int wushkv_assign_pages(const wushkv_cache *c, const wushkv_pool *pool, const int32_t *source,
                                   const int32_t *reach, int32_t *status, wushkv_stream_t stream)
{
    int st = check_pool(c, pool);
    if (st != WUSHKV_OK) return st;
    if (!status || !aligned16(status) || !aligned16(source) || !aligned16(reach)) return WUSHKV_EINVAL;
    if (c->batch > kMaxAssignBatch || (int64_t)c->batch * c->max_pages_per_seq > 0x7FFFFFFF) return WUSHKV_EUNSUPPORTED;
    AssignArgs a{};
    a.pages = c->pages;
    a.page_table = c->page_table;
    a.win_k = c->win_k;
    a.win_v = c->win_v;
    a.seq_len = c->seq_len;
    a.quant_end = c->quant_end;
    a.refs = pool->refs;
    a.held = pool->held;
    a.low = pool->low;
    a.source = source;
    a.reach = reach;
    a.status = status;
    a.batch = c->batch;
    a.n_kv = c->n_kv_heads;
    a.s_sink = c->s_sink;
    // (without pages there is no table either)
    const bool paged = c->n_pages > 0 && c->max_pages_per_seq > 0;
    a.max_pages = paged ? c->max_pages_per_seq : 0;
    a.n_pages = paged ? c->n_pages : 0;
    a.page_units = (int64_t)c->n_kv_heads * (int64_t)(wushkv_page_bytes(c->head_dim, c->bits) / 16);
    a.win_units = (int64_t)c->n_kv_heads * c->win_slots * c->head_dim / 8;
    const int64_t row_blocks = (a.max_pages + 255) / 256;
    const int64_t win_blocks = (a.win_units + 2 * kAssignThreads - 1) / (2 * kAssignThreads);
    const int64_t copy_blocks = paged ? (a.page_units + kCopyUnits - 1) / kCopyUnits : 0;
    if (win_blocks > 0x3FFFFFFF || copy_blocks * c->batch > 0x7FFFFFFF) return WUSHKV_EUNSUPPORTED;
    a.row_blocks = (int32_t)row_blocks;
    a.win_blocks = (int32_t)win_blocks;
    a.copy_blocks = (int32_t)copy_blocks;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const bool few = c->batch <= kFewSequences;
    const int64_t entries = (int64_t)c->batch * a.max_pages, copies = 2 * win_blocks * c->batch;
    const bool rows = source != nullptr && entries <= kOneAssign;
    const dim3 grid(source == nullptr ? 1u : 1u + (unsigned)(copies < 2048 ? copies : 2048)), threads(kAssignThreads);
    if (source != nullptr && !rows)
        launch("assign_rows_kernel", assign_rows_kernel, dim3((unsigned)(row_blocks * c->batch)), dim3(256), s, a);
    if (rows && few) launch("assign_pages_kernel", assign_pages_kernel<true, kFewSequences>, grid, threads, s, a);
    else if (rows) launch("assign_pages_kernel", assign_pages_kernel<true, kMaxAssignBatch>, grid, threads, s, a);
    else if (few) launch("assign_pages_kernel", assign_pages_kernel<false, kFewSequences>, grid, threads, s, a);
    else launch("assign_pages_kernel", assign_pages_kernel<false, kMaxAssignBatch>, grid, threads, s, a);
    if (source != nullptr && copy_blocks > 0)
        launch("assign_copy_kernel", assign_copy_kernel, dim3((unsigned)(copy_blocks * c->batch)), dim3(256), s, a);
    if (hipGetLastError() != hipSuccess) return WUSHKV_ELAUNCH;
    return WUSHKV_OK;
}

static size_t compact_blocks(const wushkv_cache *c)
{
    return ((size_t)c->n_pages + kBlock - 1) / kBlock;
}

extern "C" size_t wushkv_compact_workspace_bytes(const wushkv_cache *c)
{
    if (wushkv_validate_cache(c) != WUSHKV_OK || c->n_pages == 0 || c->max_pages_per_seq == 0) return 0;
    const size_t n = (size_t)c->n_pages, half = n / 2 + 1;
    return (4 + compact_blocks(c) + 3 * half + n) * sizeof(int32_t);
}

extern "C" int wushkv_compact_pages(const wushkv_cache *c, const wushkv_pool *pool, const wushkv_bounds *bounds,
                                    int32_t *table_out, int32_t *refs_out, int32_t *live_out, void *workspace,
                                    size_t workspace_bytes, wushkv_stream_t stream)
{
    int st = check_pool(c, pool);
    if (st != WUSHKV_OK) return st;
    if (c->n_pages == 0 || c->max_pages_per_seq == 0) return WUSHKV_EINVAL;  // no pages
    if (!table_out || !refs_out || !workspace) return WUSHKV_EINVAL;
    if (!aligned16(table_out) || !aligned16(refs_out) || !aligned16(live_out) || !aligned16(workspace)) return WUSHKV_EINVAL;
    if (bounds && (!bounds->codes || !bounds->scales || !aligned16(bounds->codes) || !aligned16(bounds->scales)))
        return WUSHKV_EINVAL;
    if (workspace_bytes < wushkv_compact_workspace_bytes(c)) return WUSHKV_EWORKSPACE;
    CompactArgs a{};
    a.pages = c->pages;
    if (bounds) {
        a.codes = bounds->codes;
        a.scales = bounds->scales;
    }
    a.table = c->page_table;
    a.held = pool->held;
    a.refs = pool->refs;
    a.table_out = table_out;
    a.refs_out = refs_out;
    a.live_out = live_out;
    a.batch = c->batch;
    a.n_kv = c->n_kv_heads;
    a.head_dim = c->head_dim;
    a.max_pages = c->max_pages_per_seq;
    a.n_pages = c->n_pages;
    a.page_units = (int64_t)c->n_kv_heads * (int64_t)(wushkv_page_bytes(c->head_dim, c->bits) / 16);
    a.code_units = (int64_t)c->n_kv_heads * 2 * c->head_dim / 16;
    a.n_blocks = (int32_t)compact_blocks(c);
    a.head = reinterpret_cast<int32_t *>(workspace);
    a.counts = a.head + 4;
    a.hole = a.counts + a.n_blocks;
    a.mover = a.hole + c->n_pages / 2 + 1;
    a.mover_refs = a.mover + c->n_pages / 2 + 1;
    a.rank = a.mover_refs + c->n_pages / 2 + 1;
    const int64_t entries = (int64_t)a.batch * a.max_pages;
    a.table_blocks = (int32_t)((entries + 255) / 256 < 256 ? (entries + 255) / 256 : 256);
    // at most half of the pages move
    const int64_t each = (a.page_units + kCopyUnits - 1) / kCopyUnits + 1;
    const int64_t copies = (int64_t)(a.n_pages / 2) * each;
    const unsigned move_blocks = (unsigned)(a.table_blocks + (copies < 2048 ? copies : 2048));
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const dim3 blocks((unsigned)a.n_blocks), threads(kBlock / 4);
    if (a.n_blocks <= kOwnCount) {
        launch("compact_plan_kernel", compact_plan_kernel<false>, blocks, threads, s, a);
    } else {
        launch("compact_count_kernel", compact_count_kernel, blocks, threads, s, a);
        launch("compact_plan_kernel", compact_plan_kernel<true>, blocks, threads, s, a);
    }
    launch("compact_move_kernel", compact_move_kernel, dim3(move_blocks), dim3(256), s, a);
    if (hipGetLastError() != hipSuccess) return WUSHKV_ELAUNCH;
    return WUSHKV_OK;
}
