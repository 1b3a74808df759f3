// Attention of many query rows over stored sequences, where several queries have
// a sequence, or its first pages, in common:
//   wushkv_prefix_attention    decode queries; pages shared at the start of several
//                              sequences are attended to once for all of them
//   wushkv_cross_attention     query sequences of any length over whole stored ones
//   wushkv_weighted_attention  decode queries, adding up what each page received
//
// Launches on the caller's stream:
//   rows_query_kernel  q~ = q T_K^{-1} of 16 rows at a time (fp32, for the windows)
//                      and its digit limbs (for the pages); and, in a workgroup per
//                      kv head, the plan: tiles and how they are shared out (below).
//   rows_kernel        one residency round of workgroups over the plan.
//   rows_merge_kernel / rows_join_kernel   what several workgroups have of a row,
//                      merged; the pages' weights.
//
// Plan.  A tile is up to 16 query rows ((token, query head) pairs) with a run of a
// stored sequence's pages and, where it is the rows' own sequence, its windows.
// Prefix: a tile of its own pages and windows per sequence, and tiles of the
// sequences that have a leader (sorted by what they share with it, longest first,
// so that a tile's rows end at about the same page).  Cross: the tokens of all query
// sequences of one stored sequence, 16 rows at a time.  Small tiles are dealt out
// evenly, whole; the costs of the others stand one behind the other on a line, of
// which every workgroup takes what it has room for beside its small ones: a part of
// one tile or several tiles.  No length is known to the host.  Within a workgroup the
// four waves take every fourth page each and merge in LDS at the tile's end.
//
// Pages.  As in decode_main_kernel, scores are scaled products of q~'s digit limbs
// with the key codes, here with 16 query rows as the product's rows, one product a
// limb; keys are centred (k = s (c - mid) + (z + mid s)).  A wave reads a page's
// codes and parameters from memory in operand order into registers, the next page's
// while it computes.  Lane (j, n) has rows 4 j + r of tokens 4 n + t.  A row's
// softmax has a reference, a whole number, at its maximum of the time, that moves only
// when a weight would pass 2^kGrow, so that a page costs one test.  Weights
// p s go through LDS as fp16 hi + lo parts, each formed from the exact product, to
// be the rows of the P V products with the value codes as fp16 numbers 16 (c - middle),
// middle that of the codes' own bits.  The value scales are brought to about one by a power
// of two that the wave keeps (tiny scales would leave the lo parts no bits); sums of
// p (z + middle s) and p are fp32.
//
// Windows.  q~ and weights in three bf16 parts, 64 slots at a time.
//
// What bounds it.  A page of 16 rows is about 415 vector instructions (144 of them the
// widening of its 8192 value codes), 24 scaled products and 32 fp16 ones, all issued from
// one port; two workgroups a compute unit keep the vector units 59 to 74% busy.  64
// sequences on 32768 tokens (d 128, 2-bit, 8 kv heads, G 4): rows_kernel 103 us for 65536
// page passes, 64 a SIMD; 8 sequences of 256 tokens over 1000 to 3000: 197 us; 64
// sequences weighted, 64 pages of each: 60 us, 3.4 TB/s (in traces of eight calls).  Tiles
// of 32 rows would halve the widening, but at two workgroups a compute unit their registers
// spill (116 us in the first case), and three workgroups spill with 16 rows.
#include <algorithm>
#include <atomic>

#include "query.h"

namespace wushkv {

constexpr int kMaxRowItems = 1024;  // sequences that a plan sorts
constexpr int kMaxWgs = 1024;       // workgroups of rows_kernel per kv head
constexpr int kTileLog2 = 4, kTileRows = 1 << kTileLog2;
constexpr int kReps = 2;        // most 16-row groups that a workgroup of rows_query_kernel takes
constexpr int kRowsPerCu = 2;  // workgroups of rows_kernel that a compute unit keeps

// Tiles of one stored sequence's pages for up to 16 query rows.
struct RowTile {
    int32_t seq;             // whose page table, list and windows
    int32_t first, n_pages;  // page units: logical pages (or list entries) first ..
    int32_t n_win;           // then 64-slot window units
    int32_t rows;            // query rows
    int32_t tok;             // its first entry in the token list
    int32_t limit;           // below it every row attends to a page
    int32_t part;            // its first partial row, -1: written out directly
    int32_t wg0, n_wg;       // workgroups that have a part of it
    int64_t cost0;           // its place on the line, -1: a small one
};

// Per kv head, at the start of its plan.
struct RowPlan {
    int64_t total;  // the line's length
    int32_t n_tiles, n_small;
};

enum { kPrefix = 0, kCross = 1, kWeighted = 2 };

struct RowsArgs {
    const uint8_t *pages;
    const int32_t *page_table;
    const uint16_t *win_k, *win_v;
    const int32_t *seq_len, *quant_end;
    int32_t batch, n_kv, s_sink, win_slots, max_pages, n_pages;
    int32_t mode, g_log2;         // query heads per kv head, G = 1 << g_log2
    int32_t items, max_tok;       // query sequences, and their token rows
    const uint16_t *q;            // bf16 [items][max_tok][n_kv G][D]
    const float *tinv;
    float scale, mid;             // sm_scale log2(e); the middle of the key codes
    float *out;                   // fp32 of q's shape
    const int32_t *of;            // prefix: leader; cross: source (or null)
    const int32_t *count;         // prefix: shared; cross: n_tok (or null)
    const int32_t *sel, *n_sel;   // weighted: lists, or null
    int32_t max_sel;              // entries of a list, or max_pages
    float *weights;               // weighted: [batch][n_kv][max_pages]
    // workspace
    uint8_t *qlimb;               // [n_kv][tokens][G][6][128]
    uint32_t *qaux;               // [n_kv][tokens][G][4]
    float *qt;                    // [n_kv][tokens][G][D]: q~
    uint8_t *plan;                // per kv head plan_bytes
    int64_t plan_bytes;
    // offsets in a plan: int64 [wgs + 1], where the workgroups' parts of the line begin;
    // int32 [wgs], the tile there; the tiles; int32 [tiles], the small ones in order, and
    // the costs before them; the token list and the tokens' limits; (tile, place) of each
    // sequence with a leader
    int32_t bound_at, wg_at, tile_at, small_at, before_at, tok_at, lim_at, map_at;
    int32_t wgs;                  // workgroups of rows_kernel per kv head
    uint64_t inverse;             // 2^64 / wgs, rounded up (at most 2^64 - 1)
    int32_t cus;                  // compute units
    int32_t reps;                 // 16-row groups a workgroup of rows_query_kernel takes
    float *part;                  // [n_kv][part_rows][D]
    float *part_ml;               // [n_kv][part_rows][2]
    int64_t part_rows;
    float *stat;                  // weighted: [n_kv][batch][max_sel][G][2]
};

__device__ __forceinline__ RowPlan *plan_of(const RowsArgs &a, int h)
{
    return reinterpret_cast<RowPlan *>(a.plan + h * a.plan_bytes);
}
template <typename T>
__device__ __forceinline__ T *plan_part(const RowsArgs &a, int h, int32_t at)
{
    return reinterpret_cast<T *>(a.plan + h * a.plan_bytes + at);
}

// End of sequence b's quantised positions.
__device__ __forceinline__ int32_t quantised_end(const RowsArgs &a, int32_t b)
{
    return max(min(a.quant_end[b], a.seq_len[b]), a.s_sink);
}

// Costs of a page, of a window unit and of a tile before its first unit (powers of two
// and shifts: the plan and a tile's start run once, and are as long as their code, which
// is seldom in the caches).
constexpr int kPageShift = 2, kWindowShift = 4;
constexpr int32_t kTileCost = 36;
constexpr int64_t kLeastShare = 32;
__device__ __forceinline__ int64_t tile_cost(const RowTile &t)
{
    if (t.n_pages + t.n_win == 0) return 0;
    return kTileCost + ((int64_t)t.n_pages << kPageShift) + ((int64_t)t.n_win << kWindowShift);
}
// Tiles that are not cut.
__device__ __forceinline__ bool is_small(const RowTile &t) { return t.n_pages + 2 * t.n_win <= 16; }

// The unit that begins at or after place x of a tile's cost.
__device__ __forceinline__ int32_t unit_at(const RowTile &t, int64_t x)
{
    x -= kTileCost;
    if (x <= 0) return 0;
    const int64_t pages = (int64_t)t.n_pages << kPageShift;
    if (x <= pages) return (int32_t)((x + (1 << kPageShift) - 1) >> kPageShift);
    const int64_t w = (x - pages + (1 << kWindowShift) - 1) >> kWindowShift;
    return t.n_pages + (int32_t)(w < t.n_win ? w : t.n_win);
}

// Exclusive prefix sums over the workgroup's threads, and the totals.
struct Pair {
    int64_t a, b;
};
__device__ __forceinline__ Pair block_scan(Pair x, Pair *sums, Pair &total)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = blockDim.x >> 6;
    Pair in = x;
#pragma unroll 1
    for (int s = 1; s < 64; s <<= 1) {
        const int64_t ya = __shfl_up(in.a, s), yb = __shfl_up(in.b, s);
        if (lane >= s) in = Pair{in.a + ya, in.b + yb};
    }
    __syncthreads();  // the last call's sums are read
    if (lane == 63) sums[wave] = in;
    __syncthreads();
    Pair before{0, 0}, all{0, 0};
#pragma unroll 1
    for (int w = 0; w < waves; ++w) {
        const Pair v = sums[w];
        if (w < wave) before = Pair{before.a + v.a, before.b + v.b};
        all = Pair{all.a + v.a, all.b + v.b};
    }
    total = all;
    return Pair{before.a + in.a - x.a, before.b + in.b - x.b};
}
__device__ __forceinline__ int64_t block_scan(int64_t x, Pair *sums, int64_t &total)
{
    Pair all;
    const int64_t before = block_scan(Pair{x, 0}, sums, all).a;
    total = all.a;
    return before;
}

struct PlanLds {
    int2 item[kMaxRowItems];  // leader or stored sequence (-1: none); pages shared or tokens
    int32_t most[kMaxRowItems], order[kMaxRowItems], flag[kMaxRowItems], at[kMaxRowItems], sum[kMaxRowItems], count;
    Pair sums[8];
    int64_t bound[kMaxWgs + 1];
};

// The first of n small tiles that workgroup w takes: w n / wgs, rounded up to a place
// near it.
__device__ __forceinline__ int32_t small_of(const RowsArgs &a, int32_t w, int32_t n)
{
    // (w <= 1024, n <= 2^17; inverse is 2^64 / wgs rounded up: exactly n for the last)
    const int32_t at = (int32_t)__umul64hi((uint64_t)((uint32_t)w * (uint32_t)n), a.inverse);
    return at < n && w < a.wgs ? at : n;
}

// The first w in [0, n) with bound[w] >= x (strict: > x), n if there is none.
__device__ __forceinline__ int32_t bound_of(const int64_t *bound, int32_t n, int64_t x, bool strict)
{
    int32_t lo = 0, hi = n;
    while (lo < hi) {
        const int32_t mid = (lo + hi) / 2;
        if (strict ? bound[mid] > x : bound[mid] >= x) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// The tiles' places on the line of costs, the workgroups' parts of it and the partial
// rows; all threads, after the tiles are written.
__device__ __forceinline__ void share_out(const RowsArgs &a, int h, int32_t n_tiles, PlanLds &lds)
{
    const int tid = threadIdx.x, nt = blockDim.x;
    RowTile *tiles = plan_part<RowTile>(a, h, a.tile_at);
    int32_t *wg_tile = plan_part<int32_t>(a, h, a.wg_at);
    int32_t *small = plan_part<int32_t>(a, h, a.small_at), *before = plan_part<int32_t>(a, h, a.before_at);
    const int32_t P = a.wgs;
    __syncthreads();
    RowTile mine{};  // the first of the thread's tiles (mostly its only one) stays in registers
    if (tid < n_tiles) mine = tiles[tid];
    auto tile_at = [&](int32_t t) -> RowTile { return t == tid ? mine : tiles[t]; };
    int64_t line = 0, smalls = 0;  // smalls: costs above, their number in the lower 17 bits
    for (int32_t t0 = 0; t0 < n_tiles; t0 += nt) {
        const int32_t t = t0 + tid;
        int64_t cost = 0;
        bool few = false;
        if (t < n_tiles) {
            const RowTile x = tile_at(t);
            cost = tile_cost(x);
            few = is_small(x) && cost > 0;
        }
        Pair all;
        const Pair at = block_scan(Pair{few ? 0 : cost, few ? (cost << 17) + 1 : 0}, lds.sums, all);
        const int64_t cost0 = few ? -1 : line + at.a;
        if (t < n_tiles) tiles[t].cost0 = cost0;
        if (t == tid) mine.cost0 = cost0;
        if (few) {
            const int64_t s = smalls + at.b;
            small[s & 0x1FFFF] = t;
            before[s & 0x1FFFF] = (int32_t)(s >> 17);
        }
        line += all.a;
        smalls += all.b;
    }
    const int32_t n_small = (int32_t)(smalls & 0x1FFFF);
    const int64_t cost_small = smalls >> 17;
    int64_t most = (int64_t)__umul64hi((uint64_t)(line + cost_small), a.inverse) + 1;
    most = most > kLeastShare ? most : kLeastShare;
    __syncthreads();  // (before is written)
    auto first_small = [&](int32_t w) -> int32_t { return small_of(a, w, n_small); };
    auto cost_before = [&](int32_t i) -> int64_t { return i < n_small ? before[i] : cost_small; };
    int64_t given = 0;
    for (int32_t w0 = 0; w0 < P; w0 += nt) {
        const int32_t w = w0 + tid;
        int64_t room = 0;
        if (w < P) {
            const int64_t has = cost_before(first_small(w + 1)) - cost_before(first_small(w));
            room = most > has ? most - has : 0;
        }
        int64_t all;
        const int64_t at = given + block_scan(room, lds.sums, all);
        if (w < P) lds.bound[w] = at < line ? at : line;
        given += all;
    }
    if (tid == 0) lds.bound[P] = line;
    __syncthreads();
    // a part of less than a tile's start and two pages goes to the neighbour
    for (int32_t t0 = 0; t0 < n_tiles; t0 += nt) {
        const int32_t t = t0 + tid;
        if (t >= n_tiles) continue;
        const RowTile x = tile_at(t);
        const int64_t end = x.cost0 + tile_cost(x);
        if (x.cost0 < 0 || end == x.cost0) continue;
        for (int32_t w = bound_of(lds.bound, P, x.cost0, true); w < P && lds.bound[w] < end; ++w) {
            if (lds.bound[w] - x.cost0 <= kTileCost + (2 << kPageShift)) lds.bound[w] = x.cost0;
            else if (end - lds.bound[w] <= (2 << kPageShift)) lds.bound[w] = end;
        }
    }
    __syncthreads();
    int64_t rows = 0;
    for (int32_t t0 = 0; t0 < n_tiles; t0 += nt) {
        const int32_t t = t0 + tid;
        int64_t need = 0;
        int32_t w0 = 0, n_wg = 0;
        if (t < n_tiles) {
            const RowTile x = tile_at(t);
            const int64_t end = x.cost0 + tile_cost(x);
            if (x.cost0 < 0) {
                n_wg = 1;
            } else if (end > x.cost0) {
                w0 = bound_of(lds.bound, P, x.cost0, true) - 1;
                const int32_t w1 = bound_of(lds.bound, P, end, false) - 1;
                n_wg = w1 - w0 + 1;
                for (int32_t w = bound_of(lds.bound, P, x.cost0, false); w <= w1; ++w) wg_tile[w] = t;
            }
            if (!(a.mode == kCross && n_wg == 1)) need = (int64_t)n_wg * x.rows;
        }
        int64_t all;
        const int64_t at = block_scan(need, lds.sums, all);
        if (t < n_tiles) {
            tiles[t].wg0 = w0;
            tiles[t].n_wg = n_wg;
            tiles[t].part = need > 0 ? (int32_t)(rows + at) : -1;
        }
        rows += all;
    }
    int64_t *bound = plan_part<int64_t>(a, h, a.bound_at);
    for (int32_t w = tid; w <= P; w += nt) bound[w] = lds.bound[w];
    if (tid == 0) *plan_of(a, h) = RowPlan{line, n_tiles, n_small};
}

__device__ __forceinline__ void plan_prefix(const RowsArgs &a, int h, PlanLds &lds)
{
    const int tid = threadIdx.x, nt = blockDim.x;
    const int32_t B = a.batch, G = 1 << a.g_log2, per = kTileRows >> a.g_log2;  // a power of two
    RowTile *tiles = plan_part<RowTile>(a, h, a.tile_at);
    int32_t *toks = plan_part<int32_t>(a, h, a.tok_at), *lims = plan_part<int32_t>(a, h, a.lim_at);
    int32_t *map = plan_part<int32_t>(a, h, a.map_at);
    for (int32_t b = tid; b < B; b += nt) {
        lds.item[b] = int2{a.of[b], a.count[b]};
        lds.order[b] = (quantised_end(a, b) - a.s_sink) / kPage;  // complete pages
        lds.most[b] = 0;
        lds.flag[b] = 0;
    }
    if (tid == 0) lds.count = 0;
    __syncthreads();
    for (int32_t b = tid; b < B; b += nt) {
        const int32_t l = lds.item[b].x;
        int32_t s = 0;
        if (l >= 0 && l < B && l != b) s = max(min(min(lds.item[b].y, a.max_pages), min(lds.order[b], lds.order[l])), 0);
        lds.item[b] = int2{s > 0 ? l : -1, s};
        if (s > 0) atomicMax(&lds.most[l], s);
    }
    __syncthreads();
    for (int32_t b = tid; b < B; b += nt) {
        if (lds.item[b].x < 0 && lds.most[b] > 0) lds.item[b] = int2{b, lds.most[b]};  // a leader goes with its sequences
        if (lds.item[b].x >= 0) atomicAdd(&lds.count, 1);
    }
    __syncthreads();
    // the sequences by leader, then by pages shared (longest first), then by number
    const int32_t n_sorted = lds.count;
    for (int32_t b = tid >> 6; b < B; b += nt >> 6) {  // (a wave compares it with 64 at a time)
        const int2 x = lds.item[b];
        if (x.x < 0) continue;
        int32_t before = 0, mates = 0;
        for (int32_t c0 = 0; c0 < B; c0 += 64) {
            const int32_t c = c0 + (tid & 63);
            const int2 y = c < B ? lds.item[c] : int2{-1, 0};
            mates += __popcll(__ballot(y.x == x.x && (y.y > x.y || (y.y == x.y && c < b))));
            before += __popcll(__ballot((uint32_t)y.x < (uint32_t)x.x));  // (not those of none)
        }
        if ((tid & 63) == 0) {
            lds.order[before + mates] = b;
            lds.flag[before + mates] = (mates & (per - 1)) == 0;
        }
    }
    __syncthreads();
    // tiles in that order, behind the sequences' own
    int32_t n_tiles = B;
    for (int32_t p0 = 0; p0 < n_sorted; p0 += nt) {
        const int32_t p = p0 + tid;
        const bool start = p < n_sorted && lds.flag[p] != 0;
        int64_t all;
        const int32_t before = (int32_t)block_scan(start, lds.sums, all);
        if (p < n_sorted) {
            const int32_t b = lds.order[p], t = n_tiles + before + (start ? 1 : 0) - 1;
            toks[B + p] = b;
            lims[B + p] = lds.item[b].y;
            map[2 * b] = t;
            lds.most[p] = t;  // (the counts it held are used)
            if (start) {
                int32_t n = 1;
                while (n < per && p + n < n_sorted && lds.flag[p + n] == 0) ++n;
                tiles[t] = RowTile{lds.item[b].x, 0, lds.item[b].y, 0, n * G, B + p, lds.item[lds.order[p + n - 1]].y, -1, 0, 0, 0};
            }
        }
        n_tiles += (int32_t)all;
    }
    for (int32_t b = tid; b < B; b += nt) {
        const int32_t S = a.seq_len[b], s = lds.item[b].y;
        const int32_t pages = min((quantised_end(a, b) - a.s_sink + kPage - 1) / kPage, a.max_pages);
        tiles[b] = RowTile{b, s, max(pages - s, 0), S > 0 ? a.win_slots / kPage : 0, G, b, INT32_MAX, -1, 0, 0, 0};
        toks[b] = b;
        if (lds.item[b].x < 0) map[2 * b] = -1;
    }
    __syncthreads();
    // each sorted sequence's place in its tile
    for (int32_t p = tid; p < n_sorted; p += nt) map[2 * lds.order[p] + 1] = B + p - tiles[lds.most[p]].tok;
    share_out(a, h, n_tiles, lds);
}

// Tokens of query sequence i, and the stored sequence that they attend to.
__device__ __forceinline__ int32_t item_tokens(const RowsArgs &a, int32_t i, int32_t &src)
{
    src = a.of != nullptr ? a.of[i] : i;
    if (src < 0 || src >= a.batch || a.seq_len[src] <= 0) return 0;
    return a.count != nullptr ? min(max(a.count[i], 0), a.max_tok) : a.max_tok;
}

__device__ __forceinline__ void plan_cross(const RowsArgs &a, int h, PlanLds &lds)
{
    const int tid = threadIdx.x, nt = blockDim.x;
    const int32_t N = a.items, G = 1 << a.g_log2, per = kTileRows >> a.g_log2;
    RowTile *tiles = plan_part<RowTile>(a, h, a.tile_at);
    int32_t *toks = plan_part<int32_t>(a, h, a.tok_at);
    for (int32_t i = tid; i < N; i += nt) {
        int32_t src;
        const int32_t n = item_tokens(a, i, src);
        lds.item[i] = int2{n > 0 ? src : -1, n};
    }
    if (tid == 0) lds.count = 0;
    __syncthreads();
    // the token list goes by stored sequence, then by query sequence
    // (a wave compares it with 64 at a time; the sums are below 2^24, exact in fp32)
    for (int32_t i = tid >> 6; i < N; i += nt >> 6) {
        const int2 x = lds.item[i];
        float before = 0.0f, first = 0.0f, sum = 0.0f;  // first: of the stored sequences before; before: of the same one's items
        for (int32_t c = tid & 63; c < N; c += 64) {
            const int2 y = lds.item[c];  // (those of none have no tokens)
            const float n = (float)y.y;
            first += y.x < x.x ? n : 0.0f;
            sum += y.x == x.x ? n : 0.0f;
            before += y.x == x.x && c < i ? n : 0.0f;
        }
        const int32_t f = (int32_t)wave_sum(first), t = (int32_t)wave_sum(sum), e = (int32_t)wave_sum(before);
        if ((tid & 63) == 0) {
            const int32_t n = x.y > 0 && e == 0 ? (t + per - 1) >> (kTileLog2 - a.g_log2) : 0;  // tiles, at a stored sequence's first
            lds.order[i] = f + e;
            lds.most[i] = n;
            lds.at[i] = f;
            lds.sum[i] = t;
            atomicAdd(&lds.count, n);
        }
    }
    __syncthreads();
    for (int32_t i = tid >> 6; i < N; i += nt >> 6) {
        const int32_t g = lds.item[i].x;
        float before = 0.0f;
        for (int32_t c = tid & 63; c < N; c += 64) before += lds.item[c].x < g ? (float)lds.most[c] : 0.0f;
        const int32_t f = (int32_t)wave_sum(before);
        if ((tid & 63) == 0) lds.flag[i] = f;
    }
    __syncthreads();
    const int32_t n_tiles = lds.count;
    for (int32_t i = tid >> 6; i < N; i += nt >> 6) {
        const int32_t b = lds.item[i].x;
        if (lds.most[i] == 0) continue;
        const int32_t pages = min((quantised_end(a, b) - a.s_sink + kPage - 1) / kPage, a.max_pages);
        for (int32_t x = tid & 63; x < lds.most[i]; x += 64)
            tiles[lds.flag[i] + x] = RowTile{b, 0, pages, a.win_slots / kPage, min(per, lds.sum[i] - x * per) * G,
                                             lds.at[i] + x * per, INT32_MAX, -1, 0, 0, 0};
    }
    for (int32_t i = tid >> 6; i < N; i += nt >> 6)
        for (int32_t t = tid & 63; t < lds.item[i].y; t += 64) toks[lds.order[i] + t] = i * a.max_tok + t;
    share_out(a, h, n_tiles, lds);
}

__device__ __forceinline__ void plan_weighted(const RowsArgs &a, int h, PlanLds &lds)
{
    RowTile *tiles = plan_part<RowTile>(a, h, a.tile_at);
    int32_t *toks = plan_part<int32_t>(a, h, a.tok_at);
    for (int32_t b = threadIdx.x; b < a.batch; b += blockDim.x) {
        int32_t n = min((quantised_end(a, b) - a.s_sink + kPage - 1) / kPage, a.max_pages);
        if (a.n_sel != nullptr) n = min(max(a.n_sel[(int64_t)b * a.n_kv + h], 0), a.max_sel);
        const bool any = a.seq_len[b] > 0;
        tiles[b] = RowTile{b, 0, any ? n : 0, any ? a.win_slots / kPage : 0, 1 << a.g_log2, b, INT32_MAX, -1, 0, 0, 0};
        toks[b] = b;
    }
    share_out(a, h, a.batch, lds);
}

// ------------------------------------------------------------------ q~

// Digit limbs of these rows: six base-32 digits (up to 16, whole numbers of both formats),
// 30 bits of the row's largest entry.  (decode's 24 or 25 are the larger part of a short
// sequence's error: 700 tokens, up to 8e-7 of a row's norm where a plain fp32 q~ gives up to
// 6e-7.  The sixth limb of 2-bit keys costs four of 56 products a page.)
template <int BITS>
struct RowLimbs {
    static constexpr int kCount = 6, kDigitBits = 5;
    static constexpr int kUnit = Limbs<BITS>::kUnit;
    static constexpr float kNMax = 519552480.0f;  // 15 (1 + 32 + .. + 32^5), as far as fp32 has it
};
static_assert(RowLimbs<2>::kCount <= kLimbRoom, "a row's room");

// The digit limbs as in form_limbs, for 16 rows at once: a thread has channels c .. c + 3
// of its row, D / 4 neighbours the row.  (Two rows a wave instead of one, the digits of
// N from one sum with all of them moved to 0 .. base - 1, six-bit codes packed between
// neighbours: rows_query_kernel takes 52.8 instead of 55.4 us for 65536 rows.)  Returns the
// limbs' scales; out: the row's limbs.
template <int D, int BITS>
__device__ __forceinline__ u32x2 row_limbs(const f32x4 &x, uint8_t *out, int c)
{
    using LB = RowLimbs<BITS>;
    float mx = row_max16(fmaxf(fmaxf(fabsf(x[0]), fabsf(x[1])), fmaxf(fabsf(x[2]), fabsf(x[3]))));
    if constexpr (D == 128) mx = fmaxf(mx, __shfl_xor(mx, 16));
    int F = 0;
    if (mx > 0.0f) {
        int ex;
        (void)frexpf(LB::kNMax / mx, &ex);
        F = ex - 1;
        if (ldexpf(mx, F) > LB::kNMax) F -= 1;
        if (ldexpf(mx, F + 1) <= LB::kNMax) F += 1;
        F = F < -100 ? -100 : (F > 100 ? 100 : F);
    }
    u32x2 scales = {0u, 0u};
#pragma unroll
    for (int l = 0; l < LB::kCount; ++l)
        scales[l >> 2] |= (uint32_t)(127 + LB::kUnit + LB::kDigitBits * (LB::kCount - 1 - l) - F) << (8 * (l & 3));
    constexpr int kHalf = 1 << (LB::kDigitBits - 1);
    constexpr int all_halves = [] {
        int v = 0;
        for (int l = 0; l < LB::kCount; ++l) v = (v << LB::kDigitBits) + (1 << (LB::kDigitBits - 1));
        return v;
    }();
    uint32_t N[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) N[e] = (uint32_t)((int)rintf(ldexpf(x[e], F))) + (uint32_t)all_halves;
    const int q = (c >> 2) & 3;
#pragma unroll
    for (int l = 0; l < LB::kCount; ++l) {
        int d[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            d[e] = (int)((N[e] >> (LB::kDigitBits * (LB::kCount - 1 - l))) & (2 * kHalf - 1)) - kHalf;
        if constexpr (BITS == 2) {
            // fp6 e2m3 of d / 8: sign and integer; 16 channels are three words
            uint32_t p = 0u;
#pragma unroll
            for (int e = 0; e < 4; ++e) p |= ((uint32_t)max(d[e], -d[e]) | ((uint32_t)(d[e] >> 26) & 0x20u)) << (6 * e);
            const uint32_t above = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)p, 0xF9, 0xF, 0xF, true);  // the next thread's
            if (q < 3)
                *reinterpret_cast<uint32_t *>(out + l * 128 + 32 * (c >> 5) + 12 * ((c >> 4) & 1) + 4 * q) =
                    (p >> (8 * q)) | (above << (24 - 8 * q));
        } else {
            // fp8 e4m3 of d, exact
            int w = __builtin_amdgcn_cvt_pk_fp8_f32((float)d[0], (float)d[1], 0, false);
            w = __builtin_amdgcn_cvt_pk_fp8_f32((float)d[2], (float)d[3], w, true);
            *reinterpret_cast<int *>(out + l * 128 + c) = w;
        }
        if constexpr (D == 64) {  // channels 64 .. 127 of the operands: none
            *reinterpret_cast<uint32_t *>(out + l * 128 + 64 + c) = 0u;
        }
    }
    return scales;
}

template <int D, int BITS>
__global__ void __launch_bounds__(64 * kQtWaves<D>) rows_query_kernel(RowsArgs a)
{
    constexpr int R = 16, NT = 64 * kQtWaves<D>;
    using Q = QueryLds<D, R>;
    constexpr int kRaw = (Q::kBytes + 15) / 16 * 16, kRows = kRaw + kReps * R * Q::kQPitch * 2;
    constexpr int kBytes = kRows > (int)sizeof(PlanLds) ? kRows : (int)sizeof(PlanLds);
    __shared__ __attribute__((aligned(16))) uint8_t lds[kBytes];
    uint16_t *raw = reinterpret_cast<uint16_t *>(lds + kRaw);
    const int tid = threadIdx.x, h = blockIdx.x;
    if (blockIdx.y == 0) {
        PlanLds &p = *reinterpret_cast<PlanLds *>(lds);
        if (a.mode == kPrefix) plan_prefix(a, h, p);
        else if (a.mode == kCross) plan_cross(a, h, p);
        else plan_weighted(a, h, p);
        return;
    }
    const int32_t G = 1 << a.g_log2;
    const int64_t rows = (int64_t)a.items * a.max_tok * G;  // of a kv head
    TColumns<D> tc;
    tc.load(a.tinv, h, tid);
    // all groups' queries first (in a loop their loads would wait for the stores of the
    // group before them); rows of no token get zeros
    const int pr = tid / (D / 8), pc = 8 * (tid % (D / 8));
    const int64_t first = (int64_t)(blockIdx.y - 1) * a.reps * R;
    if (tid < R * D / 8) {
        u32x4 x[kReps];
        bool there[kReps];
#pragma unroll
        for (int k = 0; k < kReps; ++k) {
            const int64_t row = min(first + k * R + pr, rows - 1);
            const int32_t tok = (int32_t)(row >> a.g_log2), g = (int32_t)row & (G - 1);
            x[k] = *reinterpret_cast<const u32x4 *>(a.q + (((int64_t)tok * a.n_kv + h) * G + g) * D + pc);
            there[k] = true;
            if (a.mode == kCross) {
                int32_t src;
                const uint32_t item = (uint32_t)tok / (uint32_t)a.max_tok;
                there[k] = tok - (int32_t)item * a.max_tok < item_tokens(a, (int32_t)item, src);
            }
        }
#pragma unroll
        for (int k = 0; k < kReps; ++k) {
            const int64_t row = first + k * R + pr;
            if (k < a.reps && row < rows && !there[k]) {
                float *to = a.out + (((row >> a.g_log2) * a.n_kv + h) * G + (row & (G - 1))) * D + pc;
                reinterpret_cast<f32x4 *>(to)[0] = f32x4{0.f, 0.f, 0.f, 0.f};
                reinterpret_cast<f32x4 *>(to)[1] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
            if (!there[k] || row >= rows) x[k] = u32x4{0u, 0u, 0u, 0u};
            *reinterpret_cast<u32x4 *>(raw + (k * R + pr) * Q::kQPitch + pc) = x[k];
        }
    }
    static_assert(NT == R * D / 4, "a thread has four channels of a row");
    const int r = tid / (D / 4), c = 4 * (tid % (D / 4));
    for (int rep = 0; rep < a.reps; ++rep) {
        const int64_t row0 = first + rep * R;
        if (row0 >= rows) return;
        const int n = (int)(rows - row0 < R ? rows - row0 : R);
        __syncthreads();
        if (tid < R * D / 8)
            *reinterpret_cast<u32x4 *>(reinterpret_cast<uint16_t *>(lds) + pr * Q::kQPitch + pc) =
                *reinterpret_cast<const u32x4 *>(raw + (rep * R + pr) * Q::kQPitch + pc);
        form_qt_mfma<D, R>(a.scale, tc, lds, tid);
        const int64_t to = (int64_t)h * rows + row0;
        const f32x4 x = reinterpret_cast<const f32x4 *>(lds)[tid];
        __syncthreads();  // (read: the limbs go there)
        if (r < n) *reinterpret_cast<f32x4 *>(a.qt + (to + r) * D + c) = x;
        const u32x2 scales = row_limbs<D, BITS>(x, lds + r * kLimbRoom * 128, c);
        if (r < n && c == 0) *reinterpret_cast<u32x2 *>(a.qaux + (to + r) * 4) = scales;
        __syncthreads();
        constexpr int kRoom = kLimbRoom * 8, kUsed = RowLimbs<BITS>::kCount * 8;  // in 16 bytes
        for (int i = tid; i < n * kUsed; i += NT) {
            const int at = i / kUsed * kRoom + i % kUsed;
            reinterpret_cast<u32x4 *>(a.qlimb + to * kLimbRoom * 128)[at] = reinterpret_cast<const u32x4 *>(lds)[at];
        }
    }
}

// ------------------------------------------------------------------ the rows

// A page's weight p s is about 2^kLift where a row's maximum is new and the value
// scale the largest (fp16 holds nothing below 2^-24, where the lo parts of small
// weights would be lost), and at most 2^(kLift + kGrow + 1) later.  A window's weights
// are taken times 2^-kRoom, so that sums of values near bf16's largest stay finite.
// Both go by factors of the values, not by the logits: an exponential's argument near
// zero has the smaller rounding (one token's row of 700: 6e-7 with references 8 below
// the maximum, up to 1.9e-6 of its norm).
constexpr float kLift = 6.0f, kGrow = 8.0f, kRoom = 12.0f;
// Rows of weights in LDS: 64 tokens of two bytes, and room that spreads the rows read
// together over the banks.
constexpr int kPitch = 144;

// LDS: the rows' limbs, and a slice per wave, which holds its weights (two planes of
// a page's, three of a window's) and in the end its sums.
template <int D, int BITS>
struct RowsLds {
    static constexpr int most(int a, int b) { return a > b ? a : b; }
    static constexpr int kWave = most(16 * D * 4, 3 * 16 * kPitch);
    static constexpr int kLimb = BITS == 2 ? 64 * 24 : 64 * 32;  // of 16 rows: [lane] 16 bytes, [lane] the rest
    static constexpr int kMl = 4 * kWave + RowLimbs<BITS>::kCount * kLimb;  // m, then l: float [4][16] each
    static constexpr int kBytes = kMl + 2 * 4 * 16 * 4;
    __host__ __device__ static constexpr int limb_at(int l) { return 4 * kWave + l * kLimb; }
};

// Physical page of page unit i of stored sequence b, or -1; lp: its logical page.
__device__ __forceinline__ int32_t page_entry(const RowsArgs &a, int32_t b, int h, int32_t i, int32_t end, int32_t &lp)
{
    lp = a.sel != nullptr ? a.sel[((int64_t)b * a.n_kv + h) * a.max_sel + i] : i;
    if (lp < 0 || lp >= a.max_pages || (int64_t)lp * kPage >= end - a.s_sink) return -1;
    const int32_t phys = a.page_table[(int64_t)b * a.max_pages + lp];
    return phys >= 0 && phys < a.n_pages ? phys : -1;
}

__device__ __forceinline__ _Float16 lo16(uint32_t x) { return __builtin_bit_cast(f16x2, x)[0]; }
__device__ __forceinline__ _Float16 hi16(uint32_t x) { return __builtin_bit_cast(f16x2, x)[1]; }

// The codes and parameters of a page as a lane holds them.
template <int D, int BITS>
struct PageRegs {
    using L = Layout<D, BITS>;
    static constexpr int kKX = L::kKWordsPerLane / 4, kVX = L::kWordsPerLane / 4;
    u32x4 k[kKX], v[kVX], kp, vp;
    __device__ __forceinline__ void load_keys(const uint8_t *pg, int lane)
    {
#pragma unroll
        for (int i = 0; i < kKX; ++i)  // (at d = 64 the upper lanes' limbs are zero)
            k[i] = *reinterpret_cast<const u32x4 *>(pg + (uint32_t)(4 * L::k_word(lane % L::kKLanes, 4 * i)));
    }
    __device__ __forceinline__ void load_values(const uint8_t *pg, int lane)
    {
#pragma unroll
        for (int i = 0; i < kVX; ++i)
            v[i] = *reinterpret_cast<const u32x4 *>(pg + (uint32_t)(L::kRegionBytes + 4 * L::v_word(lane, 4 * i)));
    }
    __device__ __forceinline__ void load_params(const uint8_t *pg, int n)
    {
        kp = *reinterpret_cast<const u32x4 *>(pg + (uint32_t)(L::kParamOffset + 16 * n));
        vp = *reinterpret_cast<const u32x4 *>(pg + (uint32_t)(L::kParamOffset + 4 * kPage + 16 * n));
    }
};

// The wave's own LDS writes come before its reads behind this, and the reverse (its
// accesses complete in order; this holds the compiler to it).
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The running softmax of rows 4 j + r: a weight is 2^(logit - m).
template <int D>
struct RowState {
    f32x4 acc[D / 16];  // sums of p s 16 (c - middle) (pages) or p v (windows), channels 16 nt + n
    f32x4 m, l, z;      // reference, sum of p, sum of p (z + middle s) (the lane's tokens)
};

// Moves the references up, and what is relative to them.
template <int D>
__device__ __forceinline__ void move_references(RowState<D> &s, const f32x4 &up)
{
    const f32x4 f = {fexp2(-up[0]), fexp2(-up[1]), fexp2(-up[2]), fexp2(-up[3])};
    s.m += up;
    s.l *= f;
    s.z *= f;
#pragma unroll
    for (int nt = 0; nt < D / 16; ++nt) s.acc[nt] *= f;
}

// Moves the references of logits x, relative to them, to the whole number at or above a
// row's largest (whole, so that what is brought from one reference to another is brought
// by a power of two).  A row that sees none of the first tokens stays: it sees none later
// either.
template <int D>
__device__ __forceinline__ void raise_references(RowState<D> &s, f32x4 (&x)[4], bool fresh)
{
    f32x4 up;
#pragma unroll
    for (int r = 0; r < 4; ++r)
        up[r] = ceilf(row_max16(fmaxf(fmaxf(x[0][r], x[1][r]), fmaxf(x[2][r], x[3][r]))));
    if (fresh) {
#pragma unroll
        for (int r = 0; r < 4; ++r) up[r] = up[r] == -INFINITY ? 0.0f : up[r];
        s.m = up;
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) up[r] = fmaxf(up[r], 0.0f);
        move_references<D>(s, up);
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) x[t] -= up;
}

template <int D, int BITS, bool WEIGH>
__device__ __forceinline__ void take_tile(const RowsArgs &a, const RowTile &tile, int32_t lo, int32_t hi, int32_t slot,
                                          uint8_t *lds, int h, bool late)
{
    using L = Layout<D, BITS>;
    using LB = RowLimbs<BITS>;
    using Lds = RowsLds<D, BITS>;
    constexpr int kNT = L::kNTiles, kC = L::kChunks, kScaleB = BITS == 2 ? 128 : 136;
    constexpr int kPlane = 16 * kPitch;
    // values as s (c - middle) + (z + middle s): the sums of both are then of the output's size.
    // (The middle goes by the codes' own bits: three-bit ones, which lie in the four-bit
    // format, centred on 8 add up to more than raw ones.)
    const float middle = BITS == 2 ? 2.0f : a.mid + 0.5f;
    // (the lane is opaque where a part begins, so that the addresses that follow from
    // it are formed there, and do not hold registers from the kernel's start on)
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int lane = tid & 63;
    asm volatile("" : "+v"(lane));
    int j = lane >> 4, n = lane & 15;
    const int32_t G = 1 << a.g_log2, b = tile.seq;
    const int64_t rows_all = (int64_t)a.items * a.max_tok << a.g_log2;
    const int32_t *toks = plan_part<int32_t>(a, h, a.tok_at) + tile.tok;
    const int32_t S = a.seq_len[b], q_hi = quantised_end(a, b);
    const uint32_t pbuf = lds_addr(lds + wave * Lds::kWave);
    // (query row r of the tile, in the workspace's order; behind them the last one again:
    // what comes of it is not used, and no load waits in a branch)
    auto row_at = [&](int r) -> int64_t {
        const int i = min(r, tile.rows - 1);
        return h * rows_all + ((int64_t)toks[i >> a.g_log2] << a.g_log2) + (i & (G - 1));
    };

    RowState<D> s;
#pragma unroll
    for (int nt = 0; nt < kNT; ++nt) s.acc[nt] = f32x4{0.f, 0.f, 0.f, 0.f};
    s.m = s.l = s.z = f32x4{0.f, 0.f, 0.f, 0.f};
    bool fresh = true;  // nothing seen, references 0
    float unit = 1.0f;  // what acc is counted in
    float in_room = 1.0f;  // what m, l and z will be, for sums with windows

    const int32_t page_hi = min(hi, tile.n_pages);
    if (lo < page_hi) {
        // ============================================ pages
        // operands: limb l of row n, in LDS (beside the sums they would not fit
        // the registers); a wave brings every fourth
        const int64_t mine = row_at(n);
        const u32x2 sc = *reinterpret_cast<const u32x2 *>(a.qaux + 4 * mine);
        constexpr int kMine = (LB::kCount + 3) / 4;
        u32x4 x0[kMine], x1[kMine];
#pragma unroll
        for (int k = 0; k < kMine; ++k) {
            const int l = min(wave + 4 * k, LB::kCount - 1);
            const u32x4 *src = reinterpret_cast<const u32x4 *>(a.qlimb + (mine * kLimbRoom + l) * 128 + 32 * j);
            x0[k] = src[0];
            x1[k] = src[1];
        }
#pragma unroll
        for (int k = 0; k < kMine; ++k) {
            const int l = min(wave + 4 * k, LB::kCount - 1);
            uint8_t *to = lds + Lds::limb_at(l);
            reinterpret_cast<u32x4 *>(to)[lane] = x0[k];
            if constexpr (BITS == 2) reinterpret_cast<u32x2 *>(to + 1024)[lane] = u32x2{x1[k][0], x1[k][1]};
            else reinterpret_cast<u32x4 *>(to + 1024)[lane] = x1[k];
        }
        __syncthreads();
        const uint32_t limbs = lds_addr(lds);
        auto limb = [&](int l) -> i32x8 {
            const uint32_t at = limbs + Lds::limb_at(l);
            const u32x4 x = lds_read16(at + 16 * lane);
            if constexpr (BITS == 2) {
                const u32x2 y = lds_read8(at + 1024 + 8 * lane);
                return i32x8{(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)y[0], (int)y[1], 0, 0};
            } else {
                const u32x4 y = lds_read16(at + 1024 + 16 * lane);
                return i32x8{(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)y[0], (int)y[1], (int)y[2], (int)y[3]};
            }
        };
        // c += the products, those of the largest digits apart from the others' sum, which
        // is rounded far below (every sum onto c would round at its size)
        auto products = [&](const i32x8 (&bop)[4], f32x4 (&c)[4]) {
            f32x4 rest[4] = {};
            limb_products<BITS, 5, kScaleB>(limb(5), bop, (int)sc[1], rest);
            limb_products<BITS, 4, kScaleB>(limb(4), bop, (int)sc[1], rest);
            limb_products<BITS, 3, kScaleB>(limb(3), bop, (int)sc[0], rest);
            limb_products<BITS, 2, kScaleB>(limb(2), bop, (int)sc[0], rest);
            limb_products<BITS, 1, kScaleB>(limb(1), bop, (int)sc[0], rest);
            limb_products<BITS, 0, kScaleB>(limb(0), bop, (int)sc[0], c);
#pragma unroll
            for (int t = 0; t < 4; ++t) c[t] += rest[t];
        };
        // the digit sums, by products with keys of code 1 (every column the same), from
        // which the products start
        f32x4 zs;
        {
            const int one = BITS == 2 ? 0x11111111 : 0x01010101;
            const i32x8 o = BITS == 2 ? i32x8{one, one, one, one, 0, 0, 0, 0} : i32x8{one, one, one, one, one, one, one, one};
            const i32x8 ones[4] = {o, o, o, o};
            f32x4 c[4] = {};
            products(ones, c);
            zs = c[0];
        }
        WidenNormal<BITS> wide;
        wide.init(middle);
        // where the lane writes its weights (rows 4 j + r, tokens 4 n ..) and reads the
        // operand of row n (tokens 32 kc + 8 j ..)
        const uint32_t pw = pbuf + 4 * j * kPitch + 8 * n, pr = pbuf + n * kPitch + 16 * j;
        // value scales up to 2^vex are served: they are taken times vscale, 2^(kLift - vex)
        int vex = 0;
        float vscale = 0.0f;
        uint32_t vmost = 0u;    // the largest (fp16 bits)

        for (int32_t base = lo; base < page_hi; base += 256) {
            int32_t lp = -1, phys = -1;
            const int32_t u = base + 4 * lane + wave;
            if (u < page_hi) phys = page_entry(a, b, h, tile.first + u, q_hi, lp);
            uint64_t todo = __ballot(phys >= 0);
            if (todo == 0) continue;
            auto page_at = [&](int i) -> const uint8_t * {
                return a.pages + ((int64_t)__builtin_amdgcn_readlane(phys, i) * a.n_kv + h) * L::kPageBytes;
            };
            PageRegs<D, BITS> pg;
            int cur = __builtin_ctzll(todo);
            {
                const uint8_t *p = page_at(cur);
                pg.load_keys(p, lane);
                pg.load_params(p, n);
                pg.load_values(p, lane);
            }
            // Of two workgroups of a compute unit the older one's waves go first and end
            // long before the other's (70 against 97 us at 64 sequences on 32K tokens): the
            // younger goes first through most of a run (the kernel: 100 -> 94 us).
            if (late) __builtin_amdgcn_s_setprio(1);
            const int until = __popcll(todo) * 2 / 3;
            for (int done = 0; todo != 0; ++done) {
                if (done == until) __builtin_amdgcn_s_setprio(0);
                todo &= todo - 1;
                const int next = todo != 0 ? __builtin_ctzll(todo) : cur;
                const uint8_t *np = page_at(next);
                const int32_t clp = __builtin_amdgcn_readlane(lp, cur);
                const int32_t nvalid = min(kPage, q_hi - (a.s_sink + clp * kPage));
                const bool part = nvalid < kPage || clp >= tile.limit;

                if (nvalid < kPage) {  // (whatever the page held before)
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        if (4 * n + t >= nvalid) pg.vp[t] = 0u;
                }
                const uint32_t big = max(max(pg.vp[0] & 0x7FFFu, pg.vp[1] & 0x7FFFu), max(pg.vp[2] & 0x7FFFu, pg.vp[3] & 0x7FFFu));
                if (__any(big > vmost)) {  // the largest scale lies in [2^(ex - 1), 2^ex)
                    int ex;
                    (void)frexpf(fminf(wave_max(f16_bits_to_f32(big)), 65504.0f), &ex);
                    if (vmost == 0u) vex = ex;  // (no sums but of zeros)
                    const float down = ldexpf(1.0f, vex - max(ex, vex));
#pragma unroll
                    for (int nt = 0; nt < kNT; ++nt) s.acc[nt] *= down;
                    vex = max(ex, vex);
                    vmost = vex >= 16 ? 0x7FFFu : f32_to_f16_bits(ldexpf(2.0f, vex));  // (and twice that)
                    vscale = ldexpf(1.0f, (int)kLift - vex);
                }
                i32x8 bop[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    uint32_t w[BITS];
#pragma unroll
                    for (int i = 0; i < BITS; ++i) w[i] = pg.k[(BITS * t + i) / 4][(BITS * t + i) % 4];
                    if constexpr (BITS == 2) {
                        bop[t] = i32x8{(int)(w[0] & 0x33333333u), (int)((w[0] >> 2) & 0x33333333u),
                                       (int)(w[1] & 0x33333333u), (int)((w[1] >> 2) & 0x33333333u), 0, 0, 0, 0};
                    } else {
                        bop[t] = i32x8{(int)(w[0] & 0x0F0F0F0Fu), (int)((w[0] >> 4) & 0x0F0F0F0Fu),
                                       (int)(w[1] & 0x0F0F0F0Fu), (int)((w[1] >> 4) & 0x0F0F0F0Fu),
                                       (int)(w[2] & 0x0F0F0F0Fu), (int)((w[2] >> 4) & 0x0F0F0F0Fu),
                                       (int)(w[3] & 0x0F0F0F0Fu), (int)((w[3] >> 4) & 0x0F0F0F0Fu)};
                    }
                }
                float mid[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) mid[t] = fmaf((float)lo16(pg.kp[t]), a.mid, (float)hi16(pg.kp[t]));
                f32x4 each = {0.f, 0.f, 0.f, 0.f};
                const f32x4 from = zs * -a.mid;
                f32x4 x[4] = {from, from, from, from};
                products(bop, x);
                pg.load_keys(np, lane);
                // logits, relative to the references: s (q~.(c - mid)) + ((z + mid s) sum(q~) - m)
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        x[t][r] = fmaf((float)lo16(pg.kp[t]), x[t][r], fmaf(mid[t], zs[r], -s.m[r]));
                if (part) {
                    // the rows and tokens that are left out
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int row = 4 * j + r;
                        bool out = false;
                        if (clp >= tile.limit && row < tile.rows)
                            out = plan_part<int32_t>(a, h, a.lim_at)[tile.tok + (row >> a.g_log2)] <= clp;
#pragma unroll
                        for (int t = 0; t < 4; ++t)
                            if (out || 4 * n + t >= nvalid) x[t][r] = -INFINITY;
                    }
                }
                float most = -INFINITY;
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    most = fmaxf(fmaxf(most, fmaxf(x[t][0], x[t][1])), fmaxf(x[t][2], x[t][3]));
                if (fresh || __any(most > kGrow)) raise_references<D>(s, x, fresh);
                float vs[4], vz[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    vs[t] = fmaf((float)lo16(pg.vp[t]), vscale, 0.0f);
                    vz[t] = fmaf((float)lo16(pg.vp[t]), middle, (float)hi16(pg.vp[t]));
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    uint32_t hi2[2], lo2[2];
                    float p[4];
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        p[t] = fexp2(x[t][r]);
                        s.z[r] = fmaf(p[t], vz[t], s.z[r]);
                    }
                    // each part is rounded from the exact product (the hi parts are opaque, so
                    // that the lo parts read them where they are, two to a register)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const float s0 = vs[2 * k], s1 = vs[2 * k + 1];
                        const f16x2 ph = {(_Float16)fmaf(p[2 * k], s0, 0.0f), (_Float16)fmaf(p[2 * k + 1], s1, 0.0f)};
                        hi2[k] = __builtin_bit_cast(uint32_t, ph);
                        asm("" : "+v"(hi2[k]));
                        const f16x2 hv = __builtin_bit_cast(f16x2, hi2[k]);
                        const f16x2 pl = {(_Float16)fmaf(p[2 * k], s0, -(float)hv[0]),
                                          (_Float16)fmaf(p[2 * k + 1], s1, -(float)hv[1])};
                        lo2[k] = __builtin_bit_cast(uint32_t, pl);
                    }
                    const float sum = (p[0] + p[1]) + (p[2] + p[3]);
                    if constexpr (WEIGH) each[r] = sum;
                    s.l[r] += sum;
                    lds_write8(pw + r * kPitch, hi2[0], hi2[1]);
                    lds_write8(pw + kPlane + r * kPitch, lo2[0], lo2[1]);
                }
                fresh = false;
                pg.load_params(np, n);
                if constexpr (WEIGH) {
                    // what the page received, with the reference that it goes by
                    float e = 0.0f, m = 0.0f;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float t = row_sum16(each[r]);
                        if (n == r) {
                            e = t;
                            m = s.m[r];
                        }
                    }
                    const int row = 4 * j + n;
                    if (n < 4 && row < tile.rows) {
                        const int64_t at = (((int64_t)h * a.batch + b) * a.max_sel + base + 4 * cur + wave) * G + row;
                        reinterpret_cast<f32x2 *>(a.stat)[at] = f32x2{e, m};
                    }
                }
                wave_fence();
#pragma unroll
                for (int kc = 0; kc < 2; ++kc) {
                    f16x8 A[2];
#pragma unroll
                    for (int p = 0; p < 2; ++p) A[p] = __builtin_bit_cast(f16x8, lds_read16(pr + p * kPlane + 64 * kc));
#pragma unroll
                    for (int uu = 0; uu < 2 * L::kNw; ++uu) {
                        const int w = kc * 2 * L::kNw + uu;
                        uint32_t op[L::kCodesPerWord / 2];
                        wide.word(pg.v[w / 4][w % 4], op);
#pragma unroll
                        for (int p = 0; p < 2; ++p)
#pragma unroll
                            for (int o = 0; o < L::kOpsPerWord; ++o) {
                                f32x4 &acc = s.acc[uu * L::kOpsPerWord + o];
                                acc = mfma16h(A[p], as_op_h(op + 4 * o), acc);
                            }
                    }
                }
                wave_fence();
                pg.load_values(np, lane);
                cur = next;
            }
        }
        unit = ldexpf(0.0625f, vex - (int)kLift);
    }

    if (hi > tile.n_pages) {
        // ============================================ windows
        asm volatile("" : "+v"(lane));
        j = lane >> 4;
        n = lane & 15;
        const uint32_t pw = pbuf + 4 * j * kPitch + 8 * n, pr = pbuf + n * kPitch + 16 * j;
        const float room = ldexpf(1.0f, -(int)kRoom);
        const int32_t ring = a.win_slots - a.s_sink;
        const int32_t a0 = S > q_hi ? (q_hi - a.s_sink) % ring : 0;
        const int32_t ring_live = S > q_hi ? S - q_hi : 0;
        const int64_t head = (int64_t)b * a.n_kv + h;
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt) s.acc[nt] *= unit * room;
        const float *q = a.qt + row_at(n) * D + 8 * j;
        unit = 1.0f;
        in_room = room;
        const int32_t from = max(lo, tile.n_pages);
        for (int32_t u = from + ((wave - (from - lo)) & 3); u < hi; u += 4) {
            const int32_t slot0 = kPage * (u - tile.n_pages);
            bool here;
            {
                const int32_t sl = slot0 + lane;
                here = sl < a.s_sink ? sl < S : ((sl - a.s_sink - a0 + ring) % ring) < ring_live;
            }
            const uint64_t live = __ballot(here);
            if (live == 0) continue;
            // keys, queries and values are requested together each (the barriers hold the
            // compiler to it: it would wait for one load after the other)
            f32x4 c[4] = {};
#pragma unroll
            for (int half = 0; half < kC; half += 2) {
                bf16x8 kx[2][4], qp[2][3];
                f32x4 qx[2][2];
#pragma unroll
                for (int ch = 0; ch < 2; ++ch) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) qx[ch][i] = *reinterpret_cast<const f32x4 *>(q + 32 * (half + ch) + 4 * i);
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        kx[ch][t] = *reinterpret_cast<const bf16x8 *>(
                            a.win_k + (head * a.win_slots + slot0 + 4 * n + t) * D + 32 * (half + ch) + 8 * j);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int ch = 0; ch < 2; ++ch)
#pragma unroll
                    for (int p = 0; p < 3; ++p) {
                        u32x4 w;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            f32x4 &x = qx[ch][i / 2];
                            const int e = 2 * (i % 2);
                            w[i] = pack_bf16_rne(x[e], x[e + 1]);
                            x[e] -= bf16_bits_to_f32(w[i] & 0xFFFFu);
                            x[e + 1] -= bf16_bits_to_f32(w[i] >> 16);
                        }
                        qp[ch][p] = __builtin_bit_cast(bf16x8, w);
                    }
#pragma unroll
                for (int ch = 0; ch < 2; ++ch)
#pragma unroll
                    for (int p = 2; p >= 0; --p)
#pragma unroll
                        for (int t = 0; t < 4; ++t) c[t] = mfma16(qp[ch][p], kx[ch][t], c[t]);
            }
            u32x4 vy[kNT];
            auto load_values = [&](int kc) {
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt)
                    vy[nt] = *reinterpret_cast<const u32x4 *>(
                        a.win_v + (head * D + 16 * nt + n) * a.win_slots + slot0 + 32 * kc + 8 * j);
                __builtin_amdgcn_sched_barrier(0);
            };
            load_values(0);
            const uint32_t seen = (uint32_t)(live >> (4 * n)) & 15u;
            float most = -INFINITY;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    c[t][r] = (seen >> t) & 1u ? c[t][r] - s.m[r] : -INFINITY;
                    most = fmaxf(most, c[t][r]);
                }
            if (fresh || __any(most > 0.0f)) raise_references<D>(s, c, fresh);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float p[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) p[t] = fexp2(c[t][r]);
                s.l[r] += (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
                for (int t = 0; t < 4; ++t) p[t] *= room;
#pragma unroll
                for (int q = 0; q < 3; ++q) {
                    const uint32_t u0 = pack_bf16_rne(p[0], p[1]), u1 = pack_bf16_rne(p[2], p[3]);
                    lds_write8(pw + (16 * q + r) * kPitch, u0, u1);
                    p[0] -= bf16_bits_to_f32(u0 & 0xFFFFu);
                    p[1] -= bf16_bits_to_f32(u0 >> 16);
                    p[2] -= bf16_bits_to_f32(u1 & 0xFFFFu);
                    p[3] -= bf16_bits_to_f32(u1 >> 16);
                }
            }
            wave_fence();
#pragma unroll
            for (int kc = 0; kc < 2; ++kc) {
                bf16x8 A[3];
#pragma unroll
                for (int p = 0; p < 3; ++p)
                    A[p] = __builtin_bit_cast(bf16x8, lds_read16(pr + 16 * p * kPitch + 64 * kc));
                if (kc == 1) load_values(kc);
                // dead slots' values are zeroed, whatever bits they hold
                const uint32_t bits = (uint32_t)(live >> (32 * kc + 8 * j)) & 255u;
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt) {
                    u32x4 y = vy[nt];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        y[i] &= (((bits >> (2 * i)) & 1u) ? 0x0000FFFFu : 0u) | (((bits >> (2 * i + 1)) & 1u) ? 0xFFFF0000u : 0u);
#pragma unroll
                    for (int p = 2; p >= 0; --p) s.acc[nt] = mfma16(A[p], __builtin_bit_cast(bf16x8, y), s.acc[nt]);
                }
            }
            wave_fence();
            fresh = false;
        }
    }

    // ---- the four waves' results, merged
    float(*o)[D] = reinterpret_cast<float(*)[D]>(lds + wave * Lds::kWave);
    float *sm = reinterpret_cast<float *>(lds + Lds::kMl), *sl = sm + 4 * 16;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int row = 4 * j + r;
        const float z = row_sum16(s.z[r]) * in_room, l = row_sum16(s.l[r]) * in_room;
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt) o[row][16 * nt + n] = fmaf(s.acc[nt][r], unit, z);
        if (n == 0) {
            sm[wave * 16 + row] = l == 0.0f ? -INFINITY : in_room < 1.0f ? s.m[r] + kRoom : s.m[r];  // (none: no token seen)
            sl[wave * 16 + row] = l;
        }
    }
    __syncthreads();
    for (int i = tid; i < tile.rows * (D / 4); i += 256) {
        const int r = i / (D / 4), c = i % (D / 4);
        float mx = -INFINITY, l = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) mx = fmaxf(mx, sm[w * 16 + r]);
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        if (mx != -INFINITY) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float m = sm[w * 16 + r];
                if (m == -INFINITY) continue;
                const float f = fexp2(m - mx);
                l = fmaf(f, sl[w * 16 + r], l);
                const f32x4 y = *reinterpret_cast<const f32x4 *>(lds + w * Lds::kWave + (r * D + 4 * c) * 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = fmaf(f, y[e], x[e]);
            }
        }
        if (slot < 0) {
            const int64_t at = (((int64_t)toks[r >> a.g_log2] * a.n_kv + h) << a.g_log2) + (r & (G - 1));
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = l != 0.0f ? x[e] / l : 0.0f;
            reinterpret_cast<f32x4 *>(a.out + at * D)[c] = x;
        } else {
            const int64_t at = h * a.part_rows + slot + r;
            reinterpret_cast<f32x4 *>(a.part + at * D)[c] = x;
            if (c == 0) reinterpret_cast<f32x2 *>(a.part_ml)[at] = f32x2{mx, l};
        }
    }
    __syncthreads();  // the waves' results are read
}

template <int D, int BITS, bool WEIGH>
__global__ void __launch_bounds__(256, kRowsPerCu) rows_kernel(RowsArgs a)
{
    __shared__ __attribute__((aligned(16))) uint8_t lds[RowsLds<D, BITS>::kBytes];
    const int h = blockIdx.x, w = blockIdx.y;
    const RowPlan plan = *plan_of(a, h);
    const int64_t *bound = plan_part<const int64_t>(a, h, a.bound_at);
    const int32_t *small = plan_part<const int32_t>(a, h, a.small_at);
    const int64_t begin = bound[w], end = bound[w + 1];
    const RowTile *tiles = plan_part<const RowTile>(a, h, a.tile_at);
    // its small tiles (latencies, mostly) and its part of the line, every other
    // workgroup of a compute unit the other way round
    int32_t s = small_of(a, w, plan.n_small);
    const int32_t s1 = small_of(a, w + 1, plan.n_small);
    int32_t t = begin < plan.total ? plan_part<const int32_t>(a, h, a.wg_at)[w] : plan.n_tiles;
    const bool late = ((h + a.n_kv * w) / a.cus) & 1;
    for (;;) {
        RowTile tile;
        int32_t lo, hi, slot;
        if (s < s1 && !(late && t < plan.n_tiles)) {
            tile = tiles[small[s++]];
            lo = 0;
            hi = tile.n_pages + tile.n_win;
            slot = tile.part;
        } else if (t < plan.n_tiles) {
            tile = tiles[t++];
            if (tile.cost0 < 0 || tile.n_wg == 0) continue;
            if (tile.cost0 >= end) {
                t = plan.n_tiles;
                continue;
            }
            // (a workgroup without room in the midst of a tile: nothing of it)
            lo = unit_at(tile, begin - tile.cost0);
            hi = unit_at(tile, end - tile.cost0);
            slot = tile.part < 0 ? -1 : tile.part + (w - tile.wg0) * tile.rows;
        } else {
            break;
        }
        take_tile<D, BITS, WEIGH>(a, tile, lo, hi, slot, lds, h, late);
    }
}

// ------------------------------------------------------------------ merges

// A wave merges n partials of a row: number i is partial row at(i) of kv head h.
// Lane l ends with channels D/64 l .. and with the row's reference and sum.
template <int D, typename At>
__device__ __forceinline__ void merge_row(const RowsArgs &a, int h, int n, At at, float (&o)[D / 64], float &M, float &l)
{
    constexpr int kPer = D / 64;
    const int lane = threadIdx.x & 63;
    M = -INFINITY;
    l = 0.0f;
#pragma unroll
    for (int e = 0; e < kPer; ++e) o[e] = 0.0f;
    for (int k0 = 0; k0 < n; k0 += 64) {
        const int m = min(n - k0, 64);
        const int64_t mine = h * a.part_rows + at(k0 + min(lane, m - 1));
        f32x2 ml = reinterpret_cast<const f32x2 *>(a.part_ml)[mine];
        if (lane >= m) ml = f32x2{-INFINITY, 0.0f};
        const float m_new = fmaxf(M, wave_max(ml[0]));
        const float f = M == -INFINITY ? 0.0f : fexp2(M - m_new);
        const float w = ml[0] == -INFINITY ? 0.0f : fexp2(ml[0] - m_new);
        l = fmaf(l, f, wave_sum(w * ml[1]));
        M = m_new;
#pragma unroll
        for (int e = 0; e < kPer; ++e) o[e] *= f;
        for (int i = 0; i < m; i += 8) {
            float x[8][kPer];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int64_t row = h * a.part_rows + at(k0 + min(i + k, m - 1));
#pragma unroll
                for (int e = 0; e < kPer; ++e) x[k][e] = a.part[row * D + kPer * lane + e];
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                // (lanes past the last partial have weight 0; i + k < 64)
                const float wk = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), i + k));
                if (i + k < m && wk != 0.0f) {
#pragma unroll
                    for (int e = 0; e < kPer; ++e) o[e] = fmaf(wk, x[k][e], o[e]);
                }
            }
        }
    }
}

// Prefix and weighted: one workgroup per (kv head, sequence).
template <int D>
__global__ void __launch_bounds__(256) rows_merge_kernel(RowsArgs a)
{
    __shared__ float sM[8], sL[8];
    constexpr int kPlaces = 4096;
    __shared__ int32_t sPage[256], sStep[4];
    __shared__ uint8_t sLast[kPlaces];
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int32_t G = 1 << a.g_log2;
    const RowTile *tiles = plan_part<const RowTile>(a, h, a.tile_at);
    const RowTile own = tiles[b];
    RowTile with{};
    int32_t pos = 0;
    if (a.mode == kPrefix) {
        const int32_t *map = plan_part<const int32_t>(a, h, a.map_at);
        const int32_t t = map[2 * b];
        if (t >= 0) {
            with = tiles[t];
            pos = map[2 * b + 1] * G;
        }
    }
    const int n = own.n_wg + with.n_wg;
    for (int g = wave; g < G; g += 4) {
        float o[D / 64], M, l;
        merge_row<D>(a, h, n, [&](int i) -> int64_t {
            return i < own.n_wg ? own.part + (int64_t)i * own.rows + g
                                : with.part + (int64_t)(i - own.n_wg) * with.rows + pos + g;
        }, o, M, l);
        float *dst = a.out + (((int64_t)b * a.n_kv + h) * G + g) * D + (D / 64) * lane;
#pragma unroll
        for (int e = 0; e < D / 64; ++e) dst[e] = l != 0.0f ? o[e] / l : 0.0f;
        if (lane == 0) {
            sM[g] = M;
            sL[g] = l;
        }
    }
    if (a.mode != kWeighted) return;
    // the pages' weights: of a page, its rows' sums brought to their rows' references
    __syncthreads();
    const int32_t end = quantised_end(a, b);
    float *weights = a.weights + ((int64_t)b * a.n_kv + h) * a.max_pages;
    for (int32_t base = 0; base < own.n_pages; base += 256) {
        const int32_t u = base + tid;
        int32_t lp = -1;
        const bool here = u < own.n_pages && page_entry(a, b, h, u, end, lp) >= 0;
        float w = 0.0f;
        if (here) {
            const f32x2 *st = reinterpret_cast<const f32x2 *>(a.stat) + (((int64_t)h * a.batch + b) * a.max_sel + u) * G;
            for (int g = 0; g < G; ++g) w += st[g][0] * fexp2(st[g][1] - sM[g]) / sL[g];
        }
        // A list may name a page several times; each adds what it received, in the list's
        // order, so that the sum is the same in every run: of the round's entries with one
        // page the n-th adds in step n.  Whether there is more than one step at all: every
        // entry leaves its number in its page's place, and finds it there if no other has
        // that place (pages 4096 apart have the same one; they only take the longer way).
        // (64 sequences, 64 entries: 68.9 us a call in any order, 72 with every page twice.)
        int mine = 0, steps = 1;
        if (a.sel != nullptr) {
            sPage[tid] = here ? lp : -1;
            if (here) sLast[lp % kPlaces] = (uint8_t)tid;
            __syncthreads();
            const uint64_t again = __ballot(here && sLast[lp % kPlaces] != tid);
            if (lane == 0) sStep[wave] = again != 0;
            __syncthreads();
            if ((sStep[0] | sStep[1] | sStep[2] | sStep[3]) != 0) {
                const int n = min(own.n_pages - base, 256);
                for (int i = 0; i < n; ++i) mine += i < tid && sPage[i] == lp;
                __syncthreads();  // (the tests are read)
                const int most = (int)wave_max(here ? (float)mine : 0.0f);
                if (lane == 0) sStep[wave] = most;
                __syncthreads();
                steps = 1 + max(max(sStep[0], sStep[1]), max(sStep[2], sStep[3]));
            }
        }
        for (int k = 0; k < steps; ++k) {
            if (here && mine == k) weights[lp] += w;
            if (a.sel != nullptr) __syncthreads();  // (and the round's pages are read)
        }
    }
}

// Cross: workgroups (h, w, ..) merge the tile that workgroup w of rows_kernel began and
// did not end, a wave a row.
template <int D>
__global__ void __launch_bounds__(256) rows_join_kernel(RowsArgs a)
{
    const int h = blockIdx.x, w = blockIdx.y, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int32_t G = 1 << a.g_log2;
    const int64_t at = plan_part<const int64_t>(a, h, a.bound_at)[w + 1];
    if (at >= plan_of(a, h)->total) return;
    const RowTile tile = plan_part<const RowTile>(a, h, a.tile_at)[plan_part<const int32_t>(a, h, a.wg_at)[w + 1]];
    if (tile.cost0 == at || tile.wg0 != w) return;
    const int32_t *toks = plan_part<const int32_t>(a, h, a.tok_at) + tile.tok;
    const int r = 4 * blockIdx.z + wave;
    if (r < tile.rows) {
        float o[D / 64], M, l;
        merge_row<D>(a, h, tile.n_wg, [&](int i) -> int64_t { return tile.part + (int64_t)i * tile.rows + r; }, o, M, l);
        const int64_t to = (((int64_t)toks[r >> a.g_log2] * a.n_kv + h) << a.g_log2) + (r & (G - 1));
#pragma unroll
        for (int e = 0; e < D / 64; ++e) a.out[to * D + (D / 64) * lane + e] = l != 0.0f ? o[e] / l : 0.0f;
    }
}

// ------------------------------------------------------------------ host

static int64_t compute_units()
{
    static std::atomic<int64_t> cache{0};
    const int64_t known = cache.load(std::memory_order_relaxed);
    if (known > 0) return known;
    int dev = 0, ncu = 0;
    int64_t v = 256;
    if (hipGetDevice(&dev) == hipSuccess &&
        hipDeviceGetAttribute(&ncu, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && ncu > 0)
        v = ncu;
    else
        (void)hipGetLastError();
    cache.store(v, std::memory_order_relaxed);
    return v;
}

}  // namespace wushkv

using namespace wushkv;

int wushkv_validate_cache(const wushkv_cache *c);

// The workspace's arrays, and their sizes in a.
static int64_t lay_out(const wushkv_cache *c, int32_t mode, int32_t n_q, int64_t items, int64_t max_tok, int64_t max_sel,
                       uint8_t *ws, RowsArgs &a)
{
    const int64_t G = n_q / c->n_kv_heads, hk = c->n_kv_heads, B = c->batch, d = c->head_dim, tokens = items * max_tok;
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t was = at;
        at += (bytes + 255) / 256 * 256;
        return ws + was;
    };
    a.cus = (int32_t)compute_units();
    a.wgs = (int32_t)std::min<int64_t>(std::max<int64_t>(kRowsPerCu * compute_units() / hk, 1), kMaxWgs);
    a.inverse = a.wgs > 1 ? UINT64_MAX / (uint64_t)a.wgs + 1 : UINT64_MAX;
    // (cross: a stored sequence's last tile may be short)
    const int64_t tiles = mode == kPrefix ? 2 * B : mode == kWeighted ? B : (tokens * G + kTileRows - 1) / kTileRows + (items < B ? items : B);
    a.part_rows = mode == kPrefix ? 2 * B * G + kTileRows * (int64_t)a.wgs
                  : mode == kWeighted ? B * G + G * (int64_t)a.wgs : 2 * kTileRows * (int64_t)a.wgs;
    a.qlimb = take(hk * tokens * G * kLimbRoom * 128);
    a.qaux = reinterpret_cast<uint32_t *>(take(hk * tokens * G * 16));
    a.qt = reinterpret_cast<float *>(take(hk * tokens * G * d * 4));
    a.part = reinterpret_cast<float *>(take(hk * a.part_rows * d * 4));
    a.part_ml = reinterpret_cast<float *>(take(hk * a.part_rows * 8));
    if (mode == kWeighted) a.stat = reinterpret_cast<float *>(take(hk * B * max_sel * G * 8));
    int64_t p = sizeof(RowPlan);
    auto within = [&](int64_t bytes) {
        const int64_t was = p;
        p += (bytes + 15) / 16 * 16;
        return (int32_t)was;
    };
    a.bound_at = within(8 * ((int64_t)a.wgs + 1));
    a.wg_at = within(4 * (int64_t)a.wgs);
    a.tile_at = within(sizeof(RowTile) * tiles);
    a.small_at = within(4 * tiles);
    a.before_at = within(4 * tiles);
    a.tok_at = within(4 * (mode == kPrefix ? 2 * B : tokens));
    a.lim_at = within(mode == kPrefix ? 8 * B : 0);
    a.map_at = within(mode == kPrefix ? 8 * B : 0);
    a.plan_bytes = (p + 255) / 256 * 256;
    a.plan = take(hk * a.plan_bytes);
    // the plans' offsets are 32 bits wide
    return p < (1ll << 31) ? at : 0;
}

static int check_rows(const wushkv_cache *c, int32_t n_q)
{
    const int st = wushkv_validate_cache(c);
    if (st != WUSHKV_OK) return st;
    if (n_q <= 0 || n_q % c->n_kv_heads != 0) return WUSHKV_EINVAL;
    const int32_t G = n_q / c->n_kv_heads;
    if (G > 8 || (G & (G - 1)) != 0 || c->n_kv_heads > 65535) return WUSHKV_EUNSUPPORTED;
    return WUSHKV_OK;
}

template <int D, int BITS>
static void launch_rows(const RowsArgs &a, hipStream_t s)
{
    const int64_t groups = (((int64_t)a.items * a.max_tok << a.g_log2) + 15) / 16;
    const dim3 gq(a.n_kv, 1 + (unsigned)((groups + a.reps - 1) / a.reps)), gm(a.n_kv, a.wgs);
    launch("rows_query_kernel", rows_query_kernel<D, BITS>, gq, dim3(64 * kQtWaves<D>), s, a);
    if (a.mode == kWeighted) launch("rows_kernel", rows_kernel<D, BITS, true>, gm, dim3(256), s, a);
    else launch("rows_kernel", rows_kernel<D, BITS, false>, gm, dim3(256), s, a);
    if (a.mode != kCross) launch("rows_merge_kernel", rows_merge_kernel<D>, dim3(a.n_kv, a.batch), dim3(256), s, a);
    else if (a.wgs > 1) launch("rows_join_kernel", rows_join_kernel<D>, dim3(a.n_kv, a.wgs - 1, kTileRows / 4), dim3(256), s, a);
}

static int attend_rows(const wushkv_cache *c, RowsArgs &a, int32_t n_q, int64_t max_sel, float sm_scale, void *workspace,
                       size_t workspace_bytes, wushkv_stream_t stream)
{
    if (!a.q || !a.tinv || !a.out || !workspace) return WUSHKV_EINVAL;
    if (((uintptr_t)a.q | (uintptr_t)a.tinv | (uintptr_t)a.out | (uintptr_t)workspace) & 15u) return WUSHKV_EINVAL;
    if (!(sm_scale > 0.0f) || sm_scale == INFINITY) return WUSHKV_EINVAL;
    const int64_t need = lay_out(c, a.mode, n_q, a.items, a.max_tok, max_sel, reinterpret_cast<uint8_t *>(workspace), a);
    if (need == 0) return WUSHKV_EUNSUPPORTED;
    if (workspace_bytes < (size_t)need) return WUSHKV_EWORKSPACE;
    a.pages = c->pages;
    a.page_table = c->page_table;
    a.win_k = c->win_k;
    a.win_v = c->win_v;
    a.seq_len = c->seq_len;
    a.quant_end = c->quant_end;
    a.batch = c->batch;
    a.n_kv = c->n_kv_heads;
    a.s_sink = c->s_sink;
    a.win_slots = c->win_slots;
    a.max_pages = c->n_pages > 0 ? c->max_pages_per_seq : 0;
    a.n_pages = c->n_pages;
    a.g_log2 = __builtin_ctz(n_q / c->n_kv_heads);
    a.scale = sm_scale * kLog2e;
    a.mid = 0.5f * ((1 << c->bits) - 1);
    const int64_t groups = (((int64_t)a.items * a.max_tok << a.g_log2) + 15) / 16;
    // (two where there is more than one round of workgroups: 49.7 us for 65536 rows, 51.3
    // with up to four, 61.9 with up to eight)
    const int64_t round = 3 * compute_units();
    a.reps = (int32_t)std::min<int64_t>((groups * a.n_kv + round - 1) / round, kReps);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    switch (c->head_dim * 10 + storage_bits(c->bits)) {
        case 1282: launch_rows<128, 2>(a, s); break;
        case 1284: launch_rows<128, 4>(a, s); break;
        case 642: launch_rows<64, 2>(a, s); break;
        case 644: launch_rows<64, 4>(a, s); break;
    }
    return hipGetLastError() != hipSuccess ? WUSHKV_ELAUNCH : WUSHKV_OK;
}

static int check_prefix(const wushkv_cache *c, int32_t n_q)
{
    const int st = check_rows(c, n_q);
    return st != WUSHKV_OK ? st : c->batch > kMaxRowItems ? WUSHKV_EUNSUPPORTED : WUSHKV_OK;
}

extern "C" size_t wushkv_prefix_workspace_bytes(const wushkv_cache *c, int32_t n_q_heads)
{
    RowsArgs a{};
    return check_prefix(c, n_q_heads) != WUSHKV_OK ? 0 : (size_t)lay_out(c, kPrefix, n_q_heads, c->batch, 1, 0, nullptr, a);
}

extern "C" int wushkv_prefix_attention(const wushkv_cache *c, const uint16_t *q, int32_t n_q_heads, const int32_t *leader,
                                       const int32_t *shared, const float *t_k_inv, float sm_scale, float *out,
                                       void *workspace, size_t workspace_bytes, wushkv_stream_t stream)
{
    const int st = check_prefix(c, n_q_heads);
    if (st != WUSHKV_OK) return st;
    if (!leader || !shared || ((uintptr_t)leader | (uintptr_t)shared) & 15u) return WUSHKV_EINVAL;
    RowsArgs a{};
    a.mode = kPrefix;
    a.items = c->batch;
    a.max_tok = 1;
    a.q = q;
    a.tinv = t_k_inv;
    a.out = out;
    a.of = leader;
    a.count = shared;
    return attend_rows(c, a, n_q_heads, 0, sm_scale, workspace, workspace_bytes, stream);
}

static int check_cross(const wushkv_cache *c, int32_t n_seqs, int32_t max_tok, int32_t n_q)
{
    const int st = check_rows(c, n_q);
    if (st != WUSHKV_OK) return st;
    if (n_seqs < 1 || max_tok < 1) return WUSHKV_EINVAL;
    // (tokens and their rows are counted in 32 bits, their groups in a grid)
    if (n_seqs > kMaxRowItems || (int64_t)n_seqs * max_tok > (1 << 17)) return WUSHKV_EUNSUPPORTED;
    return WUSHKV_OK;
}

extern "C" size_t wushkv_cross_workspace_bytes(const wushkv_cache *c, int32_t n_seqs, int32_t max_tok, int32_t n_q_heads)
{
    RowsArgs a{};
    if (check_cross(c, n_seqs, max_tok, n_q_heads) != WUSHKV_OK) return 0;
    return (size_t)lay_out(c, kCross, n_q_heads, n_seqs, max_tok, 0, nullptr, a);
}

extern "C" int wushkv_cross_attention(const wushkv_cache *c, const uint16_t *q, int32_t n_seqs, const int32_t *n_tok,
                                      int32_t max_tok, const int32_t *source, int32_t n_q_heads, const float *t_k_inv,
                                      float sm_scale, float *out, void *workspace, size_t workspace_bytes,
                                      wushkv_stream_t stream)
{
    const int st = check_cross(c, n_seqs, max_tok, n_q_heads);
    if (st != WUSHKV_OK) return st;
    if (((uintptr_t)n_tok | (uintptr_t)source) & 15u) return WUSHKV_EINVAL;
    if (!source && n_seqs > c->batch) return WUSHKV_EINVAL;
    RowsArgs a{};
    a.mode = kCross;
    a.items = n_seqs;
    a.max_tok = max_tok;
    a.q = q;
    a.tinv = t_k_inv;
    a.out = out;
    a.of = source;
    a.count = n_tok;
    return attend_rows(c, a, n_q_heads, 0, sm_scale, workspace, workspace_bytes, stream);
}

// Entries of a row's list: of all pages, a page table's row.
static int64_t weighted_width(const wushkv_cache *c, int32_t max_sel) { return max_sel < 0 ? c->max_pages_per_seq : max_sel; }

extern "C" size_t wushkv_weighted_workspace_bytes(const wushkv_cache *c, int32_t n_q_heads, int32_t max_sel)
{
    RowsArgs a{};
    if (check_rows(c, n_q_heads) != WUSHKV_OK || c->batch > 65535) return 0;
    return (size_t)lay_out(c, kWeighted, n_q_heads, c->batch, 1, weighted_width(c, max_sel), nullptr, a);
}

extern "C" int wushkv_weighted_attention(const wushkv_cache *c, const uint16_t *q, int32_t n_q_heads, const int32_t *sel,
                                         const int32_t *n_sel, int32_t max_sel, const float *t_k_inv, float sm_scale,
                                         float *weights, float *out, void *workspace, size_t workspace_bytes,
                                         wushkv_stream_t stream)
{
    const int st = check_rows(c, n_q_heads);
    if (st != WUSHKV_OK) return st;
    if (c->batch > 65535) return WUSHKV_EUNSUPPORTED;
    if (!weights || ((uintptr_t)weights | (uintptr_t)sel | (uintptr_t)n_sel) & 15u) return WUSHKV_EINVAL;
    // a list, or neither list nor counts (max_sel -1)
    if (max_sel < 0 ? max_sel != -1 || sel || n_sel : !n_sel || (!sel && max_sel > 0)) return WUSHKV_EINVAL;
    RowsArgs a{};
    a.mode = kWeighted;
    a.items = c->batch;
    a.max_tok = 1;
    a.q = q;
    a.tinv = t_k_inv;
    a.out = out;
    a.sel = sel;
    a.n_sel = n_sel;
    a.max_sel = (int32_t)weighted_width(c, max_sel);
    a.weights = weights;
    return attend_rows(c, a, n_q_heads, a.max_sel, sm_scale, workspace, workspace_bytes, stream);
}
