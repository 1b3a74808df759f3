// Attention of many query rows over stored sequences, where several queries have
// a sequence, or its first pages, in common:
//   wushkv_prefix_attention    decode queries; pages shared at the start of several
//                              sequences are attended to once for all of them
//   wushkv_cross_attention     query sequences of any length over whole stored ones
//   wushkv_weighted_attention  decode queries, adding up what each page received
//
// Launches on the caller's stream:
//   rows_query_kernel  q~ = q T_K^{-1} of 16 rows at a time with its digit limbs
//                      (for the pages) and three bf16 parts (for the windows); and,
//                      in a workgroup per kv head, the plan: tiles and how they are
//                      shared out (below).
//   rows_kernel        one residency round of workgroups over the plan.
//   rows_merge_kernel / rows_join_kernel   what several workgroups have of a row,
//                      merged; the pages' weights.
//
// Plan.  A tile is up to 32 query rows ((token, query head) pairs) with a run of a
// stored sequence's pages and, where it is the rows' own sequence, its windows.
// Prefix: a tile of its own pages and windows per sequence, and tiles of the
// sequences that have a leader (sorted by what they share with it, longest first,
// so that a tile's rows end at about the same page).  Cross: the tokens of all query
// sequences of one stored sequence, 32 rows at a time.  The tiles' costs stand one
// behind the other on a line, of which every workgroup takes the same share: a
// workgroup may take a part of one tile or several tiles, and no length is known
// to the host.  Within a workgroup the four waves take every fourth page each and
// merge in LDS at the tile's end.
//
// Pages.  As in decode_main_kernel, scores are scaled products of q~'s digit limbs
// with the key codes, here with 16 query rows as the product's rows, one product a
// limb; keys are centred (k = s (c - mid) + (z + mid s)).  A wave reads a page's
// codes and parameters from memory in operand order into registers, the next page's
// while it computes.  Lane (j, n) has rows 4 j + r of tokens 4 n + t.  A row's
// softmax has a reference that stays kLift below its maximum at the time and moves
// only when a weight would pass 2^kGrow, so that a page costs one test.  Weights
// p s go through LDS as fp16 hi + lo parts, each formed from the exact product, to
// be the rows of the P V products with the value codes as fp16 numbers 16 c.  The
// value scales are brought to about one by a power of two that the wave keeps
// (tiny scales would leave the lo parts no bits); sums of p z and p are fp32.
//
// Windows.  q~ and weights in three bf16 parts, 64 slots at a time.
#include <atomic>
#include <cfloat>

#include "query.h"

namespace wushkv {

constexpr int kMaxRowItems = 1024;  // sequences that a plan sorts
constexpr int kTileRows = 32;

// Tiles of one stored sequence's pages for up to 32 query rows.
struct RowTile {
    int32_t seq;             // whose page table, list and windows
    int32_t first, n_pages;  // page units: logical pages (or list entries) first ..
    int32_t n_win;           // then 64-slot window units
    int32_t rows;            // query rows
    int32_t tok;             // its first entry in the token list
    int32_t limit;           // below it every row attends to a page
    int32_t part;            // its first partial row, -1: written out directly
    int32_t wg0, n_wg;       // workgroups that have a part of it
    int64_t cost0;
};

// Per kv head, at the start of its plan.
struct RowPlan {
    int64_t share, total;  // of a workgroup, of all tiles
    int32_t n_tiles, pad[3];
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
    uint16_t *qpart;              // bf16 [n_kv][tokens][G][3][D]
    uint8_t *plan;                // per kv head plan_bytes
    int64_t plan_bytes;
    int32_t wg_at, tile_at, tok_at, lim_at, map_at;  // offsets in a plan
    int32_t wgs;                  // workgroups of rows_kernel per kv head
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

// Costs of a page and of a window unit, by the rows' tiles of 16.
__device__ __forceinline__ int32_t page_cost(int32_t rows) { return rows > 16 ? 3 : 2; }
__device__ __forceinline__ int32_t window_cost(int32_t rows) { return 2 * page_cost(rows); }
constexpr int64_t kLeastShare = 8;

// The unit that begins at or after place x of a tile's cost.
__device__ __forceinline__ int32_t unit_at(const RowTile &t, int64_t x)
{
    const int32_t cp = page_cost(t.rows), cw = window_cost(t.rows);
    if (x <= 0) return 0;
    const int64_t pages = (int64_t)t.n_pages * cp;
    if (x <= pages) return (int32_t)((x + cp - 1) / cp);
    const int64_t w = (x - pages + cw - 1) / cw;
    return t.n_pages + (int32_t)(w < t.n_win ? w : t.n_win);
}

// Exclusive prefix sum over the workgroup's threads, and the total.
__device__ __forceinline__ int64_t block_scan64(int64_t x, int64_t *sums, int64_t &total)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = blockDim.x >> 6;
    int64_t in = x;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const int64_t y = __shfl_up(in, s);
        if (lane >= s) in += y;
    }
    __syncthreads();  // the last call's sums are read
    if (lane == 63) sums[wave] = in;
    __syncthreads();
    int64_t before = 0, all = 0;
    for (int w = 0; w < waves; ++w) {
        const int64_t v = sums[w];
        if (w < wave) before += v;
        all += v;
    }
    total = all;
    return before + in - x;
}

struct PlanLds {
    int32_t group[kMaxRowItems], len[kMaxRowItems], most[kMaxRowItems], order[kMaxRowItems], flag[kMaxRowItems];
    int64_t sums[16];
};

// The tiles' places on the line of costs, the workgroups' shares and the partial
// rows; all threads, after the tiles are written.
__device__ __forceinline__ void share_out(const RowsArgs &a, int h, int32_t n_tiles, PlanLds &lds)
{
    const int tid = threadIdx.x, nt = blockDim.x;
    RowTile *tiles = plan_part<RowTile>(a, h, a.tile_at);
    int32_t *wg_tile = plan_part<int32_t>(a, h, a.wg_at);
    __syncthreads();
    int64_t total = 0;
    for (int32_t t0 = 0; t0 < n_tiles; t0 += nt) {
        const int32_t t = t0 + tid;
        int64_t cost = 0;
        if (t < n_tiles)
            cost = (int64_t)tiles[t].n_pages * page_cost(tiles[t].rows) + (int64_t)tiles[t].n_win * window_cost(tiles[t].rows);
        int64_t all;
        const int64_t at = block_scan64(cost, lds.sums, all);
        if (t < n_tiles) tiles[t].cost0 = total + at;
        total += all;
    }
    int64_t share = (total + a.wgs - 1) / a.wgs;
    share = share > kLeastShare ? share : kLeastShare;
    int64_t rows_before = 0;
    for (int32_t t0 = 0; t0 < n_tiles; t0 += nt) {
        const int32_t t = t0 + tid;
        int64_t need = 0;
        int32_t w0 = 0, w1 = -1;
        if (t < n_tiles) {
            const RowTile &x = tiles[t];
            const int64_t cost = (int64_t)x.n_pages * page_cost(x.rows) + (int64_t)x.n_win * window_cost(x.rows);
            if (cost > 0) {
                w0 = (int32_t)(x.cost0 / share);
                w1 = (int32_t)((x.cost0 + cost - 1) / share);
                // the workgroups whose share begins in the tile
                for (int32_t w = x.cost0 == (int64_t)w0 * share ? w0 : w0 + 1; w <= w1; ++w) wg_tile[w] = t;
            }
            if (!(a.mode == kCross && w1 <= w0)) need = (int64_t)(w1 - w0 + 1) * x.rows;
        }
        int64_t all;
        const int64_t at = block_scan64(need, lds.sums, all);
        if (t < n_tiles) {
            tiles[t].wg0 = w0;
            tiles[t].n_wg = w1 - w0 + 1;
            tiles[t].part = need > 0 ? (int32_t)(rows_before + at) : -1;
        }
        rows_before += all;
    }
    if (tid == 0) *plan_of(a, h) = RowPlan{share, total, n_tiles, {0, 0, 0}};
}

__device__ __forceinline__ void plan_prefix(const RowsArgs &a, int h, PlanLds &lds)
{
    const int tid = threadIdx.x, nt = blockDim.x;
    const int32_t B = a.batch, G = 1 << a.g_log2, per = kTileRows >> a.g_log2;
    RowTile *tiles = plan_part<RowTile>(a, h, a.tile_at);
    int32_t *toks = plan_part<int32_t>(a, h, a.tok_at), *lims = plan_part<int32_t>(a, h, a.lim_at);
    int32_t *map = plan_part<int32_t>(a, h, a.map_at);
    for (int32_t b = tid; b < B; b += nt) {
        lds.order[b] = (quantised_end(a, b) - a.s_sink) / kPage;  // complete pages
        lds.most[b] = 0;
    }
    __syncthreads();
    for (int32_t b = tid; b < B; b += nt) {
        const int32_t l = a.of[b];
        int32_t s = 0;
        if (l >= 0 && l < B && l != b) s = max(min(min(a.count[b], a.max_pages), min(lds.order[b], lds.order[l])), 0);
        lds.group[b] = s > 0 ? l : -1;
        lds.len[b] = s;
        if (s > 0) atomicMax(&lds.most[l], s);
    }
    __syncthreads();
    for (int32_t b = tid; b < B; b += nt) {
        if (lds.group[b] < 0 && lds.most[b] > 0) {  // a leader goes with its sequences
            lds.group[b] = b;
            lds.len[b] = lds.most[b];
        }
        lds.flag[b] = 0;
    }
    __syncthreads();
    // the sequences by leader, then by pages shared (longest first), then by number
    int32_t at[(kMaxRowItems + 255) / 256], in_group[(kMaxRowItems + 255) / 256];
    int k = 0;
    for (int32_t b = tid; b < B; b += nt, ++k) {
        at[k] = in_group[k] = 0;
        const int32_t g = lds.group[b], s = lds.len[b];
        if (g < 0) continue;
        for (int32_t c = 0; c < B; ++c) {
            const int32_t gc = lds.group[c], sc = lds.len[c];
            const bool mate = gc == g && (sc > s || (sc == s && c < b));
            at[k] += (gc >= 0 && gc < g) || mate;
            in_group[k] += mate;
        }
        lds.flag[at[k]] = in_group[k] % per == 0;
    }
    __syncthreads();
    k = 0;
    for (int32_t b = tid; b < B; b += nt, ++k)
        if (lds.group[b] >= 0) lds.order[at[k]] = b;
    __syncthreads();
    // tiles in that order, behind the sequences' own
    int32_t n_tiles = B, n_sorted = 0;
    for (int32_t b = 0; b < B; ++b) n_sorted += lds.group[b] >= 0;
    for (int32_t p0 = 0; p0 < B; p0 += nt) {
        const int32_t p = p0 + tid;
        const bool start = p < n_sorted && lds.flag[p] != 0;
        int64_t all;
        const int32_t before = (int32_t)block_scan64(start, lds.sums, all);
        if (p < n_sorted) {
            const int32_t b = lds.order[p], t = n_tiles + before + (start ? 1 : 0) - 1;
            toks[B + p] = b;
            lims[B + p] = lds.len[b];
            map[2 * b] = t;
            lds.most[p] = t;  // (the counts it held are used)
            if (start) {
                int32_t n = 1;
                while (n < per && p + n < n_sorted && lds.flag[p + n] == 0) ++n;
                tiles[t] = RowTile{lds.group[b], 0, lds.len[b], 0, n * G, B + p, lds.len[lds.order[p + n - 1]], -1, 0, 0, 0};
            }
        }
        n_tiles += (int32_t)all;
    }
    for (int32_t b = tid; b < B; b += nt) {
        const int32_t S = a.seq_len[b], s = lds.len[b];
        const int32_t pages = min((quantised_end(a, b) - a.s_sink + kPage - 1) / kPage, a.max_pages);
        tiles[b] = RowTile{b, s, max(pages - s, 0), S > 0 ? a.win_slots / kPage : 0, G, b, INT32_MAX, -1, 0, 0, 0};
        toks[b] = b;
        if (lds.group[b] < 0) map[2 * b] = -1;
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
        lds.len[i] = item_tokens(a, i, src);
        lds.group[i] = lds.len[i] > 0 ? src : -1;
    }
    __syncthreads();
    // the token list goes by stored sequence, then by query sequence
    int32_t start[(kMaxRowItems + 255) / 256], all_of[(kMaxRowItems + 255) / 256];
    int k = 0;
    for (int32_t i = tid; i < N; i += nt, ++k) {
        const int32_t g = lds.group[i];
        int32_t at = 0, first = 0, sum = 0;
        for (int32_t c = 0; g >= 0 && c < N; ++c) {
            const int32_t gc = lds.group[c], n = lds.len[c];
            if (gc < 0) continue;
            if (gc < g) first += n;
            if (gc == g) sum += n;
            if (gc < g || (gc == g && c < i)) at += n;
        }
        lds.order[i] = at;
        lds.most[i] = g >= 0 && at == first ? (sum + per - 1) / per : 0;  // tiles, at a stored sequence's first
        start[k] = first;
        all_of[k] = sum;
    }
    __syncthreads();
    k = 0;
    for (int32_t i = tid; i < N; i += nt, ++k) {
        int32_t before = 0;
        for (int32_t c = 0; lds.most[i] > 0 && c < N; ++c)
            if (lds.most[c] > 0 && lds.group[c] < lds.group[i]) before += lds.most[c];
        lds.flag[i] = before;
    }
    int32_t n_tiles = 0;
    for (int32_t c = 0; c < N; ++c) n_tiles += lds.most[c];
    k = 0;
    for (int32_t i = tid; i < N; i += nt, ++k) {
        const int32_t b = lds.group[i];
        if (lds.most[i] == 0) continue;
        const int32_t pages = min((quantised_end(a, b) - a.s_sink + kPage - 1) / kPage, a.max_pages);
        for (int32_t x = 0; x < lds.most[i]; ++x)
            tiles[lds.flag[i] + x] = RowTile{b, 0, pages, a.win_slots / kPage, min(per, all_of[k] - x * per) * G,
                                             start[k] + x * per, INT32_MAX, -1, 0, 0, 0};
    }
    for (int32_t i = tid >> 6; i < N; i += nt >> 6)
        for (int32_t t = tid & 63; t < lds.len[i]; t += 64) toks[lds.order[i] + t] = i * a.max_tok + t;
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

template <int D, int BITS>
__global__ void __launch_bounds__(64 * kQtWaves<D>) rows_query_kernel(RowsArgs a)
{
    constexpr int R = 16, NT = 64 * kQtWaves<D>;
    using Q = QueryLds<D, R>;
    constexpr int kBytes = Q::kBytes > (int)sizeof(PlanLds) ? Q::kBytes : (int)sizeof(PlanLds);
    __shared__ __attribute__((aligned(16))) uint8_t lds[kBytes];
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
    for (int rep = 0; rep < a.reps; ++rep) {
        const int64_t row0 = ((int64_t)(blockIdx.y - 1) * a.reps + rep) * R;
        if (row0 >= rows) return;
        const int n = (int)(rows - row0 < R ? rows - row0 : R);
        uint16_t *qs = reinterpret_cast<uint16_t *>(lds);
        __syncthreads();
        for (int i = tid; i < R * D / 8; i += NT) {
            const int r = i / (D / 8), c = 8 * (i % (D / 8));
            u32x4 x = {0u, 0u, 0u, 0u};
            if (r < n) {
                const int64_t tok = (row0 + r) >> a.g_log2;
                const int32_t g = (int32_t)(row0 + r) & (G - 1);
                const int64_t at = ((tok * a.n_kv + h) * G + g) * D + c;
                int32_t src;
                // (rows of no token: zeros out)
                const bool there = a.mode != kCross ||
                                   tok % a.max_tok < item_tokens(a, (int32_t)(tok / a.max_tok), src);
                if (there) {
                    x = *reinterpret_cast<const u32x4 *>(a.q + at);
                } else {
                    *reinterpret_cast<f32x4 *>(a.out + at) = f32x4{0.f, 0.f, 0.f, 0.f};
                    *reinterpret_cast<f32x4 *>(a.out + at + 4) = f32x4{0.f, 0.f, 0.f, 0.f};
                }
            }
            *reinterpret_cast<u32x4 *>(qs + r * Q::kQPitch + c) = x;
        }
        form_qt_mfma<D, R>(a.scale, tc, lds, tid);
        const int64_t to = (int64_t)h * rows + row0;
        const float *qt = reinterpret_cast<const float *>(lds);
        for (int i = tid; i < n * D / 4; i += NT) {
            const int r = i / (D / 4), c = 4 * (i % (D / 4));
            const f32x4 x = *reinterpret_cast<const f32x4 *>(qt + r * D + c);
            float e[4] = {x[0], x[1], x[2], x[3]};
            uint16_t *dst = a.qpart + (to + r) * 3 * D + c;
#pragma unroll
            for (int part = 0; part < 3; ++part) {
                const uint32_t u0 = pack_bf16_rne(e[0], e[1]), u1 = pack_bf16_rne(e[2], e[3]);
                *reinterpret_cast<uint2 *>(dst + part * D) = uint2{u0, u1};
                e[0] -= bf16_bits_to_f32(u0 & 0xFFFFu);
                e[1] -= bf16_bits_to_f32(u0 >> 16);
                e[2] -= bf16_bits_to_f32(u1 & 0xFFFFu);
                e[3] -= bf16_bits_to_f32(u1 >> 16);
            }
        }
        form_limbs<D, BITS, R, kQtWaves<D>>(lds, tid);
        for (int i = tid; i < n * kLimbRoom * 128 / 16; i += NT)
            reinterpret_cast<u32x4 *>(a.qlimb + to * kLimbRoom * 128)[i] = reinterpret_cast<const u32x4 *>(lds)[i];
        if (tid < n * 4) a.qaux[to * 4 + tid] = reinterpret_cast<const uint32_t *>(lds + Q::kAux)[tid];
    }
}

// ------------------------------------------------------------------ the rows

// Weights: at most 2^kGrow, about 2^kLift at a new maximum (fp16 holds nothing
// below 2^-24, where the lo parts of small weights would be lost); the windows'
// reference lies 2^kRoom above the maximum, so that sums of values near bf16's
// largest stay finite.
constexpr float kLift = 4.0f, kGrow = 8.0f, kRoom = 12.0f;

template <int D>
struct RowsLds {
    static constexpr int kWave = kTileRows * D * 4 > 3 * kTileRows * 128 ? kTileRows * D * 4 : 3 * kTileRows * 128;
    static constexpr int kMl = 4 * kWave;  // m, then l: float [4][32] each
    static constexpr int kBytes = kMl + 2 * 4 * kTileRows * 4;
};

// Physical page of page unit i of stored sequence b, or -1; lp: its logical page.
__device__ __forceinline__ int32_t page_entry(const RowsArgs &a, int32_t b, int h, int32_t i, int32_t end, int32_t &lp)
{
    lp = a.sel != nullptr ? a.sel[((int64_t)b * a.n_kv + h) * a.max_sel + i] : i;
    if (lp < 0 || lp >= a.max_pages || (int64_t)lp * kPage >= end - a.s_sink) return -1;
    const int32_t phys = a.page_table[(int64_t)b * a.max_pages + lp];
    return phys >= 0 && phys < a.n_pages ? phys : -1;
}

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
            k[i] = *reinterpret_cast<const u32x4 *>(pg + 4 * L::k_word(lane % L::kKLanes, 4 * i));
    }
    __device__ __forceinline__ void load_values(const uint8_t *pg, int lane)
    {
#pragma unroll
        for (int i = 0; i < kVX; ++i)
            v[i] = *reinterpret_cast<const u32x4 *>(pg + L::kRegionBytes + 4 * L::v_word(lane, 4 * i));
    }
    __device__ __forceinline__ void load_params(const uint8_t *pg, int n)
    {
        kp = *reinterpret_cast<const u32x4 *>(pg + L::kParamOffset + 16 * n);
        vp = *reinterpret_cast<const u32x4 *>(pg + L::kParamOffset + 4 * kPage + 16 * n);
    }
};

// The wave's own LDS writes come before its reads behind this, and the reverse (its
// accesses complete in order; this holds the compiler to it).
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// One tile of 16 rows: the running softmax of rows 4 j + r.
template <int D>
struct RowState {
    f32x4 acc[D / 16];  // sums of p s 16 c (pages) or p v (windows), channels 16 nt + n
    f32x4 m, l, z;      // reference, sum of p, sum of p z (the lane's tokens)
};

// Moves the references up: the largest logit of each row over the wave's row of
// lanes less lift.
template <int D>
__device__ __forceinline__ void raise_reference(RowState<D> &s, const f32x4 &top, float lift)
{
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float m_new = fmaxf(s.m[r], row_max16(top[r]) - lift);
        const float f = fexp2(s.m[r] - m_new);
        s.m[r] = m_new;
        s.l[r] *= f;
        s.z[r] *= f;
#pragma unroll
        for (int nt = 0; nt < D / 16; ++nt) s.acc[nt][r] *= f;
    }
}

template <int D, int BITS, int RT, bool WEIGH>
__device__ __forceinline__ void take_tile(const RowsArgs &a, const RowTile &tile, int32_t lo, int32_t hi, int32_t slot,
                                          uint8_t *lds, int h)
{
    using L = Layout<D, BITS>;
    using LB = Limbs<BITS>;
    constexpr int kNT = L::kNTiles, kC = L::kChunks, kScaleB = BITS == 2 ? 128 : 136;
    constexpr int kPlane = RT * 16 * 128;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int j = lane >> 4, n = lane & 15;
    const int32_t G = 1 << a.g_log2, b = tile.seq;
    const int64_t rows_all = (int64_t)a.items * a.max_tok << a.g_log2;
    const int32_t *toks = plan_part<int32_t>(a, h, a.tok_at) + tile.tok;
    const int32_t S = a.seq_len[b], q_hi = quantised_end(a, b);
    uint8_t *mine = lds + wave * RowsLds<D>::kWave;
    const uint32_t pbuf = lds_addr(mine);
    // (query row r of the tile, in the workspace's order)
    auto row_at = [&](int r) -> int64_t { return h * rows_all + ((int64_t)toks[r >> a.g_log2] << a.g_log2) + (r & (G - 1)); };

    RowState<D> st[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt) st[rt].acc[nt] = f32x4{0.f, 0.f, 0.f, 0.f};
        st[rt].m = f32x4{-FLT_MAX, -FLT_MAX, -FLT_MAX, -FLT_MAX};
        st[rt].l = st[rt].z = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    float unit = 1.0f;  // what acc is counted in

    const int32_t page_hi = min(hi, tile.n_pages);
    if (lo < page_hi) {
        // ============================================ pages
        // operands: limb l of row 16 rt + n, and the digit sums by products with
        // keys of code 1 (every column the same), from which the products start
        i32x8 qa[RT][LB::kCount];
        int sc03[RT], sc45[RT];
        f32x4 zs[RT], from[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int r = 16 * rt + n;
            const int64_t row = r < tile.rows ? row_at(r) : -1;
            sc03[rt] = sc45[rt] = 0x7F7F7F7F;
            if (row >= 0) {
                sc03[rt] = (int)a.qaux[4 * row];
                sc45[rt] = (int)a.qaux[4 * row + 1];
            }
#pragma unroll
            for (int l = 0; l < LB::kCount; ++l) {
                u32x4 x0 = {0u, 0u, 0u, 0u}, x1 = x0;
                if (row >= 0) {
                    const uint8_t *src = a.qlimb + (row * kLimbRoom + l) * 128 + 32 * j;
                    x0 = *reinterpret_cast<const u32x4 *>(src);
                    if constexpr (BITS == 2) {
                        const u32x2 y = *reinterpret_cast<const u32x2 *>(src + 16);
                        x1 = u32x4{y[0], y[1], 0u, 0u};
                    } else {
                        x1 = *reinterpret_cast<const u32x4 *>(src + 16);
                    }
                }
                qa[rt][l] = i32x8{(int)x0[0], (int)x0[1], (int)x0[2], (int)x0[3], (int)x1[0], (int)x1[1], (int)x1[2], (int)x1[3]};
            }
        }
        auto products = [&](int rt, const i32x8 (&bop)[4], f32x4 (&c)[4]) {
            limb_products<BITS, 0, kScaleB>(qa[rt][0], bop, sc03[rt], c);
            limb_products<BITS, 1, kScaleB>(qa[rt][1], bop, sc03[rt], c);
            limb_products<BITS, 2, kScaleB>(qa[rt][2], bop, sc03[rt], c);
            limb_products<BITS, 3, kScaleB>(qa[rt][3], bop, sc03[rt], c);
            limb_products<BITS, 4, kScaleB>(qa[rt][4], bop, sc45[rt], c);
            if constexpr (LB::kCount > 5) limb_products<BITS, 5, kScaleB>(qa[rt][5], bop, sc45[rt], c);
        };
        {
            const int one = BITS == 2 ? 0x11111111 : 0x01010101;
            const i32x8 o = BITS == 2 ? i32x8{one, one, one, one, 0, 0, 0, 0} : i32x8{one, one, one, one, one, one, one, one};
            const i32x8 ones[4] = {o, o, o, o};
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                f32x4 c[4] = {};
                products(rt, ones, c);
                zs[rt] = c[0];
                from[rt] = c[0] * -a.mid;
            }
        }
        WidenNormal<BITS> wide;
        wide.init();
        float vmul = 1.0f;      // a power of two that brings value scales to at most 8
        uint32_t vmost = 0u;    // the largest scale that it serves (fp16 bits)

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
            for (; todo != 0;) {
                todo &= todo - 1;
                const int next = todo != 0 ? __builtin_ctzll(todo) : cur;
                const uint8_t *np = page_at(next);
                const int32_t clp = __builtin_amdgcn_readlane(lp, cur);
                const int32_t nvalid = min(kPage, q_hi - (a.s_sink + clp * kPage));
                const bool part = nvalid < kPage || clp >= tile.limit;

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
                float ks[4], kz[4], vs[4], vz[4];
                if (part) {
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        if (4 * n + t >= nvalid) pg.vp[t] = 0u;  // (whatever the page held before)
                }
                const uint32_t big = max(max(pg.vp[0] & 0x7FFFu, pg.vp[1] & 0x7FFFu), max(pg.vp[2] & 0x7FFFu, pg.vp[3] & 0x7FFFu));
                if (__any(big > vmost)) {
                    // the largest scale to between 1/2 and 1, with room for eight times that
                    const float top = fminf(wave_max(f16_bits_to_f32(big)), 65504.0f);
                    int ex;
                    (void)frexpf(top, &ex);
                    const float v_new = ldexpf(1.0f, -ex), f = v_new / vmul;
                    vmul = v_new;
                    vmost = f32_to_f16_bits(fminf(ldexpf(1.0f, ex + 3), 65504.0f));
                    if (vmost >= 0x7BFFu) vmost = 0x7FFFu;
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                        for (int nt = 0; nt < kNT; ++nt) st[rt].acc[nt] *= f;
                }
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    ks[t] = f16_bits_to_f32(pg.kp[t] & 0xFFFFu);
                    kz[t] = fmaf(ks[t], a.mid, f16_bits_to_f32(pg.kp[t] >> 16));
                    vs[t] = f16_bits_to_f32(pg.vp[t] & 0xFFFFu) * vmul;
                    vz[t] = f16_bits_to_f32(pg.vp[t] >> 16);
                }
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    RowState<D> &s = st[rt];
                    f32x4 c[4] = {from[rt], from[rt], from[rt], from[rt]};
                    products(rt, bop, c);
                    if (rt + 1 == RT) {
                        pg.load_keys(np, lane);
                        pg.load_params(np, n);
                    }
                    f32x4 x[4];
                    float most = -INFINITY;
#pragma unroll
                    for (int t = 0; t < 4; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) x[t][r] = fmaf(ks[t], c[t][r], fmaf(kz[t], zs[rt][r], -s.m[r]));
                    // which of the rows and tokens are left out
                    auto hide = [&](f32x4 (&y)[4]) {
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int row = 16 * rt + 4 * j + r;
                            bool out = false;
                            if (clp >= tile.limit && row < tile.rows)
                                out = plan_part<int32_t>(a, h, a.lim_at)[tile.tok + (row >> a.g_log2)] <= clp;
#pragma unroll
                            for (int t = 0; t < 4; ++t)
                                if (out || 4 * n + t >= nvalid) y[t][r] = -INFINITY;
                        }
                    };
                    if (part) hide(x);
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        most = fmaxf(fmaxf(most, fmaxf(x[t][0], x[t][1])), fmaxf(x[t][2], x[t][3]));
                    if (__any(most > kGrow)) {
                        f32x4 y[4];
#pragma unroll
                        for (int t = 0; t < 4; ++t)
#pragma unroll
                            for (int r = 0; r < 4; ++r) y[t][r] = fmaf(ks[t], c[t][r], kz[t] * zs[rt][r]);
                        if (part) hide(y);
                        f32x4 top;
#pragma unroll
                        for (int r = 0; r < 4; ++r) top[r] = fmaxf(fmaxf(y[0][r], y[1][r]), fmaxf(y[2][r], y[3][r]));
                        raise_reference<D>(s, top, kLift);
#pragma unroll
                        for (int t = 0; t < 4; ++t)
#pragma unroll
                            for (int r = 0; r < 4; ++r) x[t][r] = y[t][r] - s.m[r];
                    }
                    f32x4 each = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        f16x2 hi2[2], lo2[2];
                        float p[4];
#pragma unroll
                        for (int t = 0; t < 4; ++t) {
                            p[t] = fexp2(x[t][r]);
                            // (each part rounded from the exact product)
                            const _Float16 ph = (_Float16)fmaf(p[t], vs[t], 0.0f);
                            hi2[t >> 1][t & 1] = ph;
                            lo2[t >> 1][t & 1] = (_Float16)fmaf(p[t], vs[t], -(float)ph);
                            s.z[r] = fmaf(p[t], vz[t], s.z[r]);
                        }
                        each[r] = (p[0] + p[1]) + (p[2] + p[3]);
                        s.l[r] += each[r];
                        const int row = 16 * rt + 4 * j + r;
                        lds_write8(pbuf + tbuf_at(row, 8 * n), __builtin_bit_cast(uint32_t, hi2[0]), __builtin_bit_cast(uint32_t, hi2[1]));
                        lds_write8(pbuf + kPlane + tbuf_at(row, 8 * n), __builtin_bit_cast(uint32_t, lo2[0]), __builtin_bit_cast(uint32_t, lo2[1]));
                    }
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
                        if (rt == 0 && n < 4 && row < tile.rows) {
                            const int64_t at = (((int64_t)h * a.batch + b) * a.max_sel + base + 4 * cur + wave) * G + row;
                            reinterpret_cast<f32x2 *>(a.stat)[at] = f32x2{e, m};
                        }
                    }
                }
                wave_fence();
#pragma unroll
                for (int kc = 0; kc < 2; ++kc) {
                    f16x8 A[RT][2];
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                        for (int p = 0; p < 2; ++p)
                            A[rt][p] = __builtin_bit_cast(f16x8, lds_read16(pbuf + p * kPlane + tbuf_at(16 * rt + n, 64 * kc + 16 * j)));
#pragma unroll
                    for (int uu = 0; uu < 2 * L::kNw; ++uu) {
                        const int w = kc * 2 * L::kNw + uu;
                        uint32_t op[L::kCodesPerWord / 2];
                        wide.word(pg.v[w / 4][w % 4], op);
#pragma unroll
                        for (int p = 0; p < 2; ++p)
#pragma unroll
                            for (int o = 0; o < L::kOpsPerWord; ++o)
#pragma unroll
                                for (int rt = 0; rt < RT; ++rt) {
                                    f32x4 &acc = st[rt].acc[uu * L::kOpsPerWord + o];
                                    acc = mfma16h(A[rt][p], as_op_h(op + 4 * o), acc);
                                }
                    }
                }
                wave_fence();
                pg.load_values(np, lane);
                cur = next;
            }
        }
        unit = 0.0625f / vmul;
    }

    if (hi > tile.n_pages) {
        // ============================================ windows
        const int32_t ring = a.win_slots - a.s_sink;
        const int32_t a0 = S > q_hi ? (q_hi - a.s_sink) % ring : 0;
        const int32_t ring_live = S > q_hi ? S - q_hi : 0;
        const int64_t head = (int64_t)b * a.n_kv + h;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int nt = 0; nt < kNT; ++nt) st[rt].acc[nt] *= unit;
        unit = 1.0f;
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
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                RowState<D> &s = st[rt];
                const int r0 = 16 * rt + n;
                const int64_t row = r0 < tile.rows ? row_at(r0) : -1;
                f32x4 c[4] = {};
#pragma unroll
                for (int ch = 0; ch < kC; ++ch) {
                    bf16x8 qp[3];
#pragma unroll
                    for (int p = 0; p < 3; ++p) {
                        u32x4 x = {0u, 0u, 0u, 0u};
                        if (row >= 0) x = *reinterpret_cast<const u32x4 *>(a.qpart + (row * 3 + p) * D + 32 * ch + 8 * j);
                        qp[p] = __builtin_bit_cast(bf16x8, x);
                    }
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const bf16x8 kx = *reinterpret_cast<const bf16x8 *>(
                            a.win_k + (head * a.win_slots + slot0 + 4 * n + t) * D + 32 * ch + 8 * j);
#pragma unroll
                        for (int p = 2; p >= 0; --p) c[t] = mfma16(qp[p], kx, c[t]);
                    }
                }
                const uint32_t seen = (uint32_t)(live >> (4 * n)) & 15u;
                f32x4 top = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                float most = -INFINITY;
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        if (!((seen >> t) & 1u)) c[t][r] = -INFINITY;
                        top[r] = fmaxf(top[r], c[t][r]);
                        most = fmaxf(most, c[t][r] - s.m[r]);
                    }
                if (__any(most > -kRoom)) raise_reference<D>(s, top, -kRoom);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int at = 16 * rt + 4 * j + r;
                    float p[4];
#pragma unroll
                    for (int t = 0; t < 4; ++t) p[t] = fexp2(c[t][r] - s.m[r]);
                    s.l[r] += (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
                    for (int q = 0; q < 3; ++q) {
                        const uint32_t u0 = pack_bf16_rne(p[0], p[1]), u1 = pack_bf16_rne(p[2], p[3]);
                        lds_write8(pbuf + q * kPlane + tbuf_at(at, 8 * n), u0, u1);
                        p[0] -= bf16_bits_to_f32(u0 & 0xFFFFu);
                        p[1] -= bf16_bits_to_f32(u0 >> 16);
                        p[2] -= bf16_bits_to_f32(u1 & 0xFFFFu);
                        p[3] -= bf16_bits_to_f32(u1 >> 16);
                    }
                }
            }
            wave_fence();
#pragma unroll
            for (int kc = 0; kc < 2; ++kc) {
                bf16x8 A[RT][3];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int p = 0; p < 3; ++p)
                        A[rt][p] = __builtin_bit_cast(bf16x8, lds_read16(pbuf + p * kPlane + tbuf_at(16 * rt + n, 64 * kc + 16 * j)));
                // dead slots' values are zeroed, whatever bits they hold
                const uint32_t bits = (uint32_t)(live >> (32 * kc + 8 * j)) & 255u;
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt) {
                    u32x4 y = *reinterpret_cast<const u32x4 *>(
                        a.win_v + (head * D + 16 * nt + n) * a.win_slots + slot0 + 32 * kc + 8 * j);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        y[i] &= (((bits >> (2 * i)) & 1u) ? 0x0000FFFFu : 0u) | (((bits >> (2 * i + 1)) & 1u) ? 0xFFFF0000u : 0u);
#pragma unroll
                    for (int p = 2; p >= 0; --p)
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt)
                            st[rt].acc[nt] = mfma16(A[rt][p], __builtin_bit_cast(bf16x8, y), st[rt].acc[nt]);
                }
            }
            wave_fence();
        }
    }

    // ---- the four waves' results, merged
    float(*o)[D] = reinterpret_cast<float(*)[D]>(mine);
    float *sm = reinterpret_cast<float *>(lds + RowsLds<D>::kMl), *sl = sm + 4 * kTileRows;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = 16 * rt + 4 * j + r;
            const float z = row_sum16(st[rt].z[r]), l = row_sum16(st[rt].l[r]);
#pragma unroll
            for (int nt = 0; nt < kNT; ++nt) o[row][16 * nt + n] = fmaf(st[rt].acc[nt][r], unit, z);
            if (n == 0) {
                sm[wave * kTileRows + row] = st[rt].m[r] == -FLT_MAX ? -INFINITY : st[rt].m[r];
                sl[wave * kTileRows + row] = l;
            }
        }
    __syncthreads();
    for (int i = tid; i < tile.rows * (D / 4); i += 256) {
        const int r = i / (D / 4), c = i % (D / 4);
        float mx = -INFINITY, l = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) mx = fmaxf(mx, sm[w * kTileRows + r]);
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        if (mx != -INFINITY) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float m = sm[w * kTileRows + r];
                if (m == -INFINITY) continue;
                const float f = fexp2(m - mx);
                l = fmaf(f, sl[w * kTileRows + r], l);
                const f32x4 y = *reinterpret_cast<const f32x4 *>(lds + w * RowsLds<D>::kWave + (r * D + 4 * c) * 4);
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
__global__ void __launch_bounds__(256, 2) rows_kernel(RowsArgs a)
{
    __shared__ __attribute__((aligned(16))) uint8_t lds[RowsLds<D>::kBytes];
    const int h = blockIdx.x, w = blockIdx.y;
    const RowPlan plan = *plan_of(a, h);
    const int64_t begin = w * plan.share, end = begin + plan.share;
    if (begin >= plan.total) return;
    const RowTile *tiles = plan_part<const RowTile>(a, h, a.tile_at);
    for (int32_t t = plan_part<const int32_t>(a, h, a.wg_at)[w]; t < plan.n_tiles; ++t) {
        const RowTile tile = tiles[t];
        if (tile.cost0 >= end) break;
        if (tile.n_wg == 0) continue;
        const int32_t lo = unit_at(tile, begin - tile.cost0), hi = unit_at(tile, end - tile.cost0);
        const int32_t slot = tile.part < 0 ? -1 : tile.part + (w - tile.wg0) * tile.rows;
        if (!WEIGH && tile.rows > 16) take_tile<D, BITS, 2, false>(a, tile, lo, hi, slot, lds, h);
        else take_tile<D, BITS, 1, WEIGH>(a, tile, lo, hi, slot, lds, h);
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
    for (int32_t u = tid; u < own.n_pages; u += 256) {
        int32_t lp;
        if (page_entry(a, b, h, u, end, lp) < 0) continue;
        const f32x2 *st = reinterpret_cast<const f32x2 *>(a.stat) + (((int64_t)h * a.batch + b) * a.max_sel + u) * G;
        float w = 0.0f;
        for (int g = 0; g < G; ++g) w += st[g][0] * fexp2(st[g][1] - sM[g]) / sL[g];
        atomicAdd(a.weights + ((int64_t)b * a.n_kv + h) * a.max_pages + lp, w);
    }
}

// Cross: workgroup w merges the tile that workgroup w of rows_kernel began and did
// not end.
template <int D>
__global__ void __launch_bounds__(256) rows_join_kernel(RowsArgs a)
{
    const int h = blockIdx.x, w = blockIdx.y, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int32_t G = 1 << a.g_log2;
    const RowPlan plan = *plan_of(a, h);
    if ((w + 1) * plan.share >= plan.total) return;
    const RowTile tile = plan_part<const RowTile>(a, h, a.tile_at)[plan_part<const int32_t>(a, h, a.wg_at)[w + 1]];
    if (tile.wg0 != w || tile.n_wg < 2) return;
    const int32_t *toks = plan_part<const int32_t>(a, h, a.tok_at) + tile.tok;
    for (int r = wave; r < tile.rows; r += 4) {
        float o[D / 64], M, l;
        merge_row<D>(a, h, tile.n_wg, [&](int i) -> int64_t { return tile.part + (int64_t)i * tile.rows + r; }, o, M, l);
        const int64_t at = (((int64_t)toks[r >> a.g_log2] * a.n_kv + h) << a.g_log2) + (r & (G - 1));
#pragma unroll
        for (int e = 0; e < D / 64; ++e) a.out[at * D + (D / 64) * lane + e] = l != 0.0f ? o[e] / l : 0.0f;
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
    a.wgs = (int32_t)(2 * compute_units() / hk > 1 ? 2 * compute_units() / hk : 1);
    // (cross: a stored sequence's last tile may be short)
    const int64_t tiles = mode == kPrefix ? 2 * B : mode == kWeighted ? B : (tokens * G + kTileRows - 1) / kTileRows + (items < B ? items : B);
    a.part_rows = mode == kPrefix ? 2 * B * G + kTileRows * (int64_t)a.wgs
                  : mode == kWeighted ? B * G + G * (int64_t)a.wgs : 2 * kTileRows * (int64_t)a.wgs;
    a.qlimb = take(hk * tokens * G * kLimbRoom * 128);
    a.qaux = reinterpret_cast<uint32_t *>(take(hk * tokens * G * 16));
    a.qpart = reinterpret_cast<uint16_t *>(take(hk * tokens * G * 3 * d * 2));
    a.part = reinterpret_cast<float *>(take(hk * a.part_rows * d * 4));
    a.part_ml = reinterpret_cast<float *>(take(hk * a.part_rows * 8));
    if (mode == kWeighted) a.stat = reinterpret_cast<float *>(take(hk * B * max_sel * G * 8));
    int64_t p = sizeof(RowPlan);
    auto within = [&](int64_t bytes) {
        const int64_t was = p;
        p += (bytes + 15) / 16 * 16;
        return (int32_t)was;
    };
    a.wg_at = within(4 * ((int64_t)a.wgs + 1));
    a.tile_at = within(sizeof(RowTile) * tiles);
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
    else if (a.wgs > 1) launch("rows_join_kernel", rows_join_kernel<D>, dim3(a.n_kv, a.wgs - 1), dim3(256), s, a);
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
    a.reps = 1;
    while (a.reps < 8 && groups * a.n_kv / (2 * a.reps) >= 2 * compute_units()) a.reps *= 2;
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
    if (n_seqs > kMaxRowItems || (int64_t)n_seqs * max_tok > (1 << 18)) return WUSHKV_EUNSUPPORTED;
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
