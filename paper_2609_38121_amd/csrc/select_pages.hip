// wushkv_page_bounds and wushkv_select_pages: a box in 8 bits round the stored
// keys of every complete page, and the pages whose box allows a decode query
// the largest logits.
//
// A box has per channel a centre c and a radius r (in units of the page's
// scale s): over the box the largest q~ . k is
//   s sum_j max(q~_j (c_j - r_j), q~_j (c_j + r_j)) = s sum_j (q~_j c_j + |q~_j| r_j),
// one product of [q~, |q~|] with [c, r].  With q~ in 15-bit fixed point N, split
// into two 8-bit digits, it is two 8-bit integer products with exact 32-bit
// sums (|sum| <= 128 16384 128 < 2^31): the scores, and so the selection, do
// not depend on an order of summation.  The rows of the 16x16x64 products are
// (query head, digit) pairs, the columns pages.
//
// page_bounds_kernel   one wave per (page, kv head).  Bound by its vector
//                      instructions (672 a wave): 8096 page-heads at d = 128,
//                      2-bit, 11.9 us, of which a launch is about 4.
// select_row_kernel    rows of at most 512 planned pages: one workgroup per (kv
//                      head, sequence), one launch.  512 rows of 380 pages 16.6
//                      us (52 MB of boxes; 10.8 at a copy's rate): q~ in fp64
//                      about 3, the selection about 3, the launch about 4.
// score_kernel         longer rows: grid (kv heads, runs of pages, sequences),
// select_kernel        then one workgroup per (kv head, sequence).  8 rows of 2046
//                      pages 16 us, two launches' fixed cost and two latency chains.
#include "common.h"
#include "merge.h"

namespace wushkv {

// ------------------------------------------------------------------ boxes

struct BoundsArgs {
    const uint8_t *pages;
    const int32_t *page_table, *seq_len, *quant_end, *since;
    int8_t *codes;
    float *scales;
    int32_t n_kv, s_sink, max_pages, n_pages, max_new;
    int32_t blocks;  // workgroups per sequence
};

// Complete pages of sequence b.
__device__ __forceinline__ int32_t complete_pages(const int32_t *seq_len, const int32_t *quant_end, int32_t b,
                                                  int32_t s_sink, int32_t max_pages)
{
    const int32_t q = min(quant_end[b], seq_len[b]);
    return q > s_sink ? min((q - s_sink) / kPage, max_pages) : 0;
}

// Four values a and four c of a lane: a becomes op(a, the partner's a) in the
// banks (groups of four lanes) A of a row and op(c, the partner's c) in the
// others, the partner being the lane that CTRL names: half of an exchange that
// leaves each lane half of the values, reduced over both lanes.  (A DPP operand
// must not have been written in the two instructions before.)
#define WUSHKV_HALVE(OP, CTRL, A, C, a, c)                                                       \
    asm volatile("s_nop 1\n\t"                                                                  \
                 OP " %0, %0, %0 " CTRL " row_mask:0xf bank_mask:" A "\n\t"                      \
                 OP " %1, %1, %1 " CTRL " row_mask:0xf bank_mask:" A "\n\t"                      \
                 OP " %2, %2, %2 " CTRL " row_mask:0xf bank_mask:" A "\n\t"                      \
                 OP " %3, %3, %3 " CTRL " row_mask:0xf bank_mask:" A "\n\t"                      \
                 OP " %0, %4, %4 " CTRL " row_mask:0xf bank_mask:" C "\n\t"                      \
                 OP " %1, %5, %5 " CTRL " row_mask:0xf bank_mask:" C "\n\t"                      \
                 OP " %2, %6, %6 " CTRL " row_mask:0xf bank_mask:" C "\n\t"                      \
                 OP " %3, %7, %7 " CTRL " row_mask:0xf bank_mask:" C                              \
                 : "+v"((a)[0]), "+v"((a)[1]), "+v"((a)[2]), "+v"((a)[3])                        \
                 : "v"((c)[0]), "v"((c)[1]), "v"((c)[2]), "v"((c)[3]))

// The least and the largest of 32 values over the 16 lanes of a row: lane n ends
// with those of values 2 n and 2 n + 1 (x[0], x[1]).  Four exchanges, with lanes
// n ^ 8, 7 - n (within eight), n ^ 2 and n ^ 1, each with half of the values
// that are left.
template <bool MAX>
__device__ __forceinline__ void row_halves(float (&x)[32], int n)
{
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
        if constexpr (MAX) WUSHKV_HALVE("v_max_f32_dpp", "row_ror:8", "0x3", "0xc", x + i, x + 16 + i);
        else WUSHKV_HALVE("v_min_f32_dpp", "row_ror:8", "0x3", "0xc", x + i, x + 16 + i);
    }
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
        if constexpr (MAX) WUSHKV_HALVE("v_max_f32_dpp", "row_half_mirror", "0x5", "0xa", x + i, x + 8 + i);
        else WUSHKV_HALVE("v_min_f32_dpp", "row_half_mirror", "0x5", "0xa", x + i, x + 8 + i);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool up = (n & 2) != 0;
        const float keep = up ? x[4 + i] : x[i], other = dpp<0x4E>(up ? x[i] : x[4 + i]);
        x[i] = MAX ? fmaxf(keep, other) : fminf(keep, other);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const bool up = (n & 1) != 0;
        const float keep = up ? x[2 + i] : x[i], other = dpp<0xB1>(up ? x[i] : x[2 + i]);
        x[i] = MAX ? fmaxf(keep, other) : fminf(keep, other);
    }
}

// Lane (j, n) of the wave holds channels 32 j .. 32 j + 31 of tokens 4 n ..
// 4 n + 3 (the page layout); with d = 64 the upper half repeats the lower.  A code
// masked where it stands in a half word, in fields F = 0 .. 6 of it, is the fp16
// subnormal c 2^(F-24): times scale 2^(24-F), one mixed-precision fma gives
// scale c + zero, rounded once, without any conversion.
template <int D, int BITS>
__global__ void __launch_bounds__(256) page_bounds_kernel(BoundsArgs a)
{
    using L = Layout<D, BITS>;
    constexpr int kWords = L::kKWordsPerLane;     // 8 (2-bit) or 16 (4-bit)
    constexpr int kSpan = L::kCodesPerWord;       // channels per word
    constexpr int kFields = 8 / BITS;             // fields of half of a half word
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t b = blockIdx.x / a.blocks;
    const int32_t item = (blockIdx.x % a.blocks) * 4 + wave;  // (new page, kv head)
    const int32_t h = item % a.n_kv;
    const int32_t q0 = a.since != nullptr ? a.since[b] : 0;
    const int32_t lp = (q0 > a.s_sink ? (q0 - a.s_sink) / kPage : 0) + item / a.n_kv;
    if (item / a.n_kv >= a.max_new || lp >= complete_pages(a.seq_len, a.quant_end, b, a.s_sink, a.max_pages)) return;
    const int32_t phys = a.page_table[(int64_t)b * a.max_pages + lp];
    if (phys < 0 || phys >= a.n_pages) return;
    const uint8_t *pg = a.pages + ((int64_t)phys * a.n_kv + h) * L::kPageBytes;
    const int src = lane % L::kKLanes, n = lane & 15;
    u32x4 w[kWords / 4];
#pragma unroll
    for (int i = 0; i < kWords / 4; ++i) w[i] = *reinterpret_cast<const u32x4 *>(pg + 4 * L::k_word(src, 4 * i));
    const u32x4 par = *reinterpret_cast<const u32x4 *>(pg + L::kParamOffset + 16 * n);
    float sc[4][kFields], zr[4];  // scale 2^(24 - F), zero
    bool odd = false;             // a parameter that is not finite
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        odd |= (par[t] & 0x7C00u) == 0x7C00u || (par[t] & 0x7C000000u) == 0x7C000000u;
        zr[t] = f16_bits_to_f32(par[t] >> 16);
#pragma unroll
        for (int f = 0; f < kFields; ++f) sc[t][f] = f16_bits_to_f32(par[t] & 0xFFFFu) * (16777216.0f / (1 << (BITS * f)));
    }
    float lo[32], hi[32];
#pragma unroll
    for (int i = 0; i < BITS; ++i)  // the word of a token
#pragma unroll
        for (int byte = 0; byte < 2; ++byte)
#pragma unroll
            for (int f = 0; f < kFields; ++f) {
                // field 8 byte + BITS f of both half words: element e and e + kSpan / 4
                const int field = 8 * byte + BITS * f;
                const int e = (f & 1) * (kSpan / 2) + field / (2 * BITS);
                const uint32_t mask = ((1u << BITS) - 1u) * 0x00010001u << (BITS * f);
                float x[4], y[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const uint32_t v = (w[(BITS * t + i) / 4][(BITS * t + i) % 4] >> (8 * byte)) & mask;
                    x[t] = fmaf(sc[t][f], f16_bits_to_f32(v & 0xFFFFu), zr[t]);
                    y[t] = fmaf(sc[t][f], f16_bits_to_f32(v >> 16), zr[t]);
                }
                const int ch = kSpan * i + e, ch2 = ch + kSpan / 4;
                lo[ch] = fminf(fminf(fminf(x[0], x[1]), x[2]), x[3]);
                hi[ch] = fmaxf(fmaxf(fmaxf(x[0], x[1]), x[2]), x[3]);
                lo[ch2] = fminf(fminf(fminf(y[0], y[1]), y[2]), y[3]);
                hi[ch2] = fmaxf(fmaxf(fmaxf(y[0], y[1]), y[2]), y[3]);
            }
    // over the tokens; lane n of a row then finishes channels 2 n and 2 n + 1 of its 32
    row_halves<false>(lo, n);
    row_halves<true>(hi, n);
    const bool any_odd = __any(odd);
    const float top = any_odd ? 0.0f
                              : wave_max(fmaxf(fmaxf(fabsf(lo[0]), fabsf(hi[0])), fmaxf(fabsf(lo[1]), fabsf(hi[1]))));
    const float s = any_odd ? INFINITY : top / 126.0f;
    int c[2] = {0, 0}, r[2] = {0, 0};
    if (top > 0.0f) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float mid = rintf(((lo[e] + hi[e]) * 0.5f) / s);
            const float ms = mid * s;
            c[e] = (int)mid;
            r[e] = (int)fminf(ceilf(fmaxf(hi[e] - ms, ms - lo[e]) / s), 127.0f);
        }
    }
    if (lane >= L::kKLanes) return;
    int8_t *out = a.codes + ((int64_t)phys * a.n_kv + h) * 2 * D + 2 * lane;
    *reinterpret_cast<uint16_t *>(out) = (uint16_t)((c[0] & 0xFF) | ((c[1] & 0xFF) << 8));
    *reinterpret_cast<uint16_t *>(out + D) = (uint16_t)(r[0] | (r[1] << 8));
    if (lane == 0) a.scales[(int64_t)h * a.n_pages + phys] = s;
}

// ------------------------------------------------------------------ scores

typedef __attribute__((ext_vector_type(4))) int i32x4;

struct SelectArgs {
    const int8_t *codes;
    const float *scales;
    const int32_t *page_table, *seq_len, *quant_end;
    const uint16_t *q;
    const float *tinv;
    int32_t *sel, *n_sel;
    float *scores;       // [batch][n_kv][max_pages], or null
    float *room;         // the same, for the long rows of a call without scores
    int32_t n_kv, G, s_sink, max_pages, n_pages;
    int32_t planned;     // pages of the longest sequence planned for
    int32_t run;         // pages per workgroup of score_kernel
    int32_t top_k;
};

// The two digits of N and |N| for the group's heads, as operand rows 2 g (the
// 256s) and 2 g + 1: [16][2 D] bytes of [N, |N|], rows 16 bytes apart in the banks.
template <int D>
struct DigitLds {
    static constexpr int kPitch = 2 * D + 16;
    int8_t rows[16 * kPitch];
    float unit[8];  // 2^-F per head
};

// q~ = q t_k_inv of the group's heads in fp64 and its digits, by all NT threads
// of the workgroup.  Thread (part, quad) sums its kRows rows of four columns for
// four heads at a time; lanes, then waves, in a fixed order.  load() requests
// T^{-1} and the first four heads' queries, so that they travel while the
// caller requests boxes.
__device__ __forceinline__ double add_pair16(double x)  // + lane ^ 16's
{
    const uint32_t lo = (uint32_t)__double2loint(x), hi = (uint32_t)__double2hiint(x);
    const auto l = __builtin_amdgcn_permlane16_swap(lo, lo, false, false);
    const auto u = __builtin_amdgcn_permlane16_swap(hi, hi, false, false);
    return __hiloint2double((int)u[0], (int)l[0]) + __hiloint2double((int)u[1], (int)l[1]);
}
__device__ __forceinline__ double add_pair32(double x)  // + lane ^ 32's
{
    const uint32_t lo = (uint32_t)__double2loint(x), hi = (uint32_t)__double2hiint(x);
    const auto l = __builtin_amdgcn_permlane32_swap(lo, lo, false, false);
    const auto u = __builtin_amdgcn_permlane32_swap(hi, hi, false, false);
    return __hiloint2double((int)u[0], (int)l[0]) + __hiloint2double((int)u[1], (int)l[1]);
}

template <int D, int NT>
struct QuerySums {
    static constexpr int kHeads = 4;
    static constexpr int kQuads = D / 4;
    static constexpr int kRows = D / (NT / kQuads);  // rows per part
    static constexpr int kWaves = NT / 64;
    f32x4 t[kRows];
    uint32_t q[kHeads][kRows / 2];
    struct __attribute__((aligned(16))) Lds {
        double red[kWaves * kHeads * D];
        double qt[8 * D];
    };
    __device__ __forceinline__ void load_q(const SelectArgs &a, int b, int h, int g0, int tid)
    {
        const uint16_t *src = a.q + (((int64_t)b * a.n_kv + h) * a.G) * D + tid / kQuads * kRows;
#pragma unroll
        for (int g = 0; g < kHeads; ++g) {
            const uint32_t *row = reinterpret_cast<const uint32_t *>(src + (int64_t)min(g0 + g, a.G - 1) * D);
#pragma unroll
            for (int r = 0; r < kRows / 2; ++r) q[g][r] = row[r];
        }
    }
    __device__ __forceinline__ void load(const SelectArgs &a, int b, int h, int tid)
    {
        const float *T = a.tinv + (int64_t)h * D * D + (int64_t)(tid / kQuads) * kRows * D + 4 * (tid % kQuads);
#pragma unroll
        for (int r = 0; r < kRows; ++r) t[r] = *reinterpret_cast<const f32x4 *>(T + (int64_t)r * D);
        load_q(a, b, h, 0, tid);
    }
    // q~ into lds.qt, without a barrier at the end, in PASSES of four heads
    template <int PASSES>
    __device__ __forceinline__ void sum(const SelectArgs &a, int b, int h, Lds &lds, int tid)
    {
        const int lane = tid & 63, wave = tid >> 6, quad = tid % kQuads;
#pragma unroll
        for (int pass = 0; pass < PASSES; ++pass) {
            const int g0 = kHeads * pass;
            if (g0 > 0) load_q(a, b, h, g0, tid);
            // (opaque, so that the conversions to fp64 are not kept for the next
            // heads in 8 registers a row)
#pragma unroll
            for (int r = 0; r < kRows; ++r) asm volatile("" : "+v"(t[r]));
            double acc[kHeads][4];
#pragma unroll
            for (int g = 0; g < kHeads; ++g)
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[g][c] = 0.0;
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                double col[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) col[c] = (double)t[r][c];
#pragma unroll
                for (int g = 0; g < kHeads; ++g) {
                    const uint32_t w = q[g][r / 2];
                    const double x = (double)__uint_as_float(r & 1 ? w & 0xFFFF0000u : w << 16);
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[g][c] = fma(x, col[c], acc[g][c]);
                }
            }
#pragma unroll
            for (int g = 0; g < kHeads; ++g)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    if constexpr (kQuads == 16) acc[g][c] = add_pair16(acc[g][c]);
                    acc[g][c] = add_pair32(acc[g][c]);
                }
            __syncthreads();  // the last heads' sums are read
            if (lane < kQuads)
#pragma unroll
                for (int g = 0; g < kHeads; ++g)
#pragma unroll
                    for (int c = 0; c < 4; ++c) lds.red[(wave * kHeads + g) * D + 4 * quad + c] = acc[g][c];
            __syncthreads();
            for (int i = tid; i < kHeads * D; i += NT) {
                double x = 0.0;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) x += lds.red[w * kHeads * D + i];
                if (g0 + i / D < a.G) lds.qt[g0 * D + i] = x;
            }
        }
    }
    // .. and its digits, between barriers
    __device__ __forceinline__ void digits(const SelectArgs &a, Lds &lds, DigitLds<D> &out, int tid)
    {
        const int lane = tid & 63, wave = tid >> 6;
        for (int i = tid; i < 16 * DigitLds<D>::kPitch / 4; i += NT) reinterpret_cast<uint32_t *>(out.rows)[i] = 0u;
        __syncthreads();
        for (int g = wave; g < a.G; g += kWaves) {
            double x[D / 64];
            uint32_t top = 0;  // the exponent of the largest magnitude
            bool zero = true;  // all entries
#pragma unroll
            for (int e = 0; e < D / 64; ++e) {
                x[e] = lds.qt[g * D + 64 * e + lane];
                top = max(top, (uint32_t)(__double2hiint(x[e]) & 0x7FF00000) >> 20);
                zero = zero && x[e] == 0.0;
            }
            top = (uint32_t)wave_max((float)top);  // (at most 2047: exact)
            const bool dead = top == 0x7FF || __all(zero);
            const int F = dead ? 0 : min(max(14 - ((int)top - 1022), -100), 100);
            const double f = __hiloint2double((1023 + F) << 20, 0);
#pragma unroll
            for (int e = 0; e < D / 64; ++e) {
                const int N = dead ? 0 : (int)fmin(fmax(rint(x[e] * f), -16384.0), 16384.0);
                const int M = N < 0 ? -N : N;
                int8_t *at = out.rows + 2 * g * DigitLds<D>::kPitch + 64 * e + lane;
                at[0] = (int8_t)((N + 128) >> 8);
                at[DigitLds<D>::kPitch] = (int8_t)N;
                at[D] = (int8_t)((M + 128) >> 8);
                at[D + DigitLds<D>::kPitch] = (int8_t)M;
            }
            if (lane == 0) out.unit[g] = ldexpf(1.0f, -F);
        }
        __syncthreads();
    }
};

// The operand rows of a lane, and what its results (heads 2 j and 2 j + 1) need.
template <int D>
struct QueryRows {
    i32x4 rows[D / 32];
    bool there[2];
    float unit[2];
    __device__ __forceinline__ void read(const SelectArgs &a, const DigitLds<D> &lds, int lane)
    {
        const int n = lane & 15, j = lane >> 4;
#pragma unroll
        for (int k = 0; k < D / 32; ++k)
            rows[k] = *reinterpret_cast<const i32x4 *>(lds.rows + n * DigitLds<D>::kPitch + 64 * k + 16 * j);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            there[e] = 2 * j + e < a.G;
            unit[e] = there[e] ? lds.unit[2 * j + e] : 1.0f;
        }
    }
};

// A tile of 16 pages: lane (j, n) holds bytes 64 k + 16 j .. + 15 of page n's
// box for every k.
template <int D>
struct BoxTile {
    i32x4 w[D / 32];
    float s;        // page n's scale
    bool inside;    // page n lies in the pool
    static __device__ __forceinline__ int32_t entry(const SelectArgs &a, int b, int32_t lp, int32_t end)
    {
        return lp < end ? a.page_table[(int64_t)b * a.max_pages + lp] : -1;
    }
    __device__ __forceinline__ void load(const SelectArgs &a, int h, int32_t phys, int lane)
    {
        inside = phys >= 0 && phys < a.n_pages;
        s = 0.0f;
#pragma unroll
        for (int k = 0; k < D / 32; ++k) w[k] = i32x4{0, 0, 0, 0};
        if (inside) {
            const int8_t *src = a.codes + ((int64_t)phys * a.n_kv + h) * 2 * D + 16 * (lane >> 4);
#pragma unroll
            for (int k = 0; k < D / 32; ++k) w[k] = *reinterpret_cast<const i32x4 *>(src + 64 * k);
            s = a.scales[(int64_t)h * a.n_pages + phys];
        }
    }
    // page n's score, in every lane of column n
    __device__ __forceinline__ float score(const QueryRows<D> &q) const
    {
        i32x4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < D / 32; ++k) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(q.rows[k], w[k], acc, 0, 0, 0);
        float best = -INFINITY;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float x = (float)(acc[2 * e] * 256 + acc[2 * e + 1]) * s;
            if (q.there[e]) best = fmaxf(best, x * q.unit[e]);
        }
        const LanePair p = pair16(best);
        const LanePair r = pair32(fmaxf(p.a, p.b));
        best = fmaxf(r.a, r.b) + 0.0f;  // (no negative zero)
        if (s == INFINITY) best = INFINITY;
        return inside ? best : -INFINITY;
    }
};

// What a sequence has: complete pages, pages in all, as far as planned.
struct SeqPages {
    int32_t full, every;
    __device__ __forceinline__ SeqPages(const SelectArgs &a, int b)
    {
        const int32_t end = min(a.quant_end[b], a.seq_len[b]), most = min(a.planned, a.max_pages);
        const int32_t span = end > a.s_sink ? end - a.s_sink : 0;
        full = min(span / kPage, most);
        every = min(span / kPage + (span % kPage != 0), most);
    }
};

// fp32 -> uint32 in the same order (no NaN); never 0.
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t u = __float_as_uint(x);
    return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}

// The largest of a wave's values, in every lane (halves, as fp32 is exact to 24 bits).
__device__ __forceinline__ uint32_t wave_most(uint32_t x)
{
    const uint32_t hi = (uint32_t)wave_max((float)(x >> 16));
    const uint32_t lo = (uint32_t)wave_max(x >> 16 == hi ? (float)(x & 0xFFFFu) : 0.0f);
    return hi << 16 | lo;
}

// The selection of a row whose keys (order_of the scores, ascending pages in
// ascending lanes and waves, 0 where there is none) the NW waves hold one per
// lane.  The k-th largest key is found from the top, after the bits that all keys
// share, eight bits at a time: a histogram of the keys that share the bits found
// so far (counted from zeroed bins, one set a pass), which every wave scans for
// itself, so that a pass is one barrier.  Then, in ascending order, the pages
// above it and as many equal ones as are missing.
template <int NW>
struct TakeLds {
    uint32_t hist[4 * 256];  // a pass each
    uint32_t range[2][NW];
    int32_t count[2][NW];
};
template <int NW>
__device__ __forceinline__ void take_largest(uint32_t key, int32_t page, int32_t n, int32_t k, int32_t *sel,
                                             TakeLds<NW> &lds, int tid)
{
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    uint32_t at = 1;   // the k-th largest key's bits so far
    int32_t left = 0;  // its rank among the keys that share them (k = n: every key is above 0)
    if (k < n) {
        uint32_t most = wave_most(key), least = ~wave_most(key != 0 ? ~key : 0u);
        if (lane == 0) {
            lds.range[0][wave] = most;
            lds.range[1][wave] = least;
        }
        __syncthreads();  // (the bins are zero too)
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            most = max(most, lds.range[0][w]);
            least = min(least, lds.range[1][w]);
        }
        int bits = most == least ? 0 : 32 - __clz(most ^ least);
        at = bits == 32 ? 0 : most >> bits << bits;
        left = k;
        for (int pass = 0; bits > 0; ++pass) {
            const int shift = max(bits - 8, 0);
            const bool in = key != 0 && (bits == 32 || (key >> bits) == (at >> bits));
            if (in) atomicAdd(&lds.hist[256 * pass + ((key >> shift) & ((1u << (bits - shift)) - 1u))], 1u);
            __syncthreads();
            // lane l: digits 252 - 4 l .. 255 - 4 l, from the top
            const uint4 c = *reinterpret_cast<const uint4 *>(&lds.hist[256 * pass + 252 - 4 * lane]);
            const int32_t up[4] = {(int32_t)c.w, (int32_t)c.z, (int32_t)c.y, (int32_t)c.x};
            int32_t above = wave_scan(up[0] + up[1] + up[2] + up[3]) - (up[0] + up[1] + up[2] + up[3]);
            int32_t digit = -1, rank = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (above < left && left <= above + up[e]) {
                    digit = 255 - 4 * lane - e;
                    rank = left - above;
                }
                above += up[e];
            }
            const int from = __ffsll((unsigned long long)__ballot(digit >= 0)) - 1;
            at |= (uint32_t)__builtin_amdgcn_readlane(digit, from) << shift;
            left = __builtin_amdgcn_readlane(rank, from);
            bits = shift;
        }
    }
    const uint64_t mg = __ballot(k < n ? key > at : key != 0), me = __ballot(k < n && key == at);
    if (lane == 0) {
        lds.count[0][wave] = __popcll(mg);
        lds.count[1][wave] = __popcll(me);
    }
    __syncthreads();
    int32_t ng = 0, ne = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        if (w < wave) {
            ng += lds.count[0][w];
            ne += lds.count[1][w];
        }
    }
    const uint64_t low = lane == 0 ? 0 : ~0ull >> (64 - lane);
    ng += __popcll(mg & low);
    ne += __popcll(me & low);
    // ng pages above and min(ne, left) equal ones come before this one
    if (((mg >> lane) & 1) != 0 || (((me >> lane) & 1) != 0 && ne < left)) sel[ng + min(ne, left)] = page;
}

// The row's entries behind the k selected pages, by all NT threads.
template <int NT>
__device__ __forceinline__ void finish_row(const SelectArgs &a, const SeqPages &sp, int32_t k, int64_t row, int32_t *sel,
                                           int tid)
{
    for (int64_t i = (int64_t)k + tid; i <= a.top_k; i += NT) sel[i] = i == k && sp.every > sp.full ? sp.full : -1;
    if (tid == 0) a.n_sel[row] = k + (sp.every > sp.full);
}

// Rows of at most 128 T planned pages: one workgroup of eight waves per (kv head,
// sequence) forms the digits, scores the pages and selects.  A wave has T tiles
// of 16 consecutive pages (T = 4: the wave's 64 lanes then hold its 64 scores):
// their table entries are requested first of all, the first tile's boxes before
// q~ is formed, the others' when its sums are done and their registers free
// (four waves per SIMD: 128 each).
template <int D, int T, int PASSES>
__global__ void __launch_bounds__(512, 4) select_row_kernel(SelectArgs a)
{
    static_assert(T == 1 || T == 4, "a score per lane");
    constexpr int NT = 512, kWaves = 8;
    using Q = QuerySums<D, NT>;
    __shared__ __attribute__((aligned(16))) DigitLds<D> digits;
    __shared__ __attribute__((aligned(16))) typename Q::Lds sums;
    __shared__ __attribute__((aligned(16))) TakeLds<kWaves> take;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, j = lane >> 4;
    const int h = blockIdx.x, b = blockIdx.y;
    const int64_t row = (int64_t)b * a.n_kv + h;
    const int32_t first = 16 * T * wave + n;
    int32_t phys[T];
#pragma unroll
    for (int i = 0; i < T; ++i) phys[i] = BoxTile<D>::entry(a, b, first + 16 * i, a.planned);
    Q in;
    in.load(a, b, h, tid);
    const SeqPages sp(a, b);
    int32_t *sel = a.sel + row * ((int64_t)a.top_k + 1);
    const int32_t k = min(a.top_k, sp.full);
    if (sp.full == 0) {  // (the same for every thread)
        finish_row<NT>(a, sp, k, row, sel, tid);
        return;
    }
    for (int i = tid; i < 4 * 256; i += NT) take.hist[i] = 0;
    BoxTile<D> tile[T];
    auto load = [&](int i) __attribute__((always_inline)) {
        tile[i].load(a, h, first + 16 * i < sp.full ? phys[i] : -1, lane);
    };
    load(0);
    in.template sum<PASSES>(a, b, h, sums, tid);
    asm volatile("" ::: "memory");  // (not earlier: their registers are T^{-1}'s and the sums' until here)
#pragma unroll
    for (int i = 1; i < T; ++i) load(i);
    in.digits(a, sums, digits, tid);
    QueryRows<D> q;
    q.read(a, digits, lane);
    float x = 0.0f;
#pragma unroll
    for (int i = 0; i < T; ++i) {
        const float y = tile[i].score(q);
        if (j == i) x = y;
    }
    const int32_t page = first + 16 * j;
    const bool mine = j < T && page < sp.full;
    if (mine && a.scores != nullptr) a.scores[row * a.max_pages + page] = x;
    if (k > 0) take_largest<kWaves>(mine ? order_of(x) : 0u, page, sp.full, k, sel, take, tid);
    finish_row<NT>(a, sp, k, row, sel, tid);
}

// Longer rows: the scores by runs of pages ..
template <int D, int NT, int PASSES>
__global__ void __launch_bounds__(NT) score_kernel(SelectArgs a)
{
    constexpr int kPre = 2;
    using Q = QuerySums<D, NT>;
    __shared__ __attribute__((aligned(16))) DigitLds<D> digits;
    __shared__ __attribute__((aligned(16))) typename Q::Lds sums;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15;
    const int h = blockIdx.x, b = blockIdx.z;
    Q in;
    in.load(a, b, h, tid);
    const int32_t full = SeqPages(a, b).full;
    const int32_t first = blockIdx.y * a.run, end = min(first + a.run, full);
    if (first >= end) return;
    BoxTile<D> tile[kPre];
#pragma unroll
    for (int i = 0; i < kPre; ++i)
        tile[i].load(a, h, BoxTile<D>::entry(a, b, first + 16 * (wave + NT / 64 * i) + n, end), lane);
    in.template sum<PASSES>(a, b, h, sums, tid);
    in.digits(a, sums, digits, tid);
    QueryRows<D> q;
    q.read(a, digits, lane);
    float *out = a.scores + ((int64_t)b * a.n_kv + h) * a.max_pages;
    for (int32_t p = first + 16 * wave; p < end; p += NT / 4) {
        const float x = tile[0].score(q);
        if (lane < 16 && p + n < end) out[p + n] = x;
        tile[0] = tile[1];
        tile[1].load(a, h, BoxTile<D>::entry(a, b, p + 2 * (NT / 4) + n, end), lane);
    }
}

// .. and the selection of one (sequence, kv head) over them: the k-th largest
// score by a histogram of the next eight bits at a time, below those that all
// scores share, among the scores that share the bits found so far; then the
// pages above it, and as many equal ones as are missing, in ascending order.
// Keys that fit LDS are read from memory once.
constexpr int kLdsKeys = 16384;
__global__ void __launch_bounds__(1024) select_kernel(SelectArgs a)
{
    __shared__ uint32_t keys[kLdsKeys];
    __shared__ uint32_t hist[256];
    __shared__ int32_t found[2];     // the digit, and how many of it are taken
    __shared__ int32_t sums[2][16];
    __shared__ uint32_t range[2][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int h = blockIdx.x, b = blockIdx.y;
    const SeqPages sp(a, b);
    const int32_t full = sp.full;
    const int64_t row = (int64_t)b * a.n_kv + h;
    const float *scores = a.scores + row * a.max_pages;
    int32_t *sel = a.sel + row * ((int64_t)a.top_k + 1);
    const int32_t k = min(a.top_k, full);
    const bool kept = full <= kLdsKeys;
    auto key = [&](int32_t i) -> uint32_t { return kept ? keys[i] : order_of(scores[i]); };
    uint32_t at = 0;        // the k-th largest score's bits so far
    int32_t left = k;       // its rank among the scores that share them
    if (k > 0 && k < full) {
        uint32_t most = 0, least = 0xFFFFFFFFu;
        for (int32_t i = tid; i < full; i += 1024) {
            const uint32_t u = order_of(scores[i]);
            if (kept) keys[i] = u;
            most = max(most, u);
            least = min(least, u);
        }
        most = wave_most(most);
        least = ~wave_most(~least);
        if (lane == 0) {
            range[0][wave] = most;
            range[1][wave] = least;
        }
        __syncthreads();
        for (int w = 0; w < 16; ++w) {
            most = max(most, range[0][w]);
            least = min(least, range[1][w]);
        }
        int bits = most == least ? 0 : 32 - __clz(most ^ least);
        at = bits == 32 ? 0 : most >> bits << bits;
        while (bits > 0) {
            const int shift = max(bits - 8, 0);
            if (tid < 256) hist[tid] = 0;
            __syncthreads();
            for (int32_t i = tid; i < full; i += 1024) {
                const uint32_t u = key(i);
                if (bits == 32 || (u >> bits) == (at >> bits)) atomicAdd(&hist[(u >> shift) & 255u & ((1u << (bits - shift)) - 1u)], 1u);
            }
            __syncthreads();
            if (wave == 0) {
                // lane l: digits 255 - 4 l down to 252 - 4 l
                int32_t c[4], sum = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) sum += c[e] = (int32_t)hist[255 - 4 * lane - e];
                int32_t above = wave_scan(sum) - sum;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (above < left && left <= above + c[e]) {
                        found[0] = 255 - 4 * lane - e;
                        found[1] = left - above;
                    }
                    above += c[e];
                }
            }
            __syncthreads();
            at |= (uint32_t)found[0] << shift;
            left = found[1];
            bits = shift;
            __syncthreads();
        }
    }
    // (k = full: everything is above)
    int32_t above = 0, equal = 0;  // pages above and pages equal before this round
    for (int32_t i0 = 0; i0 < full && k > 0; i0 += 1024) {
        const int32_t i = i0 + tid;
        const uint32_t u = i < full && k < full ? key(i) : 0u;
        const bool gt = i < full && (k == full || u > at), eq = i < full && k < full && u == at;
        const uint64_t mg = __ballot(gt), me = __ballot(eq);
        __syncthreads();
        if (lane == 0) {
            sums[0][wave] = __popcll(mg);
            sums[1][wave] = __popcll(me);
        }
        __syncthreads();
        int32_t ng = above, ne = equal;
        for (int w = 0; w < 16; ++w) {
            const int32_t g = sums[0][w], e = sums[1][w];
            if (w < wave) {
                ng += g;
                ne += e;
            }
            above += g;
            equal += e;
        }
        const uint64_t low = lane == 0 ? 0 : ~0ull >> (64 - lane);
        ng += __popcll(mg & low);
        ne += __popcll(me & low);
        // ng pages above and min(ne, left) equal ones come before this one
        if (gt || (eq && ne < left)) sel[ng + min(ne, left)] = i;
    }
    finish_row<1024>(a, sp, k, row, sel, tid);
}

}  // namespace wushkv

using namespace wushkv;

int wushkv_validate_cache(const wushkv_cache *c);  // api.hip

static bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }

static int check_bounds(const wushkv_cache *c, const wushkv_bounds *bounds)
{
    const int st = wushkv_validate_cache(c);
    if (st != WUSHKV_OK) return st;
    if (!bounds || !bounds->codes || !bounds->scales) return WUSHKV_EINVAL;
    if (!aligned16(bounds->codes) || !aligned16(bounds->scales)) return WUSHKV_EINVAL;
    return WUSHKV_OK;
}

extern "C" int wushkv_page_bounds(const wushkv_cache *c, const wushkv_bounds *bounds, const int32_t *since,
                                  int32_t max_new, wushkv_stream_t stream)
{
    const int st = check_bounds(c, bounds);
    if (st != WUSHKV_OK) return st;
    if (max_new < 0 || !aligned16(since)) return WUSHKV_EINVAL;
    if (max_new == 0 || c->n_pages == 0 || c->max_pages_per_seq == 0) return WUSHKV_OK;
    BoundsArgs a{};
    a.pages = c->pages;
    a.page_table = c->page_table;
    a.seq_len = c->seq_len;
    a.quant_end = c->quant_end;
    a.since = since;
    a.codes = bounds->codes;
    a.scales = bounds->scales;
    a.n_kv = c->n_kv_heads;
    a.s_sink = c->s_sink;
    a.max_pages = c->max_pages_per_seq;
    a.n_pages = c->n_pages;
    a.max_new = max_new < c->max_pages_per_seq ? max_new : c->max_pages_per_seq;
    const int64_t blocks = ((int64_t)a.max_new * c->n_kv_heads + 3) / 4;
    if (blocks * c->batch > 0x7FFFFFFF / 4) return WUSHKV_EUNSUPPORTED;
    a.blocks = (int32_t)blocks;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)(blocks * c->batch));
    switch (c->head_dim * 10 + storage_bits(c->bits)) {
        case 1282: launch("page_bounds_kernel", page_bounds_kernel<128, 2>, grid, dim3(256), s, a); break;
        case 1284: launch("page_bounds_kernel", page_bounds_kernel<128, 4>, grid, dim3(256), s, a); break;
        case 642: launch("page_bounds_kernel", page_bounds_kernel<64, 2>, grid, dim3(256), s, a); break;
        case 644: launch("page_bounds_kernel", page_bounds_kernel<64, 4>, grid, dim3(256), s, a); break;
    }
    if (hipGetLastError() != hipSuccess) return WUSHKV_ELAUNCH;
    return WUSHKV_OK;
}

static int check_select(const wushkv_cache *c, int32_t n_q, int32_t max_seq_len, int32_t top_k)
{
    const int st = wushkv_validate_cache(c);
    if (st != WUSHKV_OK) return st;
    if (n_q <= 0 || n_q % c->n_kv_heads != 0 || max_seq_len < 0 || top_k < 0 || top_k == INT32_MAX) return WUSHKV_EINVAL;
    const int32_t G = n_q / c->n_kv_heads;
    if (G > 8 || (G & (G - 1)) != 0) return WUSHKV_EUNSUPPORTED;
    if (c->batch > 65535) return WUSHKV_EUNSUPPORTED;
    return WUSHKV_OK;
}

extern "C" size_t wushkv_select_workspace_bytes(const wushkv_cache *c, int32_t n_q_heads, int32_t max_seq_len,
                                                int32_t top_k)
{
    if (check_select(c, n_q_heads, max_seq_len, top_k) != WUSHKV_OK) return 0;
    // the scores (and never nothing, which says that the arguments are bad)
    return (size_t)c->batch * c->n_kv_heads * c->max_pages_per_seq * sizeof(float) + 16;
}

template <int D, int PASSES>
static void launch_select(SelectArgs a, int32_t batch, hipStream_t s)
{
    constexpr int NT = 512;
    const dim3 rows((unsigned)a.n_kv, (unsigned)batch);
    // Up to 512 pages a row is one workgroup's work in one launch (8 rows of 100
    // pages 11.4 us a call, in two launches 14.6; 512 rows of 500, 21 and 28).
    // Longer ones leave too few workgroups, or too much for each (8 rows of 1000
    // pages in two launches 13.9 us, in one 20.6; 256 rows, 26.9 and 24.3).
    if (a.planned <= 128) {
        launch("select_row_kernel", select_row_kernel<D, 1, PASSES>, rows, dim3(512), s, a);
        return;
    }
    if (a.planned <= 512) {
        launch("select_row_kernel", select_row_kernel<D, 4, PASSES>, rows, dim3(512), s, a);
        return;
    }
    if (a.scores == nullptr) a.scores = a.room;
    const dim3 grid((unsigned)a.n_kv, (unsigned)((a.planned + a.run - 1) / a.run), (unsigned)batch);
    if (grid.y > 0) launch("score_kernel", score_kernel<D, NT, PASSES>, grid, dim3(NT), s, a);
    launch("select_kernel", select_kernel, rows, dim3(1024), s, a);
}

extern "C" int wushkv_select_pages(const wushkv_cache *c, const wushkv_bounds *bounds, const uint16_t *q,
                                   int32_t n_q_heads, int32_t max_seq_len, const float *t_k_inv, int32_t top_k,
                                   int32_t *sel, int32_t *n_sel, float *scores, void *workspace,
                                   size_t workspace_bytes, wushkv_stream_t stream)
{
    int st = check_bounds(c, bounds);
    if (st != WUSHKV_OK) return st;
    st = check_select(c, n_q_heads, max_seq_len, top_k);
    if (st != WUSHKV_OK) return st;
    if (!q || !t_k_inv || !sel || !n_sel || !workspace) return WUSHKV_EINVAL;
    if (!aligned16(q) || !aligned16(t_k_inv) || !aligned16(sel) || !aligned16(n_sel) || !aligned16(scores) ||
        !aligned16(workspace))
        return WUSHKV_EINVAL;
    if (workspace_bytes < wushkv_select_workspace_bytes(c, n_q_heads, max_seq_len, top_k)) return WUSHKV_EWORKSPACE;
    SelectArgs a{};
    a.codes = bounds->codes;
    a.scales = bounds->scales;
    a.page_table = c->page_table;
    a.seq_len = c->seq_len;
    a.quant_end = c->quant_end;
    a.q = q;
    a.tinv = t_k_inv;
    a.sel = sel;
    a.n_sel = n_sel;
    a.scores = scores;
    a.room = reinterpret_cast<float *>(workspace);
    a.n_kv = c->n_kv_heads;
    a.G = n_q_heads / c->n_kv_heads;
    a.s_sink = c->s_sink;
    a.max_pages = c->max_pages_per_seq;
    a.n_pages = c->n_pages;
    const int64_t span = (int64_t)max_seq_len - c->s_sink;
    const int64_t pages = span > 0 ? (span + kPage - 1) / kPage : 0;
    a.planned = (int32_t)(pages < c->max_pages_per_seq ? pages : c->max_pages_per_seq);
    if (c->page_table == nullptr) a.planned = 0;
    // a workgroup of eight waves per compute unit, a tile for each wave at least
    // (64 rows of 2000 pages 22.5 us a call; two of four waves 25)
    const int64_t rows = (int64_t)c->batch * c->n_kv_heads;
    a.run = (int32_t)((a.planned * rows + 255) / 256 + 127) / 128 * 128;
    if (a.run < 128) a.run = 128;
    while ((a.planned + a.run - 1) / a.run > 65535) a.run *= 2;
    a.top_k = top_k;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (c->head_dim == 128 && a.G > 4) launch_select<128, 2>(a, c->batch, s);
    else if (c->head_dim == 128) launch_select<128, 1>(a, c->batch, s);
    else if (a.G > 4) launch_select<64, 2>(a, c->batch, s);
    else launch_select<64, 1>(a, c->batch, s);
    if (hipGetLastError() != hipSuccess) return WUSHKV_ELAUNCH;
    return WUSHKV_OK;
}
