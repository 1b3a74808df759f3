// What the attention kernels share: query rows q~ = q^T T_K^{-1} and their digit
// limbs (the operands of the quantised-key product), LDS accesses, the scaled
// products, and value codes as fp16 operands.
#pragma once

#include "common.h"
#include "merge.h"

namespace wushkv {

constexpr float kLog2e = 1.4426950408889634f;
// Digit limbs of a query row (form_limbs): with 2-bit keys five base-32
// digits as fp6 e2m3 numbers, with 4-bit keys six base-16 digits as fp8 e4m3
// numbers.  Each limb takes 128 bytes; a row has room for six of either.
constexpr int kLimbRoom = 6;
template <int BITS>
struct Limbs {
    static constexpr int kCount = BITS == 2 ? 5 : 6;
    static constexpr int kDigitBits = BITS == 2 ? 5 : 4;
    static constexpr int kFmt = BITS == 2 ? 2 : 0;    // fp6 e2m3 or fp8 e4m3
    static constexpr int kUnit = BITS == 2 ? 3 : 0;   // log2 of the integer a digit's code 1 stands for
    // the largest N whose balanced digits (from -base/2 to base/2 - 1) fit
    static constexpr float kNMax = BITS == 2 ? 16236015.0f : 7829367.0f;
};

typedef __attribute__((ext_vector_type(8))) int i32x8;

__device__ __forceinline__ float fexp2(float x) { return __builtin_amdgcn_exp2f(x); }

// LDS of a workgroup's query rows.  One region holds, in turn, the raw bf16
// queries, q~ (fp32, scaled) and the digit limbs in operand order; the limb
// scale bytes and sum(q~) of each head follow it.
template <int D, int G>
struct QueryLds {
    // the raw queries' row pitch in bf16 elements: rows 16 bytes apart in
    // the LDS banks, so that a column read across rows does not conflict
    static constexpr int kQPitch = D + 8;
    static constexpr int kRegion = G * D * 4 > G * kLimbRoom * 128 ? G * D * 4 : G * kLimbRoom * 128;
    static constexpr int kAux = kRegion;  // uint32 [G][4]: limb scales (E8M0 bytes, limbs
                                          // 0-3 then the rest), sum(q~) (fp32 bits), unused
    static constexpr int kBytes = kRegion + G * 16;
};

// Waves of the query-row kernels: one per 16 output columns (at d = 128 each
// wave then has half the T^{-1} reads, products and limbs that four waves would
// have: 8.5 instead of 10.2 us for the 16 rows of a chunk's token groups; the
// four rows of a decode take the same 8.6 us either way).
template <int D>
constexpr int kQtWaves = D / 16;

// The T^{-1} entries lane l of wave w supplies to form_qt_mfma: column
// 16 w + l % 16 at rows 4 st + l / 16.  Loaded on their own so that a kernel
// can request them together with the raw queries (one round trip).
template <int D>
struct TColumns {
    static constexpr int kSteps = D / 4;   // k steps of 4
    float bv[kSteps];
    __device__ __forceinline__ void load(const float *t_inv, int h, int tid)
    {
        const int lane = tid & 63, wave = tid >> 6;
        const float *T = t_inv + (int64_t)h * D * D + 16 * wave + (lane & 15);
#pragma unroll
        for (int st = 0; st < kSteps; ++st) bv[st] = T[(int64_t)(4 * st + (lane >> 4)) * D];
    }
};

// q~ on the fp32 matrix instructions, for the kernels that form query rows and
// no more (with no pages to overlap they are bound by the products): q~ = q^T T^{-1} as a
// (16 x D) x (D x D) product of 16x16x4 fp32 tiles, the G query rows padded
// to 16 with zeros.  Wave w takes the output columns 16 w .. 16 w + 15; lane
// l supplies A = q[l % 16][k0 + l / 16] and
// B = T^{-1}[k0 + l / 16][n0 + l % 16] and holds the result rows
// 4 (l / 16) .. + 3 of column n0 + l % 16.  The T^{-1} column entries of
// all steps come loaded in tc.  Same contract as form_qt in decode.hip (q~
// scaled, fp32, into R; starts and ends with a barrier); the products are
// summed in the matrix unit's order, so q~ may differ from form_qt's in the
// last bits.
template <int D, int G>
__device__ __forceinline__ void form_qt_mfma(float scale, const TColumns<D> &tc, uint8_t *R, int tid)
{
    constexpr int kSteps = TColumns<D>::kSteps;
    const uint16_t *qs = reinterpret_cast<const uint16_t *>(R);
    const int lane = tid & 63, wave = tid >> 6;
    const int m = lane & 15, kk = lane >> 4;
    __syncthreads();  // the staged queries
    // (two sums, so that a product need not wait for the one before it)
    f32x4 acc[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int st = 0; st < kSteps; ++st) {
        const float av = m < G ? bf16_bits_to_f32(qs[m * QueryLds<D, G>::kQPitch + 4 * st + kk]) : 0.0f;
        acc[st & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(av, tc.bv[st], acc[st & 1], 0, 0, 0);
    }
    __syncthreads();  // the raw queries are read
    float *qt = reinterpret_cast<float *>(R);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = 4 * kk + i;
        if (row < G) qt[row * D + 16 * wave + m] = (acc[0][i] + acc[1][i]) * scale;
    }
    __syncthreads();
}

// Rewrites q~ in R (form_qt_mfma, form_qt) as the operands of the
// quantised-key product: one wave per query head writes q~ in fixed point, N = rne(q~ 2^F) with F
// the largest exponent that keeps |N| <= kNMax, as balanced digits (N =
// sum_l d_l base^(kCount - 1 - l)).  Each digit is an integer of its number
// format and limb l carries the E8M0 scale base^(kCount - 1 - l) 2^-F, so
// every product the matrix instruction forms is an integer times a power of
// two: its block sums, which it does not accumulate at full fp32 precision
// in general, are exact.  Also sum(q~) per head.  Every thread of the
// workgroup calls it; it ends with a barrier.
//
// With 2-bit (fp4) keys the digits are five base-32 ones in fp6: the
// products of fp6 with fp4 operands run at twice the rate of those with an
// fp8 one (9.2 against 17 ns on one SIMD), five limbs hold a bit more than
// six base-16 ones, and an operand takes six registers instead of eight.
// With 4-bit (fp8) keys every product runs at the fp8 rate, so the digits
// are six base-16 ones in fp8.
// Operand order: lane group j of the instruction holds channels 32 j ..
// 32 j + 31 in its 32 bytes of a limb, one byte each (fp8) or six bits each
// in the first 24 (fp6).
template <int D, int BITS, int G, int NW = 4>
__device__ __forceinline__ void form_limbs(uint8_t *R, int tid)
{
    using Q = QueryLds<D, G>;
    const int lane = tid & 63, wave = tid >> 6;
    const float *qt = reinterpret_cast<const float *>(R);
    // wave w handles query heads w, w + NW, ..; the rows are read before the
    // region is rewritten
    constexpr int kPer = D / 64;  // channels per lane
    constexpr int kMine = (G + NW - 1) / NW;
    float r[kMine][kPer];
#pragma unroll
    for (int k = 0; k < kMine; ++k)
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            r[k][e] = (wave + NW * k < G) ? qt[(wave + NW * k) * D + 64 * e + lane] : 0.0f;
    __syncthreads();
    uint8_t *qlimb = R;
    uint32_t *qaux = reinterpret_cast<uint32_t *>(R + Q::kAux);
#pragma unroll
    for (int k = 0; k < kMine; ++k) {
        const int g = wave + NW * k;
        if (g >= G) break;
        float zs = 0.0f;
#pragma unroll
        for (int e = 0; e < kPer; ++e) zs += r[k][e];
        zs = wave_sum(zs);
        uint8_t *out = qlimb + g * (kLimbRoom * 128);
        float mx = 0.0f;
#pragma unroll
        for (int e = 0; e < kPer; ++e) mx = fmaxf(mx, fabsf(r[k][e]));
        mx = wave_max(mx);
        // fixed point N = rne(q~ 2^F), exact in fp32 (|N| < 2^24)
        using LB = Limbs<BITS>;
        int F = 0;
        if (mx > 0.0f) {
            int ex;
            (void)frexpf(LB::kNMax / mx, &ex);
            F = ex - 1;
            if (ldexpf(mx, F) > LB::kNMax) F -= 1;
            if (ldexpf(mx, F + 1) <= LB::kNMax) F += 1;
            F = F < -100 ? -100 : (F > 100 ? 100 : F);
        }
        uint32_t scales[2] = {0u, 0u};
#pragma unroll
        for (int l = 0; l < LB::kCount; ++l)
            scales[l >> 2] |= (uint32_t)(127 + LB::kUnit + LB::kDigitBits * (LB::kCount - 1 - l) - F) << (8 * (l & 3));
        constexpr int kHalfBase = 1 << (LB::kDigitBits - 1);
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int ch = 64 * e + lane;
            int N = (int)rintf(ldexpf(r[k][e], F));
#pragma unroll
            for (int l = LB::kCount - 1; l >= 0; --l) {
                const int d = ((N + kHalfBase) & (2 * kHalfBase - 1)) - kHalfBase;  // balanced digit
                N = (N - d) >> LB::kDigitBits;
                const uint32_t mag = (uint32_t)(d < 0 ? -d : d);
                uint32_t code;
                if constexpr (BITS == 2) {
                    // fp6 e2m3 of d / 8: up to 16 the code is the integer itself
                    code = mag | (d < 0 ? 0x20u : 0u);
                } else {
                    // fp8 e4m3 of the integer d: exponent and top mantissa bits
                    // of its fp32 form
                    const uint32_t fb = __float_as_uint((float)mag);
                    code = (d == 0 ? 0u : ((((fb >> 23) - 120u) << 3) | ((fb >> 20) & 7u))) | (d < 0 ? 0x80u : 0u);
                }
                out[l * 128 + ch] = (uint8_t)code;
            }
        }
        if (D == 64) {
            // channels 64 .. 127 of the operands: none, zero
            for (int l = 0; l < LB::kCount; ++l) out[l * 128 + 64 + lane] = 0;
        }
        if constexpr (BITS == 2) {
            // the codes, a byte each so far, packed to six bits: lane (limb,
            // c) takes the 16 codes of channels 16 c ..  (this wave wrote
            // them and reads them all before it writes over any)
            __builtin_amdgcn_wave_barrier();
            const int l = lane >> 3, c = lane & 7;
            const bool mine = l < LB::kCount;
            uint32_t p[4] = {0u, 0u, 0u, 0u};
            if (mine) {
                const u32x4 w = *reinterpret_cast<const u32x4 *>(out + l * 128 + 16 * c);
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    p[q] = (w[q] & 0x3Fu) | ((w[q] >> 2) & 0xFC0u) | ((w[q] >> 4) & 0x3F000u) | ((w[q] >> 6) & 0xFC0000u);
            }
            __builtin_amdgcn_wave_barrier();
            if (mine) {
                uint32_t *dst = reinterpret_cast<uint32_t *>(out + l * 128 + 32 * (c >> 1) + 12 * (c & 1));
                dst[0] = p[0] | (p[1] << 24);
                dst[1] = (p[1] >> 8) | (p[2] << 16);
                dst[2] = (p[2] >> 16) | (p[3] << 8);
            }
        }
        if (lane == 0) {
            qaux[4 * g] = scales[0];
            qaux[4 * g + 1] = scales[1];
            qaux[4 * g + 2] = __float_as_uint(zs);
            qaux[4 * g + 3] = 0u;
        }
    }
    __syncthreads();
}

__device__ __forceinline__ void __attribute__((address_space(3))) *lds_ptr(void *p)
{
    return (void __attribute__((address_space(3))) *)p;
}
__device__ __forceinline__ uint32_t lds_addr(const void *p)
{
    return (uint32_t)(uintptr_t)lds_ptr(const_cast<void *>(p));
}

// LDS reads and writes are ordinary loads and stores, so the compiler tracks
// their completion (and any register copies of their results) itself.  The
// direct-to-LDS page loads (dma16 in decode.hip) are not visible to it: it would
// otherwise wait for every one of them before any LDS access, since it
// cannot tell the staging slots apart from the rest of LDS.  Ordering
// against those loads is explicit: wait_vmcnt_at_most before a slot is read,
// lds_drain before a slot is refilled; both are compiler barriers.
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) u32x2 lds_u32x2;
typedef __attribute__((address_space(3))) uint16_t lds_u16;

__device__ __forceinline__ u32x4 lds_read16(uint32_t addr)
{
    return *(const lds_u32x4 *)(uintptr_t)addr;
}
__device__ __forceinline__ u32x2 lds_read8(uint32_t addr)
{
    return *(const lds_u32x2 *)(uintptr_t)addr;
}
__device__ __forceinline__ void lds_write8(uint32_t addr, uint32_t lo, uint32_t hi)
{
    *(lds_u32x2 *)(uintptr_t)addr = u32x2{lo, hi};
}
__device__ __forceinline__ void lds_write2(uint32_t addr, uint32_t v)
{
    *(lds_u16 *)(uintptr_t)addr = (uint16_t)v;
}
// Every LDS access issued so far has completed.  The assembly form is the
// compiler barrier (no memory access moves across it); the builtin form
// tells the compiler's wait bookkeeping that nothing is outstanding, so it
// adds no waits of its own for those accesses later.  (Encoding: vmcnt 63,
// expcnt 7, lgkmcnt 0.)
__device__ __forceinline__ void lds_drain()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);
}

// Query digits (fp6 with 2-bit keys, fp8 with 4-bit ones) times key codes
// (fp4 or fp8).
template <int BITS>
__device__ __forceinline__ f32x4 mfma_scaled(const i32x8 &a, const i32x8 &b, int scale_a, int scale_b, f32x4 c)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, Limbs<BITS>::kFmt, BITS == 2 ? 4 : 0, 0, scale_a,
                                                            0, scale_b);
}

// The value codes of one word as normal fp16 numbers, 16 c: registers as
// widen_word_f16 leaves them, all at one scale, for sums whose products lose no
// bits to subnormal inputs.  A code masked into bits F .. of the fraction of
// 1024 (whose bit 0 is 1) is 1024 + c 2^F, and one fused step takes it to
// (1024 + c 2^F) 2^(4-F) - 1024 2^(4-F) = 16 c, exactly, from whatever field the
// page has it in; only fields past the fraction are shifted first.  The
// constants stay in registers (an instruction takes one that is not).  With a middle
// (a whole number below 16, so that each is an fp16 number) they are 16 (c - middle),
// as exactly.
template <int BITS>
struct WidenNormal {
    uint32_t one;       // 1024, twice
    f16x2 add[5];       // -1024 2^(4-F) - 16 middle, F = 0, 2, 4, 6, 8
    // -x in fp16, twice
    static __device__ __forceinline__ uint32_t minus(float x)
    {
        const _Float16 y = (_Float16)-x;
        return __builtin_bit_cast(uint32_t, f16x2{y, y});
    }
    __device__ __forceinline__ void init(float middle = 0.0f)
    {
        const float m = 16.0f * middle;
        uint32_t v[6] = {0x64006400u,    minus(16384.0f + m), minus(4096.0f + m),
                         minus(1024.0f + m), minus(256.0f + m), minus(64.0f + m)};
#pragma unroll
        for (int i = 0; i < 6; ++i) asm volatile("" : "+v"(v[i]));
        one = v[0];
#pragma unroll
        for (int i = 0; i < 5; ++i) add[i] = __builtin_bit_cast(f16x2, v[1 + i]);
    }
    template <int F>
    __device__ __forceinline__ uint32_t at(uint32_t x) const
    {
        constexpr uint32_t code = (1u << BITS) - 1u;
        constexpr float mul = F == 0 ? 16.0f : F == 2 ? 4.0f : F == 4 ? 1.0f : F == 6 ? 0.25f : 0.0625f;
        const f16x2 v = __builtin_bit_cast(f16x2, (x & ((code << F) | (code << (F + 16)))) | one);
        const f16x2 m = {(_Float16)mul, (_Float16)mul};
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(v, m, add[F / 2]));
    }
    __device__ __forceinline__ void word(uint32_t w, uint32_t *out) const
    {
        if constexpr (BITS == 2) {
            const uint32_t r4 = w >> 4, r6 = w >> 6;
            out[0] = at<6>(w);
            out[1] = at<6>(r4);  // field 10
            out[2] = at<8>(w);
            out[3] = at<8>(r4);  // field 12
            out[4] = at<2>(w);
            out[5] = at<0>(w);
            out[6] = at<4>(w);
            out[7] = at<8>(r6);  // field 14
        } else {
            out[0] = at<4>(w);
            out[1] = at<0>(w);
            out[2] = at<4>(w >> 4);  // field 8
            out[3] = at<4>(w >> 8);  // field 12
        }
    }
};

// Byte offset of byte `byte` of a 128-byte weight row `row`: the 16-byte
// chunks of row r are stored in the order chunk ^ (r % 8), so that the rows
// one instruction reads together fall in distinct LDS banks.
__device__ __forceinline__ uint32_t tbuf_at(int row, int byte)
{
    return (uint32_t)(row * 128 + ((((byte >> 4) ^ (row & 7)) << 4) | (byte & 15)));
}

// One limb's scaled products with four tiles of 16 tokens: A = limb L of 16
// query rows, whose E8M0 scale is byte L % 4 of the lane's packed scale word
// (the instruction's byte select), B = the tokens' key codes.
template <int BITS, int L, int SCALE_B>
__device__ __forceinline__ void limb_products(const i32x8 &a, const i32x8 (&b)[4], int scales, f32x4 (&c)[4])
{
#pragma unroll
    for (int t = 0; t < 4; ++t)
        c[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b[t], c[t], Limbs<BITS>::kFmt, BITS == 2 ? 4 : 0,
                                                                L % 4, scales, 0, SCALE_B);
}

}  // namespace wushkv
