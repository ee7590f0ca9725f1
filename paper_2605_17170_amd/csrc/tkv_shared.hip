// tkv_decode_attention_shared: decode attention for sequences that share a long prefix (a system prompt, tool definitions, a
// document).  One launch attends to the prefixes' pages for all sequences of a group together and to each sequence's own pages
// (tkv_shared_kernel), and one merges the partials by log-sum-exp (tkv_merge_shared_kernel).
//
// With one sequence, a page is read for the eight query rows at most that share its kv head, and memory bounds the kernel.
// With S sequences there are S times as many rows for the same page: arithmetic bounds it, and the page's codes are
// worth expanding.
//
//   K, V  code * scale + zero in fp16, one rounding: the values that tkv_gather_dequant gives a prefill kernel.  The page layout
//         is that of the matrix operands, so a lane expands exactly what some lane feeds to the MFMAs.
//         Own pages and items of 16 rows hold K exactly: (code - 1) * scale + (zero + scale), the products in one fp16 number (INT2)
//         or two (INT4), zero and scale as stored against the sums of q, or as keys of their own.  Logits of 20 and more make
//         2^-12 of a key up to 2^-8 of a weight, and with few rows one such row is seen in the result: 4 sequences over 1500 tokens
//         were off by up to 0.0027 in norm where bf16 alone gives 0.0019, and are by 0.0019 (10.1 -> 10.4 us; 13 over 5000 12.5 -> 12.9).
//         With 64 and 128 rows, where results are off by 0.0017 to 0.0018, it would be 12 % more MFMAs for INT2 and 59 % for INT4.
//   QK^T  D[token, row] = sum_c K[token, c] q[row, c] (v_mfma_f32_16x16x32_f16), q in fp16, each row scaled by a power of two
//         of its own that its softmax factor takes back: bf16 has 8 bits, so q is exact down to 2^-26 of the row's largest.
//   PV    D[row, channel] = sum_token W[row, token] V[token, channel]: the results of QK^T lie where PV wants its operand.
//         W = 2^(logit - m + 8) in fp16, m a reference that follows the row's own maximum lazily (within 2^4), so that W stays
//         below 2^12 and weights down to 2^-22 of the largest are exact to half a step.  The denominators are one more MFMA
//         against ones: of the rounded weights, as the numerators.
// All sums are 32 bits.  V, W and the expanded K carry 11 bits where the split kernel carries what its fp32 results need; the output is
// bf16, which has 8.
//
// Workgroups of eight wavefronts, one a compute unit (198 to 256 registers), do one of three things:
//   own pages       a wavefront for each (work item, kv head), operands in registers, rows = the query heads of the kv head
//   16 rows         the wavefronts take an item's pages in turn, operands in registers; their results are added in LDS
//   64, 128 rows    two pages a step, each expanded once into LDS by the four wavefronts that attend to it with 16 or 32 rows each;
//                   the next two are expanded and the ones after them requested between QK^T and the softmax of a step
// Which of the latter two is planned by size (tkv_plan_decode_shared).
//
// What bounds it: 128 rows, a step 2.5 us, of which the SIMD's MFMAs take 1.09, its other vector instructions 1.0 (expansion and
// softmax about half each) and LDS 0.9 (256 KiB read, 64 written).  MFMAs and vector instructions of two wavefronts overlap
// by a third at most (16 MFMAs beside 64 multiply-adds 202 ns, alone 128 and 120).  256 rows over 32768 tokens, 8 kv heads: 55 us of
// steps and some 12 of loads that wait for one another, first expansion, and results on their way out; 64.1 us with the merge, 541 TFLOP/s
// (a large product of the library reaches 1100).  16 rows: the chain item -> group -> page ids -> codes -> softmax -> sums in LDS; a page for
// each wavefront takes 8 us.
// Tried and not kept: 64 rows a wavefront in registers (copies between register files, 85 us instead of 64), 32 rows a wavefront with pages
// of its own (130 registers spilled, 23 us instead of 12 to 15), the wavefronts of a SIMD half a step apart and raised priorities
// (no change), MFMAs and vector instructions interleaved by hand (66 to 70 us).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "tkv_internal.h"
#include "tkv_layout.h"

namespace {

using namespace tkv;

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
typedef __amdgpu_buffer_rsrc_t Record;
typedef const __attribute__((address_space(4))) int32_t *ConstWords;   // words that stay as they are during a launch: scalar loads

constexpr float kTau = 4.0f;   // a row's reference moves when a logit exceeds it by this much (log2 units)
constexpr int kPExp = 8;       // weights and their sums carry 2^8, as the partials of the split kernel do
constexpr int kWaves = 8;

__device__ __forceinline__ half8 as_half8(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    const uint4v v = {a, b, c, d};
    return __builtin_bit_cast(half8, v);
}
__device__ __forceinline__ floatx4 mfma(half8 a, half8 b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ uint32_t pack_h2(float a, float b)
{
    const half2_t v = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ float bf16_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
// Two codes in bits POS .. POS + BITS - 1 of the halves of x as fp16 numbers, times s plus z with one rounding per value.  A field
// of the mantissa under the exponent 25 - POS is 2^(10 - POS) + code, and subtracting the power of two is exact.
struct Magic {   // the exponents, in vector registers: v_and_or_b32 takes one constant besides
    uint32_t e[4];
    __device__ __forceinline__ Magic()
    {
        asm("v_mov_b32 %0, 0x64006400" : "=v"(e[0]));
        asm("v_mov_b32 %0, 0x5c005c00" : "=v"(e[1]));
        asm("v_mov_b32 %0, 0x54005400" : "=v"(e[2]));
        asm("v_mov_b32 %0, 0x4c004c00" : "=v"(e[3]));
    }
};
template <int BITS, int POS> __device__ __forceinline__ uint32_t dequant2(uint32_t x, uint32_t s, uint32_t z, const Magic &mg)
{
    static_assert(POS % 2 == 0 && POS + BITS <= 8, "a field of the mantissa");
    constexpr uint32_t m = ((1u << BITS) - 1u) * 0x00010001u << POS;
    constexpr float base = 1024 >> POS;
    const half2_t k = {(_Float16)base, (_Float16)base};
    const half2_t c = __builtin_bit_cast(half2_t, (x & m) | mg.e[POS / 2]) - k;
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(c, __builtin_bit_cast(half2_t, s), __builtin_bit_cast(half2_t, z)));
}
// Eight codes: fields k of the halves of x (BITS wide) are register k.
template <int BITS> __device__ __forceinline__ half8 dequant8(uint32_t x, uint32_t s0, uint32_t s1, uint32_t s2, uint32_t s3, uint32_t z0, uint32_t z1,
                                                              uint32_t z2, uint32_t z3, const Magic &mg)
{
    if constexpr (BITS == 2) {
        return as_half8(dequant2<2, 0>(x, s0, z0, mg), dequant2<2, 2>(x, s1, z1, mg), dequant2<2, 4>(x, s2, z2, mg), dequant2<2, 6>(x, s3, z3, mg));
    } else {
        const uint32_t y = x >> 8;
        return as_half8(dequant2<4, 0>(x, s0, z0, mg), dequant2<4, 4>(x, s1, z1, mg), dequant2<4, 0>(y, s2, z2, mg), dequant2<4, 4>(y, s3, z3, mg));
    }
}
// Codes less one times s, rounded to fp16, and in `rest` what the rounding took, which is exact; with two bits nothing: -s, 0, s, 2 s.
template <int BITS, int POS> __device__ __forceinline__ uint32_t times2(uint32_t x, uint32_t s, const Magic &mg, uint32_t &rest)
{
    constexpr uint32_t m = ((1u << BITS) - 1u) * 0x00010001u << POS;
    constexpr float base = (1024 >> POS) + 1;
    const half2_t k = {(_Float16)base, (_Float16)base}, sv = __builtin_bit_cast(half2_t, s);
    const half2_t c = __builtin_bit_cast(half2_t, (x & m) | mg.e[POS / 2]) - k, p = c * sv;
    if constexpr (BITS == 4) rest = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(c, sv, -p));
    return __builtin_bit_cast(uint32_t, p);
}
// Half i & 1 of v, twice.
__device__ __forceinline__ uint32_t twice(uint32_t v, int i) { return __builtin_amdgcn_perm(v, v, (i & 1) ? 0x07060706u : 0x05040504u); }
// Orders this wavefront's LDS writes before its later LDS reads: LDS operations of a wavefront execute in order.
__device__ __forceinline__ void lds_order()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
__device__ __forceinline__ uint4 load16(Record r, uint32_t offset)
{
    const uint4v v = __builtin_amdgcn_raw_buffer_load_b128(r, (int)offset, 0, 0);
    return make_uint4(v.x, v.y, v.z, v.w);
}

__device__ __forceinline__ uint2 load8(Record r, uint32_t offset)
{
    typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
    const u32x2_t v = __builtin_amdgcn_raw_buffer_load_b64(r, (int)offset, 0, 0);
    return make_uint2(v.x, v.y);
}
__device__ __forceinline__ uint32_t load4(Record r, uint32_t offset) { return __builtin_amdgcn_raw_buffer_load_b32(r, (int)offset, 0, 0); }

struct SharedArgs {
    const uint8_t *pool;
    const uint8_t *bit_map;
    const uint16_t *q;
    const int32_t *page_indptr;   // the sequences' own tokens
    const int32_t *page_ids;
    const int32_t *n_tok_int2;
    const int32_t *n_tok_int4;
    const int32_t *items;
    int n_items;      // own items: slots [0, n_items); the prefixes' partials have [n_items, n_slots)
    int own_blocks;   // the first workgroups, a wavefront for each (own item, kv head)
    int blocks;
    tkv_prefix p;
    int n_kv_heads;
    int log2_r;
    int n_pages_int2;
    int n_pages_int4;
    int batch;
    int n_slots;
    float kappa;      // sm_scale * log2(e)
    float *acc_ws[2]; // partials of the own items, of the prefixes
    float *ml_ws[2];
    int32_t *status;
};

template <int NT> struct Rows {   // NT tiles of 16 query rows
    half8 q[NT][4];        // operand of QK^T for a group of channels: row lane % 16, channels (k, k + 4) of octet lane / 16
    half8 sums[NT];        // of q over the four groups, row lane % 16, twice: rounded (lanes 0 .. 15), what that took (16 .. 31), 0
    floatx4 acc[NT][8];    // row 4 * (lane / 16) + i, channel 16 * tile + lane % 16
    floatx4 sum[NT];       // denominators, rows as in acc
    float m[NT];           // reference of row lane % 16, log2 units, -inf at first
    float shift[NT];       // kPExp less the reference, or less 0 for -inf
    float kappa[NT];       // of row lane % 16
    bool huge;             // whether some row's reference is so large that rounding it moves a weight by more than 2^-4
    bool look;             // that, or some row has no reference yet
};
template <int NT> __device__ __forceinline__ void clear(Rows<NT> &rows)
{
    rows.huge = false;
    rows.look = true;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        rows.m[n] = -INFINITY;
        rows.shift[n] = (float)kPExp;
        rows.sum[n] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < 8; ++c) rows.acc[n][c] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
}
// q of one tile; `row`: this lane's row of q, lane % 16 of the tile.
template <int NT> __device__ __forceinline__ void load_q(Rows<NT> &rows, int n, const uint16_t *__restrict__ row, float kappa, int lane)
{
    const uint4 *src = reinterpret_cast<const uint4 *>(row) + (lane >> 4);
    uint4 x[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) x[g] = src[4 * g];
    // the largest exponent of the row, from |x| as integers plus one in the exponent: NaN and infinities are 0x8000 and more
    typedef unsigned short ushort2_t __attribute__((ext_vector_type(2)));
    ushort2_t big = {0, 0};
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const uint32_t d[4] = {x[g].x, x[g].y, x[g].z, x[g].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) big = __builtin_elementwise_max(big, __builtin_bit_cast(ushort2_t, (d[k] & 0x7fff7fffu) + 0x00800080u));
    }
    int top = big[0] > big[1] ? big[0] : big[1];
    top = max(top, __shfl_xor(top, 16));
    top = max(top, __shfl_xor(top, 32));
    // the largest lies in [2^9, 2^10), and a sum over a group below 2^15; from -118 to 136, beyond what a factor of 32 bits can be
    const int E = top <= 0x80 ? 0 : 10 - ((top >> 7) - 127);
    // (a smaller factor weighs all tokens alike too, and zero times the -inf of a token that does not count would be NaN)
    rows.kappa[n] = fmaxf(ldexpf(kappa, -E), 0x1p-126f);
    if (top >= 0x8000) {
        // every weight of the row is NaN, also where all logits are -inf; with a reference, so that the wavefront's pages do not look for one
        rows.kappa[n] = __builtin_nanf("");
        rows.m[n] = 0.0f;
    }
    auto scaled = [&](float a, float b) { return pack_h2(ldexpf(a, E), ldexpf(b, E)); };
#pragma unroll
    for (int g = 0; g < 4; ++g)
        rows.q[n][g] = as_half8(scaled(bf16_lo(x[g].x), bf16_lo(x[g].z)), scaled(bf16_hi(x[g].x), bf16_hi(x[g].z)),
                                scaled(bf16_lo(x[g].y), bf16_lo(x[g].w)), scaled(bf16_hi(x[g].y), bf16_hi(x[g].w)));
}

__device__ __forceinline__ half8 ones() { return as_half8(0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u); }
// Sums of q over the groups of channels, for what K's zero-points add.
template <int NT> __device__ __forceinline__ void sum_q(Rows<NT> &rows, int n, int lane)
{
    float sum[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        sum[g] = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[g] += (float)rows.q[n][g][k];
        sum[g] += __shfl_xor(sum[g], 16);
        sum[g] += __shfl_xor(sum[g], 32);
    }
    const int q4 = lane >> 4;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const _Float16 hi = (_Float16)sum[k & 3], lo = (_Float16)(sum[k & 3] - (float)hi);
        rows.sums[n][k] = q4 == 0 ? hi : (q4 == 1 ? lo : (_Float16)0.0f);
    }
}

// ---- codes to operands -----------------------------------------------------------------------------------------------
// K of this lane's token for a group of channels: octet lane / 16, register k holds channels (k, k + 4).  w: the group's word;
// s, z: scales and zero-points of the four registers.
template <int BITS> __device__ __forceinline__ half8 k_operand(uint32_t w, const uint32_t (&s)[4], const uint32_t (&z)[4], int q4, const Magic &mg)
{
    // INT4: codes k and k + 4 lie in the halves of the word; INT2: the bytes of this lane's octet move there
    const uint32_t x = BITS == 4 ? w : __builtin_amdgcn_perm(w, w, (q4 & 1) ? 0x0c070c06u : 0x0c050c04u);
    return dequant8<BITS>(x, s[0], s[1], s[2], s[3], z[0], z[1], z[2], z[3], mg);
}
// The same without the zero-point, of codes less one; `rest`: see times2.
template <int BITS> __device__ __forceinline__ half8 k_products(uint32_t w, const uint32_t (&s)[4], int q4, const Magic &mg, half8 &rest)
{
    uint32_t p[4], r[4] = {};
    if constexpr (BITS == 2) {
        const uint32_t x = __builtin_amdgcn_perm(w, w, (q4 & 1) ? 0x0c070c06u : 0x0c050c04u);
        p[0] = times2<2, 0>(x, s[0], mg, r[0]);
        p[1] = times2<2, 2>(x, s[1], mg, r[1]);
        p[2] = times2<2, 4>(x, s[2], mg, r[2]);
        p[3] = times2<2, 6>(x, s[3], mg, r[3]);
    } else {
        const uint32_t y = w >> 8;
        p[0] = times2<4, 0>(w, s[0], mg, r[0]);
        p[1] = times2<4, 4>(w, s[1], mg, r[1]);
        p[2] = times2<4, 0>(y, s[2], mg, r[2]);
        p[3] = times2<4, 4>(y, s[3], mg, r[3]);
    }
    rest = as_half8(r[0], r[1], r[2], r[3]);
    return as_half8(p[0], p[1], p[2], p[3]);
}
// Scales (or zero-points) of per-channel INT2 keys in that order; `plane`: 32 chunks of 8, [block][group][quarter].
__device__ __forceinline__ void channel_meta(const uint4 *plane, int blk, int g, int q4, uint32_t (&s)[4])
{
    const uint4 a = plane[(blk * 4 + g) * 4 + 2 * (q4 >> 1)], b = plane[(blk * 4 + g) * 4 + 2 * (q4 >> 1) + 1];
    const uint32_t sel = (q4 & 1) ? 0x07060302u : 0x05040100u;
    s[0] = __builtin_amdgcn_perm(b.x, a.x, sel);
    s[1] = __builtin_amdgcn_perm(b.y, a.y, sel);
    s[2] = __builtin_amdgcn_perm(b.z, a.z, sel);
    s[3] = __builtin_amdgcn_perm(b.w, a.w, sel);
}
// V of this lane's channel for the eight tokens 32 b + 16 (j >> 2) + 4 (lane / 16) + (j & 3): register k holds j = (2k, 2k + 1).
template <int BITS> __device__ __forceinline__ half8 v_operand(uint32_t w, int b, uint4 s, uint4 z, const Magic &mg)
{
    const uint32_t x = BITS == 4 ? w : w >> (8 * b);   // INT2 words hold both blocks
    return dequant8<BITS>(x, s.x, s.y, s.z, s.w, z.x, z.y, z.z, z.w, mg);
}
// What was never written counts nothing, whatever stands there: chunk (b, quad) of the V planes with the tokens from n_valid on zero.
__device__ __forceinline__ uint4 mask_meta(uint4 v, int b, int quad, int n_valid)
{
    const int t0 = 32 * b + 4 * quad;
    auto mask = [&](int t) { return (t < n_valid ? 0xffffu : 0u) | (t + 1 < n_valid ? 0xffff0000u : 0u); };
    return make_uint4(v.x & mask(t0), v.y & mask(t0 + 2), v.z & mask(t0 + 16), v.w & mask(t0 + 18));
}
__device__ __forceinline__ uint32_t word_of(uint4 v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// Softmax weights of a page.  S: logits of its 16-token tiles (token 16 e + 4 (lane / 16) + i, row lane % 16), P: operands of PV for
// its 32-token blocks.  One test for all tiles whether a reference has to move.
template <int NT> __device__ __forceinline__ void weigh(Rows<NT> &rows, floatx4 (&S)[NT][4], int n_valid, int q4, half8 (&P)[NT][2])
{
    if (__builtin_expect(n_valid < kPageTokens, 0)) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < 4; ++i) S[n][e][i] = 16 * e + 4 * q4 + i < n_valid ? S[n][e][i] : -INFINITY;
    }
    float mx[NT], factor[NT], shift[NT];
    bool move = rows.look;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        mx[n] = S[n][0][0];
#pragma unroll
        for (int k = 1; k < 16; ++k) mx[n] = __builtin_elementwise_maximum(mx[n], S[n][k >> 2][k & 3]);
        factor[n] = rows.kappa[n];
        shift[n] = rows.shift[n];
        // (a row of NaN compares false and keeps its reference: its weights are NaN)
        move = move || mx[n] * factor[n] + shift[n] > kTau + (float)kPExp;
    }
    if (__any(move)) {
        bool none = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float top = fmaxf(mx[n], __shfl_xor(mx[n], 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            // Only a row that exceeds its own reference moves: its result does not depend on the wavefront's other rows.  (8 sequences over
            // 11000 tokens 19.0 -> 19.15 us, 4 over 1500 10.4 -> 10.5 against all of them moving together.)
            const float old = rows.m[n];
            const bool moves = old == -INFINITY || top * factor[n] + shift[n] > kTau + (float)kPExp;
            const float m_new = moves ? fmaxf(old, top * factor[n]) : old;
            const float alpha = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(old - m_new);
            rows.m[n] = m_new;
            rows.huge = rows.huge || __any(fabsf(m_new) > 0x1p20f && m_new != -INFINITY);
            none = none || m_new == -INFINITY;
            const float ref = m_new == -INFINITY ? 0.0f : m_new;
            rows.shift[n] = shift[n] = (float)kPExp - ref;
            floatx4 av;
#pragma unroll
            for (int i = 0; i < 4; ++i) av[i] = __shfl(alpha, 4 * q4 + i);
#pragma unroll
            for (int c = 0; c < 8; ++c) rows.acc[n][c] *= av;
            rows.sum[n] *= av;
        }
        rows.look = rows.huge || __any(none);
        if (rows.huge) {
            // factor * logit with one rounding, as the reference has it, then the difference: the largest weight is 2^8
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const bool huge = fabsf(rows.m[n]) > 0x1p20f && rows.m[n] != -INFINITY;
                const float ref = huge ? rows.m[n] : 0.0f, f = huge ? factor[n] : 1.0f;
#pragma unroll
                for (int e = 0; e < 4; ++e) S[n][e] = S[n][e] * f - ref;
                factor[n] = huge ? 1.0f : factor[n];
                shift[n] = huge ? (float)kPExp : shift[n];
            }
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const floatx4 x = S[n][2 * b + (k >> 1)];
                w[k] = pack_h2(__builtin_amdgcn_exp2f(fmaf(x[2 * (k & 1)], factor[n], shift[n])), __builtin_amdgcn_exp2f(fmaf(x[2 * (k & 1) + 1], factor[n], shift[n])));
            }
            P[n][b] = as_half8(w[0], w[1], w[2], w[3]);
        }
}

// ---- the pages of a list, 64 at a time in registers: lane l holds page number base + l ------------------------------------
struct PageList {
    int base;
    uint32_t at;   // where the record starts in the pool, in units of kUnit; kNowhere: it cannot be read
    int valid;     // tokens of the page that count
};
constexpr uint32_t kNowhere = 0xffffffffu;
constexpr int kUnitLog2 = 11;   // record and arena sizes are multiples of it
static_assert(Rec<2>::kBytes % (1 << kUnitLog2) == 0 && Rec<4>::kBytes % (1 << kUnitLog2) == 0, "record unit");
struct ListCtx {
    const uint8_t *pool;
    const uint8_t *bit_map;
    const int32_t *pages;
    int first, step, n;                  // page number i stands at list position first + step * i; n of them
    int np2, np4, last2, last4;          // pages of either width of the list, tokens of the last ones
    int kvh, n_kv_heads, n_pages_int2, n_pages_total, lane;
    int32_t *status;
    __device__ __forceinline__ bool is2(int i) const { return first + step * i < np2; }
};
__device__ __forceinline__ void fetch_list(const ListCtx &cx, PageList &l, int base)
{
    l.base = base;
    const int i = base + cx.lane < cx.n ? base + cx.lane : cx.n - 1;
    const int pos = cx.first + cx.step * i;
    const int page = cx.pages[pos];
    const bool is2 = pos < cx.np2;
    const int lo = is2 ? 0 : cx.n_pages_int2, hi = is2 ? cx.n_pages_int2 : cx.n_pages_total;
    const bool ok = page >= lo && page < hi;
    if (!ok && cx.status) atomicOr(cx.status, page < 0 || page >= cx.n_pages_total ? TKV_STATUS_PAGE_RANGE : TKV_STATUS_BITMAP_MISMATCH);
    // a page that cannot be read counts no tokens, and nothing is read in its place (the record's size is 0, see record_of); one that
    // was never written is read, and counts none either: its request does not wait for bit_map
    const uint32_t rec = (uint32_t)(is2 ? page : page - cx.n_pages_int2) * (uint32_t)cx.n_kv_heads + (uint32_t)cx.kvh;
    constexpr uint32_t kUnits2 = Rec<2>::kBytes >> kUnitLog2, kUnits4 = Rec<4>::kBytes >> kUnitLog2;
    l.at = !ok ? kNowhere : (is2 ? rec * kUnits2 : (uint32_t)cx.n_pages_int2 * (uint32_t)cx.n_kv_heads * kUnits2 + rec * kUnits4);   // (pools below 8 TB: 32 bits)
    const bool written = ok && cx.bit_map[ok ? page : 0] == (is2 ? 2 : 4);
    if (ok && !written && cx.status) atomicOr(cx.status, TKV_STATUS_BITMAP_MISMATCH);
    l.valid = !written ? 0 : (pos == cx.np2 - 1 ? cx.last2 : pos == cx.np2 + cx.np4 - 1 ? cx.last4 : kPageTokens);
}
__device__ __forceinline__ int valid_of(const PageList &l, int i) { return __builtin_amdgcn_readlane(l.valid, i - l.base); }
__device__ __forceinline__ Record record_of(const ListCtx &cx, const PageList &l, int i, bool wanted)
{
    const uint32_t at = (uint32_t)__builtin_amdgcn_readlane((int)l.at, i - l.base);
    const bool there = wanted && at != kNowhere;
    const int bytes = cx.is2(i) ? Rec<2>::kBytes : Rec<4>::kBytes;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(cx.pool) + ((uint64_t)(there ? at : 0) << kUnitLog2), 0, there ? bytes : 0, 0x00027000);
}

// ---- few rows: a wavefront works on pages of its own -------------------------------------------------------------------
template <int BITS> struct PageRegs {   // what a lane loads of one (page, kv head) record
    uint4 kw[4];      // K codes: four group words of this lane's token of each 16-token tile
    uint4 vw[BITS];   // V codes: chunk 64 i + lane of the plane
    uint4 km, vm;     // 16 bytes of the K scale | K zero planes, of the V scale | V zero planes
};
struct alignas(16) Meta {   // of one wavefront's page
    uint4 k[64], v[64];
};
template <int BITS> __device__ __forceinline__ void load_k(PageRegs<BITS> &r, Record rec, int lane)
{
    using R = Rec<BITS>;
    r.km = load16(rec, R::kKScale + 16 * lane);
    const int at = BITS == 4 ? lane : (lane >> 5) * 16 + (lane & 15);   // INT2: the two lanes of a half group share a chunk
#pragma unroll
    for (int e = 0; e < 4; ++e) r.kw[e] = load16(rec, R::kKCodes + 16 * (e * 16 * BITS + at));
}
template <int BITS> __device__ __forceinline__ void load_v(PageRegs<BITS> &r, Record rec, int lane)
{
    using R = Rec<BITS>;
    r.vm = load16(rec, R::kVScale + 16 * lane);
#pragma unroll
    for (int i = 0; i < BITS; ++i) r.vw[i] = load16(rec, R::kVCodes + 1024 * i + 16 * lane);
}
// One page.  The K registers are free behind after_qk, the V registers behind the function.
template <int NT, int BITS, bool KC, class AfterQK>
__device__ __forceinline__ void attend_page(const PageRegs<BITS> &r, int n_valid, int lane, Rows<NT> &rows, Meta &meta, const Magic &mg, AfterQK after_qk)
{
    const int r16 = lane & 15, q4 = lane >> 4;
    meta.k[lane] = r.km;
    // this lane's chunk of the V planes: lane % 32 = (block, quad, group)
    meta.v[lane] = n_valid < kPageTokens ? mask_meta(r.vm, (lane >> 4) & 1, (lane >> 2) & 3, n_valid) : r.vm;
    lds_order();
    // K = (code - 1) * s + (z + s): the products by themselves are exact, and so are z and s, which stand for a token and a group (one MFMA
    // against the sums of q) or for a channel and 32 tokens (as keys of their own, of which all tokens have the same)
    floatx4 S[NT][4];   // token 16 e + 4 q4 + i, row r16
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        uint32_t s[4][4];
        uint2 sc[2], zc[2];
        if constexpr (KC && BITS == 2) {
#pragma unroll
            for (int n = 0; n < NT; ++n) S[n][2 * b] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                uint32_t z[4];
                channel_meta(meta.k, b, g, q4, s[g]);
                channel_meta(meta.k + 32, b, g, q4, z);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    S[n][2 * b] = mfma(as_half8(z[0], z[1], z[2], z[3]), rows.q[n][g], S[n][2 * b]);
                    S[n][2 * b] = mfma(as_half8(s[g][0], s[g][1], s[g][2], s[g][3]), rows.q[n][g], S[n][2 * b]);
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) S[n][2 * b + 1] = S[n][2 * b];
        } else {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                sc[e] = reinterpret_cast<const uint2 *>(meta.k)[32 * b + 16 * e + r16];
                zc[e] = reinterpret_cast<const uint2 *>(meta.k + 32)[32 * b + 16 * e + r16];
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    S[n][2 * b + e] = mfma(as_half8(zc[e].x, zc[e].y, sc[e].x, sc[e].y), rows.sums[n], floatx4{0.f, 0.f, 0.f, 0.f});
            }
        }
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if constexpr (!(KC && BITS == 2)) s[g][0] = s[g][1] = s[g][2] = s[g][3] = twice(g < 2 ? sc[e].x : sc[e].y, g);
                half8 rest;
                const half8 A = k_products<BITS>(word_of(r.kw[2 * b + e], g), s[g], q4, mg, rest);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    S[n][2 * b + e] = mfma(A, rows.q[n][g], S[n][2 * b + e]);
                    if constexpr (BITS == 4) S[n][2 * b + e] = mfma(rest, rows.q[n][g], S[n][2 * b + e]);
                }
            }
    }
    after_qk();
    half8 P[NT][2];
    weigh(rows, S, n_valid, q4, P);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int n = 0; n < NT; ++n) rows.sum[n] = mfma(P[n][b], ones(), rows.sum[n]);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const uint4 s = meta.v[(b * 4 + q4) * 4 + g], z = meta.v[32 + (b * 4 + q4) * 4 + g];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int tile = 2 * g + c, half = tile >> 2;
                const half8 B = v_operand<BITS>(word_of(r.vw[BITS == 4 ? b * 2 + half : half], tile & 3), b, s, z, mg);
#pragma unroll
                for (int n = 0; n < NT; ++n) rows.acc[n][tile] = mfma(P[n][b], B, rows.acc[n][tile]);
            }
        }
    }
}
// Pages [i, end), all of one width.
template <int NT, int BITS, bool KC>
__device__ __forceinline__ void run_pages(const ListCtx &cx, PageList &list, int i, int end, Rows<NT> &rows, Meta &meta)
{
    const Magic mg;
    PageRegs<BITS> r;
    Record rec = record_of(cx, list, i, true);
    load_k(r, rec, cx.lane);
    load_v(r, rec, cx.lane);
    for (; i < end; ++i) {
        const int valid = valid_of(list, i);
        const bool more = i + 1 < end;
        if (more && i + 1 - list.base >= 64) fetch_list(cx, list, i + 1);
        rec = record_of(cx, list, more ? i + 1 : i, more);
        if (valid > 0) {
            attend_page<NT, BITS, KC>(r, valid, cx.lane, rows, meta, mg, [&]() {
                __builtin_amdgcn_sched_barrier(0);
                load_k(r, rec, cx.lane);
            });
        } else {
            load_k(r, rec, cx.lane);
        }
        __builtin_amdgcn_sched_barrier(0);
        load_v(r, rec, cx.lane);
    }
}
template <int NT, bool KC> __device__ __forceinline__ void run_list(const ListCtx &cx, PageList &list, Rows<NT> &rows, Meta &meta)
{
    if (cx.n <= 0) return;
    int n2 = cx.first < cx.np2 ? (cx.np2 - cx.first + cx.step - 1) / cx.step : 0;   // INT2 pages: they come first
    n2 = n2 < cx.n ? n2 : cx.n;
    if (n2 > 0) run_pages<NT, 2, KC>(cx, list, 0, n2, rows, meta);
    if (n2 < cx.n) {
        if (n2 - list.base >= 64) fetch_list(cx, list, n2);
        run_pages<NT, 4, KC>(cx, list, n2, cx.n, rows, meta);
    }
}

// ---- many rows: four wavefronts expand a page together, and each attends to it with rows of its own ------------------------
// Wavefront (rw, th) = (wave % 4, wave / 4) owns row tiles rw * NT ... and every second page, th first.  The operands of a page
// stand in LDS as the MFMAs take them, 1 KiB each: K (token tile e, group g), V (block b, channel tile).  Of its next page
// it expands K tile rw and the V operands of chunk rw = (block, channel half) of the plane, while the others of its four
// wavefronts expand theirs.
struct alignas(16) Operands {
    uint4 k[16][64], v[16][64];
};
struct RawPage {   // this lane's part of a page as stored
    uint4 kw, vw;         // four group words of its token, four channel words of its tokens
    uint4 km;             // K scales (x, y) and zeros (z, w) of its token; per-channel INT2 keys: chunk `lane` of the K planes
    uint4 vs[2], vz[2];   // V scales and zero-points of its eight tokens, two groups
};
template <int BITS, bool KC> __device__ __forceinline__ void load_raw(RawPage &r, Record rec, int rw, int lane)
{
    using R = Rec<BITS>;
    const int r16 = lane & 15;
    r.kw = load16(rec, R::kKCodes + 16 * (BITS == 4 ? rw * 64 + lane : rw * 32 + (lane >> 5) * 16 + r16));
    if constexpr (KC && BITS == 2) {
        r.km = load16(rec, R::kKScale + 16 * lane);
    } else {
        const uint2 s = load8(rec, R::kKScale + 8 * (16 * rw + r16)), z = load8(rec, R::kKZero + 8 * (16 * rw + r16));
        r.km = make_uint4(s.x, s.y, z.x, z.y);
    }
    r.vw = load16(rec, R::kVCodes + 16 * ((BITS == 4 ? rw : rw & 1) * 64 + lane));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int chunk = ((rw >> 1) * 4 + (lane >> 4)) * 4 + 2 * (rw & 1) + i;
        r.vs[i] = load16(rec, R::kVScale + 16 * chunk);
        r.vz[i] = load16(rec, R::kVZero + 16 * chunk);
    }
}
template <int BITS, bool KC> __device__ __forceinline__ void expand(RawPage &r, int n_valid, int rw, int lane, Operands &o, uint4 *stage, const Magic &mg)
{
    const int q4 = lane >> 4, b = rw >> 1;
    if constexpr (KC && BITS == 2) {
        stage[lane] = r.km;
        lds_order();
    }
    if (__builtin_expect(n_valid < kPageTokens, 0))
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            r.vs[i] = mask_meta(r.vs[i], b, q4, n_valid);
            r.vz[i] = mask_meta(r.vz[i], b, q4, n_valid);
        }
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        uint32_t s[4], z[4];
        if constexpr (KC && BITS == 2) {
            channel_meta(stage, b, g, q4, s);
            channel_meta(stage + 32, b, g, q4, z);
        } else {
            s[0] = s[1] = s[2] = s[3] = twice(g < 2 ? r.km.x : r.km.y, g);
            z[0] = z[1] = z[2] = z[3] = twice(g < 2 ? r.km.z : r.km.w, g);
        }
        o.k[rw * 4 + g][lane] = __builtin_bit_cast(uint4, k_operand<BITS>(word_of(r.kw, g), s, z, q4, mg));
    }
#pragma unroll
    for (int c = 0; c < 4; ++c)
        o.v[b * 8 + 4 * (rw & 1) + c][lane] = __builtin_bit_cast(uint4, v_operand<BITS>(word_of(r.vw, c), b, r.vs[c >> 1], r.vz[c >> 1], mg));
}
// The logits of a page, what `between` does, and the rest.  Operands are asked for eight MFMAs ahead of the first that takes them, those
// of V ahead of the exponentials: left to the compiler's order, each read stood right in front of its MFMAs.
template <int NT, class Between> __device__ __forceinline__ void attend_operands(const Operands &o, int n_valid, int lane, Rows<NT> &rows, Between between)
{
    const int q4 = lane >> 4;
    auto k_at = [&](int g, int e) { return __builtin_bit_cast(half8, o.k[e * 4 + g][lane]); };
    auto v_at = [&](int b, int c) { return __builtin_bit_cast(half8, o.v[b * 8 + c][lane]); };
    floatx4 S[NT][4];
    half8 A[2][4];
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) A[g][e] = k_at(g, e);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int n = 0; n < NT; ++n) S[n][e] = mfma(A[g & 1][e], rows.q[n][g], g == 0 ? floatx4{0.f, 0.f, 0.f, 0.f} : S[n][e]);
        __builtin_amdgcn_sched_barrier(0);
        if (g < 2)
#pragma unroll
            for (int e = 0; e < 4; ++e) A[g & 1][e] = k_at(g + 2, e);
    }
    between();
    half8 B[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) B[c] = v_at(0, c);
    __builtin_amdgcn_sched_barrier(0);
    half8 P[NT][2];
    weigh(rows, S, n_valid, q4, P);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int n = 0; n < NT; ++n) rows.sum[n] = mfma(P[n][b], ones(), rows.sum[n]);
#pragma unroll
        for (int c = 0; c < 8; ++c) {
#pragma unroll
            for (int n = 0; n < NT; ++n) rows.acc[n][c] = mfma(P[n][b], B[c], rows.acc[n][c]);
            if (b == 0) {
                __builtin_amdgcn_sched_barrier(0);
                B[c] = v_at(1, c);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
}
struct TileLds {
    Operands page[2][2];   // [step % 2][th]
    uint4 stage[kWaves][64];
};
// Pages [i0, end) of the list, all of one width; the same number of steps, and barriers, in all wavefronts.
template <int NT, int BITS, bool KC>
__device__ __forceinline__ void run_tiles(const ListCtx &cx, PageList &list, int i0, int end, bool active, int wave, Rows<NT> &rows, TileLds &lds)
{
    const int rw = wave & 3, th = wave >> 2, lane = cx.lane;
    const Magic mg;
    RawPage raw;
    int valid = 0, valid_next = 0;   // tokens of this step's page and of the next one's; 0: none
    // (behind the last page an empty record: zeros, without a branch around the loads)
    auto request = [&](int i) -> int {
        const bool wanted = i < end;
        const int k = wanted ? i : end - 1;
        if (k - list.base >= 64) fetch_list(cx, list, k);
        load_raw<BITS, KC>(raw, record_of(cx, list, k, wanted), rw, lane);
        return wanted ? valid_of(list, k) : 0;
    };
    int i = i0 + th;
    valid = request(i);
    expand<BITS, KC>(raw, valid, rw, lane, lds.page[0][th], lds.stage[wave], mg);
    valid_next = request(i + 2);
    __syncthreads();
    // (two loops: with wavefronts with and without rows in one, the registers of either wait for the other's loads)
    auto steps = [&](auto rows_here) {
        for (int step = 0, n = (end - i0 + 1) / 2; step < n; ++step, i += 2) {
            Operands &now = lds.page[step & 1][th], &next = lds.page[(step + 1) & 1][th];
            int valid_after = 0;
            auto prepare_next = [&]() {
                expand<BITS, KC>(raw, valid_next, rw, lane, next, lds.stage[wave], mg);
                valid_after = request(i + 4);
            };
            if constexpr (decltype(rows_here)::value) attend_operands<NT>(now, valid, lane, rows, prepare_next);
            else prepare_next();
            __syncthreads();   // this step's pages are read, the next ones stand there
            valid = valid_next;
            valid_next = valid_after;
        }
    };
    if (active) steps(std::true_type());
    else steps(std::false_type());
}

// ---- work items ----------------------------------------------------------------------------------------------------------
// MODE 0: one row tile, every wavefront with pages of its own; 1, 2: MODE row tiles a wavefront, pages expanded together.  (Two row tiles
// with pages of their own do not fit the registers of two wavefronts a SIMD.)
constexpr int tiles_of(int mode) { return mode == 0 ? 1 : mode; }
constexpr int rows_of(int mode) { return mode == 0 ? 16 : 64 * mode; }
constexpr int kOutRow = kHeadDim + 4;   // floats: rows 4 q4 + i of a store fall on different banks
template <int SETS, int ROWS> struct Results {   // of SETS wavefronts for the same rows, on their way out
    float acc[SETS][ROWS][kOutRow];
    float m[SETS][ROWS], sum[SETS][ROWS];
};
template <int MODE> struct Shared {
    int64_t dest[rows_of(MODE)];   // row of each query row's partial, or -1
    static constexpr int kSets = MODE == 0 ? kWaves : 2;
    union {
        Meta meta[kWaves];
        std::conditional_t<MODE == 0, Meta, TileLds> tile;
        Results<kSets, rows_of(MODE)> out;
        union {
            Meta meta;
            float acc[8][kOutRow];
        } own[kWaves];
    };
};

// Channels 4 c4 ... of a partial's row; 32 lanes store a row.  THROUGH: the L2 passes it on to memory at once, since the merge begins behind
// the write-back of what is dirty.  64 and 128 rows: 19.2 -> 18.7 us for 8 sequences over 11000 tokens, 65.4 -> 63.6 for 32 over 32768; but not
// for the few partials of 16 rows, 10.1 -> 10.4 for 4 over 1500.
template <bool THROUGH> __device__ __forceinline__ void store_row(float *row, int c4, float4 v)
{
    if constexpr (THROUGH) {
        const floatx4 t = {v.x, v.y, v.z, v.w};
        asm volatile("global_store_dwordx4 %0, %1, off sc1\n\ts_nop 1" :: "v"(row + 4 * c4), "v"(t) : "memory");   // (the wait state: see store_once_through)
    } else {
        reinterpret_cast<float4 *>(row)[c4] = v;
    }
}
// The own tokens of a sequence: a wavefront for each (item, kv head), whose rows are the query heads of the kv head.
template <bool KC, bool THROUGH, class L> __device__ __forceinline__ void own_item(const SharedArgs &a, L &lds, int block, int wave, int lane)
{
    const int r16 = lane & 15, q4 = lane >> 4, R = 1 << a.log2_r, n_q_heads = a.n_kv_heads << a.log2_r;
    const int64_t unit = (int64_t)block * kWaves + wave;
    if (unit >= (int64_t)a.n_items * a.n_kv_heads) return;
    const int item = (int)(unit / a.n_kv_heads), kvh = (int)(unit % a.n_kv_heads);
    const ConstWords words = (ConstWords)(a.items + 4 * (size_t)item);
    const int seq = words[0], item_pb = words[1], item_pe = words[2], slot = words[3];
    const bool seq_ok = seq >= 0 && seq < a.batch, slot_ok = slot >= 0 && slot < a.n_items;
    if (!(seq_ok && slot_ok) && a.status && lane == 0) atomicOr(a.status, TKV_STATUS_BAD_ITEM);
    if (!slot_ok) return;
    const int sq = seq_ok ? seq : 0;
    const int n2 = ((ConstWords)a.n_tok_int2)[sq], n4 = ((ConstWords)a.n_tok_int4)[sq];
    const int list0 = ((ConstWords)a.page_indptr)[sq], list1 = ((ConstWords)a.page_indptr)[sq + 1];
    const int np2 = (n2 + kPageTokens - 1) / kPageTokens, np4 = (n4 + kPageTokens - 1) / kPageTokens;
    const int np = np2 + np4 < list1 - list0 ? np2 + np4 : list1 - list0;
    const int pb = item_pb > 0 ? item_pb : 0, pe = item_pe < np ? item_pe : np;
    Rows<1> rows;
    clear(rows);
    if (seq_ok && pb < pe) {
        const ListCtx cx = {a.pool, a.bit_map, a.page_ids + list0, pb, 1, pe - pb, np2, np4, n2 - (np2 - 1) * kPageTokens, n4 - (np4 - 1) * kPageTokens,
                            kvh, a.n_kv_heads, a.n_pages_int2, a.n_pages_int2 + a.n_pages_int4, lane, a.status};
        PageList list;
        fetch_list(cx, list, 0);
        load_q(rows, 0, a.q + ((size_t)sq * n_q_heads + kvh * R + (r16 & (R - 1))) * kHeadDim, a.kappa, lane);
        sum_q(rows, 0, lane);
        run_list<1, KC>(cx, list, rows, lds.own[wave].meta);
    }
    const size_t at = (size_t)slot * n_q_heads + kvh * R;
    if (q4 == 0 && r16 < R) a.ml_ws[0][2 * (at + r16)] = rows.m[0];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (r16 == 0 && 4 * q4 + i < R) a.ml_ws[0][2 * (at + 4 * q4 + i) + 1] = rows.sum[0][i];
    lds_order();   // the metadata is read
    if (q4 < 2)
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) lds.own[wave].acc[4 * q4 + i][16 * c + r16] = rows.acc[0][c][i];
    lds_order();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int r = 2 * k + (lane >> 5), c4 = lane & 31;
        if (r < R) store_row<THROUGH>(a.acc_ws[0] + (at + r) * kHeadDim, c4, *reinterpret_cast<const float4 *>(&lds.own[wave].acc[r][4 * c4]));
    }
}

// A prefix's pages [item_pb, item_pe) for rows_of(MODE) query rows of its members.
template <int MODE, bool KC> __device__ __forceinline__ void prefix_item(const SharedArgs &a, Shared<MODE> &lds, int block, int wave, int lane)
{
    constexpr int NT = tiles_of(MODE), ROWS = rows_of(MODE), SETS = Shared<MODE>::kSets;
    const int r16 = lane & 15, q4 = lane >> 4, R = 1 << a.log2_r, n_q_heads = a.n_kv_heads << a.log2_r;
    const int item = block / a.n_kv_heads, kvh = block - item * a.n_kv_heads;
    const ConstWords words = (ConstWords)(a.p.items + 5 * (size_t)item);
    const int group = words[0], item_pb = words[1], item_pe = words[2], part = words[3], row0 = words[4];
    if (group < 0 || group >= a.p.n_groups || part < 0 || row0 < 0) {
        if (a.status && threadIdx.x == 0) atomicOr(a.status, TKV_STATUS_BAD_ITEM);
        return;
    }
    int m0 = ((ConstWords)a.p.member_indptr)[group], m1 = ((ConstWords)a.p.member_indptr)[group + 1];
    const int n2 = ((ConstWords)a.p.n_tok_int2)[group], n4 = ((ConstWords)a.p.n_tok_int4)[group];
    const int list0 = ((ConstWords)a.p.page_indptr)[group], list1 = ((ConstWords)a.p.page_indptr)[group + 1];
    m0 = m0 > 0 ? m0 : 0;
    m1 = m1 < a.p.n_members ? m1 : a.p.n_members;
    const int n_rows = (m1 - m0) << a.log2_r;
    if (row0 >= n_rows) return;
    const int np2 = (n2 + kPageTokens - 1) / kPageTokens, np4 = (n4 + kPageTokens - 1) / kPageTokens;
    const int np = np2 + np4 < list1 - list0 ? np2 + np4 : list1 - list0;
    const int pb = item_pb > 0 ? item_pb : 0, pe = item_pe < np ? item_pe : np;

    const int first = MODE == 0 ? pb + wave : pb, step = MODE == 0 ? kWaves : 1;
    const ListCtx cx = {a.pool, a.bit_map, a.p.page_ids + list0, first, step, first < pe ? (pe - first + step - 1) / step : 0, np2, np4,
                        n2 - (np2 - 1) * kPageTokens, n4 - (np4 - 1) * kPageTokens,
                        kvh, a.n_kv_heads, a.n_pages_int2, a.n_pages_int2 + a.n_pages_int4, lane, a.status};
    PageList list = {0, kNowhere, 0};
    if (cx.n > 0) fetch_list(cx, list, 0);
    // where the rows' partials go, while the pages' ids are under way
    if (threadIdx.x < ROWS) {
        const int row = row0 + threadIdx.x;
        int64_t dest = -1;
        if (row < n_rows) {
            const int member = m0 + (row >> a.log2_r), seq = a.p.member_seqs[member];
            const int64_t slot = (int64_t)a.p.member_slots[member] + part;
            if (seq >= 0 && seq < a.batch && slot >= a.n_items && slot < a.n_slots)
                dest = (slot - a.n_items) * n_q_heads + kvh * R + (row & (R - 1));
            else if (a.status)
                atomicOr(a.status, TKV_STATUS_BAD_ITEM);
        }
        lds.dest[threadIdx.x] = dest;
    }
    const int wave_row = MODE == 0 ? 0 : (wave & 3) * 16 * NT;   // this wavefront's first row of the workgroup
    const bool active = row0 + wave_row < n_rows;
    Rows<NT> rows;
    clear(rows);
    if (active) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int row = row0 + wave_row + 16 * n + r16;
            int seq = row < n_rows ? a.p.member_seqs[m0 + (row >> a.log2_r)] : 0;
            if (seq < 0 || seq >= a.batch) seq = 0;   // nothing of it is stored
            load_q(rows, n, a.q + ((size_t)seq * n_q_heads + kvh * R + (row & (R - 1))) * kHeadDim, a.kappa, lane);
            if constexpr (MODE == 0) sum_q(rows, n, lane);
        }
    }
    if constexpr (MODE == 0) {
        run_list<NT, KC>(cx, list, rows, lds.meta[wave]);
    } else if (cx.n > 0) {
        int n2 = first < np2 ? np2 - first : 0;   // INT2 pages: they come first
        n2 = n2 < cx.n ? n2 : cx.n;
        if (n2 > 0) run_tiles<NT, 2, KC>(cx, list, 0, n2, active, wave, rows, lds.tile);
        if (n2 < cx.n) run_tiles<NT, 4, KC>(cx, list, n2, cx.n, active, wave, rows, lds.tile);
    }

    // ---- results of the wavefronts for the same rows are brought to a common reference, added and stored ------------------
    if constexpr (MODE == 0) __syncthreads();   // no page is being worked on
    const int set = MODE == 0 ? wave : wave >> 2;
    if (active) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int r = wave_row + 16 * n;
            if (q4 == 0) lds.out.m[set][r + r16] = rows.m[n];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (r16 == 0) lds.out.sum[set][r + 4 * q4 + i] = rows.sum[n][i];
#pragma unroll
                for (int c = 0; c < 8; ++c) lds.out.acc[set][r + 4 * q4 + i][16 * c + r16] = rows.acc[n][c][i];
            }
        }
    }
    __syncthreads();
    const int c4 = threadIdx.x & 31;   // 32 lanes store a row
#pragma unroll
    for (int k = 0; k < (ROWS + 2 * kWaves - 1) / (2 * kWaves); ++k) {
        const int r = 2 * kWaves * k + (threadIdx.x >> 5);
        const int64_t at = lds.dest[r];
        if (at < 0) continue;
        float top = lds.out.m[0][r];
#pragma unroll
        for (int i = 1; i < SETS; ++i) top = fmaxf(top, lds.out.m[i][r]);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < SETS; ++i) {
            const float m = lds.out.m[i][r], w = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - top);
            const float4 t = *reinterpret_cast<const float4 *>(&lds.out.acc[i][r][4 * c4]);
            v.x = fmaf(w, t.x, v.x);
            v.y = fmaf(w, t.y, v.y);
            v.z = fmaf(w, t.z, v.z);
            v.w = fmaf(w, t.w, v.w);
            sum = fmaf(w, lds.out.sum[i][r], sum);
        }
        store_row<MODE != 0>(a.acc_ws[1] + at * kHeadDim, c4, v);
        if (c4 == 0) reinterpret_cast<float2 *>(a.ml_ws[1])[at] = make_float2(top, sum);
    }
}
template <int MODE, bool KC>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 2))) void tkv_shared_kernel(SharedArgs a)
{
    __shared__ Shared<MODE> lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t block = blockIdx.x + blockIdx.y * gridDim.x;
    if (block >= (uint32_t)a.blocks) return;
    if ((int)block < a.own_blocks) own_item<KC, MODE != 0>(a, lds, (int)block, wave, lane);
    else prefix_item<MODE, KC>(a, lds, (int)block - a.own_blocks, wave, lane);
}

// out = sum_i 2^(m_i - M) acc_i / sum_i 2^(m_i - M) l_i over a sequence's own items and its prefixes'.  One workgroup per (sequence,
// query head); 32 lanes take every eighth partial, four channels a lane, and ask for eight of them at a time with their m and l: nothing
// waits for anything but the workspace, and that once for up to 64 partials.
constexpr int kMergeWaves = 4, kMergeSets = 2 * kMergeWaves, kMergeBatch = 8;
struct MergeArgs {
    const float *acc[2], *ml[2];     // partials of the own items, of the prefixes
    int n[2];                        // slots of either
    const int32_t *indptr;           // [2][batch + 1] slots of the sequences
    int batch;
    int n_q_heads;
    uint16_t *out;
};
__device__ __forceinline__ float merge_weight(float m, float M) { return m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - M); }
__global__ __launch_bounds__(64 * kMergeWaves) void tkv_merge_shared_kernel(MergeArgs a)
{
    __shared__ float4 num_s[kMergeSets][kHeadDim / 4];
    __shared__ float2 ml_s[kMergeSets];
    const int c4 = threadIdx.x & 31, set = threadIdx.x >> 5;
    const int h = blockIdx.x, b = blockIdx.y + blockIdx.z * gridDim.y;
    if (b >= a.batch) return;
    int i0[2], n[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int first = k ? a.n[0] : 0;   // the prefixes' slots follow the own ones
        const int x = ((ConstWords)a.indptr)[k * (a.batch + 1) + b] - first, y = ((ConstWords)a.indptr)[k * (a.batch + 1) + b + 1] - first;
        i0[k] = x > 0 ? x : 0;
        n[k] = (y < a.n[k] ? y : a.n[k]) - i0[k];
        n[k] = n[k] > 0 ? n[k] : 0;
    }
    const int all = n[0] + n[1];
    float M = -INFINITY, den = 0.0f;
    float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int base = set; base < all; base += kMergeSets * kMergeBatch) {
        float4 v[kMergeBatch];
        float2 ml[kMergeBatch];
#pragma unroll
        for (int j = 0; j < kMergeBatch; ++j) {
            const int i = base + kMergeSets * j, k = i < n[0] ? 0 : 1;
            v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
            ml[j] = make_float2(-INFINITY, 0.0f);
            if (i < all) {
                const size_t at = (size_t)(k ? i0[1] + i - n[0] : i0[0] + i) * a.n_q_heads + h;
                v[j] = reinterpret_cast<const float4 *>((k ? a.acc[1] : a.acc[0]) + at * kHeadDim)[c4];
                ml[j] = reinterpret_cast<const float2 *>(k ? a.ml[1] : a.ml[0])[at];
            }
        }
        float Mn = M;
#pragma unroll
        for (int j = 0; j < kMergeBatch; ++j) Mn = fmaxf(Mn, ml[j].x);
        const float so = merge_weight(M, Mn);
        den *= so;
        num = make_float4(num.x * so, num.y * so, num.z * so, num.w * so);
#pragma unroll
        for (int j = 0; j < kMergeBatch; ++j) {
            float w = merge_weight(ml[j].x, Mn);
            if (ml[j].y != ml[j].y) w = ml[j].y;   // NaN stays
            den = fmaf(w, ml[j].y, den);
            num.x = fmaf(w, v[j].x, num.x);
            num.y = fmaf(w, v[j].y, num.y);
            num.z = fmaf(w, v[j].z, num.z);
            num.w = fmaf(w, v[j].w, num.w);
        }
        M = Mn;
    }
    num_s[set][c4] = num;
    if (c4 == 0) ml_s[set] = make_float2(M, den);
    __syncthreads();
    const int lane = threadIdx.x;
    if (lane >= kHeadDim / 2) return;   // two channels a lane
    float Mg = ml_s[0].x;
#pragma unroll
    for (int k = 1; k < kMergeSets; ++k) Mg = fmaxf(Mg, ml_s[k].x);
    float d = 0.0f;
    float2 o = make_float2(0.f, 0.f);
#pragma unroll
    for (int k = 0; k < kMergeSets; ++k) {
        const float wk = merge_weight(ml_s[k].x, Mg);
        const float2 x = reinterpret_cast<const float2 *>(num_s[k])[lane];
        d = fmaf(wk, ml_s[k].y, d);
        o.x = fmaf(wk, x.x, o.x);
        o.y = fmaf(wk, x.y, o.y);
    }
    const float r = d == 0.0f ? 0.0f : 1.0f / d;   // no tokens: zeros; NaN stays
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v = {(__bf16)(o.x * r), (__bf16)(o.y * r)};
    reinterpret_cast<uint32_t *>(a.out + ((size_t)b * a.n_q_heads + h) * kHeadDim)[lane] = __builtin_bit_cast(uint32_t, v);
}

template <int MODE> void launch_shared(bool kc, hipStream_t s, const SharedArgs &a)
{
    constexpr unsigned kMaxX = 1 << 22;   // a grid has less than 2^32 threads in a dimension
    const unsigned blocks = (unsigned)a.blocks;
    hipLaunchKernelGGL((kc ? tkv_shared_kernel<MODE, true> : tkv_shared_kernel<MODE, false>), dim3(blocks < kMaxX ? blocks : kMaxX, (blocks + kMaxX - 1) / kMaxX),
                       dim3(64 * kWaves), 0, s, a);
}

} // namespace

int tkv_launch_shared(const tkv_desc *desc, const void *pool, const uint8_t *bit_map, const void *q, const int32_t *page_indptr,
                      const int32_t *page_ids, const int32_t *n_tok_int2, const int32_t *n_tok_int4, const int32_t *items, int32_t n_items,
                      const tkv_prefix *prefix, const int32_t *slot_indptr, int32_t n_slots, int32_t batch, int32_t n_q_heads, float sm_scale,
                      void *out, void *workspace, int32_t *status, void *stream)
{
    int log2_r = 0;
    while ((desc->n_kv_heads << log2_r) < n_q_heads) ++log2_r;
    // the rows of all slots, then their (m, l): every row begins a 128-byte line of its own, as far as the workspace does
    const size_t own_rows = (size_t)n_items * n_q_heads, rows = (size_t)n_slots * n_q_heads;
    float *const acc = (float *)workspace, *const ml = acc + rows * kHeadDim;
    SharedArgs a = {};
    a.pool = (const uint8_t *)pool;
    a.bit_map = bit_map;
    a.q = (const uint16_t *)q;
    a.page_indptr = page_indptr;
    a.page_ids = page_ids;
    a.n_tok_int2 = n_tok_int2;
    a.n_tok_int4 = n_tok_int4;
    a.items = items;
    a.n_items = n_items;
    a.p = *prefix;
    a.n_kv_heads = desc->n_kv_heads;
    a.log2_r = log2_r;
    a.n_pages_int2 = desc->n_pages_int2;
    a.n_pages_int4 = desc->n_pages_int4;
    a.batch = batch;
    a.n_slots = n_slots;
    a.kappa = sm_scale * 1.44269504088896340736f;
    a.acc_ws[0] = acc;
    a.acc_ws[1] = acc + own_rows * kHeadDim;
    a.ml_ws[0] = ml;
    a.ml_ws[1] = ml + 2 * own_rows;
    a.status = status;
    const int64_t own_blocks = ((int64_t)n_items * desc->n_kv_heads + kWaves - 1) / kWaves;
    a.own_blocks = (int)own_blocks;
    const int per = prefix->n_items > 0 ? prefix->tile_rows : 16;
    const int64_t blocks = own_blocks + (int64_t)prefix->n_items * desc->n_kv_heads;
    if (blocks > INT32_MAX) return TKV_ERR_INVALID_ARG;
    if (blocks > 0) {
        const bool kc = desc->int2_key_axis == TKV_KEYS_PER_CHANNEL;
        a.blocks = (int)blocks;
        if (per == 16) launch_shared<0>(kc, (hipStream_t)stream, a);
        else if (per == 64) launch_shared<1>(kc, (hipStream_t)stream, a);
        else launch_shared<2>(kc, (hipStream_t)stream, a);
        if (hipGetLastError() != hipSuccess) return TKV_ERR_HIP;
    }
    MergeArgs m = {};
    for (int k = 0; k < 2; ++k) {
        m.acc[k] = a.acc_ws[k];
        m.ml[k] = a.ml_ws[k];
    }
    m.n[0] = n_items;
    m.n[1] = n_slots - n_items;
    m.indptr = slot_indptr;
    m.batch = batch;
    m.n_q_heads = n_q_heads;
    m.out = (uint16_t *)out;
    constexpr int kMaxY = 65535;
    const dim3 grid((unsigned)n_q_heads, (unsigned)(batch < kMaxY ? batch : kMaxY), (unsigned)((batch + kMaxY - 1) / kMaxY));
    hipLaunchKernelGGL(tkv_merge_shared_kernel, grid, dim3(64 * kMergeWaves), 0, (hipStream_t)stream, m);
    return hipGetLastError() == hipSuccess ? TKV_OK : TKV_ERR_HIP;
}
