// tkv_decode_attention_shared: decode attention for sequences that share a long prefix (a system prompt, tool definitions, a
// document).  The prefix's pages are attended to once for all of its sequences (tkv_prefix_kernel), each sequence's own pages
// by the split kernel of tkv_decode.hip, and the partials of both are merged by log-sum-exp (tkv_merge_shared_kernel).
//
// With one sequence, a page is read for the eight query rows at most that share its kv head, and memory bounds the kernel.
// With S sequences there are S times as many rows for the same page: arithmetic bounds it, and the page's codes are
// worth expanding.  A workgroup of four wavefronts owns (work item, kv head, up to 64 query rows); the wavefronts take the
// item's pages in turn, all rows each, and their results are added in LDS at the end.
//
//   K, V  code * scale + zero in fp16, one rounding: the values that tkv_gather_dequant gives a prefill kernel.  The page layout
//         is that of the matrix operands, so a lane expands exactly what it feeds to the MFMAs, and nothing but the scales and
//         zero-points goes through LDS.
//   QK^T  D[token, row] = sum_c K[token, c] q[row, c] (v_mfma_f32_16x16x32_f16), q in fp16, each row scaled by a power of two
//         of its own that its softmax factor takes back: bf16 has 8 bits, so q is exact down to 2^-31 of the row's largest.
//   PV    D[row, channel] = sum_token W[row, token] V[token, channel]: the results of QK^T lie where PV wants its operand.
//         W = 2^(logit - m + 8) in fp16, m a reference that follows the row's maximum lazily (within 2^4), so that W stays
//         below 2^12 and weights down to 2^-22 of the largest are exact to half a step.  The denominators are one more MFMA
//         against ones: of the rounded weights, as the numerators.
// All sums are 32 bits.  K, V and W carry 11 bits where the split kernel carries what its fp32 results need; the output is
// bf16, which has 8.
#include <hip/hip_runtime.h>

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
constexpr int kWaves = 4;

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
// Two codes in bits 0.. and 16.. of x as fp16 numbers, times s plus z with one rounding per value.  (A code under the bit pattern
// 0x6400 is 1024 + code, and subtracting 1024 is exact.)
template <int BITS> __device__ __forceinline__ uint32_t dequant2(uint32_t x, uint32_t s, uint32_t z)
{
    constexpr uint32_t m = ((1u << BITS) - 1u) * 0x00010001u;
    const half2_t k = {(_Float16)1024.0f, (_Float16)1024.0f};
    const half2_t c = __builtin_bit_cast(half2_t, (x & m) | 0x64006400u) - k;
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(c, __builtin_bit_cast(half2_t, s), __builtin_bit_cast(half2_t, z)));
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

struct PrefixArgs {
    const uint8_t *pool;
    const uint8_t *bit_map;
    const uint16_t *q;
    tkv_prefix p;
    int n_kv_heads;
    int log2_r;
    int n_pages_int2;
    int n_pages_int4;
    int batch;
    int first_slot;   // slots [first_slot, n_slots) hold the prefixes' partials
    int n_slots;
    float kappa;      // sm_scale * log2(e)
    float *acc_ws;    // of slot first_slot
    float *ml_ws;
    int32_t *status;
};

// What a lane loads of one (page, kv head) record.
template <int BITS> struct PageRegs {
    uint4 kw[4];      // K codes: four group words of this lane's token of each 16-token tile
    uint4 vw[BITS];   // V codes: chunk 64 i + lane of the plane
    uint4 km, vm;     // 16 bytes of the K scale | K zero planes, of the V scale | V zero planes
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

template <int NT> struct Rows {   // NT tiles of 16 query rows
    half8 q[NT][4];        // operand of QK^T for a group of channels: row lane % 16, eight channels
    floatx4 acc[NT][8];    // row 4 * (lane / 16) + i, channel 16 * tile + lane % 16
    floatx4 sum[NT];       // denominators, rows as in acc
    float m[NT];           // reference of row lane % 16, log2 units, -inf at first
    float kappa[NT];       // of row lane % 16
    int at[NT];            // its row of q
    bool huge;             // whether some row's reference is so large that rounding it moves a weight by more than 2^-4
};
struct alignas(16) Meta {   // of one wavefront's page
    uint4 k[64], v[64];
};

// q of the lane's rows in the channel order of the codes: register k of a lane holds channels (k, k + 4) of octet lane / 16 of
// the group; SPREAD (per-channel INT2 keys): channels (k, k + 8) from 16 * (lane / 32) + 4 * (lane / 16 % 2) on.
template <int NT, bool SPREAD> __device__ __forceinline__ void load_q(Rows<NT> &rows, const uint16_t *__restrict__ q, float kappa, int lane)
{
    const int q4 = lane >> 4;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const uint16_t *row = q + (size_t)rows.at[n] * kHeadDim;
        uint2 x[4], y[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int c = 32 * g + (SPREAD ? 16 * (q4 >> 1) + 4 * (q4 & 1) : 8 * q4);
            x[g] = *reinterpret_cast<const uint2 *>(row + c);
            y[g] = *reinterpret_cast<const uint2 *>(row + c + (SPREAD ? 8 : 4));
        }
        // the largest exponent of the row; NaN and infinities do not count
        uint32_t top = 0;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const uint32_t d[4] = {x[g].x, x[g].y, y[g].x, y[g].y};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t a = d[k] & 0x7f80u, b = (d[k] >> 16) & 0x7f80u;
                top = max(top, a == 0x7f80u ? 0 : a);
                top = max(top, b == 0x7f80u ? 0 : b);
            }
        }
        top = max(top, (uint32_t)__shfl_xor((int)top, 16));
        top = max(top, (uint32_t)__shfl_xor((int)top, 32));
        int E = top == 0 ? 0 : 14 - ((int)(top >> 7) - 127);   // the largest lies in [2^14, 2^15)
        E = E > 100 ? 100 : (E < -100 ? -100 : E);
        const float f = ldexpf(1.0f, E);
        rows.kappa[n] = kappa * ldexpf(1.0f, -E);
#pragma unroll
        for (int g = 0; g < 4; ++g)
            rows.q[n][g] = as_half8(pack_h2(bf16_lo(x[g].x) * f, bf16_lo(y[g].x) * f), pack_h2(bf16_hi(x[g].x) * f, bf16_hi(y[g].x) * f),
                                    pack_h2(bf16_lo(x[g].y) * f, bf16_lo(y[g].y) * f), pack_h2(bf16_hi(x[g].y) * f, bf16_hi(y[g].y) * f));
    }
}

// One page.  The K registers are free behind after_qk, the V registers behind the function.
template <int NT, int BITS, bool KC, class AfterQK>
__device__ __forceinline__ void attend_page(const PageRegs<BITS> &r, int n_valid, int lane, Rows<NT> &rows, Meta &meta, AfterQK after_qk)
{
    constexpr bool kPerChannel = KC && BITS == 2;
    const int r16 = lane & 15, q4 = lane >> 4;
    const bool partial = n_valid < kPageTokens;
    meta.k[lane] = r.km;
    {
        uint4 vm = r.vm;
        if (partial) {
            // what was never written counts nothing, whatever stands there: chunk lane % 32 = (block, quad, group) of eight tokens
            const int t0 = 32 * ((lane >> 4) & 1) + 4 * ((lane >> 2) & 3);
            auto mask = [&](int t) { return (t < n_valid ? 0xffffu : 0u) | (t + 1 < n_valid ? 0xffff0000u : 0u); };
            vm.x &= mask(t0);
            vm.y &= mask(t0 + 2);
            vm.z &= mask(t0 + 16);
            vm.w &= mask(t0 + 18);
        }
        meta.v[lane] = vm;
    }
    lds_order();

    floatx4 S[NT][4];   // token 16 e + 4 q4 + i, row r16
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) S[n][e] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        uint2 sc, zc;
        if constexpr (!kPerChannel) {
            sc = reinterpret_cast<const uint2 *>(meta.k)[16 * e + r16];
            zc = reinterpret_cast<const uint2 *>(meta.k + 32)[16 * e + r16];
        }
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const uint32_t w = g == 0 ? r.kw[e].x : g == 1 ? r.kw[e].y : g == 2 ? r.kw[e].z : r.kw[e].w;
            uint32_t a[4];
            if constexpr (kPerChannel) {
                const uint4 s = meta.k[((e >> 1) * 4 + g) * 4 + q4], z = meta.k[32 + ((e >> 1) * 4 + g) * 4 + q4];
                const uint32_t x = w >> (8 * (q4 & 1));
                a[0] = dequant2<2>(x, s.x, z.x);
                a[1] = dequant2<2>(x >> 2, s.y, z.y);
                a[2] = dequant2<2>(x >> 4, s.z, z.z);
                a[3] = dequant2<2>(x >> 6, s.w, z.w);
            } else {
                const uint32_t s = twice(g < 2 ? sc.x : sc.y, g), z = twice(g < 2 ? zc.x : zc.y, g);
                // INT4: codes k and k + 4 lie in the halves of the word; INT2: the bytes of this lane's octet move there
                const uint32_t x = BITS == 4 ? w : __builtin_amdgcn_perm(w, w, (q4 & 1) ? 0x0c070c06u : 0x0c050c04u);
#pragma unroll
                for (int k = 0; k < 4; ++k) a[k] = dequant2<BITS>(x >> (BITS * k), s, z);
            }
            const half8 A = as_half8(a[0], a[1], a[2], a[3]);
#pragma unroll
            for (int n = 0; n < NT; ++n) S[n][e] = mfma(A, rows.q[n][g], S[n][e]);
        }
    }
    after_qk();

    // softmax weights, operands of PV: tokens 32 b + 16 (j >> 2) + 4 q4 + (j & 3), j = 0..7, of row r16
    half8 P[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        if (partial) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < 4; ++i) S[n][e][i] = 16 * e + 4 * q4 + i < n_valid ? S[n][e][i] : -INFINITY;
        }
        float mx = S[n][0][0];
#pragma unroll
        for (int k = 1; k < 16; ++k) mx = fmaxf(mx, S[n][k >> 2][k & 3]);
        if (__any(mx * rows.kappa[n] > rows.m[n] + kTau)) {
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float m_new = fmaxf(rows.m[n], mx * rows.kappa[n]);
            const float alpha = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(rows.m[n] - m_new);
            rows.m[n] = m_new;
            rows.huge = rows.huge || __any(fabsf(m_new) > 0x1p20f && m_new != -INFINITY);
            floatx4 av;
#pragma unroll
            for (int i = 0; i < 4; ++i) av[i] = __shfl(alpha, 4 * q4 + i);
#pragma unroll
            for (int c = 0; c < 8; ++c) rows.acc[n][c] *= av;
            rows.sum[n] *= av;
        }
        float factor = rows.kappa[n], shift = (float)kPExp - (rows.m[n] == -INFINITY ? 0.0f : rows.m[n]);
        if (__builtin_expect(rows.huge, 0)) {
            // factor * logit with one rounding, as the reference has it, then the difference: the largest weight is 2^8
#pragma unroll
            for (int e = 0; e < 4; ++e) S[n][e] = S[n][e] * factor - (rows.m[n] == -INFINITY ? 0.0f : rows.m[n]);
            factor = 1.0f;
            shift = (float)kPExp;
        }
        uint32_t w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float a = __builtin_amdgcn_exp2f(fmaf(S[n][k >> 1][2 * (k & 1)], factor, shift));
            const float b = __builtin_amdgcn_exp2f(fmaf(S[n][k >> 1][2 * (k & 1) + 1], factor, shift));
            w[k] = pack_h2(a, b);
        }
        P[n][0] = as_half8(w[0], w[1], w[2], w[3]);
        P[n][1] = as_half8(w[4], w[5], w[6], w[7]);
    }

    const half8 ones = as_half8(0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int n = 0; n < NT; ++n) rows.sum[n] = mfma(P[n][b], ones, rows.sum[n]);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const uint4 s = meta.v[(b * 4 + q4) * 4 + g], z = meta.v[32 + (b * 4 + q4) * 4 + g];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int tile = 2 * g + c, half = tile >> 2, comp = tile & 3;
                const uint4 v4 = r.vw[BITS == 4 ? b * 2 + half : half];
                const uint32_t w = comp == 0 ? v4.x : comp == 1 ? v4.y : comp == 2 ? v4.z : v4.w;
                const uint32_t x = BITS == 4 ? w : w >> (8 * b);
                const half8 B = as_half8(dequant2<BITS>(x, s.x, z.x), dequant2<BITS>(x >> BITS, s.y, z.y), dequant2<BITS>(x >> (2 * BITS), s.z, z.z),
                                         dequant2<BITS>(x >> (3 * BITS), s.w, z.w));
#pragma unroll
                for (int n = 0; n < NT; ++n) rows.acc[n][tile] = mfma(P[n][b], B, rows.acc[n][tile]);
            }
        }
    }
}

// The pages of a wavefront, 64 at a time in registers: lane l holds the wavefront's page number base + l.
struct PageList {
    int base;
    uint32_t at;   // where the record starts in the pool, in units of kUnit
    int valid;     // tokens of the page that count
};
constexpr int kUnitLog2 = 11;   // record and arena sizes are multiples of it
static_assert(Rec<2>::kBytes % (1 << kUnitLog2) == 0 && Rec<4>::kBytes % (1 << kUnitLog2) == 0, "record unit");
struct ItemCtx {
    const uint8_t *pool;
    const uint8_t *bit_map;
    const int32_t *pages;
    int first, n;                        // list position of the wavefront's first page; how many it has, every kWaves-th
    int np2, np4, last2, last4;          // pages of either width of the list, tokens of the last ones
    int kvh, n_kv_heads, n_pages_int2, n_pages_total, lane;
    int32_t *status;
};
__device__ __forceinline__ void fetch_list(const ItemCtx &cx, PageList &l, int base)
{
    l.base = base;
    const int i = base + cx.lane < cx.n ? base + cx.lane : cx.n - 1;
    const int pos = cx.first + kWaves * i;
    const int page = cx.pages[pos];
    const bool is2 = pos < cx.np2;
    const int lo = is2 ? 0 : cx.n_pages_int2, hi = is2 ? cx.n_pages_int2 : cx.n_pages_total;
    const bool ok = page >= lo && page < hi;
    if (!ok && cx.status) atomicOr(cx.status, page < 0 || page >= cx.n_pages_total ? TKV_STATUS_PAGE_RANGE : TKV_STATUS_BITMAP_MISMATCH);
    // a page that cannot be read counts no tokens; nothing is read in its place (the record's size is 0, see record_of)
    const uint32_t rec = (uint32_t)(is2 ? page : page - cx.n_pages_int2) * (uint32_t)cx.n_kv_heads + (uint32_t)cx.kvh;
    constexpr uint32_t kUnits2 = Rec<2>::kBytes >> kUnitLog2, kUnits4 = Rec<4>::kBytes >> kUnitLog2;
    l.at = !ok ? 0 : (is2 ? rec * kUnits2 : (uint32_t)cx.n_pages_int2 * (uint32_t)cx.n_kv_heads * kUnits2 + rec * kUnits4);   // (pools below 8 TB: 32 bits)
    const bool written = ok && cx.bit_map[ok ? page : 0] == (is2 ? 2 : 4);
    if (ok && !written && cx.status) atomicOr(cx.status, TKV_STATUS_BITMAP_MISMATCH);
    l.valid = !written ? 0 : (pos == cx.np2 - 1 ? cx.last2 : pos == cx.np2 + cx.np4 - 1 ? cx.last4 : kPageTokens);
}
template <int BITS> __device__ __forceinline__ Record record_of(const ItemCtx &cx, const PageList &l, int i, bool wanted)
{
    const uint64_t at = (uint32_t)__builtin_amdgcn_readlane((int)l.at, i - l.base);
    const int valid = __builtin_amdgcn_readlane(l.valid, i - l.base);
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(cx.pool) + (at << kUnitLog2), 0, wanted && valid > 0 ? Rec<BITS>::kBytes : 0, 0x00027000);
}

// Pages [i, end) of the wavefront, all of one width.
template <int NT, int BITS, bool KC>
__device__ __forceinline__ void run_pages(const ItemCtx &cx, PageList &list, int i, int end, Rows<NT> &rows, Meta &meta)
{
    PageRegs<BITS> r;
    Record rec = record_of<BITS>(cx, list, i, true);
    load_k(r, rec, cx.lane);
    load_v(r, rec, cx.lane);
    for (; i < end; ++i) {
        const int valid = __builtin_amdgcn_readlane(list.valid, i - list.base);
        const bool more = i + 1 < end;
        if (more && i + 1 - list.base >= 64) fetch_list(cx, list, i + 1);
        rec = record_of<BITS>(cx, list, more ? i + 1 : i, more);
        attend_page<NT, BITS, KC>(r, valid, cx.lane, rows, meta, [&]() {
            __builtin_amdgcn_sched_barrier(0);
            load_k(r, rec, cx.lane);
        });
        __builtin_amdgcn_sched_barrier(0);
        load_v(r, rec, cx.lane);
    }
}

constexpr int kOutRow = kHeadDim + 4;   // floats: rows 4 q4 + i of a store fall on different banks
template <int NT> struct Shared {
    union {
        Meta meta[kWaves];
        float acc[kWaves][16 * NT][kOutRow];
    };
    float m[kWaves][16 * NT], sum[kWaves][16 * NT];
};

template <int NT, bool KC> __device__ __forceinline__ void prefix_item(const PrefixArgs &a)
{
    __shared__ Shared<NT> lds;
    const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, q4 = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kvh = blockIdx.x, item = blockIdx.y, R = 1 << a.log2_r, n_q_heads = a.n_kv_heads << a.log2_r;
    const ConstWords words = (ConstWords)(a.p.items + 4 * (size_t)item);
    const int group = words[0], item_pb = words[1], item_pe = words[2], part = words[3];
    if (group < 0 || group >= a.p.n_groups || part < 0) {
        if (a.status && tid == 0) atomicOr(a.status, TKV_STATUS_BAD_ITEM);
        return;
    }
    int m0 = ((ConstWords)a.p.member_indptr)[group], m1 = ((ConstWords)a.p.member_indptr)[group + 1];
    const int n2 = ((ConstWords)a.p.n_tok_int2)[group], n4 = ((ConstWords)a.p.n_tok_int4)[group];
    const int list0 = ((ConstWords)a.p.page_indptr)[group], list1 = ((ConstWords)a.p.page_indptr)[group + 1];
    m0 = m0 > 0 ? m0 : 0;
    m1 = m1 < a.p.n_members ? m1 : a.p.n_members;
    const int n_rows = (m1 - m0) << a.log2_r, row0 = blockIdx.z * 16 * NT;
    if (row0 >= n_rows) return;
    if (m1 - m0 > a.p.max_members && a.status && tid == 0) atomicOr(a.status, TKV_STATUS_BAD_ITEM);   // more rows than the launch has workgroups for
    const int np2 = (n2 + kPageTokens - 1) / kPageTokens, np4 = (n4 + kPageTokens - 1) / kPageTokens;
    const int np = np2 + np4 < list1 - list0 ? np2 + np4 : list1 - list0;
    const int pb = item_pb > 0 ? item_pb : 0, pe = item_pe < np ? item_pe : np;

    Rows<NT> rows;
    rows.huge = false;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int row = row0 + 16 * n + r16, member = m0 + (row >> a.log2_r);
        int seq = row < n_rows ? a.p.member_seqs[member] : 0;
        if (seq < 0 || seq >= a.batch) seq = 0;   // nothing of it is stored
        rows.at[n] = seq * n_q_heads + kvh * R + (row & (R - 1));
        rows.m[n] = -INFINITY;
        rows.sum[n] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < 8; ++c) rows.acc[n][c] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    const int first = pb + wave, n = first < pe ? (pe - first + kWaves - 1) / kWaves : 0;   // this wavefront's pages
    if (n > 0) {
        const ItemCtx cx = {a.pool, a.bit_map, a.p.page_ids + list0, first, n, np2, np4, n2 - (np2 - 1) * kPageTokens, n4 - (np4 - 1) * kPageTokens,
                            kvh, a.n_kv_heads, a.n_pages_int2, a.n_pages_int2 + a.n_pages_int4, lane, a.status};
        PageList list;
        fetch_list(cx, list, 0);
        const int n_2 = first < np2 ? ((np2 < pe ? np2 : pe) - first + kWaves - 1) / kWaves : 0;   // INT2 pages among them: they come first
        if (n_2 > 0) {
            load_q<NT, KC>(rows, a.q, a.kappa, lane);
            run_pages<NT, 2, KC>(cx, list, 0, n_2, rows, lds.meta[wave]);
        }
        if (n_2 < n) {
            if (n_2 == 0 || KC) load_q<NT, false>(rows, a.q, a.kappa, lane);
            if (n_2 - list.base >= 64) fetch_list(cx, list, n_2);
            run_pages<NT, 4, KC>(cx, list, n_2, n, rows, lds.meta[wave]);
        }
    }

    // ---- the four wavefronts' results are brought to a common reference, added and stored --------------------------------
    if (q4 == 0)
#pragma unroll
        for (int k = 0; k < NT; ++k) lds.m[wave][16 * k + r16] = rows.m[k];
    __syncthreads();   // the references are there, and no page is being worked on
#pragma unroll
    for (int k = 0; k < NT; ++k) {
        floatx4 f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 16 * k + 4 * q4 + i;
            const float own = lds.m[wave][row];
            const float top = fmaxf(fmaxf(lds.m[0][row], lds.m[1][row]), fmaxf(lds.m[2][row], lds.m[3][row]));
            f[i] = own == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(own - top);
        }
        rows.sum[k] *= f;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            rows.acc[k][c] *= f;
#pragma unroll
            for (int i = 0; i < 4; ++i) lds.acc[wave][16 * k + 4 * q4 + i][16 * c + r16] = rows.acc[k][c][i];
        }
        if (r16 == 0)
#pragma unroll
            for (int i = 0; i < 4; ++i) lds.sum[wave][16 * k + 4 * q4 + i] = rows.sum[k][i];
    }
    __syncthreads();
    const int c4 = tid & 31;   // 32 lanes store a row
#pragma unroll 4
    for (int r = tid >> 5; r < 16 * NT; r += 8) {
        const int row = row0 + r;
        if (row >= n_rows) break;
        const int member = m0 + (row >> a.log2_r), seq = a.p.member_seqs[member];
        const int64_t slot = (int64_t)a.p.member_slots[member] + part;
        if (seq < 0 || seq >= a.batch || slot < a.first_slot || slot >= a.n_slots) {
            if (a.status) atomicOr(a.status, TKV_STATUS_BAD_ITEM);
            continue;
        }
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float4 t = *reinterpret_cast<const float4 *>(&lds.acc[w][r][4 * c4]);
            v.x += t.x;
            v.y += t.y;
            v.z += t.z;
            v.w += t.w;
        }
        const size_t at = (size_t)(slot - a.first_slot) * n_q_heads + kvh * R + (row & (R - 1));
        reinterpret_cast<float4 *>(a.acc_ws + at * kHeadDim)[c4] = v;
        if (c4 == 0)
            reinterpret_cast<float2 *>(a.ml_ws)[at] = make_float2(fmaxf(fmaxf(lds.m[0][r], lds.m[1][r]), fmaxf(lds.m[2][r], lds.m[3][r])),
                                                                  (lds.sum[0][r] + lds.sum[1][r]) + (lds.sum[2][r] + lds.sum[3][r]));
    }
}
template <int NT, bool KC>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(NT == 4 ? 1 : NT == 2 ? 2 : 3, NT == 4 ? 1 : NT == 2 ? 2 : 3)))
void tkv_prefix_kernel(PrefixArgs a)
{
    prefix_item<NT, KC>(a);
}

// out = sum_i 2^(m_i - M) acc_i / sum_i 2^(m_i - M) l_i over a sequence's own items and its prefixes'.  One workgroup of four
// wavefronts per (sequence, query head); a wavefront takes every fourth partial, a lane two channels.
struct MergeArgs {
    const float *ws[2];              // partials of the own items, of the prefixes
    int n[2];                        // slots of either
    const int32_t *indptr;           // [2][batch + 1] slots of the sequences
    int batch;
    int n_q_heads;
    uint16_t *out;
};
__device__ __forceinline__ float merge_weight(float m, float M) { return m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - M); }
__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}
__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
    return v;
}
__global__ __launch_bounds__(64 * kWaves) void tkv_merge_shared_kernel(MergeArgs a)
{
    __shared__ float2 num_s[kWaves][64];
    __shared__ float2 ml_s[kWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
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
    float2 num = make_float2(0.f, 0.f);
    auto row_of = [&](int i, const float *&acc, const float *&ml) {   // partial i of the sequence
        const int k = i < n[0] ? 0 : 1;
        const size_t at = (size_t)(k ? i0[1] + i - n[0] : i0[0] + i) * a.n_q_heads + h;
        const float *ws = k ? a.ws[1] : a.ws[0];
        acc = ws + at * kHeadDim;
        ml = ws + (size_t)(k ? a.n[1] : a.n[0]) * a.n_q_heads * kHeadDim + 2 * at;
    };
    // 64 of the wavefront's partials at a time: lane l weighs the l-th
    for (int base = wave; base < all; base += kWaves * 64) {
        const int mine = base + kWaves * lane;
        const float *acc, *mlp;
        float2 ml = make_float2(-INFINITY, 0.0f);
        if (mine < all) {
            row_of(mine, acc, mlp);
            ml = *reinterpret_cast<const float2 *>(mlp);
        }
        const float Mn = fmaxf(M, wave_max(ml.x));
        const float so = merge_weight(M, Mn);
        float w = merge_weight(ml.x, Mn);
        if (ml.y != ml.y) w = ml.y;   // NaN stays
        den = den * so + wave_sum(mine < all ? w * ml.y : 0.0f);
        num.x *= so;
        num.y *= so;
        const int count = (all - base + kWaves - 1) / kWaves < 64 ? (all - base + kWaves - 1) / kWaves : 64;
#pragma unroll 8
        for (int k = 0; k < count; ++k) {
            row_of(base + kWaves * k, acc, mlp);
            const float2 v = reinterpret_cast<const float2 *>(acc)[lane];
            const float wk = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), k));
            num.x = fmaf(wk, v.x, num.x);
            num.y = fmaf(wk, v.y, num.y);
        }
        M = Mn;
    }
    num_s[wave][lane] = num;
    if (lane == 0) ml_s[wave] = make_float2(M, den);
    __syncthreads();
    if (wave > 0) return;
    float Mg = M;
#pragma unroll
    for (int k = 1; k < kWaves; ++k) Mg = fmaxf(Mg, ml_s[k].x);
    float d = 0.0f;
    float2 o = make_float2(0.f, 0.f);
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
        const float wk = merge_weight(ml_s[k].x, Mg);
        d += wk * ml_s[k].y;
        o.x = fmaf(wk, num_s[k][lane].x, o.x);
        o.y = fmaf(wk, num_s[k][lane].y, o.y);
    }
    const float r = d == 0.0f ? 0.0f : 1.0f / d;   // no tokens: zeros; NaN stays
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v = {(__bf16)(o.x * r), (__bf16)(o.y * r)};
    reinterpret_cast<uint32_t *>(a.out + ((size_t)b * a.n_q_heads + h) * kHeadDim)[lane] = __builtin_bit_cast(uint32_t, v);
}

template <int NT> void launch_prefix(bool kc, dim3 grid, hipStream_t s, const PrefixArgs &a)
{
    hipLaunchKernelGGL((kc ? tkv_prefix_kernel<NT, true> : tkv_prefix_kernel<NT, false>), grid, dim3(64 * kWaves), 0, s, a);
}

} // namespace

int tkv_prefix_rows(int32_t rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : 64; }

int tkv_launch_prefix(const tkv_desc *desc, const void *pool, const uint8_t *bit_map, const void *q, const tkv_prefix *prefix, int32_t first_slot,
                      int32_t n_slots, int32_t batch, int32_t n_q_heads, float sm_scale, void *workspace, int32_t *status, void *stream)
{
    int log2_r = 0;
    while ((desc->n_kv_heads << log2_r) < n_q_heads) ++log2_r;
    PrefixArgs a = {};
    a.pool = (const uint8_t *)pool;
    a.bit_map = bit_map;
    a.q = (const uint16_t *)q;
    a.p = *prefix;
    a.n_kv_heads = desc->n_kv_heads;
    a.log2_r = log2_r;
    a.n_pages_int2 = desc->n_pages_int2;
    a.n_pages_int4 = desc->n_pages_int4;
    a.batch = batch;
    a.first_slot = first_slot;
    a.n_slots = n_slots;
    a.kappa = sm_scale * 1.44269504088896340736f;
    a.acc_ws = (float *)workspace;
    a.ml_ws = a.acc_ws + (size_t)(n_slots - first_slot) * n_q_heads * kHeadDim;
    a.status = status;
    const int rows = prefix->max_members << log2_r, per = tkv_prefix_rows(rows);
    const dim3 grid((unsigned)desc->n_kv_heads, (unsigned)prefix->n_items, (unsigned)((rows + per - 1) / per));
    const bool kc = desc->int2_key_axis == TKV_KEYS_PER_CHANNEL;
    if (per == 16) launch_prefix<1>(kc, grid, (hipStream_t)stream, a);
    else if (per == 32) launch_prefix<2>(kc, grid, (hipStream_t)stream, a);
    else launch_prefix<4>(kc, grid, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? TKV_OK : TKV_ERR_HIP;
}

int tkv_launch_merge_shared(const int32_t *indptr, int32_t n_own, int32_t n_prefix, int32_t batch, int32_t n_q_heads, void *out, const void *own_ws,
                            const void *prefix_ws, void *stream)
{
    MergeArgs a = {};
    a.ws[0] = (const float *)own_ws;
    a.ws[1] = (const float *)prefix_ws;
    a.n[0] = n_own;
    a.n[1] = n_prefix;
    a.indptr = indptr;
    a.batch = batch;
    a.n_q_heads = n_q_heads;
    a.out = (uint16_t *)out;
    constexpr int kMaxY = 65535;
    const dim3 grid((unsigned)n_q_heads, (unsigned)(batch < kMaxY ? batch : kMaxY), (unsigned)((batch + kMaxY - 1) / kMaxY));
    hipLaunchKernelGGL(tkv_merge_shared_kernel, grid, dim3(64 * kWaves), 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? TKV_OK : TKV_ERR_HIP;
}
