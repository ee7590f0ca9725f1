// tkv_prefill_attention: causal attention of packed sequences' new tokens over the rows of a cached prefix (fp16, as
// tkv_gather_dequant writes them) and over the new tokens themselves (Sec. 3.2.3, "Prefill").
//
//   out[i, h] = sum_j p_j v_j / sum_j p_j,   p_j = 2^(c q[i, h] . k_j - m),   c = sm_scale log2 e
//
// over the sequence's prefix rows and its new rows 0 .. i.  A workgroup takes a tile of query rows of one kv head -- row r is
// query head r mod R of token r / R, so that all heads that share a key fill one tile -- and walks over tiles of 32 or 64 keys:
// S^T = K Q^T and O^T += V^T P^T on v_mfma_f32_32x32x16, a wavefront 32 rows.  Transposed, a lane holds one query row: the running
// maximum, the sum and the mask's limit are one register each, and the weights leave the first product's accumulators in the
// order in which the second one takes its operand, if V's rows are read in that order too (ds_read_b64_tr_b16).
//
// Workgroups of 32 rows (one wavefront, four of them on a compute unit: loads of many workgroups on the way), 128 (four wavefronts, two
// workgroups: one takes the matrix cores while the other takes exponentials) and 256 (eight, one workgroup: keys and values are
// read half as often).  One MI355X, us: 2048 tokens of 64 heads behind 30 000 with 128 rows 1954, with 256 1888, now 1820 (1144 TFLOP/s, MFMAs busy 62 % of the
// cycles at the 1.4 to 1.7 GHz that power leaves; the library's bf16 product of 8192^3 runs at 1414); 8192 tokens 950 to 980 (1122 to 1157 TFLOP/s); 16
// single tokens of 64 heads behind 1500 to 5000 with 128 rows 63, with 32 41, now 37 (171 MB; 5.3 TB/s within the kernel).  In between, where there are
// few workgroups, the chain of a wavefront's steps bounds the call, each logits, weights and values of a tile: for a workgroup that has a compute unit to itself
// 0.90 us (128 rows), 1.32 (256) or 0.79 (32).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "tkv_internal.h"
#include "tkv_layout.h"

namespace {

using namespace tkv;

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kRow = kHeadDim * 2;        // bytes
constexpr int kItem = kPrefillItemWords;
constexpr float kNone = -3.4028235e38f;   // reference of a row that has seen no key
// A row's reference is set kLift below its largest logit and follows when the largest has grown by kSlack: weights reach 2^(kLift + kSlack) at most, and
// the row's largest is 2^kLift at least.  bf16 weights: 0 and 8 (8192 tokens of 64 heads 954 us, by every new maximum 1016; six ragged prompts 65.9, 68.8).  fp16
// weights end at 2^16, are whole down to 2^-14 and nothing below 2^-25: 9 and 6 keep weights down to 2^-23 of the row's largest whole and drop those below 2^-34.
// (0 and 8 dropped those below 2^-25: 60 000 keys, each e^-18 of a sink with a small value, made an output 6 % off.)  us, 0 and 8 / 7 and 8 / 9 and 6 / 11 and 4:
// four prompts of 2000 fp16 tokens 291 / 291 / 292 / 295, 8192 1004 / 1014 / 1014 / 1026, 2048 behind 30 000 1799 / 1832 / 1824 / 1831 (these two
// bound by power); other calls the same to 0.5 %, with 11 and 4 to 2 %.
template <bool BF16> constexpr float kLift = BF16 ? 0.0f : 9.0f;
template <bool BF16> constexpr float kSlack = BF16 ? 8.0f : 6.0f;

struct PrefillArgs {
    const uint16_t *q, *k[2], *v[2];      // keys and values: prefix, new tokens
    int64_t q_stride, k_stride[2], v_stride[2];
    const int32_t *items;
    uint16_t *out;
    float *partial;
    int32_t *status;
    int32_t n_items, n_slots, n_cut, n_tokens, n_prefix, group, n_kv_heads, q_bf16, out_bf16;
    float c;
};

__device__ __forceinline__ float lo_f32(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float hi_f32(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
template <bool BF16> __device__ __forceinline__ uint32_t pack(float a, float b)   // nearest even
{
    if constexpr (BF16) {
        const bf16x2 v = {(__bf16)a, (__bf16)b};
        return __builtin_bit_cast(uint32_t, v);
    } else {
        const f16x2 v = {(_Float16)a, (_Float16)b};
        return __builtin_bit_cast(uint32_t, v);
    }
}
template <bool BF16> __device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c)
{
    if constexpr (BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <bool BF16> __device__ __forceinline__ float add_pair(uint32_t p, float sum)
{
    if constexpr (BF16) {
        const bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f};
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, p), one, sum, false);
    } else {
        const f16x2 one = {(_Float16)1.0f, (_Float16)1.0f};
        return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, p), one, sum, false);
    }
}
// The other half's value of the same query row.
__device__ __forceinline__ float both_max(float x)
{
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float both_sum(float x)
{
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// LOADS times sixteen bytes a lane from global memory to LDS, zeros from beyond the buffer: load j takes offset[j % 4] (all the same, unless MIXED) + j
// `step` bytes to `lds` + j `stride` + 16 times the lane.  Written out, with the waits beside it: the compiler waits for every such load
// before any read of LDS.  In one block: scalars that a vector instruction wrote, as reloads of spilled ones do, need five wait states before the
// first load; M0 one.  M0 is named among the registers that change, so that the compiler keeps nothing in it across the block (its warning says that the register is
// its own).  (Put back by the block instead: six ragged prompts 61.7 -> 62.1 us, 2048 tokens behind 30 000 1802 -> 1845.)
//
// ONCE: non-temporal, where no other workgroup has a use for the lines.  16 single tokens behind 1500 to 5000 cached ones 41.6 -> 38.0 us, 64 of them
// 96.8 -> 86.2; but four prompts of 2000 tokens 290 -> 317 (2048 tokens behind 30000 1888 -> 1830), 1000 tokens by workgroups of 32 rows 36.8 -> 40.4.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
#define TKV_LOAD_FIRST(NT) "s_mov_b32 m0, %[lds]\n\ts_mov_b32 %[at], 0\n\ts_nop 2\n\tbuffer_load_dwordx4 %[v0], %[buffer], %[at] offen" NT " lds\n\t"
#define TKV_LOAD_NEXT(NT, V) "s_add_u32 m0, m0, %[stride]\n\ts_add_u32 %[at], %[at], %[step]\n\tbuffer_load_dwordx4 " V ", %[buffer], %[at] offen" NT " lds\n\t"
#define TKV_LOADS(TEXT) \
    asm volatile(TEXT : [at] "=&s"(at) \
                 : [lds] "s"(lds), [buffer] "s"(buffer), [step] "s"(step), [stride] "n"(STRIDE), [v0] "v"(offset[0]), [v1] "v"(offset[1]), [v2] "v"(offset[2]), [v3] "v"(offset[3]) \
                 : "memory", "scc", "m0")
template <int LOADS, int STRIDE, bool MIXED, bool ONCE> __device__ __forceinline__ void load_lds(uint32_t lds, u32x4 buffer, const uint32_t (&offset)[4], uint32_t step)
{
    static_assert(LOADS == 2 || LOADS == 4 || LOADS == 8);
    uint32_t at;
    if constexpr (LOADS == 2 && ONCE) TKV_LOADS(TKV_LOAD_FIRST(" nt") TKV_LOAD_NEXT(" nt", "%[v0]"));
    else if constexpr (LOADS == 2) TKV_LOADS(TKV_LOAD_FIRST("") TKV_LOAD_NEXT("", "%[v0]"));
    else if constexpr (LOADS == 4 && ONCE) TKV_LOADS(TKV_LOAD_FIRST(" nt") TKV_LOAD_NEXT(" nt", "%[v0]") TKV_LOAD_NEXT(" nt", "%[v0]") TKV_LOAD_NEXT(" nt", "%[v0]"));
    else if constexpr (LOADS == 4) TKV_LOADS(TKV_LOAD_FIRST("") TKV_LOAD_NEXT("", "%[v0]") TKV_LOAD_NEXT("", "%[v0]") TKV_LOAD_NEXT("", "%[v0]"));
    else if constexpr (MIXED && ONCE)
        TKV_LOADS(TKV_LOAD_FIRST(" nt") TKV_LOAD_NEXT(" nt", "%[v1]") TKV_LOAD_NEXT(" nt", "%[v2]") TKV_LOAD_NEXT(" nt", "%[v3]") TKV_LOAD_NEXT(" nt", "%[v0]") TKV_LOAD_NEXT(" nt", "%[v1]")
                      TKV_LOAD_NEXT(" nt", "%[v2]") TKV_LOAD_NEXT(" nt", "%[v3]"));
    else if constexpr (MIXED)
        TKV_LOADS(TKV_LOAD_FIRST("") TKV_LOAD_NEXT("", "%[v1]") TKV_LOAD_NEXT("", "%[v2]") TKV_LOAD_NEXT("", "%[v3]") TKV_LOAD_NEXT("", "%[v0]") TKV_LOAD_NEXT("", "%[v1]")
                      TKV_LOAD_NEXT("", "%[v2]") TKV_LOAD_NEXT("", "%[v3]"));
    else if constexpr (ONCE)
        TKV_LOADS(TKV_LOAD_FIRST(" nt") TKV_LOAD_NEXT(" nt", "%[v0]") TKV_LOAD_NEXT(" nt", "%[v0]") TKV_LOAD_NEXT(" nt", "%[v0]") TKV_LOAD_NEXT(" nt", "%[v0]") TKV_LOAD_NEXT(" nt", "%[v0]")
                      TKV_LOAD_NEXT(" nt", "%[v0]") TKV_LOAD_NEXT(" nt", "%[v0]"));
    else
        TKV_LOADS(TKV_LOAD_FIRST("") TKV_LOAD_NEXT("", "%[v0]") TKV_LOAD_NEXT("", "%[v0]") TKV_LOAD_NEXT("", "%[v0]") TKV_LOAD_NEXT("", "%[v0]") TKV_LOAD_NEXT("", "%[v0]")
                      TKV_LOAD_NEXT("", "%[v0]") TKV_LOAD_NEXT("", "%[v0]"));
}
#undef TKV_LOADS
#undef TKV_LOAD_NEXT
#undef TKV_LOAD_FIRST
#pragma clang diagnostic pop
__device__ __forceinline__ void wait_barrier() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

__device__ __forceinline__ u32x4 buffer_of(const void *p, uint32_t bytes)
{
    const uint64_t a = (uint64_t)(uintptr_t)p;
    u32x4 r;
    r.x = __builtin_amdgcn_readfirstlane((uint32_t)a);
    r.y = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32) & 0xffffu);
    r.z = __builtin_amdgcn_readfirstlane(bytes);
    r.w = 0x00020000u;
    return r;
}

struct Item {
    int32_t token0, n_new, prefix0, n_prefix, row0, begin, end, slot, part, n_parts;
};
__device__ __forceinline__ Item item_of(const int32_t *items, int k)
{
    const int32_t *p = items + (int64_t)kItem * k;
    return {p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], p[8], p[9]};
}
// Whether everything that the item names lies inside what the call has.
__device__ __forceinline__ bool item_ok(const Item &it, const PrefillArgs &a)
{
    return it.token0 >= 0 && it.n_new > 0 && (int64_t)it.token0 + it.n_new <= a.n_tokens && it.prefix0 >= 0 && it.n_prefix >= 0 &&
           (int64_t)it.prefix0 + it.n_prefix <= a.n_prefix && it.row0 >= 0 && it.row0 < (int64_t)it.n_new * a.group && it.begin >= 0 && it.begin <= it.end &&
           it.slot >= -1 && it.slot < a.n_slots && it.n_parts >= 1 && it.part >= 0 && it.part < it.n_parts && (int64_t)it.slot - it.part + it.n_parts <= a.n_slots &&
           (it.slot < 0 ? it.n_parts == 1 : it.slot >= it.part);
}

// What a wavefront knows of its 32 rows: lane l has row l % 32.
struct Rows {
    u32x4 q[8];        // channels 16 s + 8 (l / 32) .. of the row
    f32x16 o[4];       // channel 32 t + 8 (i / 4) + 4 (l / 32) + i % 4 of the row
    float m;           // reference of the exponents
    float sum;         // of this half's weights
    float c;           // logits to exponents of 2
};

// Queries of the rows, as fp16 (times a power of two for each row, if they are bf16: exact but for what lies 2^-24 below the largest)
// or as they are.
template <bool BF16> __device__ __forceinline__ void load_q(Rows &w, const uint16_t *row, bool live, const PrefillArgs &a)
{
    const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int s = 0; s < 8; ++s) w.q[s] = live ? reinterpret_cast<const u32x4 *>(row)[2 * s + half] : u32x4{};
    w.c = a.c;
    if constexpr (!BF16) {
        if (a.q_bf16) {
            // the largest finite one: with 0x80 added, infinities and NaN are negative 16-bit numbers
            typedef short s16x2 __attribute__((ext_vector_type(2)));
            s16x2 most2 = {0x80, 0x80};
#pragma unroll
            for (int s = 0; s < 8; ++s)
#pragma unroll
                for (int k = 0; k < 4; ++k) most2 = __builtin_elementwise_max(most2, __builtin_bit_cast(s16x2, w.q[s][k] & 0x7fff7fffu) + s16x2{0x80, 0x80});
            uint32_t big = (uint32_t)(most2.x > most2.y ? most2.x : most2.y) - 0x80u;
            const auto o = __builtin_amdgcn_permlane32_swap(big, big, false, false);
            big = o[0] > o[1] ? o[0] : o[1];
            int e = 14 - ((int)(big >> 7) - 127);                   // the largest becomes 2^14 .. 2^15
            const int most = (int)(__float_as_uint(a.c) >> 23) - 27;   // with which the factor of the logits stays above 2^-101
            e = e > 120 ? 120 : e;
            e = e > most ? most : e;
            e = e < -113 ? -113 : e;
            const float by = __uint_as_float((uint32_t)(e + 127) << 23);
            w.c = a.c * __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
            for (int s = 0; s < 8; ++s)
#pragma unroll
                for (int k = 0; k < 4; ++k) w.q[s][k] = pack<false>(lo_f32(w.q[s][k]) * by, hi_f32(w.q[s][k]) * by);
        }
    }
    // the loads have come back here: a wait for them inside the loop over the tiles would wait for the next tile too
#pragma unroll
    for (int s = 0; s < 8; ++s) asm volatile("" : "+v"(w.q[s]));
}

// Values of V that are finite; infinities and NaN as zero.
template <bool BF16> __device__ __forceinline__ uint32_t finite_only(uint32_t v)
{
    constexpr uint32_t top = BF16 ? 0x7f80u : 0x7c00u;
    const uint32_t low = (v & top) == top ? 0u : 0xffffu, high = (v >> 16 & top) == top ? 0u : 0xffff0000u;
    return v & (low | high);
}

struct Tiles {
    uint32_t lds;               // byte address of two buffers for tiles of K, two for tiles of V
    uint32_t k_at[8], v_at[4];  // where it reads its operands in a buffer: channels 16 j .. of K, 32 d .. of V
};
typedef __attribute__((address_space(3))) const u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

__device__ __forceinline__ u32x4 k_operand(uint32_t at, int b) { return *(lds_u32x4 *)(uintptr_t)(at + b * 32 * kRow); }
// V's operand of keys 16 s ..: two transposed reads of four keys each.
__device__ __forceinline__ u32x4 v_operand(uint32_t at, int s)
{
    u32x4 r;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)(at + s * 16 * kRow + u * 8 * kRow)));
        r[2 * u] = y.x;
        r[2 * u + 1] = y.y;
    }
    return r;
}

// Rows of a tile in LDS: 16 pieces of 16 bytes.  Piece p of key r lies at place p ^ (r & 15) in K, whose operand is read 32 keys at a
// time, and at p ^ 4 (r & 3) in V, of which a transposed read takes four keys' 64 bytes.
//
// A step takes the weights of tile i from its logits while the matrix cores make those of tile i + 1, then adds tile i's values while the
// maximum of tile i + 1 is found.  K is a tile ahead of V; there are two buffers of each, and one barrier a step.
// WAVES wavefronts share a tile of 32 KB keys.
template <bool BF16, int WAVES, int KB>
__device__ __forceinline__ void attend(Rows &w, const Tiles &t, const uint16_t *q, bool live, const PrefillArgs &a, const uint16_t *k, int64_t k_stride, const uint16_t *v,
                                       int64_t v_stride, int begin, int end, int n_keys, int limit, int least, int most, bool whole, bool first, bool once)
{
    if (begin >= end) return;
    constexpr int kKeys = 32 * KB, kTile = kKeys * kRow;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5;
    constexpr int kLoads = kKeys / 4 / WAVES;   // of a wavefront, of K and of V each
    const uint32_t k_bytes = 2 * (uint32_t)k_stride, v_bytes = 2 * (uint32_t)v_stride;
    // key r of the lane's piece in load j is 4 (WAVES j + wave) + lane / 16
    const uint32_t first_row = (uint32_t)(4 * wave + (lane >> 4)), piece = (uint32_t)(lane & 15);
    // Buffers of the next tile to fetch; keys behind the last one read as zeros.
    struct Next {
        const uint8_t *at;
        int left;
        uint32_t bytes, to;   // of a row; where in LDS
        __device__ __forceinline__ u32x4 take(int step)
        {
            const u32x4 buffer = buffer_of(at, (uint32_t)(left < step ? left : step) * bytes);
            at += (uint64_t)step * bytes;
            left -= step;
            return buffer;
        }
    };
    const uint32_t own = __builtin_amdgcn_readfirstlane(t.lds + wave * 4 * kRow);
    Next next_k = {reinterpret_cast<const uint8_t *>(k) + (int64_t)begin * kKeys * k_bytes, n_keys - begin * kKeys, k_bytes, own};
    Next next_v = {reinterpret_cast<const uint8_t *>(v) + (int64_t)begin * kKeys * v_bytes, n_keys - begin * kKeys, v_bytes, own + 2 * kTile};
    auto fetch = [&](Next &next, const uint32_t (&offset)[4], auto mixed) {
        const u32x4 buffer = next.take(kKeys);
        const uint32_t step = (uint32_t)(WAVES * 4) * next.bytes;
        if (WAVES == 1 && once) load_lds<kLoads, WAVES * 4 * kRow, mixed, true>(next.to, buffer, offset, step);
        else load_lds<kLoads, WAVES * 4 * kRow, mixed, false>(next.to, buffer, offset, step);
    };
    // (with four wavefronts or more a lane's piece of K is the same in every load)
    uint32_t k_offset[4], v_offset[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        k_offset[j] = first_row * k_bytes + (piece ^ ((WAVES >= 4 ? first_row : first_row + 4 * WAVES * j) & 15)) * 16;
        v_offset[j] = first_row * v_bytes + (piece ^ (uint32_t)(lane >> 4) << 2) * 16;
    }
    auto fetch_k = [&] {
        fetch(next_k, k_offset, std::bool_constant<(WAVES < 4)>{});
        next_k.to = 2 * own + kTile - next_k.to;   // the other one of two places
    };
    auto fetch_v = [&] {
        fetch(next_v, v_offset, std::false_type{});
        next_v.to = 2 * (own + 2 * kTile) + kTile - next_v.to;
    };
    constexpr std::integral_constant<int, 0> c0{};
    constexpr std::integral_constant<int, 2> c2{};
    constexpr std::integral_constant<int, 4> c4{};
    constexpr std::integral_constant<int, 8> c8{};
    auto hide = [&](f32x16 (&s)[KB], int i) {
        const int sees = limit - i * kKeys - 4 * half;
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[b][r] = 32 * b + 8 * (r >> 2) + (r & 3) > sees ? -INFINITY : s[b][r];
    };
    auto top_of = [&](const f32x16 (&s)[KB]) {
        float top = s[0][0];
#pragma unroll
        for (int r = 0; r < 16; ++r)
#pragma unroll
            for (int b = 0; b < KB; ++b) top = fmaxf(top, s[b][r]);
        return both_max(top) * w.c;
    };
    auto follow = [&](float top) {
        // fp16: logits of up to 2^26 are rounded by 2, and so are the reference and the bound; 2^-22 of the logit on top keeps weights below 2^15 all the same
        const bool grows = (BF16 ? top : fmaf(fabsf(top), 0x1p-22f, top)) > w.m + (kLift<BF16> + kSlack<BF16>);
        if (__any(grows)) {   // row by row: what a row gives does not depend on the others of its wavefront
            const float m = grows ? top - kLift<BF16> : w.m, by = __builtin_amdgcn_exp2f(w.m - m);
            w.m = m;
            w.sum *= by;
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) w.o[d][r] *= by;
        }
    };
    auto logits = [&](f32x16 (&s)[KB], uint32_t buffer, auto from, auto to) {
#pragma unroll
        for (int j = from; j < to; ++j)
#pragma unroll
            for (int b = 0; b < KB; ++b) s[b] = mfma<BF16>(k_operand(t.k_at[j] + buffer, b), w.q[j], j ? s[b] : f32x16{});
    };
    auto weights = [&](uint32_t (&p)[8 * KB], const f32x16 (&s)[KB]) {
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int r = 0; r < 16; r += 2) {
                const float x = __builtin_amdgcn_exp2f(fmaf(s[b][r], w.c, -w.m)), y = __builtin_amdgcn_exp2f(fmaf(s[b][r + 1], w.c, -w.m));
                p[8 * b + r / 2] = pack<BF16>(x, y);
                w.sum = add_pair<BF16>(p[8 * b + r / 2], w.sum);
            }
    };
    // `beside`: what is done beside the products of 16 keys.
    auto values = [&](const uint32_t (&p)[8 * KB], uint32_t buffer, auto cleaned, auto beside) {
#pragma unroll
        for (int j = 0; j < 2 * KB; ++j) {
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                u32x4 x = v_operand(t.v_at[d] + buffer, j);
                if constexpr (cleaned) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = finite_only<BF16>(x[e]);
                    __builtin_amdgcn_sched_barrier(0);
                }
                w.o[d] = mfma<BF16>(x, u32x4{p[4 * j], p[4 * j + 1], p[4 * j + 2], p[4 * j + 3]}, w.o[d]);
            }
            beside(j);
        }
    };
    // Whether a tile of V holds infinities or NaN.  Where not all rows see all of its keys, a weight of zero must not meet them.
    auto strange = [&](uint32_t buffer) {
        uint32_t zero = 0;
        asm("" : "+v"(zero));
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};   // of the values times zero: NaN if one of them is not finite
#pragma unroll
        for (int j = 0; j < kTile / 1024; ++j) {
            const u32x4 x = *(lds_u32x4 *)(uintptr_t)(t.lds + buffer + 1024 * j + 16 * lane);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (BF16) sum[e] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, x[e]), __builtin_bit_cast(bf16x2, zero), sum[e], false);
                else sum[e] = __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, x[e]), __builtin_bit_cast(f16x2, zero), sum[e], false);
            }
        }
        return __any(!((sum[0] + sum[1]) + (sum[2] + sum[3]) == 0.0f));
    };
    // the tiles that all rows of the wavefront see, then those that need a mask.  `whole`: all rows see all keys, and zeros stand behind these; `first`: the
    // rows have no sums yet.
    const int seen = (least + 1) / kKeys, plain = seen < begin ? begin : seen < end ? seen : end;
    // the first keys and the queries at once; what the first logits do not need waits until these are there
    fetch_k();
    load_q<BF16>(w, q, live, a);
    fetch_v();
    if (begin + 1 < end) {
        fetch_k();
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" :: "n"(2 * kLoads) : "memory");
    } else
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" :: "n"(kLoads) : "memory");
    f32x16 s[KB];
    logits(s, 0, c0, c8);
    if (begin >= plain) hide(s, begin);
    if (first) {   // nothing to rescale yet
        const float top = top_of(s);
        w.m = top > w.m ? top - kLift<BF16> : w.m;
    } else follow(top_of(s));
    int i = begin;
    auto step = [&](auto odd) {
        wait_barrier();   // K of tile i + 1 and V of tile i have arrived, and nobody reads the tiles before them
        f32x16 next[KB];
        uint32_t p[8 * KB];
        // (the scalar work of the fetches beside the first products)
        logits(next, odd ? 0 : kTile, c0, c2);
        if (i + 2 < end) fetch_k();
        logits(next, odd ? 0 : kTile, c2, c4);
        fetch_v();
        logits(next, odd ? 0 : kTile, c4, c8);
        weights(p, s);
        // (the maximum a piece beside each four products: 8192 tokens 973 -> 957 us, 4 replays 49.8 -> 49.5)
        float top = -INFINITY;
        values(p, (odd ? 3 : 2) * kTile, std::false_type{}, [&](int j) {
#pragma unroll
            for (int r = 0; r < 8; ++r) top = fmaxf(top, next[j / 2][8 * (j & 1) + r]);
        });
        follow(both_max(top) * w.c);
#pragma unroll
        for (int b = 0; b < KB; ++b) s[b] = next[b];
        ++i;
    };
    while (i + 2 < plain) {
        step(std::false_type{});
        step(std::true_type{});
    }
    if (i + 1 < plain) step(std::false_type{});   // (200 tokens of 32 heads 10.4 -> 9.9 us)
    const int from = i;
    bool left_out = false;
    for (; i < end; ++i) {
        wait_barrier();
        if (i + 2 < end) fetch_k();
        if (i + 1 < end) fetch_v();
        if (i * kKeys > most) continue;   // no row of this wavefront sees the tile
        const uint32_t odd = (uint32_t)((i - begin) & 1) * kTile;
        uint32_t p[8 * KB];
        weights(p, s);
        // (asked of every tile here: 6 ragged prompts 67.4 us, so 64.3)
        if (whole || i < plain || !strange(2 * kTile + odd)) values(p, 2 * kTile + odd, std::false_type{}, [](int) {});
        else {
            values(p, 2 * kTile + odd, std::true_type{}, [](int) {});
            left_out = true;
        }
        if (i + 1 < end) {
            logits(s, kTile - odd, c0, c8);
            hide(s, i + 1);
            follow(top_of(s));
        }
    }
    if (left_out) {   // what is not finite, for the rows that see it
        const int last = end * kKeys < most + 1 ? end * kKeys : most + 1;
#pragma unroll 1
        for (int key = from * kKeys; key < last; ++key) {
            const u32x2 *row = reinterpret_cast<const u32x2 *>(v + (int64_t)key * v_stride) + half;
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const u32x2 x = row[8 * d + r / 2];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t bits = e & 1 ? x[e >> 1] >> 16 : x[e >> 1] & 0xffffu;
                        const float value = BF16 ? __uint_as_float(bits << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
                        w.o[d][r + e] += key <= limit && !(fabsf(value) < INFINITY) ? value : 0.0f;
                    }
                }
        }
    }
    wait_barrier();   // nobody reads the last tile: its place may be filled again
}

// BF16: the new tokens' keys, values and queries are bf16; else keys and values are fp16.
template <bool BF16, int WAVES, int KB>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(2, 2))) void tkv_prefill_kernel(PrefillArgs a)
{
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    const uint32_t block = blockIdx.x + blockIdx.y * gridDim.x;
    const int kv_head = (int)(block % (uint32_t)a.n_kv_heads), number = (int)(block / (uint32_t)a.n_kv_heads);
    if (number >= a.n_items) return;
    const Item it = item_of(a.items, number);
    if (!item_ok(it, a)) {
        if (a.status && threadIdx.x == 0) atomicOr(a.status, TKV_STATUS_BAD_ITEM);
        return;
    }
    constexpr int kTileRows = 32 * WAVES, kKeys = 32 * KB;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5;
    const uint32_t n_rows = (uint32_t)it.n_new * (uint32_t)a.group, row = (uint32_t)it.row0 + 32 * wave + (lane & 31);
    const bool live = row < n_rows;
    const uint32_t use = live ? row : n_rows - 1;
    const int token = (int)(use / (uint32_t)a.group), head = kv_head * a.group + (int)(use - (uint32_t)token * (uint32_t)a.group);
    const uint32_t last = (uint32_t)it.row0 + kTileRows < n_rows ? (uint32_t)it.row0 + kTileRows : n_rows;
    const int n_see = (int)((last - 1) / (uint32_t)a.group) + 1;   // new keys that any row of the workgroup sees
    const int tiles0 = (it.n_prefix + kKeys - 1) / kKeys, tiles1 = (n_see + kKeys - 1) / kKeys;
    const int begin = it.begin, end = it.end < tiles0 + tiles1 ? it.end : tiles0 + tiles1;
    const bool idle = (uint32_t)it.row0 + 32 * wave >= n_rows;     // no row of this wavefront exists

    Tiles t;
    t.lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)smem;
    const int v_key = 4 * half + ((lane & 15) >> 2);
#pragma unroll
    for (int j = 0; j < 8; ++j) t.k_at[j] = t.lds + (uint32_t)((lane & 31) * kRow + ((2 * j + half) ^ (lane & 15)) * 16);
#pragma unroll
    for (int d = 0; d < 4; ++d)
        t.v_at[d] = t.lds + (uint32_t)(v_key * kRow + ((4 * d + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1)) ^ (v_key & 3) << 2) * 16 + (lane & 1) * 8);

    Rows w;
#pragma unroll
    for (int d = 0; d < 4; ++d) w.o[d] = f32x16{};
    w.m = kNone;
    w.sum = 0.0f;
    const bool once = n_rows <= kTileRows;   // one workgroup of a kv head reads all keys
    const uint16_t *q = a.q + (int64_t)(it.token0 + token) * a.q_stride + (int64_t)head * kHeadDim;
    // a range that goes on to the new tokens: their first tile's lines are asked for now, and found in the L2 when the prefix is through (4 chunks of 16
    // tokens behind 2000 to 6000 32.4 -> 31.7 us, 6 ragged prompts 63.8 -> 63.1)
    constexpr int kTouch = kKeys * 4 > 64 * WAVES ? kKeys * 4 / (64 * WAVES) : 1;
    uint32_t touched[kTouch] = {};
    if (begin < tiles0 && end > tiles0) {
#pragma unroll
        for (int e = 0; e < kTouch; ++e) {
            const int line = (int)threadIdx.x + e * 64 * WAVES, key = line >> 2, which = line >> 1 & 1;
            if (key < kKeys && key < n_see)
                touched[e] = *reinterpret_cast<const uint32_t *>((which ? a.v[1] : a.k[1]) + (int64_t)(it.token0 + key) * (which ? a.v_stride[1] : a.k_stride[1]) +
                                                                 (int64_t)kv_head * kHeadDim + (line & 1) * 64);
        }
    }
    if (begin < tiles0) {
        const int see = idle ? -1 : it.n_prefix - 1;
        attend<false, WAVES, KB>(w, t, q, live, a, a.k[0] + (int64_t)it.prefix0 * a.k_stride[0] + (int64_t)kv_head * kHeadDim, a.k_stride[0],
                                 a.v[0] + (int64_t)it.prefix0 * a.v_stride[0] + (int64_t)kv_head * kHeadDim, a.v_stride[0], begin, end < tiles0 ? end : tiles0, it.n_prefix,
                                 it.n_prefix - 1, see, see, true, true, once);
    }
#pragma unroll
    for (int e = 0; e < kTouch; ++e) asm volatile("" :: "v"(touched[e]));
    if (end > tiles0) {
        const int least = idle ? -1 : __builtin_amdgcn_readlane(token, 0), most = idle ? -1 : __builtin_amdgcn_readlane(token, 31);
        attend<BF16, WAVES, KB>(w, t, q, live, a, a.k[1] + (int64_t)it.token0 * a.k_stride[1] + (int64_t)kv_head * kHeadDim, a.k_stride[1],
                                a.v[1] + (int64_t)it.token0 * a.v_stride[1] + (int64_t)kv_head * kHeadDim, a.v_stride[1], begin > tiles0 ? begin - tiles0 : 0, end - tiles0,
                                n_see, token, least, most, false, begin >= tiles0, once);
    }
    const float sum = both_sum(w.sum);
    if (it.slot < 0) {
        const float by = 1.0f / sum;
        uint16_t *to = a.out + ((int64_t)(it.token0 + token) * (a.n_kv_heads * a.group) + head) * kHeadDim;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int r = 0; r < 16; r += 8) {
                uint32_t x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float u = w.o[d][r + 2 * e] * by, v = w.o[d][r + 2 * e + 1] * by;
                    x[e] = a.out_bf16 ? pack<true>(u, v) : pack<false>(u, v);
                }
                // channels 4 half .. and 8 + 4 half .. of 16: each half takes eight in a row
                const auto y = __builtin_amdgcn_permlane32_swap(x[0], x[2], false, false), z = __builtin_amdgcn_permlane32_swap(x[1], x[3], false, false);
                if (live) *reinterpret_cast<u32x4 *>(to + 32 * d + 2 * r + 8 * half) = u32x4{y[0], z[0], y[1], z[1]};
            }
    } else {
        const int64_t at = ((int64_t)it.slot * a.n_kv_heads + kv_head) * kTileRows + 32 * wave + (lane & 31);
        float *to = a.partial + at * kHeadDim;
        if (live) {
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int r = 0; r < 16; r += 4)
                    *reinterpret_cast<float4 *>(to + 32 * d + 2 * r + 4 * half) = make_float4(w.o[d][r], w.o[d][r + 1], w.o[d][r + 2], w.o[d][r + 3]);
            if (half == 0) reinterpret_cast<float2 *>(a.partial + (int64_t)a.n_slots * a.n_kv_heads * kTileRows * kHeadDim)[at] = make_float2(w.m, sum);
        }
    }
}

// Joins the parts of a tile's rows: out = sum_p 2^(m_p - m) o_p / sum_p 2^(m_p - m) l_p.  Bound by the
// loads' latency.  32 lanes take a row, four channels each, eight parts on the way; or, of many parts, eight times 32 lanes every eighth part of it.
template <bool MANY>
__global__ __launch_bounds__(256) void tkv_prefill_merge_kernel(PrefillArgs a, int32_t tile_rows)
{
    constexpr int kSets = MANY ? 8 : 1, kRows = 8 / kSets;   // of 32 lanes for a row; rows of a workgroup
    const uint32_t chunks = (uint32_t)tile_rows / kRows, block = blockIdx.x + blockIdx.y * gridDim.x;
    const uint32_t of = block / chunks;
    const int kv_head = (int)(of % (uint32_t)a.n_kv_heads), cut = (int)(of / (uint32_t)a.n_kv_heads);
    if (cut >= a.n_cut) return;
    const int32_t *what = a.items + (int64_t)kItem * cut + 10;
    const int token0 = what[0], n_new = what[1], row0 = what[2], slot = what[3], n_parts = what[4];
    if (token0 < 0 || n_new <= 0 || (int64_t)token0 + n_new > a.n_tokens || row0 < 0 || slot < 0 || n_parts < 1 || (int64_t)slot + n_parts > a.n_slots) {
        if (a.status && threadIdx.x == 0) atomicOr(a.status, TKV_STATUS_BAD_ITEM);
        return;
    }
    const int lane = threadIdx.x & 31, set = MANY ? (int)(threadIdx.x >> 5) : 0, in_tile = (int)(block % chunks) * kRows + (MANY ? 0 : (int)(threadIdx.x >> 5));
    const uint32_t row = (uint32_t)row0 + in_tile, n_rows = (uint32_t)n_new * (uint32_t)a.group;
    if (row >= n_rows) return;
    const int64_t step = (int64_t)a.n_kv_heads * tile_rows, at = ((int64_t)slot * a.n_kv_heads + kv_head) * tile_rows + in_tile;   // from part to part; of the first one
    const float2 *ml = reinterpret_cast<const float2 *>(a.partial + (int64_t)a.n_slots * step * kHeadDim) + at;
    const float4 *rows = reinterpret_cast<const float4 *>(a.partial + at * kHeadDim) + lane;
    // part k of this set is k kSets + set
    const int mine = (n_parts - set + kSets - 1) / kSets;
    auto fetch = [&](float4 (&o)[8], int p) {
#pragma unroll
        for (int k = 0; k < 8; ++k) o[k] = p + k < mine ? rows[((p + k) * kSets + set) * step * (kHeadDim / 4)] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    };
    // (m, sum) of up to 32 parts at once, a lane each, and the first rows beside them
    float m = kNone, sum = 0.0f;
    float4 x = {0.0f, 0.0f, 0.0f, 0.0f}, o[8];
    for (int first = 0; first < mine; first += 32) {
        const float2 here = first + lane < mine ? ml[((first + lane) * kSets + set) * step] : make_float2(kNone, 0.0f);
        fetch(o, first);
        float top = here.x;
#pragma unroll
        for (int k = 16; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor(top, k));
        top = fmaxf(top, m);
        const float before = __builtin_amdgcn_exp2f(m - top), by = __builtin_amdgcn_exp2f(here.x - top);
        m = top;
        sum *= before;
        x.x *= before; x.y *= before; x.z *= before; x.w *= before;
        float add = here.y * by;
#pragma unroll
        for (int k = 16; k > 0; k >>= 1) add += __shfl_xor(add, k);
        sum += add;
        for (int p = 0; p < 32 && first + p < mine; p += 8) {
            if (p > 0) fetch(o, first + p);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float f = __shfl(by, p + k, 32);
                x.x = fmaf(o[k].x, f, x.x); x.y = fmaf(o[k].y, f, x.y); x.z = fmaf(o[k].z, f, x.z); x.w = fmaf(o[k].w, f, x.w);
            }
        }
    }
    if constexpr (MANY) {
        __shared__ float4 rows_s[8][32];
        __shared__ float2 ml_s[8];
        rows_s[set][lane] = x;
        if (lane == 0) ml_s[set] = make_float2(m, sum);
        __syncthreads();
        if (set > 0) return;
        float top = kNone;
#pragma unroll
        for (int k = 0; k < 8; ++k) top = fmaxf(top, ml_s[k].x);
        sum = 0.0f;
        x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float f = __builtin_amdgcn_exp2f(ml_s[k].x - top);
            const float4 y = rows_s[k][lane];
            sum = fmaf(ml_s[k].y, f, sum);
            x.x = fmaf(y.x, f, x.x); x.y = fmaf(y.y, f, x.y); x.z = fmaf(y.z, f, x.z); x.w = fmaf(y.w, f, x.w);
        }
    }
    const float by = 1.0f / sum;
    const uint32_t token = row / (uint32_t)a.group, head = kv_head * a.group + (row - token * a.group);
    u32x2 *to = reinterpret_cast<u32x2 *>(a.out + ((int64_t)(token0 + (int)token) * (a.n_kv_heads * a.group) + head) * kHeadDim);
    to[lane] = a.out_bf16 ? u32x2{pack<true>(x.x * by, x.y * by), pack<true>(x.z * by, x.w * by)} : u32x2{pack<false>(x.x * by, x.y * by), pack<false>(x.z * by, x.w * by)};
}

template <int WAVES, int KB> hipError_t launch(const PrefillArgs &a, bool bf16, dim3 grid, hipStream_t stream)
{
    hipLaunchKernelGGL((bf16 ? tkv_prefill_kernel<true, WAVES, KB> : tkv_prefill_kernel<false, WAVES, KB>), grid, dim3(64 * WAVES), 4 * 32 * KB * kRow, stream, a);   // two buffers of K, two of V
    return hipGetLastError();
}

} // namespace

int tkv_launch_prefill(int32_t n_q_heads, int32_t n_kv_heads, const void *q, int64_t q_stride, int32_t q_type, const void *K, int64_t k_stride, const void *V,
                       int64_t v_stride, int32_t kv_type, int32_t n_tokens, const void *K_prefix, const void *V_prefix, int32_t n_prefix, const tkv_prefill *prefill,
                       float sm_scale, void *out, int32_t out_type, void *workspace, int32_t *status, void *stream)
{
    PrefillArgs a = {};
    a.q = (const uint16_t *)q;
    a.k[0] = (const uint16_t *)K_prefix; a.k[1] = (const uint16_t *)K;
    a.v[0] = (const uint16_t *)V_prefix; a.v[1] = (const uint16_t *)V;
    // (the stride of a single token is any number)
    a.q_stride = q_stride;
    if (n_tokens == 1) k_stride = v_stride = (int64_t)n_kv_heads * kHeadDim;
    a.k_stride[0] = a.v_stride[0] = (int64_t)n_kv_heads * kHeadDim;
    a.k_stride[1] = k_stride; a.v_stride[1] = v_stride;
    a.items = prefill->items;
    a.out = (uint16_t *)out;
    a.partial = (float *)workspace;
    a.status = status;
    a.n_items = prefill->n_items; a.n_slots = prefill->n_slots; a.n_cut = prefill->n_cut; a.n_tokens = n_tokens; a.n_prefix = n_prefix;
    a.group = n_q_heads / n_kv_heads; a.n_kv_heads = n_kv_heads;
    a.q_bf16 = q_type == TKV_BF16; a.out_bf16 = out_type == TKV_BF16;
    a.c = sm_scale * 1.44269504088896340736f;
    constexpr int64_t kMaxX = 1 << 22;   // a grid has less than 2^32 threads in a dimension
    auto grid = [&](int64_t blocks) { return dim3((unsigned)(blocks < kMaxX ? blocks : kMaxX), (unsigned)((blocks + kMaxX - 1) / kMaxX)); };
    const int64_t blocks = (int64_t)prefill->n_items * n_kv_heads;
    const dim3 groups = grid(blocks);
    const bool bf16 = kv_type == TKV_BF16;
    const hipError_t e = prefill->tile_rows == 32 ? launch<1, 1>(a, bf16, groups, (hipStream_t)stream)
                         : prefill->tile_rows == 128 ? launch<4, 2>(a, bf16, groups, (hipStream_t)stream) : launch<8, 2>(a, bf16, groups, (hipStream_t)stream);
    if (e != hipSuccess) return TKV_ERR_HIP;
    if (prefill->n_cut > 0) {
        const int64_t rows = (int64_t)prefill->n_cut * n_kv_heads * prefill->tile_rows;
        // Eight sets of lanes a row save half a microsecond for every eight parts behind the first, and cost two for a thousand rows: one token of one head behind 7560
        // (237 parts) 26.0 -> 11.8 us, 100000 of 64 heads (126 parts, 256 rows) 80.9 -> 72.9, 701 11.0 -> 10.0; but 16 tokens of 64 heads (8 parts, 4096 rows) 36.9 -> 46.1
        const bool many = prefill->n_slots > (8 + rows / 32) * prefill->n_cut;
        if (many) hipLaunchKernelGGL(tkv_prefill_merge_kernel<true>, grid(rows), dim3(256), 0, (hipStream_t)stream, a, prefill->tile_rows);
        else hipLaunchKernelGGL(tkv_prefill_merge_kernel<false>, grid(rows / 8), dim3(256), 0, (hipStream_t)stream, a, prefill->tile_rows);
        if (hipGetLastError() != hipSuccess) return TKV_ERR_HIP;
    }
    return TKV_OK;
}
