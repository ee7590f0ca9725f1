// tkv_quantize_rows: keys and values of chosen tokens as the cache would give them back, dense rows to dense rows: what
// tkv_quantize_append and tkv_gather_dequant do together (Sec. 3.2.1), without pages.  And tkv_head_distortion: the mean squared
// difference of two attention outputs by sequence and head (Sec. 3.1.3: what the replay of a tag at a width is compared by).
//
//   zero = fp16(min), scale = fp16((max - min) / (2^b - 1)), code = clamp(rint((x - zero) * (1 / scale)), 0, 2^b - 1),
//   0 if scale == 0;  out = fp16(code * scale + zero), one rounding
//
// IEEE binary32 without fused multiply-add up to the code, as in the append; the fp16 fused multiply-add rounds once.
// Rows are bound by HBM, 512 bytes in and 512 out for a token of a head: 65 536 tokens of 8 heads 85 us, 6.3 TB/s (171 with K
// and V of a row by two threads and plain divisions); 22 000 in blocks of per-channel keys 22 us, 6.0 TB/s, the blocks' workgroups first, which take longest.
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>

#include "tkv_internal.h"
#include "tkv_layout.h"

#pragma clang fp contract(off)

namespace {

using namespace tkv;

struct RowsArgs {
    const uint16_t *in[2];     // K, V
    uint16_t *out[2];
    int64_t stride[2];
    const uint8_t *tag_bits;
    const int32_t *blocks;
    int32_t *status;
    int32_t n_tokens, n_heads, n_blocks, channel_keys;
    uint32_t block_groups;     // workgroups of the blocks, which take longest; the rows' follow
};

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));

template <int CTRL> __device__ __forceinline__ float dpp(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float lo_f32(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float hi_f32(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
struct Grid {
    float zero, inv, levels;
    half2_t scale, shift;   // scale and zero-point, twice
};
__device__ __forceinline__ Grid grid_of(float mn, float mx, bool wide)
{
    if (mn == 0.0f) mn = 0.0f;   // -0 -> +0
    Grid g;
    g.levels = wide ? 15.0f : 3.0f;
    // Quotient by the levels and reciprocal of the scale, both correctly rounded: a product with the rounded reciprocal (the hardware's,
    // one unit off at most) and one step of Newton, whose residual the fused multiply-add gives exactly.  (Where a quotient is too small for
    // that it rounds to an fp16 zero either way.)  The plain divisions are ten instructions each.
    const float r = __fsub_rn(mx, mn), y = wide ? 1.0f / 15.0f : 1.0f / 3.0f, q = __fmul_rn(r, y);
    float quotient = __builtin_fmaf(__builtin_fmaf(-q, g.levels, r), y, q);
    asm("" : "+v"(quotient));   // rounded to 32 bits before it is rounded to 16: the compiler would do both at once, and miss ties
    const _Float16 sh = (_Float16)quotient, zh = (_Float16)mn;
    const float s = (float)sh, i = __builtin_amdgcn_rcpf(s);
    g.zero = (float)zh;
    g.inv = s == 0.0f ? 0.0f : __builtin_fmaf(__builtin_fmaf(-s, i, 1.0f), i, i);
    g.scale = half2_t{sh, sh};
    g.shift = half2_t{zh, zh};
    return g;
}
// Bits of two fp16 values that the codes of x and y stand for.
__device__ __forceinline__ uint32_t back(const Grid &g, float x, float y)
{
    const float t = __builtin_rintf(__builtin_amdgcn_fmed3f(__fmul_rn(__fsub_rn(x, g.zero), g.inv), 0.0f, g.levels));
    const float u = __builtin_rintf(__builtin_amdgcn_fmed3f(__fmul_rn(__fsub_rn(y, g.zero), g.inv), 0.0f, g.levels));
    const half2_t code = {(_Float16)t, (_Float16)u};
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(code, g.scale, g.shift));   // one rounding
}
__device__ __forceinline__ uint32_t halves(uint32_t v)   // two bf16 numbers as fp16
{
    const half2_t h = {(_Float16)lo_f32(v), (_Float16)hi_f32(v)};
    return __builtin_bit_cast(uint32_t, h);
}

// Eight channels of a row, whose group the four lanes of a quad hold.
__device__ __forceinline__ uint4 row_piece(uint4 x, uint32_t bits)
{
    const float f[8] = {lo_f32(x.x), hi_f32(x.x), lo_f32(x.y), hi_f32(x.y), lo_f32(x.z), hi_f32(x.z), lo_f32(x.w), hi_f32(x.w)};
    float mn = f[0], mx = f[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) {
        mn = fminf(mn, f[i]);
        mx = fmaxf(mx, f[i]);
    }
    mn = fminf(mn, dpp<0xB1>(mn)); mx = fmaxf(mx, dpp<0xB1>(mx));
    mn = fminf(mn, dpp<0x4E>(mn)); mx = fmaxf(mx, dpp<0x4E>(mx));
    const Grid g = grid_of(mn, mx, bits == 4);
    return make_uint4(back(g, f[0], f[1]), back(g, f[2], f[3]), back(g, f[4], f[5]), back(g, f[6], f[7]));
}

// A quad of lanes has a group of 32 channels, sixteen lanes a row of K and the same row of V, so that all reads and writes of a row are whole lines.
// PER: rows of K and of V that a thread has a piece of; ONCE: past the caches.
template <int PER, bool ONCE>
__global__ __launch_bounds__(256) void tkv_rows_kernel(RowsArgs a)
{
    uint32_t block = blockIdx.x + blockIdx.y * gridDim.x;
    if (block >= a.block_groups) {
        block -= a.block_groups;
        constexpr int kRows = 16 * PER;   // of a workgroup
        const int part = threadIdx.x & 15;
        const uint32_t first = block * kRows, heads = (uint32_t)a.n_heads, n_rows = (uint32_t)a.n_tokens * heads;
        const int token0 = (int)(first / heads), head0 = (int)(first - (uint32_t)token0 * heads);
        int token[PER], head[PER];
        uint32_t bits[PER];
        bool live[PER];
        uint4 x[PER][2];
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int local = 16 * k + (int)(threadIdx.x >> 4), at = head0 + local;
            // (below 32 heads the quotient is 1 / 64 from the next integer at least, and off by 2^-17)
            const int of = heads >= 32 ? (at >= (int)heads ? 1 : 0) : (int)(((float)at + 0.5f) * __builtin_amdgcn_rcpf((float)heads));
            live[k] = (uint64_t)first + local < n_rows;
            token[k] = live[k] ? token0 + of : 0;
            head[k] = live[k] ? at - of * (int)heads : 0;
            bits[k] = a.tag_bits[token[k]];
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const uint4 *src = reinterpret_cast<const uint4 *>(a.in[w] + token[k] * a.stride[w] + (int64_t)head[k] * kHeadDim) + part;
                x[k][w] = ONCE ? load_once(src) : *src;
            }
        }
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            if (!live[k]) continue;
            const uint32_t b = bits[k];
            const int64_t row = (int64_t)token[k] * heads + head[k];
            if (b != 0 && b != 2 && b != 4) {
                if (a.status && part == 0 && head[k] == 0) atomicOr(a.status, TKV_STATUS_TAG_MISMATCH);
                continue;
            }
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                if (w == 0 && b == 2 && a.channel_keys) continue;   // a block's
                const uint4 y = b ? row_piece(x[k][w], b) : make_uint4(halves(x[k][w].x), halves(x[k][w].y), halves(x[k][w].z), halves(x[k][w].w));
                store_once(reinterpret_cast<uint4 *>(a.out[w] + row * kHeadDim) + part, y);
            }
        }
        return;
    }
    // keys per channel: a wavefront takes a block of 32 tokens of a head, lane (i, part) its tokens i, 4 + i, .. and channels 8 part ..
    const int64_t unit = (int64_t)block * 4 + (threadIdx.x >> 6);
    if (unit >= (int64_t)a.n_blocks * a.n_heads) return;
    const int number = (int)((uint32_t)unit / (uint32_t)a.n_heads), head = (int)(unit - (int64_t)number * a.n_heads);
    const int lane = threadIdx.x & 63, part = lane & 15, i0 = lane >> 4;
    int token[8];
    bool ok = true;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        token[k] = a.blocks[(int64_t)number * kGroup + 4 * k + i0];
        const bool in = token[k] >= 0 && token[k] < a.n_tokens;
        ok = ok && in;
        if (!in) token[k] = 0;
    }
    uint4 x[8];
    uint32_t bits[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        bits[k] = a.tag_bits[token[k]];
        x[k] = reinterpret_cast<const uint4 *>(a.in[0] + token[k] * a.stride[0] + (int64_t)head * kHeadDim)[part];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) ok = ok && bits[k] == 2;
    if (!__all(ok)) {
        if (a.status && lane == 0) atomicOr(a.status, TKV_STATUS_BLOCK_PARTIAL);
        return;
    }
    uint32_t o[8][4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        float f[2][8], mn[2], mx[2];
        Grid g[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t u = c == 0 ? x[k].x : c == 1 ? x[k].y : c == 2 ? x[k].z : x[k].w;
                f[h][k] = h ? hi_f32(u) : lo_f32(u);
            }
            mn[h] = mx[h] = f[h][0];
#pragma unroll
            for (int k = 1; k < 8; ++k) {
                mn[h] = fminf(mn[h], f[h][k]);
                mx[h] = fmaxf(mx[h], f[h][k]);
            }
            mn[h] = fminf(mn[h], __shfl_xor(mn[h], 16)); mx[h] = fmaxf(mx[h], __shfl_xor(mx[h], 16));
            mn[h] = fminf(mn[h], __shfl_xor(mn[h], 32)); mx[h] = fmaxf(mx[h], __shfl_xor(mx[h], 32));
            g[h] = grid_of(mn[h], mx[h], false);
        }
        Grid both = g[0];
        both.scale.y = g[1].scale.x;
        both.shift.y = g[1].shift.x;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float t = __builtin_rintf(__builtin_amdgcn_fmed3f(__fmul_rn(__fsub_rn(f[0][k], g[0].zero), g[0].inv), 0.0f, 3.0f));
            const float u = __builtin_rintf(__builtin_amdgcn_fmed3f(__fmul_rn(__fsub_rn(f[1][k], g[1].zero), g[1].inv), 0.0f, 3.0f));
            const half2_t code = {(_Float16)t, (_Float16)u};
            o[k][c] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(code, both.scale, both.shift));
        }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        store_once(reinterpret_cast<uint4 *>(a.out[0] + ((int64_t)token[k] * a.n_heads + head) * kHeadDim) + part, make_uint4(o[k][0], o[k][1], o[k][2], o[k][3]));
}

// ------------------------------------------------------------------ distortion
struct DistortionArgs {
    const void *a, *b;
    const int32_t *seq_indptr;
    double *out, *partial;
    int32_t batch, n_tokens, n_heads, chunk;   // chunk: tokens whose squares a workgroup adds up
};
// The sequence's slots among the partial sums begin at first / chunk + b: chunks of a sequence begin at its first token, and
// ceil(n / chunk) of them end before the next one's begin.
__device__ __forceinline__ int first_slot(int first, int b, int chunk) { return (int)((uint32_t)first / (uint32_t)chunk) + b; }

__device__ __forceinline__ float f32_of(uint32_t bits, int type) { return type == TKV_BF16 ? __uint_as_float(bits << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)bits); }

// Adds to `sum` the squares of a lane's piece of rows t, t + tokens, .. of four, those before `end`.
template <int TYPE, bool ONCE>
__device__ __forceinline__ double squares(const uint4 *x, const uint4 *y, int t, int end, int tokens, int64_t step, double sum)
{
    uint4 u[4], v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int64_t at = (t + k * tokens < end ? t + k * tokens : t) * step;
        u[k] = ONCE ? load_once(x + at) : x[at];
        v[k] = ONCE ? load_once(y + at) : y[at];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (t + k * tokens >= end) break;
        const uint32_t p[4] = {u[k].x, u[k].y, u[k].z, u[k].w}, q[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (TYPE == TKV_FP32) {
                const double d = (double)__uint_as_float(p[i]) - (double)__uint_as_float(q[i]);
                sum = __builtin_fma(d, d, sum);
            } else {
#pragma unroll
                for (int h = 0; h < 32; h += 16) {
                    const double d = (double)f32_of(p[i] >> h & 0xffffu, TYPE) - (double)f32_of(q[i] >> h & 0xffffu, TYPE);
                    sum = __builtin_fma(d, d, sum);
                }
            }
        }
    }
    return sum;
}

// A workgroup takes a chunk of one sequence's tokens and sixteen (fp32: eight) heads, or all heads of several tokens at a time.  Bound by
// HBM: eight loads of 16 bytes a lane are on the way, 975 MB of bf16 rows in 148 us, 6.6 TB/s (all heads of the tokens by one workgroup, sixteen behind sixteen, 164 us).
template <int TYPE, bool ONCE>
__global__ __launch_bounds__(256) void tkv_distortion_kernel(DistortionArgs a)
{
    __shared__ double sums[16];
    constexpr int kPer = TYPE == TKV_FP32 ? 4 : 8, kLanes = kHeadDim / kPer, kGroups = 256 / kLanes;   // values of a 16-byte piece; lanes of a row; rows at once
    const int width = a.n_heads < kGroups ? a.n_heads : kGroups, tokens = kGroups / width;             // heads and tokens at once
    const uint32_t block = blockIdx.x + blockIdx.y * gridDim.x, passes = (uint32_t)((a.n_heads + width - 1) / width), slot = block / passes;
    // the sequence that the slot belongs to: every wavefront looks through all of them
    int begin = 0, end = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 64) {
        const int b = b0 + (int)(threadIdx.x & 63), at = b < a.batch ? b : a.batch - 1;
        const int lo = a.seq_indptr[at], hi = a.seq_indptr[at + 1];
        const bool ok = b < a.batch && lo >= 0 && hi > lo && hi <= a.n_tokens;
        const int first = ok ? first_slot(lo, b, a.chunk) : 0;
        const uint64_t mine = __ballot(ok && (uint32_t)first <= slot && slot - (uint32_t)first < (uint32_t)((hi - lo + a.chunk - 1) / a.chunk));
        if (mine) {
            const int lane = __builtin_ctzll(mine), l = __builtin_amdgcn_readlane(lo, lane), h = __builtin_amdgcn_readlane(hi, lane), f = __builtin_amdgcn_readlane(first, lane);
            begin = l + (int)(slot - (uint32_t)f) * a.chunk;
            end = begin + a.chunk < h ? begin + a.chunk : h;
            break;
        }
    }
    if (begin >= end) return;
    const int part = threadIdx.x % kLanes, group = threadIdx.x / kLanes, sub = group / width;
    const int head = (int)(block - slot * passes) * width + group - sub * width;
    double sum = 0.0;
    if (sub < tokens && head < a.n_heads) {
        const int64_t step = (int64_t)a.n_heads * kLanes;
        const uint4 *x = reinterpret_cast<const uint4 *>(a.a) + ((int64_t)head * kLanes + part), *y = reinterpret_cast<const uint4 *>(a.b) + ((int64_t)head * kLanes + part);
        for (int t = begin + sub; t < end; t += 4 * tokens) sum = squares<TYPE, ONCE>(x, y, t, end, tokens, step, sum);
    }
#pragma unroll
    for (int k = kLanes / 2; k > 0; k >>= 1) sum += __shfl_xor(sum, k);
    if (tokens > 1) {
        if (part == 0) sums[group] = sum;
        __syncthreads();
        for (int k = 1; k < tokens; ++k)
            if (sub == 0 && part == 0) sum += sums[group + k * width];
    }
    if (sub == 0 && part == 0 && head < a.n_heads) a.partial[(int64_t)slot * a.n_heads + head] = sum;
}
// Adds up the slots of a sequence: `width` lanes (a power of two) take a head each, 256 / width rows of them every so many slots.
__global__ __launch_bounds__(256) void tkv_distortion_join_kernel(DistortionArgs a, int32_t width)
{
    __shared__ double sums[256];
    const uint32_t block = blockIdx.x + blockIdx.y * gridDim.x, passes = (uint32_t)((a.n_heads + width - 1) / width);
    const int b = (int)(block / passes), head = (int)(block % passes) * width + (int)(threadIdx.x % width), row = (int)(threadIdx.x / width), rows = 256 / width;
    if (b >= a.batch) return;
    const int lo = a.seq_indptr[b], hi = a.seq_indptr[b + 1];
    const bool ok = lo >= 0 && hi >= lo && hi <= a.n_tokens;
    const int n = ok ? (hi - lo + a.chunk - 1) / a.chunk : 0;
    double sum = 0.0;
    if (head < a.n_heads) {
        const double *from = a.partial + (int64_t)(ok ? first_slot(lo, b, a.chunk) : 0) * a.n_heads + head;
        for (int k = row; k < n; k += 8 * rows) {
            double x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = k + j * rows < n ? from[(int64_t)(k + j * rows) * a.n_heads] : 0.0;
            sum += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
        }
    }
    sums[threadIdx.x] = sum;
    __syncthreads();
    for (int k = 128; k >= width; k >>= 1) {
        if ((int)threadIdx.x < k) sums[threadIdx.x] += sums[threadIdx.x + k];
        __syncthreads();
    }
    if ((int)threadIdx.x < width && head < a.n_heads)
        a.out[(int64_t)b * a.n_heads + head] = !ok ? __builtin_nan("") : hi > lo ? sums[threadIdx.x] / ((double)(hi - lo) * kHeadDim) : 0.0;
}

// Few tokens: a workgroup takes all of a sequence and head, and there is nothing to join.  Its sums in 64 bits take 9 us a thousand rows (more loads on the way
// change nothing).  bf16, 16 heads, one sequence, this / chunks and a join, us: 16 tokens 3.4 / 5.6, 256 4.6 / 6.1, 384 5.4 / 6.6, 512 6.4 / 6.7, 701 7.7 / 6.7; 64 heads
// 3.5 / 9.2, 4.9 / 11.9, 6.2 / 8.3, 7.8 / 8.5, 9.6 / 9.2; fp32, 64 heads, 384 8.9 / 9.2, 512 11.2 / 10.6.
template <int TYPE>
__global__ __launch_bounds__(1024) void tkv_distortion_short_kernel(DistortionArgs a)
{
    __shared__ double sums[16];
    const uint32_t block = blockIdx.x + blockIdx.y * gridDim.x;
    const int b = (int)(block / (uint32_t)a.n_heads), head = (int)(block % (uint32_t)a.n_heads);
    if (b >= a.batch) return;
    const int lo = a.seq_indptr[b], hi = a.seq_indptr[b + 1];
    const bool ok = lo >= 0 && hi >= lo && hi <= a.n_tokens;
    constexpr int kPer = TYPE == TKV_FP32 ? 4 : 8, kLanes = kHeadDim / kPer, kRows = 1024 / kLanes;
    const int part = threadIdx.x % kLanes;
    const int64_t step = (int64_t)a.n_heads * kLanes;
    const uint4 *x = reinterpret_cast<const uint4 *>(a.a) + ((int64_t)head * kLanes + part), *y = reinterpret_cast<const uint4 *>(a.b) + ((int64_t)head * kLanes + part);
    double sum = 0.0;
    if (ok)
        for (int t = lo + (int)(threadIdx.x / kLanes); t < hi; t += 4 * kRows) sum = squares<TYPE, false>(x, y, t, hi, kRows, step, sum);
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) sum += __shfl_xor(sum, k);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < 16; ++k) sum += sums[k];
        a.out[(int64_t)b * a.n_heads + head] = !ok ? __builtin_nan("") : hi > lo ? sum / ((double)(hi - lo) * kHeadDim) : 0.0;
    }
}

constexpr int64_t kMaxX = 1 << 21;   // a grid has less than 2^32 threads in a dimension
dim3 grid(int64_t blocks) { return dim3((unsigned)(blocks < kMaxX ? blocks : kMaxX), (unsigned)((blocks + kMaxX - 1) / kMaxX)); }

} // namespace

int tkv_launch_quantize_rows(const tkv_desc *desc, const void *K, int64_t k_stride, const void *V, int64_t v_stride, const uint8_t *tag_bits, int32_t n_tokens,
                             const int32_t *blocks, int32_t n_blocks, void *K_out, void *V_out, int32_t *status, void *stream)
{
    RowsArgs a = {};
    a.in[0] = (const uint16_t *)K; a.in[1] = (const uint16_t *)V;
    a.out[0] = (uint16_t *)K_out; a.out[1] = (uint16_t *)V_out;
    a.stride[0] = k_stride; a.stride[1] = v_stride;
    a.tag_bits = tag_bits; a.blocks = blocks; a.status = status;
    a.n_tokens = n_tokens; a.n_heads = desc->n_kv_heads; a.n_blocks = n_blocks;
    a.channel_keys = desc->int2_key_axis == TKV_KEYS_PER_CHANNEL;
    // Two rows of K and of V a thread keep more on the way; beyond what the Infinity Cache holds, one row, read past the caches.  us, 8 heads, rows not
    // read for two calls or more, one / two / one past the caches: 4000 tokens 7.2 / 6.7 / 8.0, 32 000 42.4 / 39.8 / 44.0, 64 000 86.0 / 90.5 / 83.9, 128 000 170 / 181 / 163;
    // per-channel keys 8000 12.9 / 12.8 / 14.3, 64 000 98.0 / 93.9 / 97.0: two.
    const bool far = n_blocks == 0 && (int64_t)n_tokens * a.n_heads > (int64_t)192 << 11;   // 512 bytes a token of a head
    const int per = far ? 1 : 2;
    a.block_groups = (uint32_t)(((int64_t)n_blocks * a.n_heads + 3) / 4);
    const int64_t groups = (int64_t)a.block_groups + ((int64_t)n_tokens * a.n_heads + 16 * per - 1) / (16 * per);
    if (far) hipLaunchKernelGGL((tkv_rows_kernel<1, true>), grid(groups), dim3(256), 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL((tkv_rows_kernel<2, false>), grid(groups), dim3(256), 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? TKV_OK : TKV_ERR_HIP;
}

int tkv_launch_distortion(const void *a_rows, const void *b_rows, int32_t type, const int32_t *seq_indptr, int32_t batch, int32_t n_tokens, int32_t n_heads,
                          double *out, void *workspace, void *stream)
{
    DistortionArgs a = {a_rows, b_rows, seq_indptr, out, (double *)workspace, batch, n_tokens, n_heads, tkv_distortion_chunk(n_tokens, n_heads)};
    if (n_tokens <= 384) {
        auto *whole = type == TKV_BF16 ? tkv_distortion_short_kernel<TKV_BF16> : type == TKV_FP16 ? tkv_distortion_short_kernel<TKV_FP16> : tkv_distortion_short_kernel<TKV_FP32>;
        hipLaunchKernelGGL(whole, grid((int64_t)batch * n_heads), dim3(1024), 0, (hipStream_t)stream, a);
        return hipGetLastError() == hipSuccess ? TKV_OK : TKV_ERR_HIP;
    }
    const int64_t slots = n_tokens / a.chunk + (int64_t)batch;
    const int32_t groups = 256 / (type == TKV_FP32 ? 32 : 16);
    // past the caches what does not fit the Infinity Cache: bf16, 8 heads, rows not read for seven calls, 256 MiB 54.6 us, past them 50.2, 512 MiB 103.2 / 93.7; but of the
    // rows of the last two calls 128 MiB 25.4 / 25.9, 192 MiB 35.5 / 36.8
    const bool far = (int64_t)n_tokens * n_heads * kHeadDim * (type == TKV_FP32 ? 8 : 4) > (int64_t)256 << 20;
    auto *kernel = type == TKV_BF16   ? (far ? tkv_distortion_kernel<TKV_BF16, true> : tkv_distortion_kernel<TKV_BF16, false>)
                   : type == TKV_FP16 ? (far ? tkv_distortion_kernel<TKV_FP16, true> : tkv_distortion_kernel<TKV_FP16, false>)
                                      : (far ? tkv_distortion_kernel<TKV_FP32, true> : tkv_distortion_kernel<TKV_FP32, false>);
    hipLaunchKernelGGL(kernel, grid(slots * (n_heads <= groups ? 1 : (n_heads + groups - 1) / groups)), dim3(256), 0, (hipStream_t)stream, a);
    if (hipGetLastError() != hipSuccess) return TKV_ERR_HIP;
    int32_t width = 1;
    while (width < n_heads && width < 16) width *= 2;
    // few sequences: more workgroups of fewer heads (one sequence of 16 heads, 4096 tokens 14.2 us, so 11.6; 32 768 59.8, 52.9)
    while (width > 2 && (int64_t)batch * ((n_heads + width - 1) / width) < 64) width /= 2;
    hipLaunchKernelGGL(tkv_distortion_join_kernel, grid((int64_t)batch * ((n_heads + width - 1) / width)), dim3(256), 0, (hipStream_t)stream, a, width);
    return hipGetLastError() == hipSuccess ? TKV_OK : TKV_ERR_HIP;
}
