// tkv_quantize_rows: keys and values of chosen tokens as the cache would give them back, dense rows to dense rows: what
// tkv_quantize_append and tkv_gather_dequant do together (Sec. 3.2.1), without pages.  And tkv_head_distortion: the mean squared
// difference of two attention outputs by sequence and head (Sec. 3.1.3: what the replay of a tag at a width is compared by).
//
//   zero = fp16(min), scale = fp16((max - min) / (2^b - 1)), code = clamp(rint((x - zero) * (1 / scale)), 0, 2^b - 1),
//   0 if scale == 0;  out = fp16(code * scale + zero), one rounding
//
// IEEE binary32 without fused multiply-add up to the code, as in the append; the fp16 fused multiply-add rounds once.
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
    uint32_t row_groups;       // workgroups of the rows of K and of V each; the blocks' follow
};

constexpr int kRowsWg = 16;    // rows (a token of a head) of a workgroup

template <int CTRL> __device__ __forceinline__ float dpp(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
struct Grid {
    float zero, inv, levels;
    _Float16 scale_h, zero_h;
};
__device__ __forceinline__ Grid grid_of(float mn, float mx, float levels)
{
    if (mn == 0.0f) mn = 0.0f;   // -0 -> +0
    Grid g;
    g.scale_h = (_Float16)__fdiv_rn(__fsub_rn(mx, mn), levels);
    g.zero_h = (_Float16)mn;
    const float s = (float)g.scale_h;
    g.zero = (float)g.zero_h;
    g.inv = s == 0.0f ? 0.0f : __fdiv_rn(1.0f, s);
    g.levels = levels;
    return g;
}
__device__ __forceinline__ uint32_t back(const Grid &g, float x)   // bits of the fp16 value
{
    const float t = __builtin_amdgcn_fmed3f(__fmul_rn(__fsub_rn(x, g.zero), g.inv), 0.0f, g.levels);
    const _Float16 code = (_Float16)__builtin_rintf(t);
    return __builtin_bit_cast(uint16_t, (_Float16)__builtin_fmaf16(code, g.scale_h, g.zero_h));
}
__device__ __forceinline__ uint32_t half_bits(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }

__global__ __launch_bounds__(256) void tkv_rows_kernel(RowsArgs a)
{
    const uint32_t block = blockIdx.x + blockIdx.y * gridDim.x;
    if (block < 2 * a.row_groups) {
        const int which = block >= a.row_groups, part = threadIdx.x & 15;
        const int64_t row = (int64_t)(block - which * a.row_groups) * kRowsWg + (threadIdx.x >> 4);
        if (row >= (int64_t)a.n_tokens * a.n_heads) return;
        const int token = (int)(row / a.n_heads), head = (int)(row - (int64_t)token * a.n_heads);
        const uint32_t bits = a.tag_bits[token];
        if (bits != 0 && bits != 2 && bits != 4) {
            if (a.status && part == 0 && head == 0) atomicOr(a.status, TKV_STATUS_TAG_MISMATCH);
            return;
        }
        if (which == 0 && bits == 2 && a.channel_keys) return;   // a block's
        const uint4 x = reinterpret_cast<const uint4 *>(a.in[which] + token * a.stride[which] + (int64_t)head * kHeadDim)[part];
        const uint32_t u[4] = {x.x, x.y, x.z, x.w};
        float f[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(u[i] << 16);
            f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
        float mn = f[0], mx = f[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) {
            mn = fminf(mn, f[i]);
            mx = fmaxf(mx, f[i]);
        }
        mn = fminf(mn, dpp<0xB1>(mn)); mx = fmaxf(mx, dpp<0xB1>(mx));   // the four lanes of a group
        mn = fminf(mn, dpp<0x4E>(mn)); mx = fmaxf(mx, dpp<0x4E>(mx));
        const Grid g = grid_of(mn, mx, bits == 4 ? 15.0f : 3.0f);
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            o[i] = bits ? back(g, f[2 * i]) | back(g, f[2 * i + 1]) << 16 : half_bits(f[2 * i]) | half_bits(f[2 * i + 1]) << 16;
        store_once(reinterpret_cast<uint4 *>(a.out[which] + row * kHeadDim) + part, make_uint4(o[0], o[1], o[2], o[3]));
        return;
    }
    // keys per channel: a wavefront takes a block of 32 tokens of a head, lane (i, part) its tokens i, 4 + i, .. and channels 8 part ..
    const int64_t unit = (int64_t)(block - 2 * a.row_groups) * 4 + (threadIdx.x >> 6);
    if (unit >= (int64_t)a.n_blocks * a.n_heads) return;
    const int number = (int)(unit / a.n_heads), head = (int)(unit - (int64_t)number * a.n_heads);
    const int lane = threadIdx.x & 63, part = lane & 15, i0 = lane >> 4;
    int token[8];
    bool ok = true;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        token[k] = a.blocks[(int64_t)number * kGroup + 4 * k + i0];
        const bool in = token[k] >= 0 && token[k] < a.n_tokens;
        if (!in) token[k] = 0;
        ok = ok && in && a.tag_bits[token[k]] == 2;
    }
    if (!__all(ok)) {
        if (a.status && lane == 0) atomicOr(a.status, TKV_STATUS_BLOCK_PARTIAL);
        return;
    }
    uint4 x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = reinterpret_cast<const uint4 *>(a.in[0] + token[k] * a.stride[0] + (int64_t)head * kHeadDim)[part];
    Grid g[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        float mn = INFINITY, mx = -INFINITY;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t u = c < 2 ? x[k].x : c < 4 ? x[k].y : c < 6 ? x[k].z : x[k].w;
            const float f = __uint_as_float(c & 1 ? u & 0xffff0000u : u << 16);
            mn = fminf(mn, f);
            mx = fmaxf(mx, f);
        }
        mn = fminf(mn, __shfl_xor(mn, 16)); mx = fmaxf(mx, __shfl_xor(mx, 16));
        mn = fminf(mn, __shfl_xor(mn, 32)); mx = fmaxf(mx, __shfl_xor(mx, 32));
        g[c] = grid_of(mn, mx, 3.0f);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint32_t u[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            o[i] = back(g[2 * i], __uint_as_float(u[i] << 16)) | back(g[2 * i + 1], __uint_as_float(u[i] & 0xffff0000u)) << 16;
        store_once(reinterpret_cast<uint4 *>(a.out[0] + ((int64_t)token[k] * a.n_heads + head) * kHeadDim) + part, make_uint4(o[0], o[1], o[2], o[3]));
    }
}

// ------------------------------------------------------------------ distortion
struct DistortionArgs {
    const void *a, *b;
    const int32_t *seq_indptr;
    double *out, *partial;
    int32_t batch, n_tokens, n_heads;
};
constexpr int kChunk = kDistortionChunk;   // tokens whose squares a workgroup adds up

// The sequence's slots among the partial sums begin at first / kChunk + b: chunks of a sequence begin at its first token, and
// ceil(n / kChunk) of them end before the next one's begin.
__device__ __forceinline__ int first_slot(int first, int b) { return first / kChunk + b; }

__device__ __forceinline__ float f32_of(uint32_t bits, int type) { return type == TKV_BF16 ? __uint_as_float(bits << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)bits); }

template <int TYPE>
__global__ __launch_bounds__(256) void tkv_distortion_kernel(DistortionArgs a)
{
    __shared__ int whose;
    const uint32_t slot = blockIdx.x + blockIdx.y * gridDim.x;
    // the last sequence whose slots begin at or before this one
    if (threadIdx.x == 0) whose = -1;
    __syncthreads();
    for (int b = threadIdx.x; b < a.batch; b += 256) {
        const int lo = a.seq_indptr[b], hi = a.seq_indptr[b + 1];
        if (lo >= 0 && hi >= lo && hi <= a.n_tokens && (uint32_t)first_slot(lo, b) <= slot && slot < (uint32_t)first_slot(lo, b) + (uint32_t)((hi - lo + kChunk - 1) / kChunk)) whose = b;
    }
    __syncthreads();
    const int b = whose;
    if (b < 0) return;
    const int lo = a.seq_indptr[b], hi = a.seq_indptr[b + 1];
    const int begin = lo + (int)(slot - first_slot(lo, b)) * kChunk, end = begin + kChunk < hi ? begin + kChunk : hi;
    constexpr int kPer = TYPE == TKV_FP32 ? 4 : 8, kLanes = kHeadDim / kPer;   // values of a 16-byte piece; lanes of a row
    const int part = threadIdx.x % kLanes;
    for (int head = threadIdx.x / kLanes; head < a.n_heads; head += 256 / kLanes) {
        double sum = 0.0;
        for (int t = begin; t < end; ++t) {
            const int64_t at = ((int64_t)t * a.n_heads + head) * kLanes + part;
            const uint4 x = reinterpret_cast<const uint4 *>(a.a)[at], y = reinterpret_cast<const uint4 *>(a.b)[at];
            const uint32_t u[4] = {x.x, x.y, x.z, x.w}, v[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (TYPE == TKV_FP32) {
                    const double d = (double)__uint_as_float(u[i]) - (double)__uint_as_float(v[i]);
                    sum = __builtin_fma(d, d, sum);
                } else {
#pragma unroll
                    for (int k = 0; k < 32; k += 16) {
                        const double d = (double)f32_of(u[i] >> k & 0xffffu, TYPE) - (double)f32_of(v[i] >> k & 0xffffu, TYPE);
                        sum = __builtin_fma(d, d, sum);
                    }
                }
            }
        }
#pragma unroll
        for (int k = kLanes / 2; k > 0; k >>= 1) sum += __shfl_xor(sum, k);
        if (part == 0) a.partial[(int64_t)slot * a.n_heads + head] = sum;
    }
}
// A wavefront adds up the slots of a sequence's head.
__global__ __launch_bounds__(256) void tkv_distortion_join_kernel(DistortionArgs a)
{
    const int64_t unit = ((int64_t)blockIdx.x + (int64_t)blockIdx.y * gridDim.x) * 4 + (threadIdx.x >> 6);
    if (unit >= (int64_t)a.batch * a.n_heads) return;
    const int b = (int)(unit / a.n_heads), head = (int)(unit - (int64_t)b * a.n_heads), lane = threadIdx.x & 63;
    const int lo = a.seq_indptr[b], hi = a.seq_indptr[b + 1];
    if (!(lo >= 0 && hi >= lo && hi <= a.n_tokens)) {
        if (lane == 0) a.out[unit] = __builtin_nan("");
        return;
    }
    const int n = (hi - lo + kChunk - 1) / kChunk;
    double sum = 0.0;
    for (int k = lane; k < n; k += 64) sum += a.partial[(int64_t)(first_slot(lo, b) + k) * a.n_heads + head];
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) sum += __shfl_xor(sum, k);
    if (lane == 0) a.out[unit] = hi > lo ? sum / ((double)(hi - lo) * kHeadDim) : 0.0;
}

constexpr int64_t kMaxX = 1 << 22;   // a grid has less than 2^32 threads in a dimension
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
    a.row_groups = (uint32_t)(((int64_t)n_tokens * a.n_heads + kRowsWg - 1) / kRowsWg);
    const int64_t groups = 2 * (int64_t)a.row_groups + ((int64_t)n_blocks * a.n_heads + 3) / 4;
    hipLaunchKernelGGL(tkv_rows_kernel, grid(groups), dim3(256), 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? TKV_OK : TKV_ERR_HIP;
}

int tkv_launch_distortion(const void *a_rows, const void *b_rows, int32_t type, const int32_t *seq_indptr, int32_t batch, int32_t n_tokens, int32_t n_heads,
                          double *out, void *workspace, void *stream)
{
    DistortionArgs a = {a_rows, b_rows, seq_indptr, out, (double *)workspace, batch, n_tokens, n_heads};
    const int64_t slots = n_tokens / kChunk + (int64_t)batch;
    auto *kernel = type == TKV_BF16 ? tkv_distortion_kernel<TKV_BF16> : type == TKV_FP16 ? tkv_distortion_kernel<TKV_FP16> : tkv_distortion_kernel<TKV_FP32>;
    hipLaunchKernelGGL(kernel, grid(slots), dim3(256), 0, (hipStream_t)stream, a);
    if (hipGetLastError() != hipSuccess) return TKV_ERR_HIP;
    hipLaunchKernelGGL(tkv_distortion_join_kernel, grid(((int64_t)batch * n_heads + 3) / 4), dim3(256), 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? TKV_OK : TKV_ERR_HIP;
}
