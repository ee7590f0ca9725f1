// tkv_norm_rope: what stands between the projections and the cache.  Queries and keys get their RMS norm per head and
// the rotation to their positions (on one to four axes) in one pass; the values of a packed projection move to rows of
// their own in the same launch.  (The paper's path takes K with positions encoded, Sec. 3.2.3.)
//
//   y = x * rsqrt(mean(x^2) + eps) * w              over the 128 channels of a head
//   (a, b) -> (a cos - b sin, a sin + b cos) * scale   for the pair (a, b) of frequency i, angle = position * f_i
//
// Eight lanes own a row (one head of one token), two 16-byte pieces each, so that an instruction of a wavefront moves
// eight whole 128-byte lines, and the pieces are chosen so that both channels of a pair lie in one lane: of paired halves
// piece l and piece l + rotary_dim / 16, of adjacent pairs pieces l and l + 8.  No row goes through LDS; the norm is three
// DPP steps.  A workgroup takes 32 consecutive rows, and while they are under way its threads turn the angles of the tokens
// that these belong to (one to three, with 16 heads or more) into cosines and sines in LDS, one frequency a thread.  (With the
// angles computed by each lane for its own pairs, and walks over many rows to make up for it, 48 heads of 2501 tokens took
// 20.9 us, and 80 of 16384 136; two and four rows a lane, all asked for at first, are no faster.)
//
// Angles: f_i / 2 pi is held as a fraction of a turn in 64 bits (tkv_rope_table), of which the lowest two hold the axis and
// count as zero here.  Position times fraction modulo 2^64 is exact but for the table's rounding (2^-63 turns a position), and rounded
// to 32 bits (2^-33 turns): the angle to 1.5 * 2^-32 turns at any position, and one of zero where the frequency is.
// Sine and cosine of the remainder in [-pi/4, pi/4] are Taylor polynomials of degree 9 and 8 (off by 2e-9 and 3e-8).
// Everything is 32 bits until the one rounding to bf16.
//
// What bounds it: HBM (every value read and written once) for prompts: 671 MB of 16384 tokens of 80 heads in 108 us, 6.2 TB/s;
// 61 MB of 2501 tokens in 11.7 us, 5.3 TB/s.  For a few tokens the launch: 32 tokens take 4.4 us, as an empty kernel does.
#include <hip/hip_runtime.h>

#include "tkv_internal.h"
#include "tkv_layout.h"

namespace {

using namespace tkv;

struct RopeArgs {
    const uint64_t *table;
    const int32_t *positions;
    const uint16_t *in[3];      // q, k, v
    const uint16_t *weight[2];  // of q and k; null: no norm
    uint16_t *out[3];
    int64_t stride[3];          // from token to token of the inputs, in elements
    int32_t heads[3];
    int32_t n_tokens;
    int32_t n_rows;
    int32_t rotary_dim;
    int32_t n_axes;
    float scale;
    float eps;
};

__device__ __forceinline__ float lo_f32(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float hi_f32(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b)   // nearest even
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
}
template <int CTRL> __device__ __forceinline__ float dpp(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// Cosine and sine of `turns` * 2^-32 turns.
__device__ __forceinline__ void cos_sin(uint32_t turns, float &c, float &s)
{
    const uint32_t quarter = (turns + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(turns - (quarter << 30)) * 1.46291807926715968e-9f;   // 2 pi / 2^32
    const float x2 = x * x;
    const float sn = fmaf(x * x2, fmaf(x2, fmaf(x2, fmaf(x2, 1.0f / 362880.0f, -1.0f / 5040.0f), 1.0f / 120.0f), -1.0f / 6.0f), x);
    const float cn = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, 1.0f / 40320.0f, -1.0f / 720.0f), 1.0f / 24.0f), -0.5f), 1.0f);
    const float cv = (quarter & 1) ? sn : cn, sv = (quarter & 1) ? cn : sn;
    c = __uint_as_float(__float_as_uint(cv) ^ (((quarter + 1) & 2) << 30));
    s = __uint_as_float(__float_as_uint(sv) ^ ((quarter & 2) << 30));
}

// Past the caches' usual order: the outputs are written once and read by other kernels, on other XCDs as a rule.
__device__ __forceinline__ void store_once(uint4 *to, uint32_t x, uint32_t y, uint32_t z, uint32_t w)
{
    typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
    __builtin_nontemporal_store(uint4v{x, y, z, w}, reinterpret_cast<uint4v *>(to));
}

constexpr int kRopeRows = 32;   // of a workgroup
struct alignas(16) Trig {   // of a token's angles, four frequencies each
    float4 c[16], s[16];
};
template <bool ADJACENT>
__global__ __launch_bounds__(256) void tkv_norm_rope_kernel(RopeArgs a)
{
    extern __shared__ Trig trig[];   // of the workgroup's tokens
    const int l = threadIdx.x & 7;
    const int rows = a.heads[0] + a.heads[1] + a.heads[2], half = a.rotary_dim >> 1;
    const int first = (int)((blockIdx.x + blockIdx.y * gridDim.x) * kRopeRows);
    if (first >= a.n_rows) return;
    const int end = a.n_rows - first < kRopeRows ? a.n_rows : first + kRopeRows;
    const int token0 = first / rows, head0 = first - token0 * rows;

    // angles: thread i has frequency i % 64 of every fourth token
    const int f = threadIdx.x & 63, n_tokens = (end - 1) / rows - token0 + 1;
    uint64_t turn = 0;
    int32_t pos[4] = {};
    auto load_pos = [&](int t) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < a.n_axes) pos[k] = a.positions[(int64_t)k * a.n_tokens + token0 + t];
    };
    int t = threadIdx.x >> 6;
    const bool turns = f < half;
    if (turns && t < n_tokens) {
        turn = a.table[f];
        load_pos(t);
    }

    // this lane's pieces of a row and its eight pairs: channels k of piece 0 and of piece 1, or 2k and 2k + 1 of either
    const int lead = a.rotary_dim >> 4;   // pieces of a half
    const int p0 = ADJACENT || l < lead ? l : 2 * l, p1 = ADJACENT ? l + 8 : (l < lead ? l + lead : 2 * l + 1);
    uint4 w[2][2] = {};
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (a.weight[k]) {
            w[k][0] = reinterpret_cast<const uint4 *>(a.weight[k])[p0];
            w[k][1] = reinterpret_cast<const uint4 *>(a.weight[k])[p1];
        }
    // (below 32 rows a token the quotient is 1 / 64 from the next integer at least, and off by 2^-17)
    const int at = threadIdx.x >> 3, of_token = rows >= kRopeRows ? (head0 + at >= rows ? 1 : 0)
                                                                  : (int)(((float)(head0 + at) + 0.5f) * __builtin_amdgcn_rcpf((float)rows));
    const int head = head0 + at - of_token * rows;
    const bool live = first + at < end;
    const int kind = head >= a.heads[0] + a.heads[1] ? 2 : (head >= a.heads[0] ? 1 : 0);
    const int h = head - (kind > 0 ? a.heads[0] : 0) - (kind > 1 ? a.heads[1] : 0);
    uint4 x[2] = {};
    if (live) {
        const uint16_t *base = kind == 0 ? a.in[0] : (kind == 1 ? a.in[1] : a.in[2]);
        const int64_t stride = kind == 0 ? a.stride[0] : (kind == 1 ? a.stride[1] : a.stride[2]);
        const uint4 *src = reinterpret_cast<const uint4 *>(base + (token0 + of_token) * stride + (int64_t)h * kHeadDim);
        x[0] = src[p0];
        x[1] = src[p1];
    }
    if (half > 0) {
        // paired halves: pairs 8l ..., two pieces of four frequencies, which lie eight pieces apart
        const int place = ADJACENT ? f : 4 * ((f >> 2 & 1) * 8 + (f >> 3)) + (f & 3);
        while (t < n_tokens) {
            float c = 1.0f, s = 0.0f;
            if (turns) {
                const int axis = (int)turn & 3;
                const int32_t p = (axis & 2) ? ((axis & 1) ? pos[3] : pos[2]) : ((axis & 1) ? pos[1] : pos[0]);
                cos_sin((uint32_t)((uint64_t)(int64_t)p * (turn & ~(uint64_t)3) + 0x80000000u >> 32), c, s);
                c *= a.scale;
                s *= a.scale;
            }
            reinterpret_cast<float *>(trig[t].c)[place] = c;
            reinterpret_cast<float *>(trig[t].s)[place] = s;
            t += 4;
            if (turns && t < n_tokens) load_pos(t);
        }
        __syncthreads();
    }
    if (!live) return;
    const uint32_t d[8] = {x[0].x, x[0].y, x[0].z, x[0].w, x[1].x, x[1].y, x[1].z, x[1].w};
    float v[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[2 * i] = lo_f32(d[i]);
        v[2 * i + 1] = hi_f32(d[i]);
    }
    const bool normed = kind == 0 ? a.weight[0] != nullptr : a.weight[1] != nullptr;
    if (normed) {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum = fmaf(v[i], v[i], sum);
        sum += dpp<0xB1>(sum);    // neighbours, pairs, halves of the eight lanes
        sum += dpp<0x4E>(sum);
        sum += dpp<0x141>(sum);
        const float r = __builtin_amdgcn_rsqf(fmaf(sum, 1.0f / kHeadDim, a.eps));
        const uint4 w0 = kind == 0 ? w[0][0] : w[1][0], w1 = kind == 0 ? w[0][1] : w[1][1];
        const uint32_t wd[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[2 * i] = v[2 * i] * r * lo_f32(wd[i]);
            v[2 * i + 1] = v[2 * i + 1] * r * hi_f32(wd[i]);
        }
    }
    if (half > 0) {
        const Trig &of = trig[of_token];
        const float4 c4[2] = {of.c[l], of.c[l + 8]}, s4[2] = {of.s[l], of.s[l + 8]};
        const float c[8] = {c4[0].x, c4[0].y, c4[0].z, c4[0].w, c4[1].x, c4[1].y, c4[1].z, c4[1].w};
        const float s[8] = {s4[0].x, s4[0].y, s4[0].z, s4[0].w, s4[1].x, s4[1].y, s4[1].z, s4[1].w};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i0 = ADJACENT ? 2 * j : j, i1 = ADJACENT ? 2 * j + 1 : j + 8;
            const bool turned = (ADJACENT ? 4 * (l + 2 * (j & 4)) + (j & 3) : 8 * l + j) < half;   // NaN and infinities of the others stay as they are
            const float p = v[i0], q = v[i1];
            v[i0] = turned ? fmaf(p, c[j], -(q * s[j])) : p;
            v[i1] = turned ? fmaf(p, s[j], q * c[j]) : q;
        }
    }
    uint32_t o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = kind == 2 ? d[i] : pack_bf16(v[2 * i], v[2 * i + 1]);
    uint16_t *base = kind == 0 ? a.out[0] : (kind == 1 ? a.out[1] : a.out[2]);
    const int n = kind == 0 ? a.heads[0] : (kind == 1 ? a.heads[1] : a.heads[2]);
    uint4 *dst = reinterpret_cast<uint4 *>(base + ((int64_t)(token0 + of_token) * n + h) * kHeadDim);
    store_once(dst + p0, o[0], o[1], o[2], o[3]);
    store_once(dst + p1, o[4], o[5], o[6], o[7]);
}
} // namespace

int tkv_launch_norm_rope(const tkv_rope *rope, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v,
                         int64_t v_stride, int32_t n_tokens, int32_t n_q_heads, int32_t n_kv_heads, const int32_t *positions,
                         const void *q_weight, const void *k_weight, float eps, void *q_out, void *k_out, void *v_out, void *stream)
{
    const int32_t rows = n_q_heads + n_kv_heads * (v ? 2 : 1);
    RopeArgs a = {};
    a.table = rope->table;
    a.positions = positions;
    a.in[0] = (const uint16_t *)q; a.in[1] = (const uint16_t *)k; a.in[2] = (const uint16_t *)v;
    a.weight[0] = (const uint16_t *)q_weight; a.weight[1] = (const uint16_t *)k_weight;
    a.out[0] = (uint16_t *)q_out; a.out[1] = (uint16_t *)k_out; a.out[2] = (uint16_t *)v_out;
    a.stride[0] = q_stride; a.stride[1] = k_stride; a.stride[2] = v_stride;
    a.heads[0] = n_q_heads; a.heads[1] = n_kv_heads; a.heads[2] = v ? n_kv_heads : 0;
    a.n_tokens = n_tokens;
    a.n_rows = n_tokens * rows;
    a.rotary_dim = rope->rotary_dim;
    a.n_axes = rope->n_axes;
    a.scale = rope->scale;
    a.eps = eps;
    const int most = (kRopeRows + rows - 2) / rows + 1;   // tokens that a workgroup's rows can touch
    constexpr unsigned kMaxX = 1 << 23;   // a grid has less than 2^32 threads in a dimension
    const unsigned blocks = (unsigned)((a.n_rows + (int64_t)kRopeRows - 1) / kRopeRows);
    const dim3 grid(blocks < kMaxX ? blocks : kMaxX, (blocks + kMaxX - 1) / kMaxX);
    hipLaunchKernelGGL(rope->adjacent ? tkv_norm_rope_kernel<true> : tkv_norm_rope_kernel<false>, grid, dim3(256), (size_t)most * sizeof(Trig),
                       (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? TKV_OK : TKV_ERR_HIP;
}
