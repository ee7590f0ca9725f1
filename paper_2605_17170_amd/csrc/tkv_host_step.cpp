// Host side of what stands around append and decode in a step of a serving loop: the rotation table, and argument validation
// in front of the launchers of tkv_rope.hip (norm and rotation) and tkv_table.hip (page tables in device memory).  Nothing
// here touches the GPU.
#include "tkv.h"
#include "tkv_internal.h"

#include <algorithm>
#include <cmath>

namespace {
constexpr int kHeadDim = 128, kPageTokens = 64;
}

extern "C" {

/* ---------------------------------------------------------------- Q1 on the GPU: page tables in device memory */

namespace {
constexpr int32_t kMaxTableTokens = 1 << 28, kMaxTablePages = 1 << 24;
int table_status(const tkv_desc *desc, const tkv_table *t)
{
    if (int st = tkv_desc_status(desc)) return st;
    if (!t || t->n_seqs < 0 || t->max_pages < 0 || t->max_pages > kMaxTablePages || (int64_t)t->n_seqs * t->max_pages > INT32_MAX) return TKV_ERR_INVALID_ARG;
    if (!t->n_free || (desc->n_pages_int2 + desc->n_pages_int4 > 0 && !t->free_pages)) return TKV_ERR_INVALID_ARG;
    if (t->n_seqs > 0 && (!t->n_tok_int2 || !t->n_tok_int4 || (t->max_pages > 0 && !t->page_ids))) return TKV_ERR_INVALID_ARG;
    const uintptr_t all = (uintptr_t)t->page_ids | (uintptr_t)t->n_tok_int2 | (uintptr_t)t->n_tok_int4 | (uintptr_t)t->free_pages | (uintptr_t)t->n_free;
    return all & 3 ? TKV_ERR_INVALID_ARG : TKV_OK;
}
} // namespace

int tkv_table_reset(const tkv_desc *desc, const tkv_table *table, void *stream)
{
    if (int st = table_status(desc, table)) return st;
    return tkv_launch_table_reset(desc, table, stream);
}

int32_t tkv_table_max_work(int32_t n_seqs, int32_t n_tokens)
{
    if (n_seqs < 0 || n_tokens < 0 || n_tokens > kMaxTableTokens) return TKV_ERR_INVALID_ARG;
    // n tokens of a sequence touch at most n pages, and at most n / 64 + 4 (tkv_plan_append_max_work)
    return (int32_t)std::min<int64_t>(n_tokens, n_tokens / kPageTokens + 4 * (int64_t)std::min(n_seqs, n_tokens));
}

size_t tkv_table_workspace_bytes(int32_t n_seqs, int32_t n_tokens)
{
    if (n_seqs < 0 || n_tokens < 0 || n_tokens > kMaxTableTokens) return 0;
    return 4 * tkv_table_words(n_seqs, n_tokens);
}

int tkv_table_append(const tkv_desc *desc, const tkv_table *table, const int32_t *keep_int2, const int32_t *keep_int4,
                     const int32_t *n_new, const uint8_t *tag_bits, int32_t n_tokens, int32_t *token_indptr, int32_t *positions,
                     int32_t *slot_ids, int32_t *work_pages, int32_t *work_src, int32_t max_work, int32_t *n_work,
                     void *workspace, size_t workspace_bytes, int32_t *status, void *stream)
{
    if (int st = table_status(desc, table)) return st;
    if (n_tokens < 0 || n_tokens > kMaxTableTokens || max_work < 0 || max_work > kMaxTableTokens) return TKV_ERR_INVALID_ARG;
    if ((n_tokens > 0 && !tag_bits) || (max_work > 0 && (!work_pages || !work_src)) || !n_work || !workspace) return TKV_ERR_INVALID_ARG;
    const uintptr_t words = (uintptr_t)keep_int2 | (uintptr_t)keep_int4 | (uintptr_t)n_new | (uintptr_t)token_indptr | (uintptr_t)positions |
                            (uintptr_t)slot_ids | (uintptr_t)work_pages | (uintptr_t)work_src | (uintptr_t)n_work | (uintptr_t)status;
    if ((words & 3) || ((uintptr_t)workspace & 15)) return TKV_ERR_INVALID_ARG;
    if (workspace_bytes < tkv_table_workspace_bytes(table->n_seqs, n_tokens)) return TKV_ERR_WORKSPACE_TOO_SMALL;
    return tkv_launch_table_append(desc, table, keep_int2, keep_int4, n_new, tag_bits, n_tokens, token_indptr, positions, slot_ids, work_pages,
                                   work_src, max_work, n_work, workspace, status, stream);
}

/* ---------------------------------------------------------------- R1: rotation table, norm and rotation */

int tkv_rope_table(int32_t rotary_dim, int32_t n_axes, const int32_t *sections, int32_t interleaved, double theta,
                   const double *inv_freq, uint64_t *table_out)
{
    if (rotary_dim < 0 || rotary_dim > kHeadDim || rotary_dim % 16 || n_axes < 1 || n_axes > 4) return TKV_ERR_BAD_SHAPE;
    if (interleaved != 0 && interleaved != 1) return TKV_ERR_INVALID_ARG;
    const int32_t pairs = rotary_dim / 2;
    if (pairs == 0) return TKV_OK;
    if (!table_out || (!sections && n_axes > 1)) return TKV_ERR_INVALID_ARG;
    if (!inv_freq && !(theta > 0.0 && std::isfinite(theta))) return TKV_ERR_INVALID_ARG;
    const int32_t all[1] = {pairs};
    if (!sections) sections = all;
    int64_t sum = 0;
    for (int32_t k = 0; k < n_axes; ++k) {
        if (sections[k] < 0) return TKV_ERR_BAD_SHAPE;
        if (interleaved && k > 0 && sections[k] > (pairs - k + n_axes - 1) / n_axes) return TKV_ERR_BAD_SHAPE;   // more than its turns
        sum += sections[k];
    }
    if (sum != pairs) return TKV_ERR_BAD_SHAPE;
    for (int32_t i = 0; inv_freq && i < pairs; ++i)
        if (!std::isfinite(inv_freq[i])) return TKV_ERR_INVALID_ARG;
    int32_t axis = 0, end = sections[0];
    for (int32_t i = 0; i < pairs; ++i) {
        if (interleaved) {
            axis = i % n_axes;
            if (i / n_axes >= sections[axis]) axis = 0;
        } else {
            while (i >= end) end += sections[++axis];
        }
        const long double f = inv_freq ? (long double)inv_freq[i] : std::pow((long double)theta, -2.0L * i / rotary_dim);
        long double turns = f / 6.283185307179586476925286766559005768L;
        turns -= std::floor(turns);
        // the lowest two bits hold the axis: 2^-63 turns at most, times a position
        const long double units = turns * 18446744073709551616.0L;
        const uint64_t word = units >= 18446744073709551614.0L ? 0 : ((uint64_t)units + 2) & ~(uint64_t)3;
        table_out[i] = word | (uint64_t)axis;
    }
    return TKV_OK;
}

int tkv_norm_rope(const tkv_rope *rope, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                  int32_t n_tokens, int32_t n_q_heads, int32_t n_kv_heads, const int32_t *positions, const void *q_weight,
                  const void *k_weight, float eps, void *q_out, void *k_out, void *v_out, void *stream)
{
    if (!rope) return TKV_ERR_INVALID_ARG;
    if (rope->rotary_dim < 0 || rope->rotary_dim > kHeadDim || rope->rotary_dim % 16 || rope->n_axes < 1 || rope->n_axes > 4) return TKV_ERR_BAD_SHAPE;
    if ((rope->adjacent != 0 && rope->adjacent != 1) || !std::isfinite(rope->scale)) return TKV_ERR_INVALID_ARG;
    if (n_tokens < 0 || n_q_heads < 0 || n_kv_heads < 0 || !(eps >= 0.0f) || !std::isfinite(eps)) return TKV_ERR_INVALID_ARG;
    const int64_t heads = (int64_t)n_q_heads + (int64_t)n_kv_heads * (v ? 2 : 1);
    if (n_tokens == 0 || heads == 0) return TKV_OK;
    if (heads > INT32_MAX - 4096 || (int64_t)n_tokens * heads > INT32_MAX - 4096) return TKV_ERR_INVALID_ARG;
    if (rope->rotary_dim > 0 && (!rope->table || !positions || ((uintptr_t)rope->table & 7))) return TKV_ERR_INVALID_ARG;
    auto tensor_ok = [&](const void *in, int64_t stride, const void *out, int32_t n) {
        return in && out && !((uintptr_t)in & 15) && !((uintptr_t)out & 15) && stride % 8 == 0 && (stride >= (int64_t)n * kHeadDim || n_tokens == 1) &&
               stride >= 0 && (in != out || stride == (int64_t)n * kHeadDim || n_tokens == 1);
    };
    if (n_q_heads > 0 && !tensor_ok(q, q_stride, q_out, n_q_heads)) return TKV_ERR_INVALID_ARG;
    if (n_kv_heads > 0 && !tensor_ok(k, k_stride, k_out, n_kv_heads)) return TKV_ERR_INVALID_ARG;
    if (n_kv_heads > 0 && v && !tensor_ok(v, v_stride, v_out, n_kv_heads)) return TKV_ERR_INVALID_ARG;
    if (((uintptr_t)q_weight & 15) || ((uintptr_t)k_weight & 15)) return TKV_ERR_INVALID_ARG;
    return tkv_launch_norm_rope(rope, q, q_stride, k, k_stride, n_kv_heads > 0 ? v : nullptr, v_stride, n_tokens, n_q_heads, n_kv_heads, positions, q_weight, k_weight,
                                eps, q_out, k_out, v_out, stream);
}

} // extern "C"
