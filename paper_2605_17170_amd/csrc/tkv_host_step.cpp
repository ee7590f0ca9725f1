// Host side of what stands around append and decode in a step of a serving loop: the rotation table, the plan of shared
// prefixes, and argument validation in front of the launchers of tkv_rope.hip (norm and rotation), tkv_table.hip (page tables
// in device memory) and tkv_shared.hip (attention over shared prefixes).  Nothing here touches the GPU.
#include "tkv.h"
#include "tkv_internal.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

namespace {
constexpr int kHeadDim = 128, kGroup = 32, kPageTokens = 64;
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
        // the nearest multiple of four units, off by two at most, 2^-63 turns: the lowest two bits hold the axis
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

/* ---------------------------------------------------------------- D8: shared prefixes */

int32_t tkv_plan_shared_capacity(int32_t n_groups, int32_t n_members, int32_t target_cus)
{
    // a workgroup for a compute unit at most, or the workgroups for the rows of every group: up to eight rows a member, at least 16 a workgroup
    const int64_t n = n_groups + (int64_t)target_cus + ((int64_t)n_members + 1) / 2;
    return n_groups < 0 || n_members < 0 || target_cus < 1 || n > INT32_MAX ? (int32_t)TKV_ERR_INVALID_ARG : (int32_t)n;
}

int32_t tkv_plan_decode_shared(const tkv_desc *desc, int32_t batch, int32_t n_q_heads, int32_t n_groups, const int32_t *n_tok_int2,
                               const int32_t *n_tok_int4, const int32_t *member_indptr, const int32_t *member_seqs, int32_t target_cus,
                               int32_t n_own_items, int32_t *items_out, int32_t capacity, int32_t *member_slots_out, int32_t *seq_slot_indptr_out,
                               int32_t *tile_rows_out)
{
    if (int st = tkv_desc_status(desc)) return st;
    if (batch < 0 || n_groups < 0 || n_own_items < 0 || capacity < 0 || n_q_heads <= 0 || !seq_slot_indptr_out || !tile_rows_out || !member_indptr) return TKV_ERR_INVALID_ARG;
    if (tkv_plan_shared_capacity(n_groups, 0, target_cus) < 0) return TKV_ERR_INVALID_ARG;
    if (n_groups > 0 && (!n_tok_int2 || !n_tok_int4)) return TKV_ERR_INVALID_ARG;
    if (n_q_heads % desc->n_kv_heads) return TKV_ERR_BAD_SHAPE;
    const int32_t r = n_q_heads / desc->n_kv_heads;
    if (r != 1 && r != 2 && r != 4 && r != 8) return TKV_ERR_BAD_SHAPE;
    if (member_indptr[0] != 0) return TKV_ERR_INVALID_ARG;
    int32_t largest = 0;
    for (int32_t g = 0; g < n_groups; ++g) {
        const int64_t members = (int64_t)member_indptr[g + 1] - member_indptr[g];
        if (members < 0 || members > batch || n_tok_int2[g] < 0 || n_tok_int4[g] < 0) return TKV_ERR_INVALID_ARG;
        if (desc->int2_key_axis == TKV_KEYS_PER_CHANNEL && n_tok_int2[g] % kGroup) return TKV_ERR_INVALID_ARG;
        largest = std::max(largest, (int32_t)members);
    }
    const int32_t n_members = member_indptr[n_groups];
    if (n_members > 0 && (!member_seqs || !member_slots_out)) return TKV_ERR_INVALID_ARG;
    if (capacity > 0 && !items_out) return TKV_ERR_INVALID_ARG;
    if ((int64_t)largest * r > INT32_MAX) return TKV_ERR_INVALID_ARG;
    try {
        std::vector<int32_t> seen((size_t)batch, -1), next((size_t)batch + 1, 0);
        for (int32_t g = 0; g < n_groups; ++g)
            for (int32_t m = member_indptr[g]; m < member_indptr[g + 1]; ++m) {
                const int32_t b = member_seqs[m];
                if (b < 0 || b >= batch || seen[(size_t)b] == g) return TKV_ERR_INVALID_ARG;
                seen[(size_t)b] = g;
            }
        // The own items' workgroups (a wavefront for each item and kv head) are launched first.  Either the prefixes' fill the compute units
        // that are left, or all, and begin behind them.
        const int64_t own = std::min(((int64_t)n_own_items * desc->n_kv_heads + 7) / 8, (int64_t)target_cus), spare = target_cus - own;
        auto pages_of = [](int32_t n) { return ((int64_t)n + kPageTokens - 1) / kPageTokens; };
        auto pages = [&](int32_t g) { return pages_of(n_tok_int2[g]) + pages_of(n_tok_int4[g]); };
        // Rows of a workgroup.  With 16 its wavefronts work on a page each, eight a step; with 64 and 128 they expand pages together, two
        // a step.  us of a call, 16 / 64 / 128 rows, 8 kv heads of 8 query heads: 4 sequences over 4000 tokens 11.7 / 12.4 / 14.7, 16000
        // 18.3 / 17.8 / 22.1; 8 over 1000 11.3 / 11.8 / 13.1, 16000 24.8 / 21.2 / 24.9; 16 over 1000 12.4 / 13.5 / 15.7, 4000 20.2 / 17.3 / 20.8,
        // 16000 39.7 / 27.2 / 29.8, 32000 72.4 / 42.4 / 39.7; 32 over 1000 16.1 / 15.4 / 18.2, 16000 61.3 / 42.4 / 40.9: about 3.2, 1.9 and
        // 2.8 us a step, and 2 and 5.5 more than with 16 rows once.  (Steps of a workgroup: those of all, over the compute units.)
        static const struct { int32_t rows, pages; double begin, step; } kinds[3] = {{16, 8, 0.0, 3.2}, {64, 2, 2.0, 1.9}, {128, 2, 5.5, 2.8}};
        int32_t rows = 0;
        int64_t unit = 1, target = target_cus;
        double least = 0.0;
        for (const auto &k : kinds) {
            int64_t all = 0;
            for (int32_t g = 0; g < n_groups; ++g)
                all += (pages(g) + k.pages - 1) / k.pages * (((int64_t)(member_indptr[g + 1] - member_indptr[g]) * r + k.rows - 1) / k.rows) * desc->n_kv_heads;
            // 6 us later, if own items come first on the same compute units
            const double with_own = spare > 0 ? k.step * (double)((all + spare - 1) / spare) : INFINITY;
            const double behind = k.step * (double)((all + target_cus - 1) / target_cus) + (own > 0 ? 6.0 : 0.0);
            const double time = k.begin + std::min(with_own, behind);
            if (rows == 0 || time < least) {
                rows = k.rows;
                unit = k.pages;
                target = with_own <= behind ? spare : target_cus;
                least = time;
            }
        }
        *tile_rows_out = rows;
        auto row_blocks = [&](int32_t g) { return ((int64_t)(member_indptr[g + 1] - member_indptr[g]) * r + rows - 1) / rows; };
        // Steps of a group, of either width by themselves or of the whole list.
        auto units = [&](int32_t g, int w, bool split) -> int64_t {
            const int64_t p2 = pages_of(n_tok_int2[g]), p4 = pages_of(n_tok_int4[g]), n = split ? (w ? p4 : p2) : (w ? 0 : p2 + p4);
            return member_indptr[g + 1] == member_indptr[g] ? 0 : (n + unit - 1) / unit;
        };
        // The fewest steps of an item with which the workgroups fit.
        auto shortest = [&](bool split) {
            int64_t lo = 1, hi = 1;
            for (int32_t g = 0; g < n_groups; ++g) hi = std::max({hi, units(g, 0, split), units(g, 1, split)});
            while (lo < hi) {
                const int64_t mid = lo + (hi - lo) / 2;
                int64_t n = 0;
                for (int32_t g = 0; g < n_groups; ++g)
                    n += ((units(g, 0, split) + mid - 1) / mid + (units(g, 1, split) + mid - 1) / mid) * row_blocks(g) * desc->n_kv_heads;
                if (n <= target) hi = mid;
                else lo = mid + 1;
            }
            return lo;
        };
        // An item with pages of both widths begins twice, which takes about as long as a step; parts of one width each may be longer, or more
        // than the target has compute units for.
        const int64_t whole = shortest(false), apart = shortest(true);
        bool split = apart <= whole + 1;
        if (split) {
            int64_t n = 0;
            for (int32_t g = 0; g < n_groups; ++g)
                n += ((units(g, 0, true) + apart - 1) / apart + (units(g, 1, true) + apart - 1) / apart) * row_blocks(g) * desc->n_kv_heads;
            split = n <= target;
        }
        const int64_t most = split ? apart : whole;
        int64_t n_items = 0, n_slots = n_own_items;
        std::vector<int32_t> parts((size_t)n_groups, 0);
        for (int32_t g = 0; g < n_groups; ++g) {
            int64_t n = 0;   // parts so far
            for (int w = 0; w < 2; ++w) {
                const int64_t all = units(g, w, split), count = (all + most - 1) / most;
                const int64_t begin = w ? pages_of(n_tok_int2[g]) : 0, end = split && w == 0 ? pages_of(n_tok_int2[g]) : pages(g);
                if (n_items + count * row_blocks(g) > capacity) return TKV_ERR_CAPACITY;
                // workgroups of the same pages follow one another: with eight kv heads they lie on one XCD, whose L2 they share
                for (int64_t k = 0; k < count; ++k)
                    for (int64_t z = 0; z < row_blocks(g); ++z) {
                        int32_t *it = items_out + 5 * n_items++;
                        it[0] = g;
                        it[1] = (int32_t)(begin + unit * (all * k / count));
                        it[2] = (int32_t)std::min(end, begin + unit * (all * (k + 1) / count));
                        it[3] = (int32_t)(n + k);
                        it[4] = (int32_t)(rows * z);
                    }
                n += count;
            }
            parts[(size_t)g] = (int32_t)n;
            for (int32_t m = member_indptr[g]; m < member_indptr[g + 1]; ++m) next[(size_t)member_seqs[m]] += (int32_t)n;
            n_slots += n * (member_indptr[g + 1] - member_indptr[g]);
            if (n_slots > INT32_MAX) return TKV_ERR_INVALID_ARG;
        }
        int32_t at = n_own_items;
        for (int32_t b = 0; b < batch; ++b) {
            seq_slot_indptr_out[b] = at;
            const int32_t n = next[(size_t)b];
            next[(size_t)b] = at;
            at += n;
        }
        seq_slot_indptr_out[batch] = at;
        for (int32_t g = 0; g < n_groups; ++g)
            for (int32_t m = member_indptr[g]; m < member_indptr[g + 1]; ++m) {
                int32_t &slot = next[(size_t)member_seqs[m]];
                member_slots_out[m] = slot;
                slot += parts[(size_t)g];
            }
        return (int32_t)n_items;
    } catch (const std::bad_alloc &) {
        return TKV_ERR_INVALID_ARG;
    }
}

int tkv_decode_attention_shared(const tkv_desc *desc, const void *pool, const uint8_t *bit_map, const void *q, const int32_t *page_indptr,
                                const int32_t *page_ids, const int32_t *n_tok_int2, const int32_t *n_tok_int4, const int32_t *items,
                                int32_t n_items, const tkv_prefix *prefix, const int32_t *slot_indptr, int32_t n_slots, int32_t batch,
                                int32_t n_q_heads, float sm_scale, void *out, void *workspace, size_t workspace_bytes, int32_t *status,
                                void *stream)
{
    if (!prefix || n_items < 0 || n_slots < n_items) return tkv_desc_status(desc) ? tkv_desc_status(desc) : TKV_ERR_INVALID_ARG;
    if (int st = tkv_decode_check_args(desc, n_slots, batch, n_q_heads, workspace, workspace_bytes)) return st;
    const tkv_prefix &p = *prefix;
    if (p.n_groups < 0 || p.n_members < 0 || p.n_items < 0) return TKV_ERR_INVALID_ARG;
    if (batch == 0) return TKV_OK;
    if (!(sm_scale > 0.0f) || !(sm_scale < 3.0e38f)) return TKV_ERR_INVALID_ARG;
    if (!q || !out || !slot_indptr) return TKV_ERR_INVALID_ARG;
    if ((n_items > 0 || p.n_items > 0) && (!pool || !bit_map)) return TKV_ERR_INVALID_ARG;
    if (n_items > 0 && (!page_indptr || !page_ids || !n_tok_int2 || !n_tok_int4 || !items)) return TKV_ERR_INVALID_ARG;
    if (((uintptr_t)pool & 255) || ((uintptr_t)q & 15) || ((uintptr_t)out & 15)) return TKV_ERR_INVALID_ARG;
    const int32_t r = n_q_heads / desc->n_kv_heads;
    if (p.n_items > 0) {
        if (!p.page_indptr || !p.page_ids || !p.n_tok_int2 || !p.n_tok_int4 || !p.member_indptr || !p.member_seqs || !p.member_slots || !p.items ||
            p.n_groups == 0 || p.n_members == 0)
            return TKV_ERR_INVALID_ARG;
        if (p.tile_rows != 16 && p.tile_rows != 64 && p.tile_rows != 128) return TKV_ERR_INVALID_ARG;
        if ((int64_t)p.n_members * r > INT32_MAX / 2 || (int64_t)p.n_items * desc->n_kv_heads > INT32_MAX / 2) return TKV_ERR_INVALID_ARG;
    }
    return tkv_launch_shared(desc, pool, bit_map, q, page_indptr, page_ids, n_tok_int2, n_tok_int4, items, n_items, prefix, slot_indptr, n_slots,
                             batch, n_q_heads, sm_scale, out, workspace, status, stream);
}

} // extern "C"
