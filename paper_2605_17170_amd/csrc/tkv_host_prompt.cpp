// Host side of prompts and calibration: the plan of prompt attention, the blocks of per-channel keys, and argument validation in
// front of the launchers of tkv_prefill.hip and tkv_rows.hip.  Nothing here touches the GPU.
#include "tkv.h"
#include "tkv_internal.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

namespace {
constexpr int kHeadDim = 128, kGroup = 32;
constexpr int64_t kMaxStride = 1 << 23;

int group_of(const tkv_desc *desc, int32_t n_q_heads, int32_t &group)
{
    if (int st = tkv_desc_status(desc)) return st;
    if (n_q_heads <= 0) return TKV_ERR_INVALID_ARG;
    if (n_q_heads % desc->n_kv_heads) return TKV_ERR_BAD_SHAPE;
    group = n_q_heads / desc->n_kv_heads;
    return TKV_OK;
}
bool rows_ok(const void *p, int64_t stride, int64_t heads, int32_t n_tokens)
{
    return p && !((uintptr_t)p & 15) && stride >= 0 && stride % 8 == 0 && stride < kMaxStride && (stride >= heads * kHeadDim || n_tokens == 1);
}
// Sizes that the plan returns and the call takes.
bool heads_ok(const tkv_desc *desc) { return (int64_t)desc->n_kv_heads * kHeadDim < kMaxStride; }
bool tokens_ok(int64_t n_tokens, int32_t group) { return n_tokens * group <= INT32_MAX; }
bool items_ok(const tkv_desc *desc, int64_t n_items, int64_t n_cut, int32_t tile_rows)
{
    return n_items * desc->n_kv_heads <= INT32_MAX / 64 && n_cut <= n_items && n_cut * desc->n_kv_heads * tile_rows <= INT32_MAX;
}
int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }
// Workgroups of tkv_prefill_attention.  Times in us, fitted to 792 measured plans of 94 calls on rows that are not in the caches (1 to 64 sequences of 1 to 16384 tokens behind 0 to 100000,
// 1 to 8 key heads, groups of 1 to 8): the plan chosen is 0.6 % behind the best of a call's in the mean, 22 % at most.
struct Kind {
    int32_t rows, keys, resident;   // rows, keys of a tile, workgroups that a compute unit holds at once
    double begin, again;            // what a workgroup takes beside its steps: the first one of a place, those behind it
    double alone, step;             // a step (a tile of keys) of a workgroup by itself; steps of a full compute unit, one behind the other
};
constexpr Kind kKinds[3] = {{32, 32, 4, 4.5, 10.8, 0.70, 0.173}, {128, 64, 2, 6.0, 6.4, 0.96, 0.98}, {256, 64, 1, 6.0, 8.1, 1.32, 1.90}};
constexpr double kMergeUs = 3.1, kCrossUs = 2.0;   // a second launch; going on from a prefix to the new tokens
constexpr double kBytesPerUs = 6.1e6, kPartialBytesPerUs = 3.4e6;   // keys and values; partial results
bool kind_of(int32_t rows)
{
    for (const Kind &k : kKinds)
        if (k.rows == rows) return true;
    return false;
}
} // namespace

extern "C" {

/* ---------------------------------------------------------------- P2: attention of prompts */

int32_t tkv_plan_prefill_capacity(const tkv_desc *desc, int32_t batch, int32_t n_tokens, int32_t n_q_heads, int32_t target_cus)
{
    int32_t group = 0;
    if (int st = group_of(desc, n_q_heads, group)) return st;
    if (batch < 0 || n_tokens < 0 || target_cus < 1) return TKV_ERR_INVALID_ARG;
    // a tile of each sequence and kind of workgroup, and as many parts again as are resident at once
    const int64_t n = (int64_t)n_tokens * group / kKinds[0].rows + batch + 4 * (int64_t)target_cus;
    return n > INT32_MAX ? (int32_t)TKV_ERR_INVALID_ARG : (int32_t)n;
}

int32_t tkv_plan_prefill(const tkv_desc *desc, int32_t batch, int32_t n_q_heads, const int32_t *seq_indptr, const int32_t *prefix_indptr,
                         int32_t target_cus, int32_t *items_out, int32_t capacity, int32_t *tile_rows_out, int32_t *n_slots_out, int32_t *n_cut_out)
{
    int32_t group = 0;
    if (int st = group_of(desc, n_q_heads, group)) return st;
    if (batch < 0 || target_cus < 1 || capacity < 0 || !seq_indptr || !tile_rows_out || !n_slots_out || !n_cut_out || (capacity > 0 && !items_out)) return TKV_ERR_INVALID_ARG;
    if (seq_indptr[0] != 0 || (prefix_indptr && prefix_indptr[0] != 0)) return TKV_ERR_INVALID_ARG;
    for (int32_t b = 0; b < batch; ++b) {
        if (seq_indptr[b + 1] < seq_indptr[b] || (prefix_indptr && prefix_indptr[b + 1] < prefix_indptr[b])) return TKV_ERR_INVALID_ARG;
        if (((int64_t)seq_indptr[b + 1] - seq_indptr[b]) * group > 1 << 30) return TKV_ERR_INVALID_ARG;
    }
    if (!heads_ok(desc) || ((int64_t)n_q_heads * kHeadDim >= kMaxStride && seq_indptr[batch] > 1)) return TKV_ERR_BAD_SHAPE;   // the token stride of more
    if (!tokens_ok(seq_indptr[batch], group)) return TKV_ERR_INVALID_ARG;
    try {
        struct Tile { int32_t seq, row, keys, parts; };   // keys: tiles of keys that its rows see
        const Kind *best = nullptr;
        std::vector<Tile> tiles, mine;
        double least = 0.0;
        for (const Kind &kind : kKinds) {
            mine.clear();
            int64_t all = 0, longest = 0;
            double bytes = 0.0;
            bool crosses = false;
            for (int32_t b = 0; b < batch; ++b) {
                const int32_t n = seq_indptr[b + 1] - seq_indptr[b], pre = prefix_indptr ? prefix_indptr[b + 1] - prefix_indptr[b] : 0;
                const int64_t rows = (int64_t)n * group;
                crosses = crosses || (n > 0 && pre > 0);
                for (int64_t r = 0; r < rows; r += kind.rows) {
                    const int64_t see = (std::min(r + kind.rows, rows) - 1) / group + 1, keys = up(pre, kind.keys) + up(see, kind.keys);
                    mine.push_back({b, (int32_t)r, (int32_t)keys, 1});
                    all += keys;
                    longest = std::max(longest, keys);
                }
                // the first tile's keys and values come from memory, most of the next three tiles' from the caches (4 chunks of 16 tokens of 64 heads
                // behind 2000 to 6000 38.6 us with 32 rows, which the plan took without this, 33.8 with 128); 0.13 of the bytes for each, fitted with the constants above
                if (rows > 0) bytes += ((double)pre + n) * 4.0 * kHeadDim * (1.0 + 0.13 * std::min<double>(3.0, (double)(up(rows, kind.rows) - 1)));
            }
            if (mine.empty()) break;
            const double heads = desc->n_kv_heads, slots = std::max(1.0, kind.resident * (double)target_cus / heads);
            // What a call is expected to take with ranges of at most `most` tiles.
            auto expect = [&](int64_t most) {
                int64_t n = 0;
                double partial = 0.0;
                for (const Tile &t : mine) {
                    const int64_t k = up(t.keys, most);
                    n += k;
                    if (k > 1) partial += (double)k * (double)std::min<int64_t>(kind.rows, ((int64_t)seq_indptr[t.seq + 1] - seq_indptr[t.seq]) * group - t.row);
                }
                // the chip's work and the longest chain of steps: the longer one, and of the shorter 0.16 that do not fall beside it (fitted likewise), less the more rounds there are
                const double work = std::max((double)all * heads / target_cus * kind.step, bytes * heads / kBytesPerUs), line = (double)std::min(most, longest) * kind.alone + (crosses && most > 1 ? kCrossUs : 0.0);
                const double rounds = std::max(1.0, (double)n * heads / (kind.resident * (double)target_cus));
                return kind.begin + (rounds - 1.0) * kind.again + std::max(work, line) + 0.16 * std::min(work, line) / rounds +
                       (partial > 0.0 ? kMergeUs + partial * heads * 8.0 * (kHeadDim + 2) / kPartialBytesPerUs : 0.0);
            };
            auto parts = [&](int64_t most) { int64_t n = 0; for (const Tile &t : mine) n += up(t.keys, most); return n; };
            // whole ranges, or as short ones as give no more workgroups than are resident at once, or a half, a quarter, ... as many; whole ones without a look at others,
            // where there are more tiles than that
            int64_t most = longest;
            double time = expect(longest);
            for (double share = 1.0; share > 0.05; share *= 0.5) {
                if ((double)mine.size() > slots * share) break;
                int64_t lo = 1, hi = longest;
                while (lo < hi) {
                    const int64_t mid = lo + (hi - lo) / 2;
                    if ((double)parts(mid) <= slots * share) hi = mid;
                    else lo = mid + 1;
                }
                const double t = lo < longest ? expect(lo) : time;
                if (t < time) {
                    most = lo;
                    time = t;
                }
            }
            if (!best || time < least) {
                best = &kind;
                least = time;
                for (Tile &t : mine) t.parts = (int32_t)up(t.keys, most);
                tiles.swap(mine);
            }
        }
        int64_t n_items = 0, n_cut = 0;
        for (const Tile &t : tiles) {
            n_items += t.parts;
            n_cut += t.parts > 1;
        }
        if (n_items > capacity) return TKV_ERR_CAPACITY;
        if (best && !items_ok(desc, n_items, n_cut, best->rows)) return TKV_ERR_INVALID_ARG;
        std::stable_sort(tiles.begin(), tiles.end(), [](const Tile &x, const Tile &y) { return (int64_t)x.keys * y.parts > (int64_t)y.keys * x.parts; });
        // Two workgroups of 128 rows are dealt to each compute unit, number k and k + target_cus: the longest ranges stand beside the shortest, or
        // alone, if there are fewer than two for each unit.  (Falling from the first on, the longest share theirs with the next
        // longest: six sequences of 21 to 724 tokens behind prefixes 71.8 us, this way 68.4; 1000 tokens of 64 heads 29.7, 28.8.)
        const size_t units = (size_t)std::max(1, target_cus / desc->n_kv_heads);
        if (best && best->resident == 2 && n_cut == 0 && tiles.size() > units) std::reverse(tiles.begin(), tiles.begin() + (int64_t)units);
        int32_t slot = 0, cut = 0, number = 0;
        for (const Tile &t : tiles) {
            if (t.parts > 1) {
                int32_t *of = items_out + kPrefillItemWords * (int64_t)cut++ + 10;
                of[0] = seq_indptr[t.seq];
                of[1] = seq_indptr[t.seq + 1] - seq_indptr[t.seq];
                of[2] = t.row;
                of[3] = slot;
                of[4] = t.parts;
            }
            for (int32_t k = 0; k < t.parts; ++k, ++number) {
                const int32_t b = t.seq;
                int32_t *it = items_out + kPrefillItemWords * (int64_t)number;
                it[0] = seq_indptr[b];
                it[1] = seq_indptr[b + 1] - seq_indptr[b];
                it[2] = prefix_indptr ? prefix_indptr[b] : 0;
                it[3] = prefix_indptr ? prefix_indptr[b + 1] - prefix_indptr[b] : 0;
                it[4] = t.row;
                it[5] = (int32_t)((int64_t)t.keys * k / t.parts);
                it[6] = (int32_t)((int64_t)t.keys * (k + 1) / t.parts);
                it[7] = t.parts > 1 ? slot++ : -1;
                it[8] = k;
                it[9] = t.parts;
            }
        }
        for (int32_t k = 0; k < number; ++k) {
            int32_t *of = items_out + kPrefillItemWords * (int64_t)k;
            for (int32_t j = k < cut ? 15 : 10; j < 16; ++j) of[j] = 0;
        }
        *tile_rows_out = best ? best->rows : kKinds[0].rows;
        *n_slots_out = slot;
        *n_cut_out = cut;
        return number;
    } catch (const std::bad_alloc &) {
        return TKV_ERR_INVALID_ARG;
    }
}

size_t tkv_prefill_workspace_bytes(const tkv_desc *desc, int32_t n_slots, int32_t tile_rows)
{
    if (tkv_desc_status(desc) || n_slots < 0 || !kind_of(tile_rows)) return 0;
    return (size_t)n_slots * desc->n_kv_heads * tile_rows * (kHeadDim + 2) * sizeof(float);
}

int tkv_prefill_attention(const tkv_desc *desc, int32_t n_q_heads, const void *q, int64_t q_stride, int32_t q_type, const void *K, int64_t k_stride,
                          const void *V, int64_t v_stride, int32_t kv_type, int32_t n_tokens, const void *K_prefix, const void *V_prefix, int32_t n_prefix,
                          const tkv_prefill *prefill, float sm_scale, void *out, int32_t out_type, void *workspace, size_t workspace_bytes, int32_t *status,
                          void *stream)
{
    int32_t group = 0;
    if (int st = group_of(desc, n_q_heads, group)) return st;
    if (!prefill || n_tokens < 0 || n_prefix < 0 || prefill->n_items < 0 || prefill->n_slots < 0 || prefill->n_cut < 0 || prefill->n_cut > prefill->n_slots) return TKV_ERR_INVALID_ARG;
    if ((q_type != TKV_BF16 && q_type != TKV_FP16) || (kv_type != TKV_BF16 && kv_type != TKV_FP16) || (out_type != TKV_BF16 && out_type != TKV_FP16) ||
        (q_type == TKV_FP16 && kv_type == TKV_BF16))
        return TKV_ERR_INVALID_ARG;
    if (!(sm_scale > 0.0f) || !(sm_scale < 2.0e38f)) return TKV_ERR_INVALID_ARG;
    if (prefill->n_items == 0 || n_tokens == 0) return TKV_OK;
    if (!kind_of(prefill->tile_rows) || !prefill->items || ((uintptr_t)prefill->items & 3)) return TKV_ERR_INVALID_ARG;
    if (!rows_ok(q, q_stride, n_q_heads, n_tokens) || !rows_ok(K, k_stride, desc->n_kv_heads, n_tokens) || !rows_ok(V, v_stride, desc->n_kv_heads, n_tokens)) return TKV_ERR_INVALID_ARG;
    if (n_prefix > 0 && (!rows_ok(K_prefix, 0, 0, n_prefix) || !rows_ok(V_prefix, 0, 0, n_prefix))) return TKV_ERR_INVALID_ARG;
    if (!heads_ok(desc)) return TKV_ERR_BAD_SHAPE;
    if (!out || ((uintptr_t)out & 15) || ((uintptr_t)workspace & 15) || ((uintptr_t)status & 3)) return TKV_ERR_INVALID_ARG;
    if (!tokens_ok(n_tokens, group) || !items_ok(desc, prefill->n_items, prefill->n_cut, prefill->tile_rows)) return TKV_ERR_INVALID_ARG;
    if (prefill->n_slots > 0) {
        if (!workspace) return TKV_ERR_INVALID_ARG;
        if (workspace_bytes < tkv_prefill_workspace_bytes(desc, prefill->n_slots, prefill->tile_rows)) return TKV_ERR_WORKSPACE_TOO_SMALL;
    }
    return tkv_launch_prefill(n_q_heads, desc->n_kv_heads, q, q_stride, q_type, K, k_stride, V, v_stride, kv_type, n_tokens, K_prefix, V_prefix, n_prefix, prefill,
                              sm_scale, out, out_type, workspace, status, stream);
}

/* ---------------------------------------------------------------- C1: rows as the cache gives them back, distortion */

int32_t tkv_plan_row_blocks(const uint8_t *tag_bits, const int32_t *seq_indptr, int32_t batch, int32_t *blocks_out, int32_t capacity)
{
    if (!seq_indptr || batch < 0 || capacity < 0 || (capacity > 0 && !blocks_out) || seq_indptr[0] != 0) return TKV_ERR_INVALID_ARG;
    int64_t n = 0;
    for (int32_t b = 0; b < batch; ++b) {
        if (seq_indptr[b + 1] < seq_indptr[b]) return TKV_ERR_INVALID_ARG;
        if (seq_indptr[b + 1] > seq_indptr[b] && !tag_bits) return TKV_ERR_INVALID_ARG;
        int64_t mine = 0;
        for (int32_t t = seq_indptr[b]; t < seq_indptr[b + 1]; ++t) mine += tag_bits[t] == 2;
        if (mine % kGroup) return TKV_ERR_INVALID_ARG;
        n += mine;
    }
    if (n > kGroup * (int64_t)capacity) return TKV_ERR_CAPACITY;
    int32_t *to = blocks_out;
    for (int32_t t = 0; t < seq_indptr[batch]; ++t)
        if (tag_bits[t] == 2) *to++ = t;
    return (int32_t)(n / kGroup);
}

int tkv_quantize_rows(const tkv_desc *desc, const void *K, int64_t k_stride, const void *V, int64_t v_stride, const uint8_t *tag_bits, int32_t n_tokens,
                      const int32_t *blocks, int32_t n_blocks, void *K_out, void *V_out, int32_t *status, void *stream)
{
    if (int st = tkv_desc_status(desc)) return st;
    if (n_tokens < 0 || n_blocks < 0 || n_blocks > n_tokens / kGroup) return TKV_ERR_INVALID_ARG;
    if (n_tokens == 0) return TKV_OK;
    if (n_blocks > 0 && (!blocks || ((uintptr_t)blocks & 3) || desc->int2_key_axis != TKV_KEYS_PER_CHANNEL)) return TKV_ERR_INVALID_ARG;
    if (!rows_ok(K, k_stride, desc->n_kv_heads, n_tokens) || !rows_ok(V, v_stride, desc->n_kv_heads, n_tokens)) return TKV_ERR_INVALID_ARG;
    if (!tag_bits || !K_out || !V_out || ((uintptr_t)K_out & 15) || ((uintptr_t)V_out & 15) || ((uintptr_t)status & 3)) return TKV_ERR_INVALID_ARG;
    if ((int64_t)n_tokens * desc->n_kv_heads > INT32_MAX) return TKV_ERR_INVALID_ARG;
    return tkv_launch_quantize_rows(desc, K, k_stride, V, v_stride, tag_bits, n_tokens, blocks, n_blocks, K_out, V_out, status, stream);
}

size_t tkv_distortion_workspace_bytes(int32_t batch, int32_t n_tokens, int32_t n_heads)
{
    if (batch < 0 || n_tokens < 0 || n_heads < 0) return 0;
    return ((size_t)(n_tokens / tkv_distortion_chunk(n_tokens, n_heads)) + (size_t)batch) * (size_t)n_heads * sizeof(double);
}

int tkv_head_distortion(const void *x, const void *y, int32_t type, const int32_t *seq_indptr, int32_t batch, int32_t n_tokens, int32_t n_heads, double *out,
                        void *workspace, size_t workspace_bytes, void *stream)
{
    if (type != TKV_BF16 && type != TKV_FP16 && type != TKV_FP32) return TKV_ERR_INVALID_ARG;
    if (batch < 0 || n_tokens < 0 || n_heads < 0) return TKV_ERR_INVALID_ARG;
    if (batch == 0 || n_heads == 0) return TKV_OK;
    if (!seq_indptr || ((uintptr_t)seq_indptr & 3) || !out || ((uintptr_t)out & 7)) return TKV_ERR_INVALID_ARG;
    if (n_tokens > 0 && (!x || !y || (((uintptr_t)x | (uintptr_t)y) & 15))) return TKV_ERR_INVALID_ARG;
    if (!workspace || ((uintptr_t)workspace & 15)) return TKV_ERR_INVALID_ARG;
    if ((int64_t)batch * n_heads > INT32_MAX || (int64_t)n_tokens * n_heads > INT32_MAX) return TKV_ERR_INVALID_ARG;
    if (workspace_bytes < tkv_distortion_workspace_bytes(batch, n_tokens, n_heads)) return TKV_ERR_WORKSPACE_TOO_SMALL;
    return tkv_launch_distortion(x, y, type, seq_indptr, batch, n_tokens, n_heads, out, workspace, stream);
}

} // extern "C"
