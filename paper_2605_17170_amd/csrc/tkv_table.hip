// tkv_table_append: the page tables of a batch kept on the GPU.  One call cuts sequences back to what they keep, gives the
// arriving tokens slots in the page streams of their widths and writes what append and decode read: slots, positions, the
// list of pages that receive tokens, page lists, token counts, free lists (paper Sec. 3.2.2 for the pools and their
// allocators, Sec. 3.2.3 for the page table; the host's tkv_plan_append does the same for one sequence at a time).
//
// With C(t) the number of INT4 tags before token t, a token of sequence b at INT4 stands at place
//   keep4[b] + C(t) - C(first token of b)      of the sequence's INT4 stream, one at INT2 at
//   keep2[b] + (t - first) - (C(t) - C(first)) of its INT2 stream,
// so one prefix sum over the tags and one over the sequences (tokens, pages given back and taken of either pool, pages that
// receive tokens) decide everything.  Free lists are stacks: the pages given back are pushed with the first sequence's
// first page on top, those taken are popped from there, and every one of them is known from the sums without a loop over
// sequences.
//
// What bounds it is latency: a few hundred KiB move at most.  One workgroup forms the sums, a sequence and 64 tokens a thread, and
// asks for everything it may need (open pages, tops of the free lists) before the first of them.
//   up to 1024 sequences, 6144 tokens and 1024 work entries: one launch, which also updates rows and places tokens.  32 sequences
//     with a token each 5.7 us (an empty kernel 3.9 to 4.4), 200 with five 6.9; 9 thousand tokens would take 12.7, and 11.0 in two launches.
//   up to 1024 sequences and 65536 tokens: rows and tokens in a second launch over many workgroups, and pages given back by rows of more
//     than 8192 entries together in one between them.  6 prompts with 63 thousand tokens
//     11.6 us (in four launches 15.6), 12 with 9 thousand 10.9 (15.2).
//   beyond: three launches, four where sequences may be cut; tags to bit masks, sums in a loop, pages given back, rows and tokens.  2048
//     sequences with a token each 22.5 us, with eight 24, 8192 with four 61 (sums of 1024 sequences at a time); 2 prompts with 131 thousand
//     tokens together 16.5, 32 with a million 36.
#include <hip/hip_runtime.h>

#include "tkv_internal.h"
#include "tkv_layout.h"

namespace {

using namespace tkv;

struct TableArgs {
    int32_t *page_ids, *n_tok[2], *free_pages, *n_free;
    const int32_t *keep[2];
    const int32_t *n_new;
    const uint8_t *tag_bits;
    int32_t *token_indptr, *positions, *slot_ids, *work_pages, *work_src, *n_work, *status;
    int32_t *ws;
    int32_t n_seqs, max_pages, n_tokens, max_work;
    int32_t pool_pages[2];
    int32_t channel_keys;
};

constexpr int kThreads = 1024, kWaves = kThreads / 64;

// What is known of a sequence; kept as arrays, one word of each sequence after the other.
enum { kTok0, kWide0, kKeep2, kKeep4, kPop2, kPop4, kWork, kTouch2, kOpen2, kOpen4, kOld2, kOld4, kPush2, kPush4, kNow2, kNow4, kWords };

struct Info {   // arrays of n words each
    int32_t *w;
    int n;
    __device__ __forceinline__ int32_t &at(int k, int b) const { return w[(size_t)k * n + b]; }
};
struct Totals { int32_t push[2], pop[2], work, tokens, bad; };   // bad: TKV_STATUS bits

__device__ __forceinline__ int pages_of(int n) { return (n + kPageTokens - 1) / kPageTokens; }

template <int CTRL, int ROWS> __device__ __forceinline__ int dpp_add(int v) { return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int row_scan(int v)   // over the 16 lanes of a row
{
    v = dpp_add<0x111, 0xf>(v);   // row_shr 1, 2, 4, 8
    v = dpp_add<0x112, 0xf>(v);
    v = dpp_add<0x114, 0xf>(v);
    return dpp_add<0x118, 0xf>(v);
}
// Sums over the workgroup of what the threads before this one hold; `all` receives the sums over all of them.  `shared` is read
// until the next barrier.  (Scans by DPP: through LDS one took 0.5 us.)
template <int N> __device__ __forceinline__ void block_before(int (&v)[N], int (&all)[N], int (*shared)[kWaves])
{
    static_assert(kWaves == 16, "the sums of the wavefronts are one row");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int own[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        own[k] = v[k];
        v[k] = row_scan(v[k]);
        v[k] = dpp_add<0x142, 0xa>(v[k]);   // the sum of row 0 to row 1, of 2 to 3; then of the lower half to the upper
        v[k] = dpp_add<0x143, 0xc>(v[k]);
    }
    if (lane == 63)
#pragma unroll
        for (int k = 0; k < N; ++k) shared[k][wave] = v[k];
    __syncthreads();
    const int mine = __builtin_amdgcn_readfirstlane(wave);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int t = row_scan(shared[k][lane & (kWaves - 1)]);
        all[k] = __builtin_amdgcn_readlane(t, kWaves - 1);
        v[k] += (mine > 0 ? __builtin_amdgcn_readlane(t, mine - 1) : 0) - own[k];
    }
}

// One sequence's pages.  Returns status bits.
struct SeqPages {
    int keep[2], old[2], kept[2], now[2], touch[2];
};
__device__ __forceinline__ int plan_sequence(const TableArgs &a, const int (&had)[2], const int (&want)[2], int n_new, int wide, SeqPages &s)
{
    const int fresh[2] = {n_new - wide, wide}, most = a.max_pages * kPageTokens;
    int bad = 0;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const bool ok = had[w] >= 0 && had[w] <= most && want[w] >= 0;
        if (!ok) bad |= TKV_STATUS_TABLE_REFUSED;
        const int have = ok ? had[w] : 0;
        s.keep[w] = ok && want[w] < have ? want[w] : have;
        s.old[w] = pages_of(have);
        s.kept[w] = pages_of(s.keep[w]);
        s.now[w] = pages_of(s.keep[w] + fresh[w]);
        s.touch[w] = fresh[w] > 0 ? s.now[w] - s.keep[w] / kPageTokens : 0;
    }
    if (s.old[0] + s.old[1] > a.max_pages) bad |= TKV_STATUS_TABLE_REFUSED;
    else if (s.now[0] + s.now[1] > a.max_pages) bad |= TKV_STATUS_CAPACITY;
    if (a.channel_keys && (fresh[0] % kGroup || s.keep[0] % kGroup)) bad |= TKV_STATUS_TABLE_REFUSED;
    return bad;
}
// Whether the whole call can be done.
__device__ __forceinline__ int refusal(const TableArgs &a, const Totals &t, const int (&n_free)[2])
{
    int bad = t.bad;
    if (t.tokens < 0) bad |= TKV_STATUS_TABLE_REFUSED;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        if (n_free[w] < 0 || n_free[w] > a.pool_pages[w] || (int64_t)n_free[w] + t.push[w] > a.pool_pages[w]) bad |= TKV_STATUS_TABLE_REFUSED;
        else if (t.pop[w] > n_free[w] + t.push[w]) bad |= TKV_STATUS_POOL_EXHAUSTED;
    }
    if (t.work > a.max_work) bad |= TKV_STATUS_CAPACITY;
    return bad;
}
__device__ __forceinline__ int32_t *free_list(const TableArgs &a, int w) { return a.free_pages + (w ? a.pool_pages[0] : 0); }

// Ids [from, from + n) of a row move by `by`, one wavefront; eight blocks of 64 at a time, from the end that is not written into.
__device__ __forceinline__ void move_ids(int32_t *row, int from, int n, int by, int lane)
{
    constexpr int kStep = 8 * 64;
    for (int done = 0; done < n; done += kStep) {
        const int m = n - done < kStep ? n - done : kStep;
        int32_t *p = row + from + (by > 0 ? n - done - m : done);
        int32_t v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = 64 * k + lane < m ? p[64 * k + lane] : 0;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // every lane has its ids before one of them is written over
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (64 * k + lane < m) p[64 * k + lane + by] = v[k];
    }
}
// The pages that sequence b gives back, by `n` threads of which this is number `me`; given(width, depth below the new top, page).
template <class Given>
__device__ __forceinline__ void push_pages(const TableArgs &a, const Info &s, const Totals &t, const int (&n_free)[2], int b, int me, int n, Given given)
{
    const int32_t *row = a.page_ids + (size_t)b * a.max_pages;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const int kept = pages_of(s.at(kKeep2 + w, b)), old = s.at(kOld2 + w, b), lead = w ? s.at(kOld2, b) : 0;
        const int depth = s.at(kPush2 + w, b);
        int32_t *top = free_list(a, w) + n_free[w] + t.push[w] - 1 - depth;
#pragma unroll 4
        for (int i = me; i < old - kept; i += n) {
            const int page = row[lead + kept + i];
            top[-i] = page;
            given(w, depth + i, page);
        }
    }
}
// The row of sequence b, by one wavefront (WAVE) or one thread; popped(width, depth): a page of the free list as it is with those given back.
template <bool WAVE, class Popped> __device__ __forceinline__ void update_row(const TableArgs &a, const Info &s, int b, int lane, Popped popped)
{
    constexpr int kStep = WAVE ? 64 : 1;
    int32_t *row = a.page_ids + (size_t)b * a.max_pages;
    const int old2 = s.at(kOld2, b), old4 = s.at(kOld4, b), now2 = s.at(kNow2, b), now4 = s.at(kNow4, b);
    const int kept2 = pages_of(s.at(kKeep2, b)), kept4 = pages_of(s.at(kKeep4, b));
    if (WAVE && now2 != old2 && kept4 > 0) move_ids(row, old2, kept4, now2 - old2, lane);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const int kept = w ? kept4 : kept2, n = (w ? now4 : now2) - kept;
        const int depth = s.at(kPop2 + w, b);
        for (int i = lane; i < n; i += kStep) row[(w ? now2 : 0) + kept + i] = popped(w, depth + i);
    }
    for (int i = now2 + now4 + lane; i < old2 + old4; i += kStep) row[i] = -1;
}
// Whether one thread does with the row of a sequence.
__device__ __forceinline__ bool is_light(const SeqPages &s)
{
    return (s.now[0] == s.old[0] || s.kept[1] == 0) && s.old[0] - s.kept[0] + s.old[1] - s.kept[1] <= 2 && s.now[0] - s.kept[0] + s.now[1] - s.kept[1] <= 2;
}
// Token t of sequence b, `wide` INT4 tokens before it.
template <class Popped> __device__ __forceinline__ void place_token(const TableArgs &a, const Info &s, int b, int token, bool is4, int wide, Popped popped)
{
    const int rank = token - s.at(kTok0, b), rank4 = wide - s.at(kWide0, b), w = is4;
    const int keep2 = s.at(kKeep2, b), keep4 = s.at(kKeep4, b), keep = w ? keep4 : keep2;
    const int place = keep + (w ? rank4 : rank - rank4), index = place / kPageTokens, kept = pages_of(keep);
    const int page = index < kept ? s.at(kOpen2 + w, b) : popped(w, s.at(kPop2 + w, b) + index - kept);
    const int entry = s.at(kWork, b) + (w ? s.at(kTouch2, b) : 0) + index - keep / kPageTokens;
    const int slot = place % kPageTokens;
    if (a.slot_ids) a.slot_ids[token] = page * kPageTokens + slot;
    if (a.positions) a.positions[token] = keep2 + keep4 + rank;
    a.work_src[(size_t)entry * kPageTokens + slot] = token;
    // the first token of a page names it: nothing of the page was written by this call before it
    if (slot == 0 || place == keep) a.work_pages[entry] = page;
}
// The pages that hold the last kept tokens of sequence b, which may have room.  Counts that cannot be: any id.
__device__ __forceinline__ void open_pages(const TableArgs &a, int b, const int (&had)[2], const int (&want)[2], int (&open)[2])
{
    int lead = 0;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const bool ok = had[w] >= 0 && had[w] <= a.max_pages * kPageTokens;
        const int have = ok ? had[w] : 0, keep = want[w] < have ? want[w] : have, at = lead + pages_of(keep > 0 ? keep : 0) - 1;
        open[w] = keep > 0 && at < a.max_pages ? a.page_ids[(size_t)b * a.max_pages + at] : 0;
        lead = pages_of(have);
    }
}
// The sequence of a token: the last b with first token <= t (later ones of the same first token own it, earlier ones are empty).
template <class First> __device__ __forceinline__ int sequence_of(First first, int n, int t)
{
    int lo = 0, hi = n;   // first(lo) <= t < first(hi)
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first(mid) <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Workspace, words: header | INT4 masks (two words per 64 tokens) | INT4 tokens before each 64 | sequences.
struct Header { Totals t; int32_t n_free[2]; int32_t odd_from; };   // odd_from: the first token with a tag that is neither 2 nor 4
constexpr int kHeaderWords = 16;
static_assert(sizeof(Header) <= kHeaderWords * 4, "header");
struct Workspace {
    Header *h;
    uint64_t *masks;
    int32_t *before;
    Info s;
};
__host__ __device__ inline size_t table_chunks(int32_t n_tokens) { return ((size_t)n_tokens + 63) / 64; }
__device__ __forceinline__ Workspace workspace_of(const TableArgs &a)
{
    const size_t c = table_chunks(a.n_tokens);
    Workspace w;
    w.h = reinterpret_cast<Header *>(a.ws);
    w.masks = reinterpret_cast<uint64_t *>(a.ws + kHeaderWords);
    w.before = a.ws + kHeaderWords + 2 * c;
    w.s = Info{w.before + c + 1, a.n_seqs};
    return w;
}
// ---- one workgroup for the sums --------------------------------------------------------------------------------------
// PLACE: the same workgroup updates the rows and places the tokens.  Otherwise tkv_table_place_kernel does, from the workspace, the
// other workgroups of this launch clear the lists, and with `push` 0 a launch between the two gives the pages back.
constexpr int kPlanSeqs = kThreads, kPlanTokens = 64 * kThreads, kSmallTokens = 6 * kThreads, kSmallWork = kThreads;
__device__ __forceinline__ void clear_lists(const TableArgs &a, int64_t i, int64_t step)
{
    const int64_t n = (int64_t)a.max_work * kPageTokens;
    if (((uintptr_t)a.work_src & 15) == 0) {
        for (int64_t k = i; k < n / 4; k += step) reinterpret_cast<int4 *>(a.work_src)[k] = make_int4(-1, -1, -1, -1);
    } else {
        for (int64_t k = i; k < n; k += step) a.work_src[k] = -1;
    }
    for (int64_t k = i; k < a.max_work; k += step) a.work_pages[k] = 0;
}
template <bool PLACE> __global__ __launch_bounds__(kThreads) void tkv_table_plan_kernel(TableArgs a, int push)
{
    __shared__ int32_t words[PLACE ? kWords * kPlanSeqs : 1];
    __shared__ int32_t popped_s[2][PLACE ? kSmallWork : 1];   // pages by their depth below the top of the free lists, those given back on top
    __shared__ int sums[7][kWaves];
    __shared__ int before[kThreads + 1];                      // per 64 tokens: INT4 tokens before them
    __shared__ alignas(16) uint64_t masks[kThreads];          // ... and which of them are INT4
    __shared__ int32_t heavy[kPlanSeqs], n_heavy, bad_s, odd_s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = a.n_seqs;
    if (!PLACE && blockIdx.x > 0) {
        clear_lists(a, (int64_t)(blockIdx.x - 1) * kThreads + tid, (int64_t)(gridDim.x - 1) * kThreads);
        return;
    }
    Workspace ws = {};
    if constexpr (!PLACE) ws = workspace_of(a);
    const Info s = PLACE ? Info{words, kPlanSeqs} : ws.s;
    const bool mine = tid < n;
    int had[2] = {0, 0}, want[2] = {0, 0}, n_new = 0;
    if (mine) {
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            had[w] = a.n_tok[w][tid];
            want[w] = a.keep[w] ? a.keep[w][tid] : had[w];
        }
        if (a.n_new) n_new = a.n_new[tid];
    }
    const int n_free[2] = {a.n_free[0], a.n_free[1]};
    if (tid == 0) {
        n_heavy = bad_s = 0;
        odd_s = INT32_MAX;
    }
    // eight tags at a time to eight bits
    const bool aligned = ((uintptr_t)a.tag_bits & 7) == 0;
    int odd = INT32_MAX;   // the first token with a tag that is neither 2 nor 4
    auto tags_of = [&](int at) -> uint64_t {
        const int left = a.n_tokens - at;
        if (left >= 8 && aligned) return *reinterpret_cast<const uint64_t *>(a.tag_bits + at);
        uint64_t x = 0;
        for (int i = 0; i < 8; ++i) x |= (uint64_t)(i < left ? a.tag_bits[at + i] : 2) << (8 * i);
        return x;
    };
    auto mask_of = [&](int at, uint64_t x) {
        const uint64_t k1 = 0x0101010101010101ull, is2 = (x >> 1) & k1, is4 = (x >> 2) & k1, bad = (x & ~(6 * k1)) | ((is2 ^ is4) ^ k1);
        if (bad) odd = min(odd, at + (int)(__builtin_ctzll(bad) >> 3));
        reinterpret_cast<uint8_t *>(masks)[at >> 3] = (uint8_t)((is4 * 0x0102040810204080ull) >> 56);
    };
    constexpr int kAhead = PLACE ? 1 : 8;
    uint64_t tags[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) tags[k] = 8 * (kThreads * k + tid) < a.n_tokens ? tags_of(8 * (kThreads * k + tid)) : 0x0202020202020202ull;
    // what the next steps need, while the counts are summed
    int open[2] = {0, 0}, top[2] = {0, 0};
    if (mine) open_pages(a, tid, had, want, open);
    if constexpr (PLACE)
#pragma unroll
        for (int w = 0; w < 2; ++w)
            if (tid < n_free[w] && n_free[w] <= a.pool_pages[w]) top[w] = free_list(a, w)[n_free[w] - 1 - tid];
    if constexpr (PLACE) clear_lists(a, tid, kThreads);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) mask_of(8 * (kThreads * k + tid), tags[k]);
    if constexpr (PLACE)   // behind them there are none
        for (int k = kThreads + tid; k < 8 * kThreads; k += kThreads) reinterpret_cast<uint8_t *>(masks)[k] = 0;
    __syncthreads();
    if (odd != INT32_MAX) atomicMin(&odd_s, odd);
    int bad = 0;
    if (n_new < 0 || n_new > a.n_tokens) {
        bad = TKV_STATUS_TABLE_REFUSED;
        n_new = 0;
    }
    int v[2] = {n_new, (int)__popcll(masks[tid])}, all[2];
    block_before(v, all, sums);
    const int tok0 = v[0], total = all[0];   // (at most 1024 times 65536)
    before[tid] = v[1];
    if (tid == 0) before[kThreads] = all[1];
    if (total > a.n_tokens || odd_s < total) bad |= TKV_STATUS_TABLE_REFUSED;   // (tokens behind the last sequence are no tokens)
    __syncthreads();
    auto wide_before = [&](int t) {
        const int left = t & 63;
        return before[t >> 6] + (left ? (int)__popcll(masks[t >> 6] & ((1ull << left) - 1)) : 0);
    };
    SeqPages p = {};
    int wide0 = 0;
    if (mine && total <= a.n_tokens) {
        wide0 = wide_before(tok0);
        bad |= plan_sequence(a, had, want, n_new, wide_before(tok0 + n_new) - wide0, p);
    }
    if (bad) {
        atomicOr(&bad_s, bad);
        p = {};
    }
    int u[5] = {p.old[0] - p.kept[0], p.old[1] - p.kept[1], p.now[0] - p.kept[0], p.now[1] - p.kept[1], p.touch[0] + p.touch[1]}, sum[5];
    block_before(u, sum, sums + 2);
    Totals t = {{sum[0], sum[1]}, {sum[2], sum[3]}, sum[4], total, bad_s};
    const int refused = refusal(a, t, n_free);
    if constexpr (!PLACE)
        if (tid == 0) {
            ws.h->t = t;
            ws.h->t.bad = refused;
#pragma unroll
            for (int w = 0; w < 2; ++w) ws.h->n_free[w] = n_free[w];
        }
    if (refused) {
        if (tid == 0 && a.status) atomicOr(a.status, refused);
        if (tid == 0) *a.n_work = 0;
        if constexpr (PLACE)
            for (int i = tid; i < a.n_tokens; i += kThreads) {
                if (a.slot_ids) a.slot_ids[i] = -1;
                if (a.positions) a.positions[i] = -1;
            }
        if (a.token_indptr)
            for (int i = tid; i <= n; i += kThreads) a.token_indptr[i] = 0;
        return;
    }
    if (mine) {
        if (a.token_indptr) a.token_indptr[tid] = tok0;
        s.at(kTok0, tid) = tok0;
        s.at(kWide0, tid) = wide0;
        s.at(kWork, tid) = u[4];
        s.at(kTouch2, tid) = p.touch[0];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            s.at(kKeep2 + w, tid) = p.keep[w];
            s.at(kPush2 + w, tid) = u[w];
            s.at(kPop2 + w, tid) = u[2 + w];
            s.at(kOld2 + w, tid) = p.old[w];
            s.at(kNow2 + w, tid) = p.now[w];
            s.at(kOpen2 + w, tid) = open[w];
        }
    }
    if constexpr (!PLACE) {
        const int chunks = (int)table_chunks(a.n_tokens);
        if (tid < chunks) {
            ws.masks[tid] = masks[tid];
            ws.before[tid] = before[tid];
        }
        if (tid == 0) ws.before[chunks] = all[1];
    }
    const bool light = is_light(p);
    auto given = [&](int w, int depth, int page) {
        if constexpr (PLACE)
            if (depth < kSmallWork) popped_s[w][depth] = page;
    };
    if constexpr (PLACE)
#pragma unroll
        for (int w = 0; w < 2; ++w)
            if (t.push[w] + tid < kSmallWork) popped_s[w][t.push[w] + tid] = top[w];
    if (mine) {
        if (!light) heavy[atomicAdd(&n_heavy, 1)] = tid;
        else if (push) push_pages(a, s, t, n_free, tid, 0, 1, given);
    }
    if (tid == 0) {
        if (a.token_indptr) a.token_indptr[n] = total;
        *a.n_work = t.work;
        a.n_free[0] = n_free[0] + t.push[0] - t.pop[0];
        a.n_free[1] = n_free[1] + t.push[1] - t.pop[1];
    }
    if (!PLACE && (!push || t.push[0] + t.push[1] == 0)) return;
    __syncthreads();
    if (t.push[0] + t.push[1] > 0) {
        for (int i = wave; i < n_heavy; i += kWaves) push_pages(a, s, t, n_free, heavy[i], lane, 64, given);
        if constexpr (PLACE) __syncthreads();   // every page that was given back is known, and every id that moves is still in its place
    }
    if constexpr (PLACE) {
        auto popped = [&](int w, int depth) { return popped_s[w][depth]; };   // (no more are taken than work entries)
        if (mine) {
            const int wide = wide_before(tok0 + n_new) - wide0;
            a.n_tok[0][tid] = p.keep[0] + n_new - wide;
            a.n_tok[1][tid] = p.keep[1] + wide;
            if (light) update_row<false>(a, s, tid, 0, popped);
        }
        for (int i = wave; i < n_heavy; i += kWaves) update_row<true>(a, s, heavy[i], lane, popped);
        for (int i = tid; i < a.n_tokens; i += kThreads) {
            if (i < total) {
                const int b = sequence_of([&](int k) { return s.at(kTok0, k); }, n, i);
                place_token(a, s, b, i, masks[i >> 6] >> (i & 63) & 1, wide_before(i), popped);
            } else {
                if (a.slot_ids) a.slot_ids[i] = -1;
                if (a.positions) a.positions[i] = -1;
            }
        }
    }
}

// ---- many sequences or tokens ----------------------------------------------------------------------------------------
// Tags to masks of 64 tokens, and nothing listed yet.
__global__ __launch_bounds__(256) void tkv_table_tags_kernel(TableArgs a)
{
    const Workspace w = workspace_of(a);
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
    for (int64_t k = i; k < (int64_t)table_chunks(a.n_tokens) * 64; k += step) {
        const int tag = k < a.n_tokens ? a.tag_bits[k] : 2;
        const uint64_t m = __ballot(tag == 4), odd = __ballot(tag != 2 && tag != 4);
        if ((k & 63) == 0) {
            w.masks[k >> 6] = m;
            w.before[k >> 6] = odd ? -__builtin_ctzll(odd) - 1 : __popcll(m);   // a chunk with other tags: minus the first of them, minus one
        }
    }
    clear_lists(a, i, step);
}
// Sums over the tags and the sequences, one workgroup; the verdict, and what can be written from here.
__global__ __launch_bounds__(kThreads) void tkv_table_sums_kernel(TableArgs a)
{
    __shared__ int sums[7][kWaves];
    __shared__ int32_t bad_s, odd_s;
    const Workspace ws = workspace_of(a);
    const int tid = threadIdx.x, chunks = (int)table_chunks(a.n_tokens);
    if (tid == 0) {
        bad_s = 0;
        odd_s = INT32_MAX;
    }
    __syncthreads();
    int carry = 0;
    for (int c = 0; c < chunks; c += kThreads) {
        const int k = c + tid;
        const int raw = k < chunks ? ws.before[k] : 0;
        if (raw < 0) atomicMin(&odd_s, 64 * k - raw - 1);
        int v[1] = {raw < 0 ? (int)__popcll(ws.masks[k]) : raw}, all[1];
        block_before(v, all, sums);
        __syncthreads();   // `sums` is read
        if (k < chunks) ws.before[k] = carry + v[0];
        carry += all[0];
    }
    if (tid == 0) ws.before[chunks] = carry;
    __syncthreads();
    auto wide_before = [&](int t) {
        const int left = t & 63;
        return ws.before[t >> 6] + (left ? __popcll(ws.masks[t >> 6] & ((1ull << left) - 1)) : 0);
    };
    const int n_free[2] = {a.n_free[0], a.n_free[1]};
    int64_t tokens = 0;   // so far
    int at[5] = {};       // pages given back and taken, work entries so far
    for (int c = 0; c < a.n_seqs; c += kThreads) {
        const int b = c + tid;
        const bool mine = b < a.n_seqs;
        int n_new = mine && a.n_new ? a.n_new[b] : 0, bad = 0, had[2] = {0, 0}, want[2] = {0, 0}, open[2] = {0, 0};
        if (mine) {
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                had[w] = a.n_tok[w][b];
                want[w] = a.keep[w] ? a.keep[w][b] : had[w];
            }
            open_pages(a, b, had, want, open);
        }
        if (n_new < 0 || n_new > a.n_tokens) {
            bad = TKV_STATUS_TABLE_REFUSED;
            n_new = 0;
        }
        int v[2] = {n_new & 0x3fff, n_new >> 14}, all[2];   // lengths up to 2^28: 1024 of either part fit
        block_before(v, all, sums + 5);
        const int64_t tok0 = tokens + v[0] + ((int64_t)v[1] << 14);
        SeqPages p = {};
        int wide0 = 0;
        if (mine && tok0 + n_new <= a.n_tokens) {
            wide0 = wide_before((int)tok0);
            bad |= plan_sequence(a, had, want, n_new, wide_before((int)tok0 + n_new) - wide0, p);
        } else if (mine) {
            bad |= TKV_STATUS_TABLE_REFUSED;
        }
        if (bad) {
            atomicOr(&bad_s, bad);
            p = {};
        }
        int u[5] = {p.old[0] - p.kept[0], p.old[1] - p.kept[1], p.now[0] - p.kept[0], p.now[1] - p.kept[1], p.touch[0] + p.touch[1]}, sum[5];
        block_before(u, sum, sums);   // (its barrier stands between the reads of sums + 5 and their next writes, as the other one does for these)
        if (mine && !bad) {
            ws.s.at(kTok0, b) = (int)tok0;
            ws.s.at(kWide0, b) = wide0;
            ws.s.at(kWork, b) = at[4] + u[4];
            ws.s.at(kTouch2, b) = p.touch[0];
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                ws.s.at(kKeep2 + w, b) = p.keep[w];
                ws.s.at(kPush2 + w, b) = at[w] + u[w];
                ws.s.at(kPop2 + w, b) = at[2 + w] + u[2 + w];
                ws.s.at(kOld2 + w, b) = p.old[w];
                ws.s.at(kNow2 + w, b) = p.now[w];
                ws.s.at(kOpen2 + w, b) = open[w];
            }
        }
        tokens += all[0] + ((int64_t)all[1] << 14);
#pragma unroll
        for (int k = 0; k < 5; ++k) at[k] += sum[k];
    }
    __syncthreads();
    // (sums of pages fit 32 bits: each row has at most max_pages, and rows times max_pages do)
    Totals t = {{at[0], at[1]}, {at[2], at[3]}, at[4], tokens <= a.n_tokens ? (int)tokens : -1, bad_s};
    if (odd_s < t.tokens) t.bad |= TKV_STATUS_TABLE_REFUSED;
    const int refused = refusal(a, t, n_free);
    for (int b = tid; b < a.n_seqs; b += kThreads)
        if (a.token_indptr) a.token_indptr[b] = refused ? 0 : ws.s.at(kTok0, b);
    if (tid == 0) {
        if (a.token_indptr) a.token_indptr[a.n_seqs] = refused ? 0 : t.tokens;
        *a.n_work = refused ? 0 : t.work;
        if (refused && a.status) atomicOr(a.status, refused);
        t.bad = refused;
        ws.h->t = t;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            ws.h->n_free[w] = n_free[w];
            if (!refused) a.n_free[w] = n_free[w] + t.push[w] - t.pop[w];
        }
    }
}
__global__ __launch_bounds__(256) void tkv_table_push_kernel(TableArgs a)
{
    const Workspace w = workspace_of(a);
    const Totals t = w.h->t;
    if (t.bad || t.push[0] + t.push[1] == 0) return;
    const int n_free[2] = {w.h->n_free[0], w.h->n_free[1]};
    for (int b = blockIdx.x; b < a.n_seqs; b += gridDim.x) push_pages(a, w.s, t, n_free, b, threadIdx.x, 256, [](int, int, int) {});
}
// The first `seq_blocks` workgroups update rows, a wavefront for each, the others place tokens.
__global__ __launch_bounds__(256) void tkv_table_place_kernel(TableArgs a, int seq_blocks)
{
    const Workspace w = workspace_of(a);
    const Totals t = w.h->t;
    const int n_free[2] = {w.h->n_free[0], w.h->n_free[1]};
    const int lane = threadIdx.x & 63;
    auto popped = [&](int k, int depth) { return free_list(a, k)[n_free[k] + t.push[k] - 1 - depth]; };
    if ((int)blockIdx.x < seq_blocks) {
        if (t.bad) return;
        for (int b = blockIdx.x * 4 + (threadIdx.x >> 6); b < a.n_seqs; b += seq_blocks * 4) {
            update_row<true>(a, w.s, b, lane, popped);
            if (lane == 0) {
                const int end = b + 1 < a.n_seqs ? w.s.at(kTok0, b + 1) : t.tokens, n_new = end - w.s.at(kTok0, b);
                const int left = end & 63;
                const int wide = w.before[end >> 6] + (left ? __popcll(w.masks[end >> 6] & ((1ull << left) - 1)) : 0) - w.s.at(kWide0, b);
                a.n_tok[0][b] = w.s.at(kKeep2, b) + n_new - wide;
                a.n_tok[1][b] = w.s.at(kKeep4, b) + wide;
            }
        }
        return;
    }
    const int64_t step = (int64_t)(gridDim.x - seq_blocks) * 256;
    for (int64_t i = (int64_t)(blockIdx.x - seq_blocks) * 256 + threadIdx.x; i < a.n_tokens; i += step) {
        if (!t.bad && i < t.tokens) {
            const int b = sequence_of([&](int k) { return w.s.at(kTok0, k); }, a.n_seqs, (int)i);
            const uint64_t m = w.masks[i >> 6];
            place_token(a, w.s, b, (int)i, m >> (i & 63) & 1, w.before[i >> 6] + __popcll(m & ((1ull << (i & 63)) - 1)), popped);
        } else {
            if (a.slot_ids) a.slot_ids[i] = -1;
            if (a.positions) a.positions[i] = -1;
        }
    }
}

__global__ __launch_bounds__(256) void tkv_table_reset_kernel(TableArgs a)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
    for (int64_t k = i; k < (int64_t)a.n_seqs * a.max_pages; k += step) a.page_ids[k] = -1;
    for (int64_t k = i; k < a.n_seqs; k += step) a.n_tok[0][k] = a.n_tok[1][k] = 0;
    // popped from the end: pages are handed out in increasing order
    for (int64_t k = i; k < a.pool_pages[0]; k += step) a.free_pages[k] = a.pool_pages[0] - 1 - (int32_t)k;
    for (int64_t k = i; k < a.pool_pages[1]; k += step) a.free_pages[a.pool_pages[0] + k] = a.pool_pages[0] + a.pool_pages[1] - 1 - (int32_t)k;
    if (i == 0) {
        a.n_free[0] = a.pool_pages[0];
        a.n_free[1] = a.pool_pages[1];
    }
}

TableArgs table_args(const tkv_desc *desc, const tkv_table *table)
{
    TableArgs a = {};
    a.page_ids = table->page_ids;
    a.n_tok[0] = table->n_tok_int2;
    a.n_tok[1] = table->n_tok_int4;
    a.free_pages = table->free_pages;
    a.n_free = table->n_free;
    a.n_seqs = table->n_seqs;
    a.max_pages = table->max_pages;
    a.pool_pages[0] = desc->n_pages_int2;
    a.pool_pages[1] = desc->n_pages_int4;
    a.channel_keys = desc->int2_key_axis == TKV_KEYS_PER_CHANNEL;
    return a;
}
unsigned blocks_for(int64_t n, int64_t most) { const int64_t b = (n + 255) / 256; return (unsigned)(b < 1 ? 1 : (b > most ? most : b)); }

} // namespace

size_t tkv_table_words(int32_t n_seqs, int32_t n_tokens)
{
    return kHeaderWords + 3 * table_chunks(n_tokens) + 2 + (size_t)kWords * n_seqs;
}

int tkv_launch_table_reset(const tkv_desc *desc, const tkv_table *table, void *stream)
{
    const TableArgs a = table_args(desc, table);
    hipLaunchKernelGGL(tkv_table_reset_kernel, dim3(blocks_for((int64_t)a.n_seqs * a.max_pages + a.pool_pages[0] + a.pool_pages[1], 1024)), dim3(256), 0,
                       (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? TKV_OK : TKV_ERR_HIP;
}

int tkv_launch_table_append(const tkv_desc *desc, const tkv_table *table, const int32_t *keep_int2, const int32_t *keep_int4, const int32_t *n_new,
                            const uint8_t *tag_bits, int32_t n_tokens, int32_t *token_indptr, int32_t *positions, int32_t *slot_ids,
                            int32_t *work_pages, int32_t *work_src, int32_t max_work, int32_t *n_work, void *workspace, int32_t *status, void *stream)
{
    TableArgs a = table_args(desc, table);
    a.keep[0] = keep_int2;
    a.keep[1] = keep_int4;
    a.n_new = n_new;
    a.tag_bits = tag_bits;
    a.n_tokens = n_tokens;
    a.token_indptr = token_indptr;
    a.positions = positions;
    a.slot_ids = slot_ids;
    a.work_pages = work_pages;
    a.work_src = work_src;
    a.max_work = max_work;
    a.n_work = n_work;
    a.status = status;
    a.ws = (int32_t *)workspace;
    hipStream_t s = (hipStream_t)stream;
    if (a.n_seqs <= kPlanSeqs && n_tokens <= kSmallTokens && max_work <= kSmallWork) {
        hipLaunchKernelGGL(tkv_table_plan_kernel<true>, dim3(1), dim3(kThreads), 0, s, a, 1);
        return hipGetLastError() == hipSuccess ? TKV_OK : TKV_ERR_HIP;
    }
    const int64_t lists = (int64_t)max_work * kPageTokens;
    bool push = keep_int2 || keep_int4;
    if (a.n_seqs <= kPlanSeqs && n_tokens <= kPlanTokens) {
        // Pages given back in the launch of the sums, by its one workgroup, or in one of their own.  Few of them: a launch (3.9 us) less.
        // 8000: 17.6 us inside and 14.4 in a launch of their own, 64000: 39 and 16.  How many there are is known on the GPU only.
        const bool inside = (int64_t)a.n_seqs * a.max_pages <= 8192;
        hipLaunchKernelGGL(tkv_table_plan_kernel<false>, dim3(1 + blocks_for(lists / 16, 255)), dim3(kThreads), 0, s, a, inside ? 1 : 0);
        push = push && !inside;
    } else {
        hipLaunchKernelGGL(tkv_table_tags_kernel, dim3(blocks_for(n_tokens > lists ? n_tokens : lists, 1024)), dim3(256), 0, s, a);
        hipLaunchKernelGGL(tkv_table_sums_kernel, dim3(1), dim3(kThreads), 0, s, a);
    }
    if (push) hipLaunchKernelGGL(tkv_table_push_kernel, dim3(a.n_seqs < 1 ? 1 : (a.n_seqs < 1024 ? a.n_seqs : 1024)), dim3(256), 0, s, a);
    const int seq_blocks = (int)blocks_for((int64_t)a.n_seqs * 64, 512);
    hipLaunchKernelGGL(tkv_table_place_kernel, dim3(seq_blocks + blocks_for(n_tokens, 1024)), dim3(256), 0, s, a, seq_blocks);
    return hipGetLastError() == hipSuccess ? TKV_OK : TKV_ERR_HIP;
}
