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
// What bounds it is latency: a hundred KiB move at most.  Few sequences and tokens are one launch of one workgroup
// (tkv_table_small_kernel); the rest is four: tags to bit masks, sums over the sequences, pages given back, rows and tokens.
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

// Sums over the workgroup of what the threads before this one hold; `all` receives the sums over all of them.
template <int N> __device__ __forceinline__ void block_before(int (&v)[N], int (&all)[N], int (*shared)[kWaves])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int own[N];
#pragma unroll
    for (int k = 0; k < N; ++k) own[k] = v[k];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int t = __shfl_up(v[k], d);
            v[k] += lane >= d ? t : 0;
        }
    }
    if (lane == 63)
#pragma unroll
        for (int k = 0; k < N; ++k) shared[k][wave] = v[k];
    __syncthreads();
    // the sixteen sums of the wavefronts, one a lane
    int t[N];
#pragma unroll
    for (int k = 0; k < N; ++k) t[k] = shared[k][lane & (kWaves - 1)];
#pragma unroll
    for (int d = 1; d < kWaves; d <<= 1) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int u = __shfl_up(t[k], d);
            t[k] += (lane & (kWaves - 1)) >= d ? u : 0;
        }
    }
    const int mine = __builtin_amdgcn_readfirstlane(wave);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        all[k] = __builtin_amdgcn_readlane(t[k], kWaves - 1);
        v[k] += (mine > 0 ? __builtin_amdgcn_readlane(t[k], mine - 1) : 0) - own[k];
    }
    __syncthreads();
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
__device__ __forceinline__ int judge(const TableArgs &a, const Totals &t, const int (&n_free)[2])
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
// The pages that sequence b gives back, by `n` threads of which this is number `me`.
__device__ __forceinline__ void push_pages(const TableArgs &a, const Info &s, const Totals &t, const int (&n_free)[2], int b, int me, int n)
{
    const int32_t *row = a.page_ids + (size_t)b * a.max_pages;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const int kept = pages_of(s.at(kKeep2 + w, b)), old = s.at(kOld2 + w, b), lead = w ? s.at(kOld2, b) : 0;
        int32_t *top = free_list(a, w) + n_free[w] + t.push[w] - 1 - s.at(kPush2 + w, b);
        for (int i = me; i < old - kept; i += n) top[-i] = row[lead + kept + i];
    }
}
// The row and the counts of sequence b, by one wavefront (WAVE) or one thread.
template <bool WAVE> __device__ __forceinline__ void update_row(const TableArgs &a, const Info &s, const Totals &t, const int (&n_free)[2], int b, int lane)
{
    constexpr int kStep = WAVE ? 64 : 1;
    int32_t *row = a.page_ids + (size_t)b * a.max_pages;
    const int old2 = s.at(kOld2, b), old4 = s.at(kOld4, b), now2 = s.at(kNow2, b), now4 = s.at(kNow4, b);
    const int kept2 = pages_of(s.at(kKeep2, b)), kept4 = pages_of(s.at(kKeep4, b));
    if (WAVE && now2 != old2 && kept4 > 0) move_ids(row, old2, kept4, now2 - old2, lane);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const int kept = w ? kept4 : kept2, n = (w ? now4 : now2) - kept;
        const int32_t *top = free_list(a, w) + n_free[w] + t.push[w] - 1 - s.at(kPop2 + w, b);
        for (int i = lane; i < n; i += kStep) row[(w ? now2 : 0) + kept + i] = top[-i];
    }
    for (int i = now2 + now4 + lane; i < old2 + old4; i += kStep) row[i] = -1;
}
// Whether one thread does with the row of a sequence.
__device__ __forceinline__ bool is_light(const SeqPages &s)
{
    return (s.now[0] == s.old[0] || s.kept[1] == 0) && s.old[0] - s.kept[0] + s.old[1] - s.kept[1] <= 2 && s.now[0] - s.kept[0] + s.now[1] - s.kept[1] <= 2;
}
// Token t of sequence b, `wide` INT4 tokens before it.
__device__ __forceinline__ void place_token(const TableArgs &a, const Info &s, const Totals &t, const int (&n_free)[2], int b, int token, bool is4, int wide)
{
    const int rank = token - s.at(kTok0, b), rank4 = wide - s.at(kWide0, b), w = is4;
    const int keep2 = s.at(kKeep2, b), keep4 = s.at(kKeep4, b), keep = w ? keep4 : keep2;
    const int place = keep + (w ? rank4 : rank - rank4), index = place / kPageTokens, kept = pages_of(keep);
    const int page = index < kept ? s.at(kOpen2 + w, b) : free_list(a, w)[n_free[w] + t.push[w] - 1 - s.at(kPop2 + w, b) - (index - kept)];
    const int entry = s.at(kWork, b) + (w ? s.at(kTouch2, b) : 0) + index - keep / kPageTokens;
    const int slot = place % kPageTokens;
    if (a.slot_ids) a.slot_ids[token] = page * kPageTokens + slot;
    if (a.positions) a.positions[token] = keep2 + keep4 + rank;
    a.work_src[(size_t)entry * kPageTokens + slot] = token;
    // the first token of a page names it: nothing of the page was written by this call before it
    if (slot == 0 || place == keep) a.work_pages[entry] = page;
}
// The page that holds the last kept token of sequence b at either width, which may have room.
__device__ __forceinline__ int open_page(const TableArgs &a, int b, int lead, int keep)
{
    return keep > 0 ? a.page_ids[(size_t)b * a.max_pages + lead + pages_of(keep) - 1] : 0;
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

// ---- one workgroup for everything ------------------------------------------------------------------------------------
constexpr int kSmallSeqs = kThreads, kSmallTokens = 8 * kThreads;
__global__ __launch_bounds__(kThreads) void tkv_table_small_kernel(TableArgs a)
{
    __shared__ int32_t words[kWords * kSmallSeqs];
    __shared__ int sums[5][kWaves];
    __shared__ uint32_t before[kThreads + 1];   // per eight tokens: INT4 tokens before them
    __shared__ uint8_t masks[kThreads];         // ... and which of them are INT4
    __shared__ int32_t heavy[kSmallSeqs], n_heavy, bad_s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = a.n_seqs;
    const Info s = {words, kSmallSeqs};
    if (tid == 0) n_heavy = bad_s = 0;
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
    uint32_t m8 = 0;
    uint64_t tags = 0;
    const int left = a.n_tokens - 8 * tid;
    if (left > 0) {
        if (left >= 8 && ((uintptr_t)a.tag_bits & 7) == 0) {
            tags = reinterpret_cast<const uint64_t *>(a.tag_bits)[tid];
        } else {
            for (int i = 0; i < 8; ++i) tags |= (uint64_t)(i < left ? a.tag_bits[8 * tid + i] : 2) << (8 * i);
        }
    }
    // nothing is listed yet
    for (int i = tid; i < a.max_work * kPageTokens; i += kThreads) a.work_src[i] = -1;
    for (int i = tid; i < a.max_work; i += kThreads) a.work_pages[i] = 0;
    __syncthreads();   // n_heavy, bad_s
    int bad = 0;
    if (n_new < 0 || n_new > a.n_tokens) {
        bad = TKV_STATUS_TABLE_REFUSED;
        n_new = 0;
    }
    uint32_t odd8 = 0;   // tags that are neither 2 nor 4
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t t = (uint32_t)(tags >> (8 * i)) & 0xff;
        m8 |= (i < left && t == 4 ? 1u : 0u) << i;
        odd8 |= (i < left && t != 2 && t != 4 ? 1u : 0u) << i;
    }
    int v[2] = {n_new, (int)__popc(m8)}, all[2];
    block_before(v, all, sums);
    const int tok0 = v[0], total = all[0];
    before[tid] = (uint32_t)v[1];
    masks[tid] = (uint8_t)m8;
    if (mine) s.at(kTok0, tid) = tok0;
    // tokens behind the last sequence are no tokens
    for (int i = 0; i < 8; ++i)
        if ((odd8 >> i & 1) && 8 * tid + i < total) bad |= TKV_STATUS_TABLE_REFUSED;
    if (total > a.n_tokens) bad |= TKV_STATUS_TABLE_REFUSED;
    if (tid == 0) before[kThreads] = (uint32_t)all[1];
    __syncthreads();
    auto wide_before = [&](int t) { return (int)(before[t >> 3] + __popc((uint32_t)masks[t >> 3 < kThreads ? t >> 3 : 0] & ((1u << (t & 7)) - 1))); };
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
    block_before(u, sum, sums);
    const Totals t = {{sum[0], sum[1]}, {sum[2], sum[3]}, sum[4], total, bad_s};
    const int refused = judge(a, t, n_free);
    if (refused) {
        if (tid == 0 && a.status) atomicOr(a.status, refused);
        if (tid == 0) *a.n_work = 0;
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
            s.at(kOpen2 + w, tid) = open_page(a, tid, w ? p.old[0] : 0, p.keep[w]);
        }
        if (is_light(p)) push_pages(a, s, t, n_free, tid, 0, 1);
        else heavy[atomicAdd(&n_heavy, 1)] = tid;
    }
    if (tid == 0) {
        if (a.token_indptr) a.token_indptr[n] = total;
        *a.n_work = t.work;
    }
    __syncthreads();
    if (t.push[0] + t.push[1] > 0) {
        for (int i = wave; i < n_heavy; i += kWaves) push_pages(a, s, t, n_free, heavy[i], lane, 64);
        __syncthreads();   // every page that was given back is on the free lists, and every id that moves is still in its place
    }
    if (mine) {
        const int wide = wide_before(tok0 + n_new) - wide0;
        a.n_tok[0][tid] = p.keep[0] + n_new - wide;
        a.n_tok[1][tid] = p.keep[1] + wide;
        if (is_light(p)) update_row<false>(a, s, t, n_free, tid, 0);
    }
    for (int i = wave; i < n_heavy; i += kWaves) update_row<true>(a, s, t, n_free, heavy[i], lane);
    if (tid == 0) {
        a.n_free[0] = n_free[0] + t.push[0] - t.pop[0];
        a.n_free[1] = n_free[1] + t.push[1] - t.pop[1];
    }
    for (int i = tid; i < a.n_tokens; i += kThreads) {
        if (i < total) {
            const int b = sequence_of([&](int k) { return s.at(kTok0, k); }, n, i);
            place_token(a, s, t, n_free, b, i, masks[i >> 3] >> (i & 7) & 1, wide_before(i));
        } else {
            if (a.slot_ids) a.slot_ids[i] = -1;
            if (a.positions) a.positions[i] = -1;
        }
    }
}

// ---- many sequences or tokens ----------------------------------------------------------------------------------------
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
    for (int64_t k = i; k < (int64_t)a.max_work * kPageTokens; k += step) a.work_src[k] = -1;
    for (int64_t k = i; k < a.max_work; k += step) a.work_pages[k] = 0;
}
// Sums over the tags and the sequences, one workgroup; the verdict, and what can be written from here.
__global__ __launch_bounds__(kThreads) void tkv_table_sums_kernel(TableArgs a)
{
    __shared__ int sums[5][kWaves];
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
        int n_new = mine && a.n_new ? a.n_new[b] : 0, bad = 0;
        if (n_new < 0 || n_new > a.n_tokens) {
            bad = TKV_STATUS_TABLE_REFUSED;
            n_new = 0;
        }
        int v[2] = {n_new & 0x3fff, n_new >> 14}, all[2];   // lengths up to 2^28: 1024 of either part fit
        block_before(v, all, sums);
        const int64_t tok0 = tokens + v[0] + ((int64_t)v[1] << 14);
        SeqPages p = {};
        int wide0 = 0;
        if (mine && tok0 + n_new <= a.n_tokens) {
            int had[2], want[2];
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                had[w] = a.n_tok[w][b];
                want[w] = a.keep[w] ? a.keep[w][b] : had[w];
            }
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
        block_before(u, sum, sums);
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
                ws.s.at(kOpen2 + w, b) = open_page(a, b, w ? p.old[0] : 0, p.keep[w]);
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
    const int refused = judge(a, t, n_free);
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
    for (int b = blockIdx.x; b < a.n_seqs; b += gridDim.x) push_pages(a, w.s, t, n_free, b, threadIdx.x, 256);
}
// The first `seq_blocks` workgroups update rows, a wavefront for each, the others place tokens.
__global__ __launch_bounds__(256) void tkv_table_place_kernel(TableArgs a, int seq_blocks)
{
    const Workspace w = workspace_of(a);
    const Totals t = w.h->t;
    const int n_free[2] = {w.h->n_free[0], w.h->n_free[1]};
    const int lane = threadIdx.x & 63;
    if ((int)blockIdx.x < seq_blocks) {
        if (t.bad) return;
        for (int b = blockIdx.x * 4 + (threadIdx.x >> 6); b < a.n_seqs; b += seq_blocks * 4) {
            update_row<true>(a, w.s, t, n_free, b, lane);
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
            place_token(a, w.s, t, n_free, b, (int)i, m >> (i & 63) & 1, w.before[i >> 6] + __popcll(m & ((1ull << (i & 63)) - 1)));
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
    if (a.n_seqs <= kSmallSeqs && n_tokens <= kSmallTokens && max_work <= 1024) {
        hipLaunchKernelGGL(tkv_table_small_kernel, dim3(1), dim3(kThreads), 0, s, a);
        return hipGetLastError() == hipSuccess ? TKV_OK : TKV_ERR_HIP;
    }
    hipLaunchKernelGGL(tkv_table_tags_kernel, dim3(blocks_for(n_tokens > (int64_t)max_work * kPageTokens ? n_tokens : (int64_t)max_work * kPageTokens, 1024)), dim3(256), 0, s, a);
    hipLaunchKernelGGL(tkv_table_sums_kernel, dim3(1), dim3(kThreads), 0, s, a);
    if (keep_int2 || keep_int4) hipLaunchKernelGGL(tkv_table_push_kernel, dim3(a.n_seqs < 1 ? 1 : (a.n_seqs < 1024 ? a.n_seqs : 1024)), dim3(256), 0, s, a);
    const int seq_blocks = (int)blocks_for((int64_t)a.n_seqs * 64, 512);
    hipLaunchKernelGGL(tkv_table_place_kernel, dim3(seq_blocks + blocks_for(n_tokens, 1024)), dim3(256), 0, s, a, seq_blocks);
    return hipGetLastError() == hipSuccess ? TKV_OK : TKV_ERR_HIP;
}
