// The checks in front of tkv_prefill_attention, tkv_quantize_rows and tkv_head_distortion (csrc/tkv_host_prompt.cpp) under AddressSanitizer /
// UndefinedBehaviorSanitizer: what is launched, what is refused and how, and whether the workspace of distortions holds what its kernels write.
// Built and run by tests/test_host_prompt_calls.py with the host compiler only; the launchers are stubs that count.
#include <cstdint>
#include <cstdio>
#include <functional>
#include <limits>
#include <vector>

#include "tkv.h"
#include "tkv_internal.h"

static int launched = 0;
int tkv_desc_status(const tkv_desc *d) { return !d ? TKV_ERR_INVALID_ARG : d->n_kv_heads > 0 ? TKV_OK : TKV_ERR_BAD_SHAPE; }
int tkv_launch_prefill(int32_t, int32_t, const void *, int64_t, int32_t, const void *, int64_t, const void *, int64_t, int32_t, int32_t, const void *, const void *, int32_t,
                       const tkv_prefill *, float, void *, int32_t, void *, int32_t *, void *) { ++launched; return TKV_OK; }
int tkv_launch_quantize_rows(const tkv_desc *, const void *, int64_t, const void *, int64_t, const uint8_t *, int32_t, const int32_t *, int32_t, void *, void *, int32_t *, void *) { ++launched; return TKV_OK; }
int tkv_launch_distortion(const void *, const void *, int32_t, const int32_t *, int32_t, int32_t, int32_t, double *, void *, void *) { ++launched; return TKV_OK; }

#define CHECK(x) do { if (!(x)) { std::printf("FAILED line %d: %s\n", __LINE__, #x); return 1; } } while (0)

static uint64_t rng_state = 88172645463325252ull;
static uint32_t rnd() { rng_state ^= rng_state << 13; rng_state ^= rng_state >> 7; rng_state ^= rng_state << 17; return (uint32_t)(rng_state >> 32); }

// Aligned addresses that nothing here reads.
alignas(64) static char place[4096];
static void *at(int k) { return place + 64 * k; }

struct Prefill {
    tkv_desc d = {};
    tkv_prefill p = {};
    int32_t n_q_heads = 8, q_type = TKV_BF16, kv_type = TKV_BF16, out_type = TKV_BF16, n_tokens = 10, n_prefix = 5;
    int64_t q_stride = 1024, k_stride = 256, v_stride = 256;
    const void *q = at(0), *K = at(1), *V = at(2), *K_prefix = at(3), *V_prefix = at(4);
    void *out = at(5), *workspace = at(6);
    int32_t *status = (int32_t *)at(7);
    float sm = 0.1f;
    size_t bytes = 0;
    Prefill()
    {
        d.n_kv_heads = 2;
        p.tile_rows = 128; p.n_items = 4; p.n_slots = 3; p.n_cut = 1;
        p.items = (const int32_t *)at(8);
        bytes = tkv_prefill_workspace_bytes(&d, p.n_slots, p.tile_rows);
    }
    int call(bool with_desc = true, bool with_plan = true)
    {
        return tkv_prefill_attention(with_desc ? &d : nullptr, n_q_heads, q, q_stride, q_type, K, k_stride, V, v_stride, kv_type, n_tokens, K_prefix, V_prefix, n_prefix,
                                     with_plan ? &p : nullptr, sm, out, out_type, workspace, bytes, status, nullptr);
    }
};
static int prefill(const std::function<void(Prefill &)> &change)
{
    Prefill c;
    change(c);
    return c.call();
}

struct Rows {
    tkv_desc d = {};
    int32_t n_tokens = 70, n_blocks = 2;
    int64_t k_stride = 256, v_stride = 512;
    const void *K = at(0), *V = at(1);
    const uint8_t *bits = (const uint8_t *)place + 3;
    const int32_t *blocks = (const int32_t *)at(2);
    void *K_out = at(3), *V_out = at(4);
    int32_t *status = nullptr;
    Rows() { d.n_kv_heads = 2; d.int2_key_axis = TKV_KEYS_PER_CHANNEL; }
    int call() { return tkv_quantize_rows(&d, K, k_stride, V, v_stride, bits, n_tokens, blocks, n_blocks, K_out, V_out, status, nullptr); }
};
static int rows(const std::function<void(Rows &)> &change)
{
    Rows c;
    change(c);
    return c.call();
}

struct Distortion {
    const void *x = at(0), *y = at(1);
    int32_t type = TKV_FP16, batch = 3, n_tokens = 100, n_heads = 5;
    const int32_t *ip = (const int32_t *)at(2);
    double *out = (double *)at(3);
    void *workspace = at(4);
    size_t bytes = 0;
    Distortion() { bytes = tkv_distortion_workspace_bytes(batch, n_tokens, n_heads); }
    int call() { return tkv_head_distortion(x, y, type, ip, batch, n_tokens, n_heads, out, workspace, bytes, nullptr); }
};
static int distortion(const std::function<void(Distortion &)> &change)
{
    Distortion c;
    change(c);
    return c.call();
}

static int workspace_of_distortions()
{
    for (int round = 0; round < 2000; ++round) {
        const int32_t heads = round % 2 ? 1 + (int32_t)(rnd() % 3) : 4 + (int32_t)(rnd() % 80), batch = 1 + (int32_t)(rnd() % 40);
        const uint32_t longest = round % 3 == 0 ? 5 : round % 3 == 1 ? 300 : 2000;      // 8192 tokens in all on either side
        std::vector<int32_t> ip(1, 0);
        for (int32_t b = 0; b < batch; ++b) ip.push_back(ip.back() + (int32_t)(rnd() % longest));
        const int32_t tokens = ip.back() + (int32_t)(rnd() % 20), chunk = tkv_distortion_chunk(tokens, heads);
        const size_t slots = tkv_distortion_workspace_bytes(batch, tokens, heads) / sizeof(double) / (size_t)heads;
        int64_t next = 0;
        for (int32_t b = 0; b < batch; ++b) {
            const int64_t n = ((int64_t)ip[(size_t)b + 1] - ip[(size_t)b] + chunk - 1) / chunk, first = ip[(size_t)b] / chunk + b;
            CHECK(first >= next);
            if (n > 0) next = first + n;
            CHECK((size_t)next <= slots);
        }
    }
    return 0;
}

// A plan that is returned can be launched, and one that cannot is refused: `n` sequences of one token of `heads` kv heads and as many query heads.
static int plan_and_call(int32_t heads, int32_t n, int want)
{
    tkv_desc d = {};
    d.n_kv_heads = heads;
    std::vector<int32_t> ip;
    for (int32_t b = 0; b <= n; ++b) ip.push_back(b);
    std::vector<int32_t> items((size_t)n * 16 + 4096 * 16);
    int32_t rows = 0, slots = 0, cut = 0;
    const int32_t got = tkv_plan_prefill(&d, n, heads, ip.data(), nullptr, 1, items.data(), n + 4096, &rows, &slots, &cut);
    Prefill c;
    c.d = d;
    c.n_q_heads = heads;
    c.n_tokens = n;
    c.n_prefix = 0;
    c.q_stride = c.k_stride = c.v_stride = n > 1 ? (int64_t)heads * 128 : 0;
    c.p = {rows, got < 0 ? n : got, slots, cut, c.p.items};
    if (got < 0) c.p.tile_rows = 32;
    c.bytes = (size_t)1 << 40;
    CHECK(want == TKV_OK ? got >= 0 : got == want);
    CHECK(c.call() == want);
    return 0;
}

// Queries of more rows in all than 32 bits count.
static int rows_of_all_sequences()
{
    tkv_desc d = {};
    d.n_kv_heads = 1;
    const int32_t ip[] = {0, 1 << 20, 2 << 20, 3 << 20};
    int32_t rows = 0, slots = 0, cut = 0, word = 0;
    CHECK(tkv_plan_prefill(&d, 2, 1024, ip, nullptr, 1, &word, 0, &rows, &slots, &cut) == TKV_ERR_INVALID_ARG);
    CHECK(prefill([](Prefill &c) { c.d.n_kv_heads = 1; c.n_q_heads = 1024; c.q_stride = 1024 * 128; c.n_tokens = 2 << 20; }) == TKV_ERR_INVALID_ARG);
    CHECK(prefill([](Prefill &c) { c.d.n_kv_heads = 1; c.n_q_heads = 1023; c.q_stride = 1023 * 128; c.n_tokens = 2 << 20; }) == TKV_OK);
    return 0;
}

// Query heads whose rows are as long as a token stride can be, and one more, which a single token may have.
static int rows_as_long_as_strides()
{
    tkv_desc d = {};
    d.n_kv_heads = 1;
    const int32_t ip[] = {0, 1, 2};
    std::vector<int32_t> items((size_t)16 * 10000);
    int32_t rows = 0, slots = 0, cut = 0;
    for (int32_t heads : {65535, 65536})
        for (int32_t n : {1, 2}) {
            const int want = heads == 65536 && n > 1 ? TKV_ERR_BAD_SHAPE : TKV_OK;
            const int32_t got = tkv_plan_prefill(&d, n, heads, ip, nullptr, 1, items.data(), 10000, &rows, &slots, &cut);
            CHECK(want == TKV_OK ? got > 0 : got == want);
            if (want != TKV_OK) continue;
            Prefill c;
            c.d = d;
            c.n_q_heads = heads;
            c.n_tokens = n;
            c.n_prefix = 0;
            c.q_stride = n > 1 ? (int64_t)heads * 128 : 0;
            c.p = {rows, got, slots, cut, c.p.items};
            c.bytes = tkv_prefill_workspace_bytes(&d, slots, rows);
            CHECK(c.call() == TKV_OK);
        }
    return 0;
}

// Of many heads and units: what the plan returns can be launched.
static int plans_of_many_heads()
{
    int returned = 0;
    for (int32_t heads : {1000, 65535})
        for (int32_t n : {1, 60, 140, 250})
            for (int32_t units : {1, 100, 400}) {
                tkv_desc d = {};
                d.n_kv_heads = heads;
                std::vector<int32_t> ip, pp;
                for (int32_t b = 0; b <= n; ++b) {
                    ip.push_back(b * 256);
                    pp.push_back(b * 64000);
                }
                std::vector<int32_t> items((size_t)16 * 100000);
                int32_t rows = 0, slots = 0, cut = 0;
                const int32_t got = tkv_plan_prefill(&d, n, heads, ip.data(), pp.data(), units * heads, items.data(), 100000, &rows, &slots, &cut);
                CHECK(got > 0 || got == TKV_ERR_INVALID_ARG);
                if (got < 0) continue;
                ++returned;
                Prefill c;
                c.d = d;
                c.n_q_heads = heads;
                c.n_tokens = n * 256;
                c.n_prefix = n * 64000;
                c.q_stride = c.k_stride = c.v_stride = (int64_t)heads * 128;
                c.p = {rows, got, slots, cut, c.p.items};
                c.bytes = tkv_prefill_workspace_bytes(&d, slots, rows);
                CHECK(c.call() == TKV_OK);
            }
    CHECK(returned > 0);
    return 0;
}

int main()
{
    if (plan_and_call(65535, 512, TKV_OK) || plan_and_call(65535, 513, TKV_ERR_INVALID_ARG)) return 1;      // 2^25 - 1 workgroups are 512 times 65535 and some
    if (plan_and_call(1024, 32767, TKV_OK) || plan_and_call(1024, 32768, TKV_ERR_INVALID_ARG)) return 1;
    if (plan_and_call(65536, 1, TKV_ERR_BAD_SHAPE)) return 1;
    if (rows_as_long_as_strides() || rows_of_all_sequences() || plans_of_many_heads()) return 1;
    const float nan = std::numeric_limits<float>::quiet_NaN(), inf = std::numeric_limits<float>::infinity();
    if (workspace_of_distortions()) return 1;

    // what is launched
    launched = 0;
    CHECK(prefill([](Prefill &) {}) == TKV_OK && launched == 1);
    CHECK(prefill([](Prefill &c) { c.n_prefix = 0; c.K_prefix = c.V_prefix = nullptr; }) == TKV_OK && launched == 2);
    CHECK(prefill([](Prefill &c) { c.q_type = c.kv_type = c.out_type = TKV_FP16; c.status = nullptr; }) == TKV_OK && launched == 3);
    CHECK(prefill([](Prefill &c) { c.p.n_slots = c.p.n_cut = 0; c.workspace = nullptr; c.bytes = 0; }) == TKV_OK && launched == 4);
    CHECK(prefill([](Prefill &c) { c.n_tokens = 1; c.q_stride = c.k_stride = c.v_stride = 0; }) == TKV_OK && launched == 5);
    CHECK(prefill([](Prefill &c) { c.q_stride = c.k_stride = c.v_stride = (1 << 23) - 8; }) == TKV_OK && launched == 6);
    CHECK(rows([](Rows &) {}) == TKV_OK && launched == 7);
    CHECK(rows([](Rows &c) { c.n_blocks = 0; c.blocks = nullptr; c.d.int2_key_axis = TKV_KEYS_PER_TOKEN; }) == TKV_OK && launched == 8);
    CHECK(distortion([](Distortion &) {}) == TKV_OK && launched == 9);
    CHECK(distortion([](Distortion &c) { c.n_tokens = 0; c.x = c.y = nullptr; }) == TKV_OK && launched == 10);
    // what has nothing to do
    CHECK(prefill([](Prefill &c) { c.n_tokens = 0; c.q = c.K = c.V = nullptr; c.out = nullptr; }) == TKV_OK);
    CHECK(prefill([](Prefill &c) { c.p.n_items = 0; c.p.items = nullptr; }) == TKV_OK);
    CHECK(rows([](Rows &c) { c.n_tokens = c.n_blocks = 0; c.K = c.V = nullptr; }) == TKV_OK);
    CHECK(distortion([](Distortion &c) { c.batch = 0; c.ip = nullptr; }) == TKV_OK);
    CHECK(distortion([](Distortion &c) { c.n_heads = 0; c.out = nullptr; }) == TKV_OK);
    CHECK(launched == 10);

    // what is refused
    CHECK(Prefill().call(false) == TKV_ERR_INVALID_ARG && Prefill().call(true, false) == TKV_ERR_INVALID_ARG);
    CHECK(prefill([](Prefill &c) { c.n_q_heads = 7; }) == TKV_ERR_BAD_SHAPE);
    CHECK(prefill([](Prefill &c) { c.d.n_kv_heads = c.n_q_heads = 65536; c.q_stride = c.k_stride = c.v_stride = 0; c.n_tokens = 1; }) == TKV_ERR_BAD_SHAPE);
    CHECK(prefill([](Prefill &c) { --c.bytes; }) == TKV_ERR_WORKSPACE_TOO_SMALL);
    const std::function<void(Prefill &)> bad_prefill[] = {
        [](Prefill &c) { c.n_q_heads = 0; }, [](Prefill &c) { c.n_tokens = -1; }, [](Prefill &c) { c.n_prefix = -1; }, [](Prefill &c) { c.p.n_items = -1; },
        [](Prefill &c) { c.p.n_slots = -1; }, [](Prefill &c) { c.p.n_cut = -1; }, [](Prefill &c) { c.p.n_cut = 4; }, [](Prefill &c) { c.p.n_items = 0x7fffffff; },
        [](Prefill &c) { c.p.n_cut = c.p.n_slots = 5; c.bytes *= 2; }, [](Prefill &c) { c.p.tile_rows = 64; }, [](Prefill &c) { c.p.items = nullptr; },
        [](Prefill &c) { c.p.items = (const int32_t *)((const char *)c.p.items + 2); }, [](Prefill &c) { c.q_type = TKV_FP32; }, [](Prefill &c) { c.kv_type = 3; },
        [](Prefill &c) { c.out_type = TKV_FP32; }, [](Prefill &c) { c.q_type = TKV_FP16; }, [](Prefill &c) { c.sm = 0.0f; }, [](Prefill &c) { c.sm = -1.0f; },
        [nan](Prefill &c) { c.sm = nan; }, [inf](Prefill &c) { c.sm = inf; }, [](Prefill &c) { c.q = nullptr; }, [](Prefill &c) { c.K = (const char *)c.K + 8; },
        [](Prefill &c) { c.V = nullptr; }, [](Prefill &c) { c.q_stride = 1016; }, [](Prefill &c) { c.k_stride = 260; }, [](Prefill &c) { c.v_stride = 1 << 23; },
        [](Prefill &c) { c.k_stride = -256; }, [](Prefill &c) { c.K_prefix = nullptr; }, [](Prefill &c) { c.V_prefix = (const char *)c.V_prefix + 2; },
        [](Prefill &c) { c.out = nullptr; }, [](Prefill &c) { c.out = (char *)c.out + 8; }, [](Prefill &c) { c.workspace = nullptr; }, [](Prefill &c) { c.workspace = (char *)c.workspace + 4; },
        [](Prefill &c) { c.status = (int32_t *)((char *)c.status + 1); }, [](Prefill &c) { c.n_tokens = 0x7fffffff; }};
    for (const auto &change : bad_prefill) CHECK(prefill(change) == TKV_ERR_INVALID_ARG);
    CHECK(rows([](Rows &c) { c.d.n_kv_heads = 0; }) == TKV_ERR_BAD_SHAPE);
    const std::function<void(Rows &)> bad_rows[] = {
        [](Rows &c) { c.n_tokens = -1; }, [](Rows &c) { c.n_blocks = -1; }, [](Rows &c) { c.n_blocks = 3; }, [](Rows &c) { c.blocks = nullptr; }, [](Rows &c) { c.K = nullptr; },
        [](Rows &c) { c.d.int2_key_axis = TKV_KEYS_PER_TOKEN; }, [](Rows &c) { c.V = (const char *)c.V + 8; }, [](Rows &c) { c.k_stride = 128; }, [](Rows &c) { c.v_stride = 516; },
        [](Rows &c) { c.bits = nullptr; }, [](Rows &c) { c.K_out = nullptr; }, [](Rows &c) { c.V_out = (char *)c.V_out + 4; }, [](Rows &c) { c.status = (int32_t *)(place + 1); },
        [](Rows &c) { c.blocks = (const int32_t *)(place + 2); }, [](Rows &c) { c.n_tokens = 0x7fffffff; }};
    for (const auto &change : bad_rows) CHECK(rows(change) == TKV_ERR_INVALID_ARG);
    CHECK(distortion([](Distortion &c) { --c.bytes; }) == TKV_ERR_WORKSPACE_TOO_SMALL);
    const std::function<void(Distortion &)> bad_distortion[] = {
        [](Distortion &c) { c.type = 3; }, [](Distortion &c) { c.batch = -1; }, [](Distortion &c) { c.n_tokens = -1; }, [](Distortion &c) { c.n_heads = -1; }, [](Distortion &c) { c.ip = nullptr; },
        [](Distortion &c) { c.ip = (const int32_t *)(place + 2); }, [](Distortion &c) { c.out = nullptr; }, [](Distortion &c) { c.out = (double *)(place + 4); }, [](Distortion &c) { c.x = nullptr; },
        [](Distortion &c) { c.y = (const char *)c.y + 8; }, [](Distortion &c) { c.workspace = nullptr; }, [](Distortion &c) { c.workspace = (char *)c.workspace + 8; },
        [](Distortion &c) { c.batch = c.n_heads = 65536; }, [](Distortion &c) { c.n_tokens = 0x7fffffff; }};
    for (const auto &change : bad_distortion) CHECK(distortion(change) == TKV_ERR_INVALID_ARG);
    CHECK(tkv_distortion_workspace_bytes(-1, 5, 5) == 0 && tkv_distortion_workspace_bytes(5, -1, 5) == 0 && tkv_distortion_workspace_bytes(5, 5, -1) == 0);
    CHECK(launched == 10);
    std::printf("host prompt calls ok\n");
    return 0;
}
