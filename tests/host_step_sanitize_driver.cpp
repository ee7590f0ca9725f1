// Exercises csrc/tkv_host_step.cpp (rotation table, plan of shared prefixes, argument checks) under AddressSanitizer /
// UndefinedBehaviorSanitizer.  Built and run by tests/test_host_step_sanitizers.py with the host compiler only; the kernel
// launchers are stubs (nothing here needs a GPU).
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <vector>

#include "tkv.h"
#include "tkv_internal.h"

int tkv_launch_append(const tkv_desc *, void *, uint8_t *, const void *, const void *, const uint8_t *, int32_t,
                      const int32_t *, const int32_t *, int32_t, int32_t *, void *) { return TKV_OK; }
int tkv_launch_gather(const tkv_desc *, const void *, const uint8_t *, const int32_t *, const int32_t *, int32_t, void *,
                      void *, int32_t, int32_t *, void *) { return TKV_OK; }
int tkv_launch_probe_read(const void *, size_t, uint32_t *, void *) { return TKV_OK; }
int tkv_launch_probe_records(const tkv_desc *, const void *, const int32_t *, const int32_t *, const int32_t *, const int32_t *,
                             const int32_t *, int32_t, int32_t, int32_t, uint32_t *, void *) { return TKV_OK; }
int tkv_launch_probe_mix(const void *, void *, size_t, int32_t, int32_t, void *) { return TKV_OK; }
int tkv_launch_decode_split(const tkv_desc *, const void *, const uint8_t *, const void *, const int32_t *, const int32_t *,
                            const int32_t *, const int32_t *, const int32_t *, int32_t, int32_t, int32_t, float, void *,
                            int32_t *, void *) { return TKV_OK; }
int tkv_launch_decode_reduce(const tkv_desc *, const int32_t *, int32_t, int32_t, int32_t, float *, const void *, void *) { return TKV_OK; }
int tkv_launch_norm_rope(const tkv_rope *, const void *, int64_t, const void *, int64_t, const void *, int64_t, int32_t, int32_t, int32_t,
                         const int32_t *, const void *, const void *, float, void *, void *, void *, void *) { return TKV_OK; }
size_t tkv_table_words(int32_t n_seqs, int32_t n_tokens) { return (size_t)n_seqs + n_tokens; }
int tkv_launch_table_reset(const tkv_desc *, const tkv_table *, void *) { return TKV_OK; }
int tkv_launch_table_append(const tkv_desc *, const tkv_table *, const int32_t *, const int32_t *, const int32_t *, const uint8_t *, int32_t, int32_t *,
                            int32_t *, int32_t *, int32_t *, int32_t *, int32_t, int32_t *, void *, int32_t *, void *) { return TKV_OK; }
int tkv_launch_shared(const tkv_desc *, const void *, const uint8_t *, const void *, const int32_t *, const int32_t *, const int32_t *, const int32_t *,
                      const int32_t *, int32_t, const tkv_prefix *, const int32_t *, int32_t, int32_t, int32_t, float, void *, void *, int32_t *,
                      void *) { return TKV_OK; }

#define CHECK(x) do { if (!(x)) { std::printf("FAILED line %d: %s\n", __LINE__, #x); return 1; } } while (0)

static uint64_t rng_state = 88172645463325252ull;
static uint32_t rnd() { rng_state ^= rng_state << 13; rng_state ^= rng_state >> 7; rng_state ^= rng_state << 17; return (uint32_t)(rng_state >> 32); }

int main()
{
    for (int rotary = 0; rotary <= 128; rotary += 16)
        for (int axes = 1; axes <= 4; ++axes)
            for (int interleaved = 0; interleaved < 2; ++interleaved) {
                std::vector<int32_t> sections((size_t)axes, rotary / 2 / axes);
                sections[0] += rotary / 2 - rotary / 2 / axes * axes;
                std::vector<uint64_t> table((size_t)rotary / 2);
                CHECK(tkv_rope_table(rotary, axes, sections.data(), interleaved, 1e4, nullptr, table.data()) == TKV_OK);
                std::vector<double> f((size_t)rotary / 2);
                for (auto &x : f) x = ((int)(rnd() % 2000) - 1000) * 1e-2;
                CHECK(tkv_rope_table(rotary, axes, sections.data(), interleaved, 1e4, f.data(), table.data()) == TKV_OK);
                for (auto &x : f) x = (rnd() & 1 ? 1 : -1) * std::ldexp(1.0, (int)(rnd() % 2000) - 1000);
                CHECK(tkv_rope_table(rotary, axes, sections.data(), interleaved, 1e4, f.data(), table.data()) == TKV_OK);
            }
    for (int round = 0; round < 300; ++round) {
        const int batch = 1 + (int)(rnd() % 40), n = (int)(rnd() % 6), r = 1 << (rnd() % 4);
        tkv_desc d = {1 + (int)(rnd() % 8), 128, 32, 64, 100, 100, 0};
        std::vector<int32_t> n2, n4, indptr(1, 0), seqs;
        for (int g = 0; g < n; ++g) {
            n2.push_back((int32_t)(rnd() % 3 ? rnd() % 100000 : 0));
            n4.push_back((int32_t)(rnd() % 3 ? rnd() % 100000 : 0));
            for (int b = 0; b < batch; ++b)
                if (rnd() & 1) seqs.push_back(b);
            indptr.push_back((int32_t)seqs.size());
        }
        int32_t tile = 0;
        const int target = 1 + (int)(rnd() % 400), cap = tkv_plan_shared_capacity(n, (int)seqs.size(), target);
        std::vector<int32_t> items(5 * (size_t)cap), slots(seqs.size()), out((size_t)batch + 1);
        const int got = tkv_plan_decode_shared(&d, batch, d.n_kv_heads * r, n, n2.data(), n4.data(), indptr.data(), seqs.data(), target, 5, items.data(), cap,
                                               slots.data(), out.data(), &tile);
        CHECK(got >= 0 && got <= cap && out[0] == 5);
        if (got > 0)
            CHECK(tkv_plan_decode_shared(&d, batch, d.n_kv_heads * r, n, n2.data(), n4.data(), indptr.data(), seqs.data(), target, 5, items.data(), got - 1,
                                         slots.data(), out.data(), &tile) == TKV_ERR_CAPACITY);
    }
    CHECK(tkv_plan_shared_capacity(INT32_MAX, 0, INT32_MAX) == TKV_ERR_INVALID_ARG);
    CHECK(tkv_table_max_work(INT32_MAX, 1 << 28) == 1 << 28);
    CHECK(tkv_table_max_work(1 << 20, 1 << 28) == (1 << 22) + (1 << 22));
    std::printf("host step sanitizer run ok\n");
    return 0;
}
