// Exercises csrc/tkv_host_prompt.cpp (plan of prompt attention, blocks of per-channel keys, argument checks) under AddressSanitizer /
// UndefinedBehaviorSanitizer.  Built and run by tests/test_host_prompt_sanitizers.py with the host compiler only; the kernel launchers and
// the descriptor's check are stubs (nothing here needs a GPU).
#include <cstdint>
#include <cstdio>
#include <vector>

#include "tkv.h"
#include "tkv_internal.h"

int tkv_desc_status(const tkv_desc *d) { return !d ? TKV_ERR_INVALID_ARG : d->n_kv_heads > 0 ? TKV_OK : TKV_ERR_BAD_SHAPE; }
int tkv_launch_prefill(int32_t, int32_t, const void *, int64_t, int32_t, const void *, int64_t, const void *, int64_t, int32_t, int32_t, const void *, const void *, int32_t,
                       const tkv_prefill *, float, void *, int32_t, void *, int32_t *, void *) { return TKV_OK; }
int tkv_launch_quantize_rows(const tkv_desc *, const void *, int64_t, const void *, int64_t, const uint8_t *, int32_t, const int32_t *, int32_t, void *, void *, int32_t *, void *) { return TKV_OK; }
int tkv_launch_distortion(const void *, const void *, int32_t, const int32_t *, int32_t, int32_t, int32_t, double *, void *, void *) { return TKV_OK; }

#define CHECK(x) do { if (!(x)) { std::printf("FAILED line %d: %s\n", __LINE__, #x); return 1; } } while (0)

static uint64_t rng_state = 88172645463325252ull;
static uint32_t rnd() { rng_state ^= rng_state << 13; rng_state ^= rng_state >> 7; rng_state ^= rng_state << 17; return (uint32_t)(rng_state >> 32); }

int main()
{
    for (int round = 0; round < 300; ++round) {
        const int32_t hk = 1 << rnd() % 4, group = 1 + (int32_t)(rnd() % 9), batch = (int32_t)(rnd() % 20), cus = 1 + (int32_t)(rnd() % 300);
        tkv_desc d = {};
        d.n_kv_heads = hk;
        std::vector<int32_t> ip(1, 0), pp(1, 0);
        for (int32_t b = 0; b < batch; ++b) {
            ip.push_back(ip.back() + (int32_t)(rnd() % (round % 3 ? 40 : 3000)));
            pp.push_back(pp.back() + (int32_t)(rnd() % (round % 5 ? 500 : 100000)));
        }
        const int32_t cap = tkv_plan_prefill_capacity(&d, batch, ip.back(), hk * group, cus);
        CHECK(cap >= 0);
        std::vector<int32_t> items((size_t)cap * 16);
        int32_t rows = -1, slots = -1, cut = -1;
        const int32_t n = tkv_plan_prefill(&d, batch, hk * group, ip.data(), round % 2 ? pp.data() : nullptr, cus, items.data(), cap, &rows, &slots, &cut);
        CHECK(n >= 0 && n <= cap && (rows == 32 || rows == 128 || rows == 256) && slots >= 0 && cut >= 0 && 2 * cut <= slots);
        std::vector<char> used((size_t)slots, 0);
        for (int32_t k = 0; k < n; ++k) {
            const int32_t *it = &items[(size_t)k * 16];
            CHECK(it[5] < it[6] && it[8] >= 0 && it[8] < it[9] && (it[9] == 1) == (it[7] < 0));
            if (it[7] >= 0) CHECK(it[7] < slots && !used[(size_t)it[7]]++);
            CHECK(k < cut ? it[14] > 1 && it[13] >= 0 && it[13] + it[14] <= slots : it[14] == 0);
        }
        if (n > 0) CHECK(tkv_plan_prefill(&d, batch, hk * group, ip.data(), round % 2 ? pp.data() : nullptr, cus, items.data(), n - 1, &rows, &slots, &cut) == TKV_ERR_CAPACITY);
        // blocks
        std::vector<uint8_t> bits((size_t)ip.back(), 0);
        std::vector<int32_t> want;
        for (int32_t b = 0; b < batch; ++b)
            for (int32_t k = 0, left = (ip[(size_t)b + 1] - ip[(size_t)b]) / 32 * 32 / (1 + (int32_t)(rnd() % 3)) / 32 * 32; k < left; ++k) {
                bits[(size_t)(ip[(size_t)b + 1] - left + k)] = 2;
                want.push_back(ip[(size_t)b + 1] - left + k);
            }
        std::vector<int32_t> blocks(want.size());
        const int32_t nb = tkv_plan_row_blocks(bits.data(), ip.data(), batch, blocks.data(), (int32_t)want.size() / 32);
        CHECK(nb == (int32_t)want.size() / 32 && blocks == want);
    }
    CHECK(tkv_distortion_workspace_bytes(3, 100, 5) >= 8u * 5 * (100 / 16 + 3));
    std::printf("host prompt sanitizer run ok\n");
    return 0;
}
