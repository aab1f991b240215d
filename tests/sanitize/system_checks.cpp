// Host-side checks, under sanitizers, of how the ragged delta rule numbers its chunk
// systems: room for every chunk of every long sequence, none shared, a workgroup finds its
// sequence by the last first number at most its own, and short sequences cost no workspace;
// and of the largest launches.
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <random>
#include <vector>

#include "serve_stubs.hpp"
#include "stateflow.h"

static int failures = 0;
#define EXPECT(cond)                                                        \
    do {                                                                    \
        if (!(cond)) {                                                      \
            std::fprintf(stderr, "%s:%d: FAILED %s (%s)\n", __FILE__, __LINE__, #cond, sf_last_error()); \
            ++failures;                                                     \
        }                                                                   \
    } while (0)

static size_t workspace(int N, int64_t T, int64_t max_len, int Hv) {
    sf_gdn_ragged_shape s = {Hv, Hv, 128, 128, SF_BF16, 0, Hv * 128, 128, Hv * 128, 128, Hv * 128, 128, Hv, 1, Hv * 128 * 128};
    sf_ragged b = {N, N, T, max_len, (const int32_t *)(uintptr_t)0x1000, nullptr, nullptr};
    return sf_gdn_ragged_workspace_bytes(&s, &b);
}

int main() {
    // 1000 single tokens beside a prompt of 2000, 40 heads: systems of the tokens over 25, not of 1001 sequences
    EXPECT(workspace(1001, 3000, 2000, 40) <= (size_t)(3000 / 25) * 40 * sf::RAG_SYS + 4 * 1003);
    // prompts alone: a system for every 64 tokens and one a sequence
    EXPECT(workspace(8, 8192, 2000, 40) == (size_t)(8192 / 64 + 8) * 40 * sf::RAG_SYS + 4 * 10);
    // no sequence can be long
    EXPECT(workspace(4, 12, 4096, 1) == 0);
    EXPECT(workspace(300, 24, 4096, 40) == 0);
    std::mt19937 rng(7);
    auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
    int with_few = 0;
    for (int n = 0; n < 4000; ++n) {
        sf::GdnRaggedArgs a{};
        a.r.N = pick(1, 200);
        a.longer = n % 2 ? sf::RAG_LONG : sf::RAG_LONG_FEW;
        const int kind = pick(0, 2), top = kind == 0 ? 3 : kind == 1 ? 40 : 300;
        std::vector<int64_t> cu(a.r.N + 1, pick(0, 30));
        for (int i = 0; i < a.r.N; ++i) cu[i + 1] = cu[i] + (pick(0, 9) ? pick(0, top) : pick(0, 700));
        a.r.T = cu.back() + pick(0, 30);
        if (n % 5 == 0) std::shuffle(cu.begin(), cu.end(), rng);  // decreasing bounds: in range all the same
        const bool rising = std::is_sorted(cu.begin(), cu.end());
        sf::gdn_number(a);
        with_few += a.sys_add == 0;
        EXPECT(a.n_chunks <= a.r.T / 64 + a.r.N && a.n_chunks <= a.r.T / (a.longer + 1));
        std::vector<int> owner(a.n_chunks, -1);
        for (int i = 0; i < a.r.N; ++i) {
            const int64_t len = cu[i + 1] - cu[i], first = sf::gdn_first_system(a, cu[i], i);
            if (len <= a.longer) continue;
            for (int64_t c = 0; c < (len + 63) / 64; ++c) {
                EXPECT(first + c < a.n_chunks);
                if (first + c >= a.n_chunks || !rising) continue;
                EXPECT(owner[first + c] == -1);
                owner[first + c] = i;
            }
        }
        for (int64_t id = 0; rising && id < a.n_chunks; ++id) {
            int found = 0;
            for (int i = 0; i < a.r.N; ++i)
                if (sf::gdn_first_system(a, cu[i], i) <= id) found = i;
            EXPECT(owner[id] == -1 || owner[id] == found);
        }
    }
    // a launch holds fewer than 2^32 threads: more are refused before anything is launched
    for (int over = 0; over < 2; ++over) {
        sf::ServeRecord rec;
        sf::serve_record = over ? nullptr : &rec;
        auto at = [](uint64_t i) { return (void *)(uintptr_t)(i << 48); };
        sf_conv_ragged_shape c = {4096, 1, SF_BF16, SF_ACT_NONE, 0, 0, 4096, 0};
        const int N = over ? 1 << 23 : (1 << 23) - 8192;
        sf_ragged b = {N, 1, 64, 1, (const int32_t *)at(1), (const int32_t *)at(2), nullptr};
        EXPECT(sf_conv_ragged_fwd(&c, &b, at(3), (const float *)at(4), nullptr, at(5), nullptr, nullptr) ==
               (over ? SF_E_UNSUPPORTED : SF_OK));
        sf_gdn_ragged_shape s = {16, 16, 128, 128, SF_BF16, 0, 0, 0, 0, 0, 16 * 128, 128, 0, 0, 16 * 128 * 128};
        b.N = over ? 1 << 20 : (1 << 20) - 1024;
        EXPECT(sf_gdn_ragged_fwd(&s, &b, at(3), at(4), at(6), (const float *)at(7), (const float *)at(8), (float *)at(9),
                                 at(5), nullptr, 0, nullptr, nullptr) == (over ? SF_E_UNSUPPORTED : SF_OK));
    }
    EXPECT(with_few > 500 && with_few < 3500);
    if (failures) return 1;
    std::printf("system checks passed\n");
    return 0;
}
