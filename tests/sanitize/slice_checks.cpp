// Host-side checks, under sanitizers, of which outputs of the norms of queries and keys may
// lie between each other: named layouts, and small random ones whose elements are counted.
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <random>
#include <set>

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

static char *P(int i) { return (char *)(uintptr_t)(0x100000000000ull + (uint64_t)i * (1ull << 40)); }

static sf_qk_shape shape(int B, int64_t L, int Hq, int Hk, int D) {
    sf_qk_shape s;
    std::memset(&s, 0, sizeof s);
    s.B = B, s.L = L, s.Hq = Hq, s.Hk = Hk, s.D = D, s.io_dtype = SF_BF16, s.norm = SF_NORM_L2;
    s.eps = 1e-6f, s.q_scale = 1.f;
    s.q = {L * Hq * D, (int64_t)Hq * D, D};
    s.k = {L * Hk * D, (int64_t)Hk * D, D};
    s.yq = s.dq = s.q, s.yk = s.dk = s.k;
    return s;
}
// outputs at element offsets oq, ok of one buffer
static sf_status fwd(const sf_qk_shape &s, int64_t oq, int64_t ok) {
    return sf_qk_norm_fwd(&s, P(1), P(2), nullptr, nullptr, nullptr, nullptr, P(3) + 2 * oq, P(3) + 2 * ok, nullptr, nullptr);
}
static sf_status bwd(const sf_qk_shape &s, int64_t oq, int64_t ok) {
    return sf_qk_norm_bwd(&s, P(1), P(2), nullptr, nullptr, nullptr, nullptr, P(4), P(5), P(3) + 2 * oq, P(3) + 2 * ok,
                          nullptr, nullptr, nullptr, 0, nullptr, nullptr);
}

int main() {
    sf::ServeRecord rec;
    sf::serve_record = &rec;
    const int B = 2, Hq = 4, Hk = 2, D = 128;
    const int64_t L = 10;
    {  // slices of one [B, Hq + Hk, L, D] buffer, seen as [B, L, H, D]
        sf_qk_shape s = shape(B, L, Hq, Hk, D);
        s.yq = s.yk = s.dq = s.dk = {(Hq + Hk) * L * D, D, L * D};
        EXPECT(fwd(s, 0, Hq * L * D) == SF_OK);
        EXPECT(fwd(s, Hk * L * D, 0) == SF_OK);
        EXPECT(bwd(s, 0, Hq * L * D) == SF_OK);
        EXPECT(fwd(s, 0, Hq * L * D - 8) == SF_E_ALIAS);
        EXPECT(fwd(s, 0, Hq * L * D + 8) == SF_E_ALIAS);  // into the next batch
        EXPECT(bwd(s, 0, (Hq - 1) * L * D) == SF_E_ALIAS);
    }
    {  // queries and keys in turn, head by head
        sf_qk_shape s = shape(B, L, Hk, Hk, D);
        s.yq = s.yk = {L * Hk * 2 * D, Hk * 2 * D, 2 * D};
        EXPECT(fwd(s, 0, D) == SF_OK);
        EXPECT(fwd(s, 0, D - 8) == SF_E_ALIAS);
        EXPECT(fwd(s, 0, D + 8) == SF_E_ALIAS);
    }
    {  // batches in turn, each a block of its own
        sf_qk_shape s = shape(B, L, Hk, Hk, D);
        s.yq = s.yk = {2 * L * Hk * D, Hk * D, D};
        EXPECT(fwd(s, 0, L * Hk * D) == SF_OK);
        EXPECT(fwd(s, 0, L * Hk * D - 8) == SF_E_ALIAS);
    }
    {  // a single token's stride may be anything
        sf_qk_shape s = shape(B, 1, Hq, Hk, D);
        s.yq = {(Hq + Hk) * D, INT64_MAX - 7, D}, s.yk = {(Hq + Hk) * D, 8, D};
        EXPECT(fwd(s, 0, Hq * D) == SF_OK);
        EXPECT(fwd(s, 0, Hq * D - 8) == SF_E_ALIAS);
    }
    // whatever is accepted shares no element
    std::mt19937 rng(1);
    auto pick = [&](int lo, int hi) { return (int64_t)std::uniform_int_distribution<int>(lo, hi)(rng); };
    int accepted = 0, between = 0, free_ = 0;
    for (int n = 0; n < 40000; ++n) {
        sf_qk_shape s = shape((int)pick(1, 3), pick(1, 3), (int)pick(1, 3), (int)pick(1, 3), 16);
        auto strides = [&]() -> sf_strides { return {8 * pick(1, 30), 8 * pick(1, 30), 8 * pick(1, 12)}; };
        s.yq = strides();
        s.yk = n % 4 ? s.yq : strides();
        if (n % 3 == 0) s.Hk = s.Hq, s.k = s.q;
        const int64_t ok = 8 * pick(0, 60), oq = 8 * pick(0, 10);
        std::set<int64_t> q, both;
        int64_t lo = INT64_MAX, hi = 0;
        size_t clash = 0;
        for (int b = 0; b < s.B; ++b)
            for (int l = 0; l < s.L; ++l) {
                for (int h = 0; h < s.Hq; ++h)
                    for (int c = 0; c < 16; c += 8) clash += !q.insert(oq + b * s.yq.b + l * s.yq.l + h * s.yq.h + c).second;
            }
        both = q;
        for (int b = 0; b < s.B; ++b)
            for (int l = 0; l < s.L; ++l)
                for (int h = 0; h < s.Hk; ++h)
                    for (int c = 0; c < 16; c += 8) {
                        const int64_t at = ok + b * s.yk.b + l * s.yk.l + h * s.yk.h + c;
                        clash += !both.insert(at).second;
                        lo = std::min(lo, at), hi = std::max(hi, at);
                    }
        const sf_status rc = fwd(s, oq, ok);
        EXPECT(rc == SF_OK || rc == SF_E_ALIAS || rc == SF_E_SHAPE);
        EXPECT(rc != SF_OK || clash == 0);
        free_ += clash == 0;
        accepted += rc == SF_OK;
        between += rc == SF_OK && lo < *q.rbegin() && hi > *q.begin();
    }
    std::printf("%d accepted of %d without a clash, %d of them between each other\n", accepted, free_, between);
    EXPECT(accepted > 1000 && between > 100);
    if (failures) return 1;
    std::printf("slice checks passed\n");
    return 0;
}
