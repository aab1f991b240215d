// Host-side checks of the ragged-batch calls and of the norms of queries and keys under
// AddressSanitizer and UndefinedBehaviorSanitizer: refused calls reach no launch (fake
// device pointers, never dereferenced), accepted ones hand the kernels a plan that fits
// the arguments.
#include <climits>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>

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

static void *P(int i) { return (void *)(uintptr_t)(0x100000000000ull + (uint64_t)i * (1ull << 46)); }
static float *F(int i) { return (float *)P(i); }

struct Gdn {
    sf_gdn_ragged_shape s;
    sf_ragged b;
    void *q = P(1), *k = P(2), *v = P(3), *o = P(7), *ws = P(8);
    float *g = F(4), *beta = F(5), *state = F(6);
    size_t ws_bytes = (size_t)1 << 39;
    const sf_tuning *t = nullptr;
    Gdn() {
        s = {4, 8, 128, 128, SF_BF16, 0, 512, 128, 1024, 128, 1024, 128, 8, 1, 8 * 128 * 128};
        b = {3, 5, 100, 90, (const int32_t *)P(9), (const int32_t *)P(10), (const uint8_t *)P(11)};
    }
    sf_status run() const { return sf_gdn_ragged_fwd(&s, &b, q, k, v, g, beta, state, o, ws, ws_bytes, t, nullptr); }
};
struct Conv {
    sf_conv_ragged_shape s;
    sf_ragged b;
    void *x = P(1), *y = P(2);
    float *w = F(3), *tails = F(4);
    Conv() {
        s = {256, 4, SF_BF16, SF_ACT_SILU, 0, 256, 256, 3 * 256};
        b = {3, 5, 100, 90, (const int32_t *)P(9), (const int32_t *)P(10), (const uint8_t *)P(11)};
    }
    sf_status run() const { return sf_conv_ragged_fwd(&s, &b, x, w, tails, y, nullptr, nullptr); }
};
struct Qk {
    sf_qk_shape s;
    void *q = P(1), *k = P(2), *yq = P(3), *yk = P(4), *dq = P(5), *dk = P(6), *ws = P(7);
    float *wq = F(8), *wk = F(9), *dwq = F(10), *dwk = F(11);
    const double *f = (const double *)P(12);
    const int64_t *pos = (const int64_t *)P(13);
    size_t ws_bytes = 1 << 30;
    Qk() {
        std::memset(&s, 0, sizeof s);
        s.B = 2, s.L = 10, s.Hq = 4, s.Hk = 2, s.D = 128, s.io_dtype = SF_BF16, s.norm = SF_NORM_RMS, s.R = 64;
        s.eps = 1e-6f, s.q_scale = 1.f, s.sp_b = 10, s.sp_l = 1;
        s.q = s.yq = s.dq = {10 * 512, 512, 128};
        s.k = s.yk = s.dk = {10 * 256, 256, 128};
    }
    sf_status fwd() const { return sf_qk_norm_fwd(&s, q, k, wq, wk, f, pos, yq, yk, nullptr, nullptr); }
    sf_status bwd() const {
        return sf_qk_norm_bwd(&s, q, k, wq, wk, f, pos, yq, yk, dq, dk, dwq, dwk, ws, ws_bytes, nullptr, nullptr);
    }
};

#define REFUSED(T, call, status, ...) \
    {                                 \
        T c;                          \
        __VA_ARGS__;                  \
        EXPECT(c.call() == status);   \
        EXPECT(status == SF_OK || sf_last_error()[0]); \
    }

int main() {
    // ---- gated delta rule: refusals
    EXPECT(sf_gdn_ragged_fwd(nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr,
                             0, nullptr, nullptr) == SF_E_NULL);
    REFUSED(Gdn, run, SF_E_SHAPE, c.s.Hk = 3)
    REFUSED(Gdn, run, SF_E_SHAPE, c.s.Hk = 0)
    REFUSED(Gdn, run, SF_E_SHAPE, c.s.Hv = -8)
    REFUSED(Gdn, run, SF_E_UNSUPPORTED, c.s.Dk = 96)
    REFUSED(Gdn, run, SF_E_UNSUPPORTED, c.s.Dv = 32)
    REFUSED(Gdn, run, SF_E_DTYPE, c.s.io_dtype = 2)
    REFUSED(Gdn, run, SF_E_SHAPE, c.s.reserved = 1)
    REFUSED(Gdn, run, SF_E_SHAPE, c.b.N = -1)
    REFUSED(Gdn, run, SF_E_SHAPE, c.b.T = -1)
    REFUSED(Gdn, run, SF_E_SHAPE, c.b.max_len = -1)
    REFUSED(Gdn, run, SF_E_SHAPE, c.b.n_slots = -1)
    REFUSED(Gdn, run, SF_E_UNSUPPORTED, c.b.T = INT64_MAX)
    REFUSED(Gdn, run, SF_E_UNSUPPORTED, c.b.T = (int64_t)1 << 31)
    REFUSED(Gdn, run, SF_E_NULL, c.b.cu = nullptr)
    REFUSED(Gdn, run, SF_E_ALIGN, c.b.cu = (const int32_t *)((const char *)c.b.cu + 2))
    REFUSED(Gdn, run, SF_E_SHAPE, c.b.slot = nullptr; c.b.n_slots = 2)
    REFUSED(Gdn, run, SF_E_NULL, c.q = nullptr)
    REFUSED(Gdn, run, SF_E_NULL, c.state = nullptr)
    REFUSED(Gdn, run, SF_E_NULL, c.beta = nullptr)
    REFUSED(Gdn, run, SF_E_NULL, c.o = nullptr)
    REFUSED(Gdn, run, SF_E_ALIGN, c.v = (char *)c.v + 8)
    REFUSED(Gdn, run, SF_E_ALIGN, c.state = c.state + 2)
    REFUSED(Gdn, run, SF_E_ALIGN, c.g = (float *)((char *)c.g + 2))
    REFUSED(Gdn, run, SF_E_SHAPE, c.s.sq_t = -512)
    REFUSED(Gdn, run, SF_E_ALIGN, c.s.sq_t = 516)
    REFUSED(Gdn, run, SF_E_SHAPE, c.s.sv_t = INT64_MAX - 7)
    REFUSED(Gdn, run, SF_E_SHAPE, c.s.so_t = 0)
    REFUSED(Gdn, run, SF_E_SHAPE, c.s.so_t = 512)
    REFUSED(Gdn, run, SF_E_SHAPE, c.s.ss = 100)
    REFUSED(Gdn, run, SF_E_SHAPE, c.s.ss = INT64_MAX / 4 * 4)
    REFUSED(Gdn, run, SF_E_ALIGN, c.s.ss += 2)
    REFUSED(Gdn, run, SF_E_ALIAS, c.o = c.v)
    REFUSED(Gdn, run, SF_E_ALIAS, c.o = c.state)
    REFUSED(Gdn, run, SF_E_ALIAS, c.state = (float *)c.k)
    REFUSED(Gdn, run, SF_E_ALIAS, c.state = (float *)c.b.slot)
    REFUSED(Gdn, run, SF_E_UNSUPPORTED, c.b.N = INT_MAX; c.s.Hv = 400; c.s.sv_h = c.s.sg_h = 0; c.b.slot = (const int32_t *)P(30);
            c.s.so_t = 400 * 128; c.s.ss = 400 * 128 * 128; c.b.fresh = nullptr; c.b.max_len = 1)
    {
        sf_tuning t;
        std::memset(&t, 0, sizeof t);
        t.overlap = 9;
        REFUSED(Gdn, run, SF_E_SHAPE, c.t = &t)
    }
    // nothing to do: no launch
    REFUSED(Gdn, run, SF_OK, c.b.N = 0; c.b.cu = nullptr)
    REFUSED(Gdn, run, SF_OK, c.b.T = 0; c.q = c.k = c.v = c.o = nullptr)
    REFUSED(Gdn, run, SF_OK, c.b.n_slots = 0; c.state = nullptr)
    // ---- convolution
    REFUSED(Conv, run, SF_E_UNSUPPORTED, c.s.C = 12)
    REFUSED(Conv, run, SF_E_UNSUPPORTED, c.s.C = 0)
    REFUSED(Conv, run, SF_E_UNSUPPORTED, c.s.W = 5)
    REFUSED(Conv, run, SF_E_UNSUPPORTED, c.s.W = 0)
    REFUSED(Conv, run, SF_E_DTYPE, c.s.act = 2)
    REFUSED(Conv, run, SF_E_DTYPE, c.s.io_dtype = -1)
    REFUSED(Conv, run, SF_E_SHAPE, c.s.reserved = 1)
    REFUSED(Conv, run, SF_E_SHAPE, c.s.sy_t = 128)
    REFUSED(Conv, run, SF_E_ALIGN, c.s.sx_t = 257)
    REFUSED(Conv, run, SF_E_SHAPE, c.s.ss = 256)
    REFUSED(Conv, run, SF_E_ALIGN, c.s.ss = 769)
    REFUSED(Conv, run, SF_E_NULL, c.tails = nullptr)
    REFUSED(Conv, run, SF_E_NULL, c.w = nullptr)
    REFUSED(Conv, run, SF_E_ALIGN, c.tails += 1)
    REFUSED(Conv, run, SF_E_ALIAS, c.y = c.x)
    REFUSED(Conv, run, SF_E_ALIAS, c.tails = (float *)c.y)
    REFUSED(Conv, run, SF_E_ALIAS, c.w = c.tails)
    REFUSED(Conv, run, SF_OK, c.b.T = 0)
    // ---- norms
    EXPECT(sf_qk_norm_fwd(nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr,
                          nullptr) == SF_E_NULL);
    EXPECT(sf_qk_norm_bwd_workspace_bytes(nullptr, 1) == 0);
    REFUSED(Qk, fwd, SF_E_UNSUPPORTED, c.s.D = 120)
    REFUSED(Qk, fwd, SF_E_UNSUPPORTED, c.s.D = 272)
    REFUSED(Qk, fwd, SF_E_UNSUPPORTED, c.s.R = 24)
    REFUSED(Qk, fwd, SF_E_UNSUPPORTED, c.s.R = 144)
    REFUSED(Qk, fwd, SF_E_DTYPE, c.s.norm = 3)
    REFUSED(Qk, fwd, SF_E_DTYPE, c.s.interleaved = 2)
    REFUSED(Qk, fwd, SF_E_SHAPE, c.s.eps = 0.f)
    REFUSED(Qk, fwd, SF_E_SHAPE, c.s.eps = NAN)
    REFUSED(Qk, fwd, SF_E_SHAPE, c.s.q_scale = INFINITY)
    REFUSED(Qk, fwd, SF_E_SHAPE, c.s.Hk = 0)
    REFUSED(Qk, fwd, SF_E_SHAPE, c.s.L = -1)
    REFUSED(Qk, fwd, SF_E_UNSUPPORTED, c.s.B = INT_MAX; c.s.L = INT64_MAX)
    REFUSED(Qk, fwd, SF_E_NULL, c.wk = nullptr)
    REFUSED(Qk, fwd, SF_E_NULL, c.f = nullptr)
    REFUSED(Qk, fwd, SF_E_ALIGN, c.pos = (const int64_t *)((const char *)c.pos + 4))
    REFUSED(Qk, fwd, SF_E_NULL, c.yk = nullptr)
    REFUSED(Qk, fwd, SF_E_ALIGN, c.q = (char *)c.q + 8)
    REFUSED(Qk, fwd, SF_E_ALIGN, c.s.q.l = 513)
    REFUSED(Qk, fwd, SF_E_SHAPE, c.s.k.h = -128)
    REFUSED(Qk, fwd, SF_E_SHAPE, c.s.yq.h = 64)
    REFUSED(Qk, fwd, SF_E_SHAPE, c.s.yq.b = 0)
    REFUSED(Qk, fwd, SF_E_ALIAS, c.yq = c.q)
    REFUSED(Qk, fwd, SF_E_ALIAS, c.yk = c.yq)
    REFUSED(Qk, fwd, SF_E_ALIAS, c.wq = (float *)c.yk)
    REFUSED(Qk, bwd, SF_E_NULL, c.dwk = nullptr)
    REFUSED(Qk, bwd, SF_E_NULL, c.dq = nullptr)
    REFUSED(Qk, bwd, SF_E_WORKSPACE, c.ws_bytes = 16)
    REFUSED(Qk, bwd, SF_E_WORKSPACE, c.ws = nullptr)
    REFUSED(Qk, bwd, SF_E_ALIGN, c.dwq = (float *)((char *)c.dwq + 1))
    REFUSED(Qk, bwd, SF_E_ALIAS, c.dwq = c.dwk)
    REFUSED(Qk, bwd, SF_E_ALIAS, c.dq = c.yq)
    REFUSED(Qk, bwd, SF_E_ALIAS, c.ws = c.dk)
    REFUSED(Qk, bwd, SF_E_SHAPE, c.s.dk.l = 128)
    REFUSED(Qk, fwd, SF_OK, c.s.L = 0)
    // slices of one row lie side by side; one channel further they clash
    const sf_strides wide = {10 * 1024, 1024, 128};
    sf::ServeRecord rec;
    sf::serve_record = &rec;
    REFUSED(Qk, fwd, SF_OK, c.s.yq = c.s.yk = wide; c.yk = (char *)c.yq + 4 * 128 * 2)
    REFUSED(Qk, fwd, SF_OK, c.s.yq = c.s.yk = wide; c.yk = c.yq; c.yq = (char *)c.yk + 2 * 128 * 2)
    REFUSED(Qk, bwd, SF_OK, c.s.dq = c.s.dk = c.s.q = wide; c.dk = (char *)c.dq + 512 * 2; c.q = (char *)c.dq + 768 * 2;
            c.s.Hq = 2; c.s.yq = {10 * 512, 512, 128})
    REFUSED(Qk, fwd, SF_E_ALIAS, c.s.yq = c.s.yk = wide; c.yk = (char *)c.yq + 4 * 128 * 2 - 16)
    REFUSED(Qk, fwd, SF_E_ALIAS, c.s.yq = c.s.yk = wide; c.yk = (char *)c.yq + 6 * 128 * 2 + 16)
    // batches inside a token's row: its heads of all batches must stay clear of each other
    REFUSED(Qk, fwd, SF_OK, c.s.B = 2; c.s.yq = c.s.yk = {1024, 4096, 128}; c.yk = (char *)c.yq + 4 * 128 * 2)
    REFUSED(Qk, fwd, SF_E_ALIAS, c.s.B = 2; c.s.yq = c.s.yk = {768, 4096, 128}; c.yk = (char *)c.yq + 768 * 2)
    REFUSED(Qk, fwd, SF_E_ALIAS, c.s.B = 2; c.s.L = 1; c.s.yq = c.s.yk = {768, 4096, 128}; c.yk = (char *)c.yq + 768 * 2)
    // a single token's stride means nothing
    REFUSED(Qk, fwd, SF_OK, c.s.B = 2; c.s.L = 1; c.s.yq = {1024, 0, 128}; c.s.yk = {1024, 8, 128}; c.yk = (char *)c.yq + 512 * 2)
    rec = {};

    // ---- accepted calls
    REFUSED(Gdn, run, SF_OK, )
    REFUSED(Gdn, run, SF_OK, c.s.sq_t = c.s.sq_h = c.s.sv_t = c.s.sv_h = c.s.sg_t = c.s.sg_h = 0)  // broadcast inputs
    REFUSED(Gdn, run, SF_OK, c.b.n_slots = 1; c.s.ss = 0)
    // a long sequence: the systems and the plan, then the walk with the other tokens
    EXPECT(rec.gdn.empty() && rec.prep.size() == 3 && rec.walk.size() == 3);
    EXPECT(rec.walk[0].Hv == 8 && rec.walk[0].r.N == 3 && rec.walk[1].sq_t == 0);
    EXPECT(rec.walk[0].n_chunks == 100 / 64 + 3 && rec.walk[0].longer == sf::RAG_LONG_FEW);
    EXPECT(sf::gdn_token_waves(rec.walk[0]) == 3 * 8 * 4);
    {
        Gdn c;
        const size_t need = sf_gdn_ragged_workspace_bytes(&c.s, &c.b);
        EXPECT(need == (size_t)4 * 8 * sf::RAG_SYS + 4 * 5);
        EXPECT((char *)rec.walk[0].plan == rec.walk[0].ws + 4 * 8 * sf::RAG_SYS);
        c.ws_bytes = need;
        EXPECT(c.run() == SF_OK);
        c.ws_bytes = need - 1;
        EXPECT(c.run() == SF_E_WORKSPACE);
        c.ws_bytes = need, c.ws = (char *)c.ws + 8;
        EXPECT(c.run() == SF_E_ALIGN);
        c.ws = c.o;
        EXPECT(c.run() == SF_E_ALIAS);
        c.ws = nullptr;
        EXPECT(c.run() == SF_E_WORKSPACE);
        c.b.max_len = sf::RAG_LONG_FEW;  // token by token: no workspace
        EXPECT(sf_gdn_ragged_workspace_bytes(&c.s, &c.b) == 0 && c.run() == SF_OK);
        c.b.max_len = 90, c.s.io_dtype = SF_F32;
        EXPECT(sf_gdn_ragged_workspace_bytes(&c.s, &c.b) == 0 && c.run() == SF_OK);
        c.s.io_dtype = SF_BF16, c.s.sq_t = 1 << 23;  // 64 rows of 1 GiB: token by token
        EXPECT(sf_gdn_ragged_workspace_bytes(&c.s, &c.b) == 0 && c.run() == SF_OK);
        EXPECT(rec.prep.size() == 4 && rec.gdn.size() == 3 && rec.gdn[2].longer == 0);
    }
    // every item has a workgroup or follows one, whatever the sizes; columns cover Dv
    for (int N : {1, 7, 3000})
        for (int Hv : {1, 3, 40})
            for (int Dv : {64, 128, 256})
                for (int nc : {1, 2}) {
                    sf::GdnRaggedArgs a = rec.walk[0];
                    a.r.N = N, a.Hv = Hv, a.Dv = Dv;
                    const int64_t items = sf::gdn_walk_items(a, N, nc), groups = sf::gdn_walk_groups(a);
                    EXPECT(groups % 8 == 0 && groups >= 8 && (groups >= items || groups == 8 * a.n_cu));
                    EXPECT(items % (8 * (Dv / (16 * nc))) == 0 && items >= (int64_t)N * Hv * (Dv / (16 * nc)));
                }
    // chunk numbers stay below n_chunks whatever the bounds, decreasing ones too
    for (int b = 0; b <= 200; ++b)
        for (int e = b + 1; e <= 200; ++e) EXPECT(b / 64 + 4 + (e - b + 63) / 64 <= 200 / 64 + 5);
    REFUSED(Conv, run, SF_OK, )
    REFUSED(Conv, run, SF_OK, c.s.W = 1; c.tails = nullptr; c.s.ss = 0)
    for (const auto &a : rec.conv)  // every run of every sequence has a number below n_runs
        for (int n0 = 0; n0 <= 100; n0 += 7) {
            const int cu[4] = {n0 / 3, n0 / 2, n0, 100};
            for (int i = 0; i < 3; ++i) {
                const int runs = (cu[i + 1] - cu[i] + a.run - 1) / a.run, base = cu[i] / a.run + i;
                EXPECT(base + runs <= (i < 2 ? cu[i + 1] / a.run + i + 1 : a.n_runs));
            }
        }
    for (int n : {1, 3, 1000, 1 << 20, 1 << 30})
        for (int Hq : {1, 5, 40})
            for (int D : {16, 96, 256}) {
                Qk c;
                c.s.B = 1, c.s.L = n, c.s.Hq = Hq, c.s.Hk = 1, c.s.D = D, c.s.R = 16;
                c.s.q = c.s.yq = c.s.dq = {0, (int64_t)Hq * D, D};
                c.s.k = c.s.yk = c.s.dk = {0, D, D};
                c.ws_bytes = sf_qk_norm_bwd_workspace_bytes(&c.s, 1);
                EXPECT(sf_qk_norm_bwd_workspace_bytes(&c.s, 0) == 0);
                EXPECT(c.fwd() == SF_OK && c.bwd() == SF_OK);
                const sf::QkArgs &a = rec.qk.back().second;
                EXPECT(rec.qk.back().first && a.blocks >= 1 && a.parts >= 1);
                EXPECT(c.ws_bytes == (size_t)a.blocks * 2 * D * 4);
                EXPECT(a.blocks <= 4 * 256 && a.parts <= 2 * Hq + 2);
            }
    if (failures) return 1;
    std::printf("serve checks passed\n");
    return 0;
}
