// sf_abi_serve.hip -- host side of the ragged-batch calls (gated delta rule, short
// convolution) and of the norms of queries and keys: argument checks, workspace
// sizes, launches.
#include <climits>
#include <cmath>

#include "sf_host.hpp"
#include "sf_launch.hpp"
#include "stateflow.h"

namespace {

using namespace sf::host;

size_t elem_size(int io) { return io == SF_BF16 ? 2 : 4; }

// No C++ exception (an allocation that fails inside a check) leaves an entry point.
template <typename F>
sf_status guarded(F f) {
    try {
        g_err.clear();
        return f();
    } catch (...) {
        return SF_E_HIP;
    }
}

sf_status check_io(int io) {
    return io == SF_F32 || io == SF_BF16 ? SF_OK : fail(SF_E_DTYPE, "unknown io_dtype %d", io);
}

// an input's strides: not negative, 16-byte multiples, no address beyond 2^62 bytes
sf_status check_in(const char *name, std::initializer_list<Dim> dims, size_t esz, int64_t step = 16) {
    double last = 0;
    for (const Dim &d : dims) {
        if (d.stride < 0) return fail(SF_E_SHAPE, "%s: strides must not be negative", name);
        if (d.size > 1 && (d.stride % (step / std::min<int64_t>(step, (int64_t)esz))))
            return fail(SF_E_ALIGN, "%s: strides must be multiples of %lld bytes", name, (long long)step);
        if (d.size > 1) last += (double)(d.size - 1) * (double)d.stride;
    }
    return last * (double)esz < 4e18 ? SF_OK : fail(SF_E_SHAPE, "%s: strides too large", name);
}
sf_status check_out(const char *name, std::initializer_list<Dim> dims, int64_t inner, size_t esz) {
    TRY(check_in(name, dims, esz));
    return non_overlapping(dims, inner) ? SF_OK : fail(SF_E_SHAPE, "%s: strides make elements overlap", name);
}
Range strided(const void *p, std::initializer_list<Dim> dims, int64_t inner, size_t esz, const char *name) {
    int64_t last = inner;
    for (const Dim &d : dims) {
        if (d.size <= 0) return span(p, 0, name);
        last += (d.size - 1) * d.stride;
    }
    return span(p, last * (int64_t)esz, name);
}

sf_status check_batch(const sf_ragged *b) {
    if (!b) return fail(SF_E_NULL, "batch is NULL");
    if (b->N < 0 || b->T < 0 || b->n_slots < 0 || b->max_len < 0)
        return fail(SF_E_SHAPE, "need N, n_slots, T, max_len >= 0 (got %d, %d, %lld, %lld)", b->N, b->n_slots,
                    (long long)b->T, (long long)b->max_len);
    if (b->T > INT32_MAX) return fail(SF_E_UNSUPPORTED, "T must be below 2^31 (got %lld)", (long long)b->T);
    if (b->N > 0 && !b->cu) return fail(SF_E_NULL, "batch.cu is required");
    if ((uintptr_t)b->cu % 4 || (uintptr_t)b->slot % 4) return fail(SF_E_ALIGN, "cu and slot must be 4-byte aligned");
    if (!b->slot && b->n_slots < b->N)
        return fail(SF_E_SHAPE, "without a slot list every sequence needs its own slot (N = %d, n_slots = %d)", b->N,
                    b->n_slots);
    return SF_OK;
}
sf::RaggedArgs ragged_args(const sf_ragged &b) { return {b.cu, b.slot, b.fresh, b.N, b.n_slots, b.T}; }
Range cu_range(const sf_ragged &b) { return span(b.cu, 4 * ((int64_t)b.N + 1), "cu"); }
Range slot_range(const sf_ragged &b) { return span(b.slot, 4 * (int64_t)b.N, "slot"); }
Range fresh_range(const sf_ragged &b) { return span(b.fresh, b.N, "fresh"); }

// slots of `per` floats, ss apart
sf_status check_pool(const char *name, const float *p, int32_t n_slots, int64_t per, int64_t ss, bool used) {
    if (used && n_slots > 0 && !p) return fail(SF_E_NULL, "%s is required", name);
    if (n_slots > 1 && (ss < per || (double)ss * n_slots > 1e18))
        return fail(SF_E_SHAPE, "%s: slots overlap or lie too far apart", name);
    if (n_slots > 1 && ss % 4) return fail(SF_E_ALIGN, "%s: the slot stride must be a multiple of 4", name);
    return SF_OK;
}
Range pool_range(const char *name, const float *p, int32_t n_slots, int64_t per, int64_t ss) {
    return span(p, n_slots > 0 ? 4 * ((n_slots - 1) * ss + per) : 0, name);
}

// a launch counts its threads in 32 bits
sf_status grid_fits(double threads) {
    return threads < 4294967296.0 ? SF_OK : fail(SF_E_UNSUPPORTED, "batch too large for one call");
}
sf_status launched(hipError_t e) { return e == hipSuccess ? SF_OK : hip_fail(e, "kernel launch"); }

// ------------------------------------------------------------- gated delta rule
sf_status check_gdn(const sf_gdn_ragged_shape *s, const sf_ragged *b) {
    if (!s) return fail(SF_E_NULL, "shape is NULL");
    TRY(check_batch(b));
    TRY(check_io(s->io_dtype));
    if (s->reserved != 0) return fail(SF_E_SHAPE, "shape.reserved must be 0");
    if (s->Hk < 1 || s->Hv < 1 || s->Hv % s->Hk)
        return fail(SF_E_SHAPE, "Hk must divide Hv (got Hk = %d, Hv = %d)", s->Hk, s->Hv);
    if (s->Dk != 64 && s->Dk != 128) return fail(SF_E_UNSUPPORTED, "supported Dk: 64, 128 (got %d)", s->Dk);
    if (s->Dv != 64 && s->Dv != 128 && s->Dv != 256)
        return fail(SF_E_UNSUPPORTED, "supported Dv: 64, 128, 256 (got %d)", s->Dv);
    const size_t e = elem_size(s->io_dtype);
    TRY(check_in("q, k", {{b->T, s->sq_t}, {s->Hk, s->sq_h}}, e));
    TRY(check_in("v", {{b->T, s->sv_t}, {s->Hv, s->sv_h}}, e));
    TRY(check_in("g, beta", {{b->T, s->sg_t}, {s->Hv, s->sg_h}}, 4, 4));
    return check_out("o", {{b->T, s->so_t}, {s->Hv, s->so_h}}, s->Dv, e);
}

sf::GdnRaggedArgs gdn_args(const sf_gdn_ragged_shape &s, const sf_ragged &b) {
    sf::GdnRaggedArgs a{};
    a.r = ragged_args(b);
    a.Hk = s.Hk;
    a.Hv = s.Hv;
    a.Dk = s.Dk;
    a.Dv = s.Dv;
    a.io = s.io_dtype;
    a.n_cu = device_cus();
    a.sq_t = s.sq_t;
    a.sq_h = s.sq_h;
    a.sv_t = s.sv_t;
    a.sv_h = s.sv_h;
    a.so_t = s.so_t;
    a.so_h = s.so_h;
    a.sg_t = s.sg_t;
    a.sg_h = s.sg_h;
    a.ss = s.ss;
    // Long sequences are taken in chunks where the operands are bf16, the host knows of
    // such a sequence and 64 rows span less than 2 GiB (the walk's offsets inside a chunk
    // are 32 bits); fp32 operands go token by token.
    const int few = sf::gdn_long(a);
    if (s.io_dtype == SF_BF16 && std::min(b.max_len, b.T) > few && std::max(s.sq_t, s.sv_t) < (int64_t)1 << 23) a.longer = few;
    sf::gdn_number(a);
    return a;
}
size_t gdn_ragged_ws_bytes(const sf_gdn_ragged_shape &s, const sf_ragged &b) {
    if (b.N == 0 || b.T == 0) return 0;
    const sf::GdnRaggedArgs a = gdn_args(s, b);
    return a.longer ? sf::gdn_chunk_ws_bytes(a) : 0;
}

// ------------------------------------------------------------- norms and rotation
sf_status check_qk(const sf_qk_shape *s, bool bwd) {
    if (!s) return fail(SF_E_NULL, "shape is NULL");
    TRY(check_io(s->io_dtype));
    if (s->B < 0 || s->L < 0 || s->Hq < 1 || s->Hk < 1)
        return fail(SF_E_SHAPE, "need B, L >= 0 and Hq, Hk >= 1 (got %d, %lld, %d, %d)", s->B, (long long)s->L, s->Hq,
                    s->Hk);
    if (s->norm != SF_NORM_NONE && s->norm != SF_NORM_L2 && s->norm != SF_NORM_RMS)
        return fail(SF_E_DTYPE, "unknown norm %d", s->norm);
    if (s->interleaved != 0 && s->interleaved != 1) return fail(SF_E_DTYPE, "interleaved must be 0 or 1");
    if (s->D < 16 || s->D > 256 || s->D % 16)
        return fail(SF_E_UNSUPPORTED, "D must be a multiple of 16 from 16 to 256 (got %d)", s->D);
    if (s->R < 0 || s->R > s->D || s->R % 16)
        return fail(SF_E_UNSUPPORTED, "R must be a multiple of 16 from 0 to D (got %d)", s->R);
    if (s->norm != SF_NORM_NONE && !(s->eps >= 1.17549435e-38f && std::isfinite(s->eps)))
        return fail(SF_E_SHAPE, "eps must be positive and finite");
    if (!std::isfinite(s->q_scale)) return fail(SF_E_SHAPE, "q_scale must be finite");
    if ((double)s->B * (double)s->L >= 2147483647.0) return fail(SF_E_UNSUPPORTED, "B * L must be below 2^31");
    const size_t e = elem_size(s->io_dtype);
    auto dims = [&](const sf_strides &t, int H, const char *name, bool out) -> sf_status {
        return out ? check_out(name, {{s->B, t.b}, {s->L, t.l}, {H, t.h}}, s->D, e)
                   : check_in(name, {{s->B, t.b}, {s->L, t.l}, {H, t.h}}, e);
    };
    TRY(dims(s->q, s->Hq, "q", false));
    TRY(dims(s->k, s->Hk, "k", false));
    TRY(dims(s->yq, s->Hq, bwd ? "dyq" : "yq", !bwd));
    TRY(dims(s->yk, s->Hk, bwd ? "dyk" : "yk", !bwd));
    if (bwd) {
        TRY(dims(s->dq, s->Hq, "dq", true));
        TRY(dims(s->dk, s->Hk, "dk", true));
    }
    return check_in("pos", {{s->B, s->sp_b}, {s->L, s->sp_l}}, 8, 8);
}

sf::QkArgs qk_args(const sf_qk_shape &s, bool bwd, bool weights) {
    sf::QkArgs a{};
    a.B = s.B;
    a.Hq = s.Hq;
    a.Hk = s.Hk;
    a.D = s.D;
    a.io = s.io_dtype;
    a.norm = s.norm;
    a.R = s.R;
    a.inter = s.interleaved;
    a.eps = s.eps;
    a.q_scale = s.q_scale;
    a.n_tok = (int32_t)(s.B * s.L);
    a.L = s.L;
    a.pos0 = s.pos0;
    a.sp_b = s.sp_b;
    a.sp_l = s.sp_l;
    a.sq = s.q;
    a.sk = s.k;
    a.syq = bwd ? s.dq : s.yq;
    a.syk = bwd ? s.dk : s.yk;
    a.sdyq = s.yq;
    a.sdyk = s.yk;
    sf::qk_plan(a, bwd, weights, device_cus());
    return a;
}
// a workgroup's part of dwq and dwk, for every workgroup
size_t qk_ws_bytes(const sf_qk_shape &s, bool weights) {
    return weights && s.B * s.L > 0 ? (size_t)qk_args(s, true, true).blocks * 2 * (size_t)s.D * 4 : 0;
}
sf_status check_qk_weights(const float *wq, const float *wk) {
    if (!wq != !wk) return fail(SF_E_NULL, "wq and wk go together");
    return (uintptr_t)wq % 4 || (uintptr_t)wk % 4 ? fail(SF_E_ALIGN, "wq and wk must be 4-byte aligned") : SF_OK;
}
sf_status check_qk_turn(const sf_qk_shape &s, const double *inv_freq, const int64_t *pos) {
    if (s.R > 0 && !inv_freq) return fail(SF_E_NULL, "inv_freq is required for R > 0");
    return (uintptr_t)inv_freq % 8 || (uintptr_t)pos % 8 ? fail(SF_E_ALIGN, "inv_freq and pos must be 8-byte aligned")
                                                          : SF_OK;
}

// One tensor of heads.  Two whose spans overlap may still share no element: slices of one
// projection, or of one buffer with the heads outermost.
struct Heads {
    const void *p;
    sf_strides t;
    int H;
    const char *name;
};
// Whether some of the dims that both tensors step through alike (size and stride) leave,
// taken away, spans that lie one behind the other and fit together into those dims' cells.
bool side_by_side(const Heads &a, const Heads &b, const sf_qk_shape &s, size_t e) {
    if ((uintptr_t)a.p > (uintptr_t)b.p) return side_by_side(b, a, s, e);
    const uint64_t d = (uintptr_t)b.p - (uintptr_t)a.p;
    const int64_t E = (int64_t)e;
    auto dim = [&](int64_t size, int64_t stride) { return Dim{size, size > 1 ? stride * E : 0}; };  // of one: never stepped
    const Dim da[3] = {dim(s.B, a.t.b), dim(s.L, a.t.l), dim(a.H, a.t.h)};
    const Dim db[3] = {dim(s.B, b.t.b), dim(s.L, b.t.l), dim(b.H, b.t.h)};
    for (int outer = 1; outer < 8; ++outer) {
        std::vector<Dim> cells;
        uint64_t ea = (uint64_t)(s.D * E), eb = ea;
        bool alike = true;
        for (int i = 0; i < 3; ++i) {
            if (outer >> i & 1) {
                alike = alike && da[i].size == db[i].size && da[i].stride == db[i].stride;
                cells.push_back(da[i]);
            } else {
                ea += (uint64_t)((da[i].size - 1) * da[i].stride);
                eb += (uint64_t)((db[i].size - 1) * db[i].stride);
            }
        }
        if (alike && d >= ea && d + eb <= (uint64_t)INT64_MAX && non_overlapping(cells, (int64_t)(d + eb))) return true;
    }
    return false;
}
sf_status check_qk_alias(const sf_qk_shape &s, const std::vector<Heads> &ins, const std::vector<Heads> &outs,
                         std::vector<Range> in, const std::vector<Range> &out) {
    const size_t e = elem_size(s.io_dtype);
    auto range = [&](const Heads &h) {
        return strided(h.p, {{s.B, h.t.b}, {s.L, h.t.l}, {h.H, h.t.h}}, s.D, e, h.name);
    };
    auto clash = [&](const Heads &a, const Heads &b) { return overlap(range(a), range(b)) && !side_by_side(a, b, s, e); };
    for (size_t i = 0; i < outs.size(); ++i) {
        for (auto &x : ins)
            if (clash(outs[i], x)) return fail(SF_E_ALIAS, "output %s overlaps input %s", outs[i].name, x.name);
        for (size_t j = i + 1; j < outs.size(); ++j)
            if (clash(outs[i], outs[j])) return fail(SF_E_ALIAS, "output %s overlaps output %s", outs[i].name, outs[j].name);
    }
    // the vectors against everything, the tensors' spans among them
    for (auto &h : outs) TRY(check_alias(in, {range(h)}));
    for (auto &h : outs) in.push_back(range(h));
    for (auto &h : ins) in.push_back(range(h));
    TRY(check_alias(in, out));
    return SF_OK;
}

}  // namespace

extern "C" {

size_t sf_gdn_ragged_workspace_bytes(const sf_gdn_ragged_shape *shape, const sf_ragged *batch) {
    size_t n = 0;
    (void)guarded([&]() -> sf_status {
        TRY(check_gdn(shape, batch));
        n = gdn_ragged_ws_bytes(*shape, *batch);
        return SF_OK;
    });
    return n;
}

sf_status sf_gdn_ragged_fwd(const sf_gdn_ragged_shape *shape, const sf_ragged *batch, const void *q, const void *k,
                            const void *v, const float *g, const float *beta, float *state, void *o, void *ws,
                            size_t ws_bytes, const sf_tuning *tuning, sf_stream stream) {
    return guarded([&]() -> sf_status {
        TRY(check_gdn(shape, batch));
        TRY(check_timing(tuning));
        const sf_gdn_ragged_shape &s = *shape;
        const sf_ragged &b = *batch;
        const size_t need = gdn_ragged_ws_bytes(s, b);
        if (b.N == 0 || b.T == 0) return SF_OK;  // no sequence has a token
        const int64_t per = (int64_t)s.Hv * s.Dk * s.Dv;
        TRY(check_pool("state", state, b.n_slots, per, s.ss, true));
        if (!q || !k || !v || !g || !beta || !o) return fail(SF_E_NULL, "q, k, v, g, beta and o are required");
        if (need > 0 && (!ws || ws_bytes < need))
            return fail(SF_E_WORKSPACE, "workspace of %zu bytes needed (got %zu)", need, ws ? ws_bytes : (size_t)0);
        TRY(check_align({{q, "q"}, {k, "k"}, {v, "v"}, {o, "o"}, {state, "state"}, {need ? ws : nullptr, "ws"}}));
        if ((uintptr_t)g % 4 || (uintptr_t)beta % 4) return fail(SF_E_ALIGN, "g and beta must be 4-byte aligned");
        const size_t e = elem_size(s.io_dtype);
        TRY(check_alias({strided(q, {{b.T, s.sq_t}, {s.Hk, s.sq_h}}, s.Dk, e, "q"),
                         strided(k, {{b.T, s.sq_t}, {s.Hk, s.sq_h}}, s.Dk, e, "k"),
                         strided(v, {{b.T, s.sv_t}, {s.Hv, s.sv_h}}, s.Dv, e, "v"),
                         strided(g, {{b.T, s.sg_t}, {s.Hv, s.sg_h}}, 1, 4, "g"),
                         strided(beta, {{b.T, s.sg_t}, {s.Hv, s.sg_h}}, 1, 4, "beta"), cu_range(b), slot_range(b),
                         fresh_range(b)},
                        {strided(o, {{b.T, s.so_t}, {s.Hv, s.so_h}}, s.Dv, e, "o"),
                         pool_range("state", state, b.n_slots, per, s.ss), wsrange(need ? ws : nullptr, need)}));
        if (b.n_slots == 0) return SF_OK;  // every slot is out of range
        sf::GdnRaggedArgs a = gdn_args(s, b);
        a.q = q;
        a.k = k;
        a.v = v;
        a.g = g;
        a.beta = beta;
        a.state = state;
        a.o = o;
        a.ws = (char *)ws;
        a.plan = need ? (int32_t *)(a.ws + sf::gdn_plan_at(a)) : nullptr;
        // waves of 64, a workgroup's four at most idle
        const double tok = 64.0 * (double)(sf::gdn_token_waves(a) + 4), walk = 256.0 * (double)sf::gdn_walk_groups(a);
        TRY(grid_fits(a.longer ? std::max(tok + walk, 256.0 * ((double)a.n_chunks * s.Hk + 1)) : tok));
        sf_timing *const tm = timing_of(tuning);
        hipEvent_t e0, e1;
        if (!a.longer) {
            take_pair(tm, SF_K_GDN_TOKENS, e0, e1);
            return launched(sf::launch_gdn_tokens(a, (hipStream_t)stream, e0, e1));
        }
        take_pair(tm, SF_K_GDN_CHUNK_PREP, e0, e1);
        TRY(launched(sf::launch_gdn_chunk_prep(a, (hipStream_t)stream, e0, e1)));
        take_pair(tm, SF_K_GDN_CHUNK_WALK, e0, e1);
        return launched(sf::launch_gdn_chunk_walk(a, (hipStream_t)stream, e0, e1));
    });
}

sf_status sf_conv_ragged_fwd(const sf_conv_ragged_shape *shape, const sf_ragged *batch, const void *x, const float *w,
                             float *tails, void *y, const sf_tuning *tuning, sf_stream stream) {
    return guarded([&]() -> sf_status {
        if (!shape) return fail(SF_E_NULL, "shape is NULL");
        const sf_conv_ragged_shape &s = *shape;
        TRY(check_batch(batch));
        const sf_ragged &b = *batch;
        TRY(check_timing(tuning));
        TRY(check_io(s.io_dtype));
        if (s.act != SF_ACT_NONE && s.act != SF_ACT_SILU) return fail(SF_E_DTYPE, "unknown act %d", s.act);
        if (s.reserved != 0) return fail(SF_E_SHAPE, "shape.reserved must be 0");
        if (s.W < 1 || s.W > 4) return fail(SF_E_UNSUPPORTED, "supported taps: 1 <= W <= 4 (got %d)", s.W);
        if (s.C < 8 || s.C % 8) return fail(SF_E_UNSUPPORTED, "C must be a positive multiple of 8 (got %d)", s.C);
        const size_t e = elem_size(s.io_dtype);
        TRY(check_in("x", {{b.T, s.sx_t}}, e));
        TRY(check_out("y", {{b.T, s.sy_t}}, s.C, e));
        const bool tail = s.W > 1;
        const int64_t per = (int64_t)(s.W - 1) * s.C;
        if (b.N == 0 || b.T == 0) return SF_OK;
        if (tail) TRY(check_pool("tails", tails, b.n_slots, per, s.ss, true));
        if (!x || !w || !y) return fail(SF_E_NULL, "x, w and y are required");
        TRY(check_align({{x, "x"}, {y, "y"}, {tail ? tails : nullptr, "tails"}}));
        if ((uintptr_t)w % 4) return fail(SF_E_ALIGN, "w must be 4-byte aligned");
        TRY(check_alias({strided(x, {{b.T, s.sx_t}}, s.C, e, "x"), span(w, 4 * (int64_t)s.C * s.W, "w"), cu_range(b),
                         slot_range(b), fresh_range(b)},
                        {strided(y, {{b.T, s.sy_t}}, s.C, e, "y"),
                         pool_range("tails", tail ? tails : nullptr, b.n_slots, per, s.ss)}));
        if (b.n_slots == 0) return SF_OK;
        sf::ConvRaggedArgs a{};
        a.r = ragged_args(b);
        a.x = x;
        a.w = w;
        a.tails = tails;
        a.y = y;
        a.C = s.C;
        a.W = s.W;
        a.act = s.act;
        a.io = s.io_dtype;
        a.run = sf::conv_ragged_run(b.T, b.N, s.C, device_cus());
        a.n_runs = b.T / a.run + b.N;
        a.sx_t = s.sx_t;
        a.sy_t = s.sy_t;
        a.ss = s.ss;
        TRY(grid_fits((double)a.n_runs * ((s.C / 8 + 255) / 256 * 256)));
        hipEvent_t e0, e1;
        take_pair(timing_of(tuning), SF_K_CONV_RAGGED, e0, e1);
        return launched(sf::launch_conv_ragged(a, (hipStream_t)stream, e0, e1));
    });
}

sf_status sf_qk_norm_fwd(const sf_qk_shape *shape, const void *q, const void *k, const float *wq, const float *wk,
                         const double *inv_freq, const int64_t *pos, void *yq, void *yk, const sf_tuning *tuning,
                         sf_stream stream) {
    return guarded([&]() -> sf_status {
        TRY(check_qk(shape, false));
        TRY(check_timing(tuning));
        const sf_qk_shape &s = *shape;
        TRY(check_qk_weights(wq, wk));
        TRY(check_qk_turn(s, inv_freq, pos));
        if (s.B * s.L == 0) return SF_OK;
        if (!q || !k || !yq || !yk) return fail(SF_E_NULL, "q, k, yq and yk are required");
        TRY(check_align({{q, "q"}, {k, "k"}, {yq, "yq"}, {yk, "yk"}}));
        TRY(check_qk_alias(s, {{q, s.q, s.Hq, "q"}, {k, s.k, s.Hk, "k"}}, {{yq, s.yq, s.Hq, "yq"}, {yk, s.yk, s.Hk, "yk"}},
                           {span(wq, 4 * (int64_t)s.D, "wq"), span(wk, 4 * (int64_t)s.D, "wk"),
                            span(s.R ? inv_freq : nullptr, 4 * (int64_t)s.R, "inv_freq"),
                            strided(s.R ? pos : nullptr, {{s.B, s.sp_b}, {s.L, s.sp_l}}, 1, 8, "pos")},
                           {}));
        sf::QkArgs a = qk_args(s, false, wq != nullptr);
        a.q = q;
        a.k = k;
        a.wq = wq;
        a.wk = wk;
        a.inv_freq = inv_freq;
        a.pos = pos;
        a.yq = yq;
        a.yk = yk;
        hipEvent_t e0, e1;
        take_pair(timing_of(tuning), SF_K_QK_FWD, e0, e1);
        return launched(sf::launch_qk(false, a, (hipStream_t)stream, e0, e1));
    });
}

size_t sf_qk_norm_bwd_workspace_bytes(const sf_qk_shape *shape, int32_t weights) {
    size_t n = 0;
    (void)guarded([&]() -> sf_status {
        TRY(check_qk(shape, true));
        n = qk_ws_bytes(*shape, weights != 0);
        return SF_OK;
    });
    return n;
}

sf_status sf_qk_norm_bwd(const sf_qk_shape *shape, const void *q, const void *k, const float *wq, const float *wk,
                         const double *inv_freq, const int64_t *pos, const void *dyq, const void *dyk, void *dq,
                         void *dk, float *dwq, float *dwk, void *ws, size_t ws_bytes, const sf_tuning *tuning,
                         sf_stream stream) {
    return guarded([&]() -> sf_status {
        TRY(check_qk(shape, true));
        TRY(check_timing(tuning));
        const sf_qk_shape &s = *shape;
        TRY(check_qk_weights(wq, wk));
        TRY(check_qk_turn(s, inv_freq, pos));
        const bool weights = wq != nullptr, empty = s.B * s.L == 0;
        if (weights && (!dwq || !dwk)) return fail(SF_E_NULL, "dwq and dwk are required with weights");
        if (empty && !weights) return SF_OK;
        if (!empty && (!q || !k || !dyq || !dyk || !dq || !dk))
            return fail(SF_E_NULL, "q, k, dyq, dyk, dq and dk are required");
        TRY(check_align({{q, "q"}, {k, "k"}, {dyq, "dyq"}, {dyk, "dyk"}, {dq, "dq"}, {dk, "dk"}}));
        const size_t need = qk_ws_bytes(s, weights);
        if (need > 0 && (!ws || ws_bytes < need))
            return fail(SF_E_WORKSPACE, "workspace of %zu bytes needed (got %zu)", need, ws ? ws_bytes : (size_t)0);
        if ((uintptr_t)(weights ? dwq : nullptr) % 4 || (uintptr_t)(weights ? dwk : nullptr) % 4 || (need && (uintptr_t)ws % 4))
            return fail(SF_E_ALIGN, "dwq, dwk and the workspace must be 4-byte aligned");
        const int64_t nw = 4 * (int64_t)s.D;
        const std::vector<Heads> none;
        const std::vector<Heads> ins = {{q, s.q, s.Hq, "q"}, {k, s.k, s.Hk, "k"}, {dyq, s.yq, s.Hq, "dyq"}, {dyk, s.yk, s.Hk, "dyk"}};
        const std::vector<Heads> outs = {{dq, s.dq, s.Hq, "dq"}, {dk, s.dk, s.Hk, "dk"}};
        TRY(check_qk_alias(s, empty ? none : ins, empty ? none : outs,
                           {span(wq, nw, "wq"), span(wk, nw, "wk"),
                            span(s.R ? inv_freq : nullptr, 4 * (int64_t)s.R, "inv_freq"),
                            strided(s.R ? pos : nullptr, {{s.B, s.sp_b}, {s.L, s.sp_l}}, 1, 8, "pos")},
                           {span(weights ? dwq : nullptr, nw, "dwq"), span(weights ? dwk : nullptr, nw, "dwk"),
                            wsrange(need ? ws : nullptr, need)}));
        sf::QkArgs a = qk_args(s, true, weights);
        a.q = q;
        a.k = k;
        a.dyq = dyq;
        a.dyk = dyk;
        a.wq = wq;
        a.wk = wk;
        a.inv_freq = inv_freq;
        a.pos = pos;
        a.yq = dq;
        a.yk = dk;
        a.dwq = dwq;
        a.dwk = dwk;
        a.ws = (float *)ws;
        hipEvent_t e0, e1;
        take_pair(timing_of(tuning), SF_K_QK_BWD, e0, e1);
        return launched(sf::launch_qk(true, a, (hipStream_t)stream, e0, e1));
    });
}

}  // extern "C"
