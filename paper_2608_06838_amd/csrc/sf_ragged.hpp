// sf_ragged.hpp -- sequences of a ragged batch, as the kernels see them.
#pragma once
#include "sf_chunk.hpp"

namespace sf {

// A sequence's rows [begin, end) and slot; end <= begin or slot < 0: nothing to do.
struct Seq {
    int64_t begin, end;
    int slot;
};
__device__ __forceinline__ int64_t clamp_row(int64_t x, int64_t T) { return x < 0 ? 0 : x > T ? T : x; }
__device__ __forceinline__ Seq seq_of(const RaggedArgs &r, int i) {
    Seq s;
    s.begin = clamp_row(r.cu[i], r.T);
    s.end = clamp_row(r.cu[i + 1], r.T);
    s.slot = r.slot ? r.slot[i] : i;
    if (s.slot >= r.n_slots) s.slot = -1;
    return s;
}

// Runs of `run` tokens, none across a sequence's end.  Run numbers of sequence i start
// at cu[i] / run + i, which leaves it room for its own ceil(n / run) runs (its last one
// may be short, and one number may stay unused), so a launch of T / run + N numbers
// needs neither the lengths on the host nor a table.
// the last sequence i in [0, N) whose first run, cu[i] / run + add i, is <= id; 64 candidates a step
__device__ __forceinline__ int find_seq(const RaggedArgs &r, int run, int64_t id, int add = 1) {
    const int lane = threadIdx.x & 63;
    int lo = 0, n = r.N;
    while (n > 1) {
        const int step = (n + 63) / 64, i = lo + lane * step;
        const bool in = lane * step < n && (int64_t)((uint32_t)clamp_row(r.cu[lane * step < n ? i : lo], r.T) / (uint32_t)run) + (int64_t)add * i <= id;
        const int m = __popcll(__ballot(in));
        const int at = m > 0 ? (m - 1) * step : 0;
        lo += at;
        n = n - at < step ? n - at : step;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}
__device__ __forceinline__ int64_t first_run(const Seq &s, int run, int i) { return (uint32_t)s.begin / (uint32_t)run + (int64_t)i; }

// Gated delta rule, token by token (S <- e^g S, u = beta (v - S^T k), S <- S + k u^T,
// o = S^T q).  A single token reads and writes the whole state for 6 flops an
// element: the roofline is HBM.  State columns (value channels) never mix, so a
// wave owns CW columns of one head of one sequence and keeps them in registers from
// the sequence's first token to its last; no LDS, no barrier.  Lane (rg, cl) holds
// rows rg RPL .. + RPL - 1 of columns 4 cl .. + 3: a row's columns are 16 bytes of
// 8 consecutive lanes, one 128-byte line, and k and q come as the lane's own run of
// rows, one or two 16-byte loads that its neighbours share.  With a = e^g and the old
// state S,
//     S^T k and S^T q are summed together,   u = beta (v - a S^T k),
//     o = a S^T q + (k . q) u,               S <- a S + k u^T,
// so a token costs one reduction over the row groups, of nine sums.  Several tokens' decay
// is kept as one factor beside the state (a quarter of a token's work would go into
// applying it), applied when it leaves [1e-9, 16] and at the end.  The state goes past
// the caches (256 sequences of 40 heads of 128 x 128: 235 us, 5.7 TB/s; 258 through them).
constexpr int TOK_NT = 256;

// sum over the row groups (lanes that differ in the bits from CL up), in every lane
template <int CL>
__device__ __forceinline__ float group_sum(float x) {
    static_assert(CL == 4 || CL == 8, "column lanes");
    x += dpp_or0<0x128>(x);                       // row_ror:8
    if constexpr (CL == 4) x += dpp_or0<0x124>(x);  // row_ror:4
    return sum_rows(x);
}

template <typename T, int N> struct Vec { typedef T type __attribute__((ext_vector_type(N))); };

// one wave: tile unit % (Dv / CW) of head unit / (Dv / CW) % Hv of the sequence
template <typename T, int DK, int CL>
__device__ __forceinline__ void gdn_tokens(const GdnRaggedArgs &a, int64_t unit) {
    constexpr int CW = 4 * CL, RG = 64 / CL, RPL = DK / RG;
    typedef typename Vec<T, RPL>::type rows_t;
    typedef typename Vec<T, 4>::type cols_t;
    const int lane = threadIdx.x & 63, nt = a.Dv / CW;
    const int tile = (int)(unit % nt);
    const int64_t ih = unit / nt;
    const int h = (int)(ih % a.Hv);
    const int64_t i = ih / a.Hv;
    if (i >= a.r.N) return;
    const Seq sq = seq_of(a.r, (int)i);
    if (sq.end <= sq.begin || sq.slot < 0 || (a.longer && sq.end - sq.begin > a.longer)) return;
    const int rg = lane / CL, col = tile * CW + 4 * (lane % CL), hk = h / (a.Hv / a.Hk);
    float *const sp = a.state + sq.slot * a.ss + (int64_t)h * DK * a.Dv + (int64_t)rg * RPL * a.Dv + col;
    f32x4 S[RPL];
    const bool fresh = a.r.fresh && a.r.fresh[i];
#pragma unroll
    for (int m = 0; m < RPL; ++m)
        S[m] = fresh ? f32x4{0.f, 0.f, 0.f, 0.f} : __builtin_nontemporal_load(reinterpret_cast<const f32x4 *>(sp + (int64_t)m * a.Dv));
    const T *kp = (const T *)a.k + hk * a.sq_h + rg * RPL, *qp = (const T *)a.q + hk * a.sq_h + rg * RPL;
    const T *vp = (const T *)a.v + h * a.sv_h + col;
    T *op = (T *)a.o + h * a.so_h + col;
    const float *gp = a.g + h * a.sg_h, *bp = a.beta + h * a.sg_h;
    // tokens come two steps ahead
    struct Token {
        rows_t k, q;
        cols_t v;
        float g, beta;
    };
    auto fetch = [&](int64_t t) {
        t = t < sq.end ? t : sq.end - 1;
        return Token{*reinterpret_cast<const rows_t *>(kp + t * a.sq_t), *reinterpret_cast<const rows_t *>(qp + t * a.sq_t),
                     *reinterpret_cast<const cols_t *>(vp + t * a.sv_t), gp[t * a.sg_t], bp[t * a.sg_t]};
    };
    Token n0 = fetch(sq.begin), n1 = fetch(sq.begin + 1);
    float scale = 1.f;  // the state is scale S
    for (int64_t t = sq.begin; t < sq.end; ++t) {
        const Token x = n0;
        n0 = n1;
        if (t + 2 < sq.end) n1 = fetch(t + 2);
        scale *= fexp2(x.g * LOG2E);
        auto apply = [&] {
#pragma unroll
            for (int m = 0; m < RPL; ++m) S[m] *= scale;
            scale = 1.f;
        };
        if (!(scale > 1e-9f && scale < 16.f)) apply();  // one value in the whole wave
        float inv = 1.f / scale;
        const float most = 1e36f * scale;
        f32x4 sk = {0.f, 0.f, 0.f, 0.f}, sv = sk;
        float kq = 0.f;
#pragma unroll
        for (int m = 0; m < RPL; ++m) {
            const float km = (float)x.k[m], qm = (float)x.q[m];
            kq = fmaf(km, qm, kq);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                sk[c] = fmaf(S[m][c], km, sk[c]);
                sv[c] = fmaf(S[m][c], qm, sv[c]);
            }
        }
        kq = group_sum<CL>(kq);
        f32x4 u = {0.f, 0.f, 0.f, 0.f}, o = u;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            u[c] = x.beta * ((float)x.v[c] - scale * group_sum<CL>(sk[c]));
            o[c] = fmaf(kq, u[c], scale * group_sum<CL>(sv[c]));
        }
        // u / scale stays in range: the factor is applied first where it would not (the test
        // costs a token 1 to 3%)
        if (__any(fmaxf(fmaxf(fabsf(u[0]), fabsf(u[1])), fmaxf(fabsf(u[2]), fabsf(u[3]))) > most)) {
            apply();
            inv = 1.f;
        }
        u *= inv;
#pragma unroll
        for (int m = 0; m < RPL; ++m) {
            const float km = (float)x.k[m];
#pragma unroll
            for (int c = 0; c < 4; ++c) S[m][c] = fmaf(km, u[c], S[m][c]);
        }
        if (rg == 0) {
            T *p = op + t * a.so_t;
            if constexpr (sizeof(T) == 2) st4(p, o[0], o[1], o[2], o[3]);
            else *reinterpret_cast<f32x4 *>(p) = o;
        }
    }
#pragma unroll
    for (int m = 0; m < RPL; ++m) __builtin_nontemporal_store(S[m] * scale, reinterpret_cast<f32x4 *>(sp + (int64_t)m * a.Dv));
}

}  // namespace sf
