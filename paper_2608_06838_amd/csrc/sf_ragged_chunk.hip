// sf_ragged_chunk.hip -- gfx950 kernels of the gated delta rule over the long
// sequences of a ragged batch, 64 tokens at a time.
//
// Chunk algebra (S the state entering the chunk, b_t the chunk's running sum of g,
// rows past the sequence's end with beta = 0 and g = 0):
//   A[t][s] = beta_t e^(b_t - b_s) k_t.k_s  (s < t),   T = (I + A)^-1
//   P[t][s] = e^(b_t - b_s) q_t.k_s         (s <= t)
//   U = T diag(beta) (V - diag(e^b) K S),   O = diag(e^b) Q S + P U
//   S <- e^(b_63) S + K^T diag(e^(b_63 - b)) U
// T and P need no state: k_rag_prep forms them for every chunk at once, and k_rag_walk
// takes the chunks of one sequence and value head in order.
//
// The state leaves this call in fp32 and enters the next one, thousands of times in a
// decoded sequence, so it is carried as precisely as the token-by-token kernel carries
// it: every matrix product runs on bf16 MFMA with its fp32 operands cut into three
// bf16 pieces of eight bits (exact: 24 bits), keys entering as the bf16 they are.  The
// pieces' products that lie below 2^-24 are left out (T's times X's: six of nine), and
// the output, which is rounded to bf16, takes two pieces.  Against fp32 matrix
// instructions that is 3 to 6 instructions at 16 times the rate.
//
// State columns never mix, so a wave of the walk owns 16 of them and shares only the
// staged tiles (K, Q, V, T, P) with its workgroup; U, X and S pass from one product to
// the next inside registers: the accumulator pairs (2m, 2m + 1) hold, in lane row
// q = lane / 16, rows 32 m + 8 q .. + 7 of the wave's column lane % 16, the slot order
// of an operand fragment.  The products that build them read their A rows in that
// order (fragment row n of tile i is 32 (i / 2) + 8 (n / 4) + 4 (i % 2) + n % 4).
#include "sf_ragged.hpp"

#include <type_traits>

namespace sf {

namespace {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// x = hi + mid + lo, 8 bits each, exactly: the upper halves of x, of x - hi and of what
// then remains
__device__ __forceinline__ void split3(const float (&x)[8], bf16x8 &hi, bf16x8 &mid, bf16x8 &lo) {
    u32x4 h = {0u, 0u, 0u, 0u}, m = h, l = h;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        unsigned r[2], s[2], x0[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            x0[e] = __float_as_uint(x[2 * p + e]);
            r[e] = __float_as_uint(x[2 * p + e] - __uint_as_float(x0[e] & 0xffff0000u));
            s[e] = __float_as_uint(__uint_as_float(r[e]) - __uint_as_float(r[e] & 0xffff0000u));
        }
        h[p] = __builtin_amdgcn_perm(x0[1], x0[0], 0x07060302u);
        m[p] = __builtin_amdgcn_perm(r[1], r[0], 0x07060302u);
        l[p] = __builtin_amdgcn_perm(s[1], s[0], 0x07060302u);
    }
    hi = __builtin_bit_cast(bf16x8, h);
    mid = __builtin_bit_cast(bf16x8, m);
    lo = __builtin_bit_cast(bf16x8, l);
}
__device__ __forceinline__ void split3(const f32x4 &a, const f32x4 &b, bf16x8 &hi, bf16x8 &mid, bf16x8 &lo) {
    const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    split3(x, hi, mid, lo);
}

// e^-104 is below the smallest fp32: a gate of -inf (forget everything) becomes one
// whose running sum stays finite
__device__ __forceinline__ float gate_log2(float g) { return fmaxf(g, -104.f) * LOG2E; }

// Rows [0, 64) of a chunk tile of D channels, in 16-byte blocks over NT threads, rows
// from m on zero; to LDS with pitch LD, rows of bit 3 swizzled by SW channels (see
// ldfragTR).
template <int D, int NT, int LD, int SW>
struct RowTile {
    static constexpr int BPR = D / 8, RPP = NT / BPR, N = 64 / RPP;
    static_assert(NT % BPR == 0 && 64 % RPP == 0, "tile shape");
    u32x4 r[N];
    __device__ __forceinline__ void load(const __bf16 *p, int64_t ld, int m, int tid) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int row = tid / BPR + RPP * i;
            r[i] = u32x4{0u, 0u, 0u, 0u};
            if (row < m) r[i] = *reinterpret_cast<const u32x4 *>(p + row * ld + 8 * (tid % BPR));
        }
    }
    __device__ __forceinline__ void store(__bf16 *lds, int tid) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int row = tid / BPR + RPP * i, ch = 8 * (tid % BPR);
            *reinterpret_cast<u32x4 *>(lds + row * LD + swz_col(row, ch, SW)) = r[i];
        }
    }
};

// fragment (tt, ks) of a lower triangle: tiles 0, 1 have columns 0..31 only
__device__ __forceinline__ constexpr int tri_frag(int tt, int ks) { return tt < 2 ? tt : 2 + 2 * (tt - 2) + ks; }

// ---------------------------------------------------------------- T and P of a chunk
template <int DK>
__global__ void __launch_bounds__(256) k_rag_prep(GdnRaggedArgs a) {
    constexpr int NT = 256, LD = DK + 16, SW = swx<__bf16, DK>(), LA = 68;
    __shared__ __attribute__((aligned(16))) __bf16 sK[64 * LD], sQ[64 * LD];
    __shared__ __attribute__((aligned(16))) float sA[64 * LA], sT[64 * LA];
    __shared__ __attribute__((aligned(16))) float sb[64], sbeta[64];
    const int tid = threadIdx.x, lane = tid & 63, q4 = lane >> 4, n16 = lane & 15;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hk = blockIdx.x % a.Hk, group = a.Hv / a.Hk;
    const int64_t id = blockIdx.x / a.Hk;
    const int i = find_seq(a.r, 64, id);
    const Seq sq = seq_of(a.r, i);
    const int64_t c0 = (id - first_run(sq, 64, i)) * 64, n = sq.end - sq.begin;
    if (c0 < 0 || c0 >= n || n <= a.longer || sq.slot < 0) return;
    const int m = n - c0 < 64 ? (int)(n - c0) : 64;
    const int64_t row0 = sq.begin + c0;
    RowTile<DK, NT, LD, SW> t;
    t.load((const __bf16 *)a.k + row0 * a.sq_t + hk * a.sq_h, a.sq_t, m, tid);
    t.store(sK, tid);
    t.load((const __bf16 *)a.q + row0 * a.sq_t + hk * a.sq_h, a.sq_t, m, tid);
    t.store(sQ, tid);
    __syncthreads();
    // wave w: rows 16 w .. of k.k and q.k, columns s in plain pairs
    const LaneOff swo = swz_off<__bf16, LD, SW>(lane);
    const int ar = 8 * (n16 >> 2) + (n16 & 3), sgn = ((n16 >> 2) & 1) * SW;
    f32x4 kk[4], qk[4];
#pragma unroll
    for (int st = 0; st < 4; ++st) kk[st] = qk[st] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < DK / 32; ++ks) {
        const bf16x8 kt = ldfrag_swz<__bf16, LD, SW>(sK, swo, 16 * w, 32 * ks);
        const bf16x8 qt = ldfrag_swz<__bf16, LD, SW>(sQ, swo, 16 * w, 32 * ks);
#pragma unroll
        for (int st = 0; st < 4; ++st) {
            if (st >= 2 && w < 2) continue;  // above the diagonal
            const bf16x8 kf = *reinterpret_cast<const bf16x8 *>(
                &sK[(ar + 32 * (st >> 1) + 4 * (st & 1)) * LD + 8 * q4 + 32 * ks + (((32 * ks) & SW) ? -sgn : sgn)]);
            mma(kk[st], kf, kt);
            mma(qk[st], kf, qt);
        }
    }
    const int tok = 16 * w + n16;
    for (int hv = hk * group; hv < (hk + 1) * group; ++hv) {
        __syncthreads();  // the last head is done with the gates and with T
        if (w == 0) {
            const bool in = lane < m;
            const int64_t go = (row0 + lane) * a.sg_t + hv * a.sg_h;
            sb[lane] = wave_scan_dpp(in ? gate_log2(a.g[go]) : 0.f);
            sbeta[lane] = in ? a.beta[go] : 0.f;
        }
        __syncthreads();
        __bf16 *const sys = reinterpret_cast<__bf16 *>(a.ws + (id * a.Hv + hv) * (int64_t)RAG_SYS);
        const float bt = sb[tok], be = sbeta[tok];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            if (ks > (w >> 1)) continue;
            float av[8], pv[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int s = 32 * ks + 8 * q4 + j;
                const float d = fexp2(bt - sb[s]);
                av[j] = s < tok ? be * kk[2 * ks + (j >> 2)][j & 3] * d : 0.f;
                pv[j] = s <= tok ? qk[2 * ks + (j >> 2)][j & 3] * d : 0.f;
            }
            float *p = &sA[tok * LA + 32 * ks + 8 * q4];
            *reinterpret_cast<f32x4 *>(p) = f32x4{av[0], av[1], av[2], av[3]};
            *reinterpret_cast<f32x4 *>(p + 4) = f32x4{av[4], av[5], av[6], av[7]};
            bf16x8 hi, lo;
            split8<__bf16, true>(pv, hi, lo);
            __bf16 *out = sys + (RAG_TP * RAG_FRAGS + tri_frag(w, ks)) * 512 + 8 * lane;
            *reinterpret_cast<bf16x8 *>(out) = hi;
            *reinterpret_cast<bf16x8 *>(out + RAG_FRAGS * 512) = lo;
        }
        __syncthreads();
        // Diagonal blocks by forward substitution, a column a thread: x_r = [r == c] -
        // sum_{s < r} A[r][s] x_s.  (A series in powers of A would lose its digits where
        // neighbouring keys are nearly parallel.)
        if (w == 0) {
            const int o = 16 * q4;
            float x[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                float acc[4] = {r == n16 ? 1.f : 0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s4 = 0; s4 < (r + 3) / 4; ++s4) {
                    const f32x4 v = *reinterpret_cast<const f32x4 *>(&sA[(o + r) * LA + o + 4 * s4]);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (4 * s4 + e < r) acc[e] = fmaf(-v[e], x[4 * s4 + e], acc[e]);
                }
                x[r] = (acc[0] + acc[1]) + (acc[2] + acc[3]);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) sT[(o + r) * LA + o + n16] = x[r];
        }
        __syncthreads();
        // Block column w below the diagonal: T_iw = -T_ii sum_{k = w}^{i - 1} A_ik T_kw in
        // fp32 MFMA.  The blocks stay in their accumulators, which are the B operands of
        // the next rows' products.
        {
            f32x4 col[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) col[0][r] = sT[(16 * w + 4 * q4 + r) * LA + 16 * w + n16];
#pragma unroll
            for (int d = 1; d < 4; ++d) {
                col[d] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (w + d < 4) {
                    const int bi = w + d;
                    f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int k = 0; k < d; ++k) {
                        const f32x4 av = *reinterpret_cast<const f32x4 *>(&sA[(16 * bi + n16) * LA + 16 * (w + k) + 4 * q4]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) y = __builtin_amdgcn_mfma_f32_16x16x4f32(av[e], col[k][e], y, 0, 0, 0);
                    }
                    const f32x4 tv = *reinterpret_cast<const f32x4 *>(&sT[(16 * bi + n16) * LA + 16 * bi + 4 * q4]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) col[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(-tv[e], y[e], col[d], 0, 0, 0);
#pragma unroll
                    for (int r = 0; r < 4; ++r) sT[(16 * bi + 4 * q4 + r) * LA + 16 * w + n16] = col[d][r];
                }
            }
            // blocks (0, 1) and (2, 3) lie in fragments: zero
            if (w & 1) {
#pragma unroll
                for (int r = 0; r < 4; ++r) sT[(16 * (w - 1) + 4 * q4 + r) * LA + 16 * w + n16] = 0.f;
            }
        }
        __syncthreads();
        // fragments of tile w: rows in the walk's order, columns 32 ks + 8 q4 ..
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            if (ks > (w >> 1)) continue;
            const float *p = &sT[(32 * (w >> 1) + ar + 4 * (w & 1)) * LA + 32 * ks + 8 * q4];
            bf16x8 f[3];
            split3(*reinterpret_cast<const f32x4 *>(p), *reinterpret_cast<const f32x4 *>(p + 4), f[0], f[1], f[2]);
#pragma unroll
            for (int pl = 0; pl < RAG_TP; ++pl)
                *reinterpret_cast<bf16x8 *>(sys + (pl * RAG_FRAGS + tri_frag(w, ks)) * 512 + 8 * lane) = f[pl];
        }
    }
}

// ----------------------------------------------------------------------- the walk
template <int DK, int NW>
__global__ void __launch_bounds__(64 * NW, 2) k_rag_walk(GdnRaggedArgs a) {
    constexpr int NT = 64 * NW, NK = DK / 16, LD = DK + 16, SW = swx<__bf16, DK>();
    constexpr int VW = 16 * NW, LDV = VW + 16, SWV = NW == 2 ? 16 : 32;
    constexpr int BLK = RAG_SYS / 16, SYS = (BLK + NT - 1) / NT;  // 16-byte blocks of a system, of a thread
    __shared__ __attribute__((aligned(16))) __bf16 sK[64 * LD], sQ[64 * LD], sV[64 * LDV];
    __shared__ __attribute__((aligned(16))) u32x4 sS[BLK];
    __shared__ __attribute__((aligned(16))) float sq[64], se[64], sbeta[64];
    const int tid = threadIdx.x, lane = tid & 63, q4 = lane >> 4, n16 = lane & 15;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ncb = a.Dv / VW;
    const int cb = blockIdx.x % ncb, h = (blockIdx.x / ncb) % a.Hv, i = blockIdx.x / ncb / a.Hv;
    const Seq s = seq_of(a.r, i);
    const int64_t n = s.end - s.begin;
    if (n <= a.longer || s.slot < 0) return;
    const int hk = h / (a.Hv / a.Hk), col = cb * VW + 16 * w + n16;
    const __bf16 *K = (const __bf16 *)a.k + s.begin * a.sq_t + hk * a.sq_h;
    const __bf16 *Q = (const __bf16 *)a.q + s.begin * a.sq_t + hk * a.sq_h;
    const __bf16 *V = (const __bf16 *)a.v + s.begin * a.sv_t + h * a.sv_h + cb * VW;
    __bf16 *O = (__bf16 *)a.o + s.begin * a.so_t + h * a.so_h + cb * VW + 16 * w + 4 * q4;
    const float *G = a.g + s.begin * a.sg_t + h * a.sg_h, *BE = a.beta + s.begin * a.sg_t + h * a.sg_h;
    const char *sys = a.ws + (first_run(s, 64, i) * a.Hv + h) * (int64_t)RAG_SYS;
    float *const st = a.state + s.slot * a.ss + (int64_t)h * DK * a.Dv + col;

    // S[t][r] = state row 32 (t / 2) + 8 q4 + 4 (t % 2) + r, column col
    auto row = [&](int t, int r) { return 32 * (t >> 1) + 8 * q4 + 4 * (t & 1) + r; };
    f32x4 S[NK];
    const bool fresh = a.r.fresh && a.r.fresh[i];
#pragma unroll
    for (int t = 0; t < NK; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) S[t][r] = fresh ? 0.f : st[(int64_t)row(t, r) * a.Dv];

    RowTile<DK, NT, LD, SW> tk, tq;
    RowTile<VW, NT, LDV, SWV> tv;
    u32x4 ts[SYS] = {};
    float gl = 0.f, bl = 0.f;
    auto fetch = [&](int64_t c) {
        const int m = n - c < 64 ? (int)(n - c) : 64;
        tk.load(K + c * a.sq_t, a.sq_t, m, tid);
        tq.load(Q + c * a.sq_t, a.sq_t, m, tid);
        tv.load(V + c * a.sv_t, a.sv_t, m, tid);
        const u32x4 *p = reinterpret_cast<const u32x4 *>(sys + (c / 64) * a.Hv * (int64_t)RAG_SYS) + tid;
#pragma unroll
        for (int j = 0; j < SYS; ++j)
            if (j * NT + NT <= BLK || j * NT + tid < BLK) ts[j] = p[j * NT];
        if (w == 0) {
            gl = lane < m ? gate_log2(G[(c + lane) * a.sg_t]) : 0.f;
            bl = lane < m ? BE[(c + lane) * a.sg_t] : 0.f;
        }
    };
    fetch(0);
    const LaneOff swo = swz_off<__bf16, LD, SW>(lane), tr8 = tr_off8<__bf16, LD, SW>(lane);
    const LaneOff trv = tr_off<__bf16, LDV, SWV>(lane);
    const int ar = 8 * (n16 >> 2) + (n16 & 3), sgn = ((n16 >> 2) & 1) * SW;
    const bf16x8 *const T = reinterpret_cast<const bf16x8 *>(sS) + lane;
    const bf16x8 *const P = T + RAG_TP * RAG_FRAGS * 64;
    for (int64_t c = 0; c < n; c += 64) {
        __syncthreads();  // the last chunk is done with the tiles
        tk.store(sK, tid);
        tq.store(sQ, tid);
        tv.store(sV, tid);
#pragma unroll
        for (int j = 0; j < SYS; ++j)
            if (j * NT + NT <= BLK || j * NT + tid < BLK) sS[j * NT + tid] = ts[j];
        if (w == 0) {
            const float b = wave_scan_dpp(gl);
            sq[lane] = fexp2(b);
            se[lane] = fexp2(lane_value(b, 63) - b);
            sbeta[lane] = bl;
        }
        __syncthreads();
        if (c + 64 < n) fetch(c + 64);

        f32x4 X[4], Y[4];  // K S (rows: tokens), (Q S)^T (columns: tokens)
#pragma unroll
        for (int t = 0; t < 4; ++t) X[t] = Y[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < DK / 32; ++ks) {
            bf16x8 f[3];
            split3(S[2 * ks], S[2 * ks + 1], f[0], f[1], f[2]);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const bf16x8 kf = *reinterpret_cast<const bf16x8 *>(
                    &sK[(ar + 32 * (t >> 1) + 4 * (t & 1)) * LD + 8 * q4 + 32 * ks + (((32 * ks) & SW) ? -sgn : sgn)]);
                mma(X[t], kf, f[2]);
                mma(X[t], kf, f[1]);
                mma(X[t], kf, f[0]);
                const bf16x8 qf = ldfrag_swz<__bf16, LD, SW>(sQ, swo, 16 * t, 32 * ks);
                mma(Y[t], f[2], qf);
                mma(Y[t], f[1], qf);
                mma(Y[t], f[0], qf);
            }
        }
        // X = beta (V - e^b K S); the transposing read returns V in X's own slots
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            const bf16x8 vf = ldfragTR<__bf16, LDV, SWV>(sV, trv, 32 * ks, 16 * w);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int t = 2 * ks + u;
                const f32x4 eb = *reinterpret_cast<const f32x4 *>(&sq[row(t, 0)]);
                const f32x4 be = *reinterpret_cast<const f32x4 *>(&sbeta[row(t, 0)]);
#pragma unroll
                for (int r = 0; r < 4; ++r) X[t][r] = be[r] * ((float)vf[4 * u + r] - eb[r] * X[t][r]);
            }
        }
        f32x4 U[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) U[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            bf16x8 f[3];
            split3(X[2 * ks], X[2 * ks + 1], f[0], f[1], f[2]);
#pragma unroll
            for (int t = 2 * ks; t < 4; ++t) {
                const int fr = tri_frag(t, ks) * 64;
                const bf16x8 t0 = T[fr], t1 = T[fr + RAG_FRAGS * 64], t2 = T[fr + 2 * RAG_FRAGS * 64];
                mma(U[t], t2, f[0]);
                mma(U[t], t1, f[1]);
                mma(U[t], t0, f[2]);
                mma(U[t], t1, f[0]);
                mma(U[t], t0, f[1]);
                mma(U[t], t0, f[0]);
            }
        }
        // O^T = e^b (Q S)^T + U^T P^T
#pragma unroll
        for (int t = 0; t < 4; ++t) Y[t] *= sq[16 * t + n16];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            bf16x8 uh, ul;
            split_acc<__bf16, true>(U[2 * ks], U[2 * ks + 1], uh, ul);
#pragma unroll
            for (int t = 2 * ks; t < 4; ++t) {
                const int fr = tri_frag(t, ks) * 64;
                const bf16x8 p0 = P[fr], p1 = P[fr + RAG_FRAGS * 64];
                mma(Y[t], uh, p1);
                mma(Y[t], ul, p0);
                mma(Y[t], uh, p0);
            }
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int64_t tok = c + 16 * t + n16;
            if (tok < n) st4(O + tok * a.so_t, Y[t][0], Y[t][1], Y[t][2], Y[t][3]);
        }
        // S = e^(b_63) S + K^T e^(b_63 - b) U
        const float gam = sq[63];
#pragma unroll
        for (int t = 0; t < NK; ++t) S[t] *= gam;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
            for (int t = 2 * ks; t < 2 * ks + 2; ++t) U[t] *= *reinterpret_cast<const f32x4 *>(&se[row(t, 0)]);
            bf16x8 f[3];
            split3(U[2 * ks], U[2 * ks + 1], f[0], f[1], f[2]);
#pragma unroll
            for (int t = 0; t < NK; ++t) {
                const bf16x8 kf = ldfragTR<__bf16, LD, SW>(sK, tr8, 32 * ks, 32 * (t >> 1) + 4 * (t & 1));
                mma(S[t], kf, f[2]);
                mma(S[t], kf, f[1]);
                mma(S[t], kf, f[0]);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < NK; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) st[(int64_t)row(t, r) * a.Dv] = S[t][r];
}

}  // namespace

hipError_t launch_gdn_chunk_prep(const GdnRaggedArgs &a, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
    const dim3 grid((unsigned)(a.n_chunks * a.Hk));
    if (a.Dk == 128) hipExtLaunchKernelGGL((k_rag_prep<128>), grid, dim3(256), 0, s, e0, e1, 0, a);
    else hipExtLaunchKernelGGL((k_rag_prep<64>), grid, dim3(256), 0, s, e0, e1, 0, a);
    return hipGetLastError();
}

hipError_t launch_gdn_chunk_walk(const GdnRaggedArgs &a, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
    const dim3 grid((unsigned)((int64_t)a.r.N * a.Hv * (a.Dv / (16 * RAG_NW)))), block(64 * RAG_NW);
    if (a.Dk == 128) hipExtLaunchKernelGGL((k_rag_walk<128, RAG_NW>), grid, block, 0, s, e0, e1, 0, a);
    else hipExtLaunchKernelGGL((k_rag_walk<64, RAG_NW>), grid, block, 0, s, e0, e1, 0, a);
    return hipGetLastError();
}

}  // namespace sf
