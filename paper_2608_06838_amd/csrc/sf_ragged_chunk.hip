// sf_ragged_chunk.hip -- gfx950 kernels of the gated delta rule over the long
// sequences of a ragged batch, 64 tokens at a time.
//
// Chunk algebra (S the state entering the chunk, b_t the chunk's running sum of g,
// rows past the sequence's end with beta = 0 and g = 0):
//   A[t][s] = beta_t e^(b_t - b_s) k_t.k_s  (s < t),   T = (I + A)^-1
//   P[t][s] = e^(b_t - b_s) q_t.k_s         (s <= t),  R = P T
//   X = diag(beta) (V - diag(e^b) K S),   U = T X,   O = diag(e^b) Q S + R X  (P U = R X)
//   S <- e^(b_63) S + K^T diag(e^(b_63 - b)) U
// T and R need no state: k_rag_prep forms them for every chunk at once, and k_rag_walk
// takes the chunks of one sequence and value head in order.
//
// The state leaves this call in fp32 and enters the next one, thousands of times in a
// decoded sequence, so it is carried as precisely as the token-by-token kernel carries
// it, and outputs are as exact before their rounding: every product of the walk runs on
// bf16 MFMA with its fp32 operands cut into three bf16 pieces of eight bits (exact: 24
// bits), keys and queries entering as the bf16 they are.  Of the nine products of two
// operands' pieces the three below 2^-24 are left out.  Against fp32 matrix instructions
// that is 3 to 6 instructions at 16 times the rate.  Outputs take X, whose pieces U needs
// anyway: U's own would be a second set through LDS (8259 packed tokens of 20 heads: 229 us
// that way, 224 this).
//
// State columns never mix, so a workgroup of the walk owns 16 NC of them.  Its four
// waves share each chunk's chain of products by rows: wave w forms the rows of its 16
// tokens of K S, Q S, U and O, and keeps a quarter of the state's key rows.  Between
// the products the operands pass through LDS as their three pieces (S, then X, then U).
// A wave that kept 16 columns for itself would need no exchange, and took 5.8 us a
// chunk, most of it waiting on its own chain of 200 matrix instructions: a sequence's
// chunks follow one another, so the chain is what a long prompt waits for.  As it is, a
// step takes 2.2 us with one column tile on a CU of its own.
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
__device__ __forceinline__ void split3(const f32x4 &x, bf16x4 &hi, bf16x4 &mid, bf16x4 &lo) {
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    const f32x4 z = {0.f, 0.f, 0.f, 0.f};
    f32x4 r = z, s = z;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        r[e] = x[e] - __uint_as_float(__float_as_uint(x[e]) & 0xffff0000u);
        s[e] = r[e] - __uint_as_float(__float_as_uint(r[e]) & 0xffff0000u);
    }
    auto upper = [](const f32x4 &v) {
        const u32x2 u = {__builtin_amdgcn_perm(__float_as_uint(v[1]), __float_as_uint(v[0]), 0x07060302u),
                         __builtin_amdgcn_perm(__float_as_uint(v[3]), __float_as_uint(v[2]), 0x07060302u)};
        return __builtin_bit_cast(bf16x4, u);
    };
    hi = upper(x);
    mid = upper(r);
    lo = upper(s);
}
__device__ __forceinline__ void split3(const f32x4 &a, const f32x4 &b, bf16x8 &hi, bf16x8 &mid, bf16x8 &lo) {
    const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    split3(x, hi, mid, lo);
}

// A chunk's running sum of gates (in powers of two) is formed in 64 bits and kept as a
// pair of floats: a decay is the difference of two sums, and behind strong gates both are
// large (some thousands where documents reset the state), so that sums in 32 bits would
// leave a weak gate's decay with the large sums' error: 1e-4 of the state behind four
// resets, 1e-6 with gates near -0.1; the pair leaves 1e-7.  e^-104 is below the smallest
// fp32: a gate of -inf (forget everything) becomes one whose sum stays finite (and NaN
// stays NaN).
__device__ __forceinline__ double gate_log2(float g) { return (double)(g < -104.f ? -104.f : g) * 1.4426950408889634; }
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ double dpp_or0(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)u, CTRL, ROWS, 0xf, true);
    const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)(u >> 32), CTRL, ROWS, 0xf, true);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_scan_dpp(double x) {  // as for floats
    x += dpp_or0<0x111>(x);
    x += dpp_or0<0x112>(x);
    x += dpp_or0<0x114>(x);
    x += dpp_or0<0x118>(x);
    x += dpp_or0<0x142, 0xa>(x);
    x += dpp_or0<0x143, 0xc>(x);
    return x;
}
__device__ __forceinline__ double lane_value(double x, int l) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)u, l);
    const unsigned hi = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)(u >> 32), l);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// Rows [0, 64) of a chunk tile of D channels, in 16-byte blocks over NT threads, rows
// from m on the last one again; to LDS with pitch LD, rows of bit 3 swizzled by SW channels (see
// ldfragTR).
template <int D, int NT, int LD, int SW>
struct RowTile {
    static constexpr int BPR = D / 8, RPP = NT / BPR, N = 64 / RPP;
    static_assert(NT % BPR == 0 && 64 % RPP == 0, "tile shape");
    u32x4 r[N];
    __device__ __forceinline__ void load(const __bf16 *p, int64_t ld, int m, int tid) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int row = min(tid / BPR + RPP * i, m - 1);
            r[i] = *reinterpret_cast<const u32x4 *>(p + row * ld + 8 * (tid % BPR));
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
// tile (tt, c) of such a triangle, two to a fragment
__device__ __forceinline__ constexpr int tri_tile16(int tt, int c) { return 2 * tri_frag(tt, c >> 1) + (c & 1); }

// The sequences that are taken in chunks, longest first: the walk's time is that of
// its longest sequence once the others no longer fill the chip, so that one starts
// first.  Sorted by buckets, four to a doubling (the order inside a bucket is free: it
// steers the schedule alone).  A sequence with more chunks than a CU's share of all
// chunk steps is what the launch waits for: it is walked in single column tiles, whose
// step is shorter, as long as each has a CU of its own; the others in pairs of tiles,
// which share what a chunk loads.  (Chunk steps, us: alone on a CU 2.2 single, 3.1 in
// pairs; with the CUs full 2.1 a single tile, 3.1 a pair.)  One workgroup.
constexpr int PLAN_B = 128;
__device__ __forceinline__ int plan_bucket(int64_t n) {
    const unsigned c = (unsigned)((n + 63) / 64);  // 1 .. 2^25
    const int lg = 31 - __builtin_clz(c);
    return PLAN_B - 1 - (4 * lg + (int)(((uint64_t)c << 2 >> lg) & 3));
}
// the fewest chunks of a bucket
__device__ __forceinline__ int64_t bucket_chunks(int b) {
    const int e = PLAN_B - 1 - b, lg = e >> 2;
    return (((int64_t)(4 + (e & 3)) << lg) + 3) >> 2;
}
__device__ __forceinline__ void make_plan(const GdnRaggedArgs &a, int *at, int tid) {
    int *const sum = at + PLAN_B, *const single = sum + 1;
    if (tid < PLAN_B + 2) at[tid] = 0;
    __syncthreads();
    auto length = [&](int i) {
        const Seq s = seq_of(a.r, i);
        return s.slot < 0 || s.end - s.begin <= a.longer ? (int64_t)0 : s.end - s.begin;
    };
    for (int i = tid; i < a.r.N; i += 256)
        if (const int64_t n = length(i)) {
            atomicAdd(&at[plan_bucket(n)], 1);
            atomicAdd(sum, (int)((n + 63) / 64));
        }
    __syncthreads();
    if (tid < 64) {  // counts become first places, two buckets a lane
        const int c0 = at[2 * tid], c1 = at[2 * tid + 1];
        int first = c0 + c1;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(first, o, 64);
            if (tid >= o) first += y;
        }
        const int64_t share = (int64_t)*sum * a.Hv * (a.Dv / 32) / a.n_cu, most = a.n_cu / (a.Hv * (a.Dv / 16));
        int own = 0;  // sequences of this lane's buckets that get single tiles
        if (bucket_chunks(2 * tid) > share && first - c1 <= most) own = c0;
        if (bucket_chunks(2 * tid + 1) > share && first <= most) own += c1;
        if (own) atomicAdd(single, own);
        at[2 * tid] = first - c0 - c1;
        at[2 * tid + 1] = first - c1;
        if (tid == 63) a.plan[0] = first;
    }
    __syncthreads();
    if (tid == 0) a.plan[1] = *single;
    for (int i = tid; i < a.r.N; i += 256)
        if (const int64_t n = length(i)) a.plan[2 + atomicAdd(&at[plan_bucket(n)], 1)] = i;
}

// ---------------------------------------------------------------- T and R of a chunk
template <int DK>
__global__ void __launch_bounds__(256, 4) k_rag_prep(GdnRaggedArgs a) {
    constexpr int NT = 256, LD = DK + 16, SW = swx<__bf16, DK>(), LA = 68;
    // A lies where K's tile was: its products are in registers by then
    constexpr int KB = 64 * LD * 2 > 64 * LA * 4 ? 64 * LD * 2 : 64 * LA * 4;
    __shared__ __attribute__((aligned(16))) char mem[KB];
    __bf16 *const sK = reinterpret_cast<__bf16 *>(mem);
    float *const sA = reinterpret_cast<float *>(mem);
    __shared__ __attribute__((aligned(16))) float sT[64 * LA];
    __shared__ __attribute__((aligned(16))) float sb[64], sbl[64], sbeta[64];  // sums (high, low), beta
    const int tid = threadIdx.x, lane = tid & 63, q4 = lane >> 4, n16 = lane & 15;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (blockIdx.x == 0) {
        make_plan(a, reinterpret_cast<int *>(mem), tid);
        return;
    }
    const unsigned block = blockIdx.x - 1;
    const int hk = block % a.Hk, group = a.Hv / a.Hk;
    const int64_t id = block / a.Hk;
    const int i = find_seq(a.r, a.sys_div, id, a.sys_add);
    const Seq sq = seq_of(a.r, i);
    const int64_t c0 = (id - gdn_first_system(a, sq.begin, i)) * 64, n = sq.end - sq.begin;
    if (c0 < 0 || c0 >= n || n <= a.longer || sq.slot < 0) return;
    const int m = n - c0 < 64 ? (int)(n - c0) : 64;
    const int64_t row0 = sq.begin + c0;
    // rows past the end stand for the last one: beta is 0 there, and their rows of P
    // make outputs that are not stored
    RowTile<DK, NT, LD, SW> t;
    t.load((const __bf16 *)a.k + row0 * a.sq_t + hk * a.sq_h, a.sq_t, m, tid);
    bf16x8 qt[DK / 32];
    {
        const __bf16 *q = (const __bf16 *)a.q + (row0 + min(16 * w + n16, m - 1)) * a.sq_t + hk * a.sq_h + 8 * q4;
#pragma unroll
        for (int ks = 0; ks < DK / 32; ++ks) qt[ks] = *reinterpret_cast<const bf16x8 *>(q + 32 * ks);
    }
    t.store(sK, tid);
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
#pragma unroll
        for (int st = 0; st < 4; ++st) {
            if (st >= 2 && w < 2) continue;  // above the diagonal
            const bf16x8 kf = *reinterpret_cast<const bf16x8 *>(
                &sK[(ar + 32 * (st >> 1) + 4 * (st & 1)) * LD + 8 * q4 + 32 * ks + (((32 * ks) & SW) ? -sgn : sgn)]);
            mma(kk[st], kf, kt);
            mma(qk[st], kf, qt[ks]);
        }
    }
    for (int hv = hk * group; hv < (hk + 1) * group; ++hv) {
        int ln = lane;
        asm volatile("" : "+v"(ln));  // addresses are formed for each head, not held in registers all the while
        const int lane = ln, q4 = lane >> 4, n16 = lane & 15, tok = 16 * w + n16;
        __syncthreads();  // the last head is done with the gates, with A and T (the first: all with K)
        if (w == 0) {
            const bool in = lane < m;
            const int64_t go = (row0 + lane) * a.sg_t + hv * a.sg_h;
            const double b = wave_scan_dpp(in ? gate_log2(a.g[go]) : 0.0);
            const float be = in ? a.beta[go] : 0.f, hi = (float)b;
            sb[lane] = hi;
            sbl[lane] = (float)(b - hi);
            sbeta[lane] = be;
            float *const gates = reinterpret_cast<float *>(a.ws + (id * a.Hv + hv) * (int64_t)RAG_SYS + RAG_GATES) + lane;
            gates[0] = fexp2(hi);
            gates[64] = fexp2((float)(lane_value(b, 63) - b));
            gates[128] = be;
        }
        __syncthreads();
        __bf16 *const sys = reinterpret_cast<__bf16 *>(a.ws + (id * a.Hv + hv) * (int64_t)RAG_SYS);
        const float bt = sb[tok], btl = sbl[tok], be = sbeta[tok];
        float pv[2][8] = {};  // P's row tok, columns 32 ks + 8 q4 ..
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            if (ks > (w >> 1)) continue;
            float av[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int s = 32 * ks + 8 * q4 + j;
                const float d = fexp2((bt - sb[s]) + (btl - sbl[s]));  // e^(b_tok - b_s)
                av[j] = s < tok ? be * kk[2 * ks + (j >> 2)][j & 3] * d : 0.f;
                pv[ks][j] = s <= tok ? qk[2 * ks + (j >> 2)][j & 3] * d : 0.f;
            }
            float *p = &sA[tok * LA + 32 * ks + 8 * q4];
            *reinterpret_cast<f32x4 *>(p) = f32x4{av[0], av[1], av[2], av[3]};
            *reinterpret_cast<f32x4 *>(p + 4) = f32x4{av[4], av[5], av[6], av[7]};
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
        // Rows 16 w .. of R = P T in fp32 MFMA, as R^T = T^T P^T: lane (q4, n16) gets four
        // columns of row 16 w + n16.  P lies in the wave's own rows of sA (A has had its last
        // read).  The wave with the most blocks here had the fewest above.
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            if (ks > (w >> 1)) continue;
            float *p = &sA[tok * LA + 32 * ks + 8 * q4];
            *reinterpret_cast<f32x4 *>(p) = f32x4{pv[ks][0], pv[ks][1], pv[ks][2], pv[ks][3]};
            *reinterpret_cast<f32x4 *>(p + 4) = f32x4{pv[ks][4], pv[ks][5], pv[ks][6], pv[ks][7]};
        }
        f32x4 acc[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            acc[k] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (k > w) continue;
            const f32x4 pk = *reinterpret_cast<const f32x4 *>(&sA[tok * LA + 16 * k + 4 * q4]);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int c = 0; c <= k; ++c)
                    acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(sT[(16 * k + 4 * q4 + e) * LA + 16 * c + n16], pk[e], acc[c], 0, 0, 0);
        }
        // T's fragments of tile w: rows 16 w + n16, columns 32 ks + 8 q4 ..
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            if (ks > (w >> 1)) continue;
            const float *p = &sT[tok * LA + 32 * ks + 8 * q4];
            bf16x8 f[3];
            split3(*reinterpret_cast<const f32x4 *>(p), *reinterpret_cast<const f32x4 *>(p + 4), f[0], f[1], f[2]);
#pragma unroll
            for (int pl = 0; pl < RAG_TP; ++pl)
                *reinterpret_cast<bf16x8 *>(sys + (pl * RAG_FRAGS + tri_frag(w, ks)) * 512 + 8 * lane) = f[pl];
        }
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (c <= (w | 1))
                *reinterpret_cast<f32x4 *>(reinterpret_cast<char *>(sys) + RAG_R + tri_tile16(w, c) * 1024 + 16 * lane) = acc[c];
    }
}

// ----------------------------------------------------------------------- the walk
// Per chunk, with barriers between the phases:
//   S's pieces to LDS | K S, Q S of the wave's tokens, X = beta (V - e^b K S) to LDS |
//   U = T X, to LDS in three pieces times e^(b_63 - b) | O, S
// K, Q, T and R are needed by one wave each, in fragment order: they come from memory
// into registers a chunk ahead and pass LDS only where K is read transposed.  R comes as
// it is, 12 KB instead of 18, and is cut beside the first products.
// Everything a chunk loads is waited for at one place, before the last chunk's outputs
// are stored: loads and stores share a counter (see vm_wait_all).

// LDS of a walk workgroup.  NC >= 2: K's tile and U's pieces lie where S's pieces were,
// which keeps the whole within 64 KB; one barrier more keeps the next chunk's S behind
// their last reads.
template <int DK, int NC>
struct WalkLds {
    static constexpr int LD = DK + 16, CW = 16 * NC, LS = DK + 16, LT = 64 + 16;
    static constexpr bool ALIAS = NC >= 2;
    static constexpr int NSP = 3 * CW * LS, NX = 3 * CW * LT, NU = 3 * CW * LT, NKT = 64 * LD;
    static constexpr int SIZE = NX + (ALIAS ? (NSP > NU + NKT ? NSP : NU + NKT) : NSP + NU + NKT);
};

// One item: 16 NC columns of one value head of sequence i; reach: fetch lines further ahead.
template <int DK, int NC>
__device__ __forceinline__ void rag_walk(const GdnRaggedArgs &a, __bf16 *mem, int i, int h, int cb, bool reach) {
    const int ncb = a.Dv / (16 * NC);
    constexpr int NK = DK / 32, NS = DK / 64;              // k-steps; state tiles of a wave
    constexpr int SW = swx<__bf16, DK>(), CW = 16 * NC;    // K tile's swizzle; columns
    typedef WalkLds<DK, NC> L;
    constexpr bool ALIAS = L::ALIAS;
    __bf16 *const sX = mem, *const sS = mem + L::NX, *const sU = ALIAS ? sS : sS + L::NSP, *const sK = sU + L::NU;
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));  // what follows from the lane is formed for each item, not held in registers between them
    const int lane = tid & 63, q4 = lane >> 4, n16 = lane & 15;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Seq s = seq_of(a.r, i);
    const int64_t n = s.end - s.begin;
    const int hk = h / (a.Hv / a.Hk), tok = 16 * w + n16;
    // bases are uniform, a chunk's rows 32-bit offsets from them
    const char *const K = (const char *)a.k + 2 * (s.begin * a.sq_t + hk * a.sq_h);
    const char *const Q = (const char *)a.q + 2 * (s.begin * a.sq_t + hk * a.sq_h);
    const char *const V = (const char *)a.v + 2 * (s.begin * a.sv_t + h * a.sv_h + cb * CW);
    __bf16 *const O = (__bf16 *)a.o + (s.begin + tok) * a.so_t + h * a.so_h + cb * CW + 4 * q4;
    const char *const sys = a.ws + (gdn_first_system(a, s.begin, i) * a.Hv + h) * (int64_t)RAG_SYS;
    const int64_t sys_step = (int64_t)a.Hv * RAG_SYS;
    float *const st = a.state + s.slot * a.ss + (int64_t)h * DK * a.Dv + (int64_t)(16 * NS * w + 4 * q4) * a.Dv + cb * CW + n16;

    // S[t][c][r] = state row 16 (NS w + t) + 4 q4 + r, column 16 c + n16 of the block
    f32x4 S[NS][NC];
    const bool fresh = a.r.fresh && a.r.fresh[i];
#pragma unroll
    for (int t = 0; t < NS; ++t)
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][c][r] = fresh ? 0.f : st[(int64_t)(16 * t + r) * a.Dv + 16 * c];

    bf16x8 kf[NK], qf[NK], t0[RAG_TP], t1[RAG_TP];
    f32x4 rf[2][2];  // R's row tok, columns 32 ks + 8 q4 ..
    unsigned short vf[NC][4];
    f32x4 eb, ee, be;  // of the wave's rows 16 w + 4 q4 + r
    float et, gam;     // e^b of token 16 w + n16, of the chunk
    const bool two = w >= 2;  // the wave's tile of T and R has a second k-step
    // rows past the sequence's end stand for its last one: their beta is 0, so they
    // change nothing
    auto last_row = [&](int64_t c) { return n - c < 64 ? (int)(n - c) - 1 : 63; };
    auto fetch_k = [&](int64_t c) {
        const char *const p = K + 2 * c * a.sq_t;
        const uint32_t o = 2u * ((uint32_t)min(tok, last_row(c)) * (uint32_t)a.sq_t + 8 * q4);
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) kf[ks] = *reinterpret_cast<const bf16x8 *>(p + o + 64 * ks);
    };
    auto fetch_qv = [&](int64_t c) {
        const char *const p = Q + 2 * c * a.sq_t, *const v = V + 2 * c * a.sv_t;
        const uint32_t o = 2u * ((uint32_t)min(tok, last_row(c)) * (uint32_t)a.sq_t + 8 * q4);
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) qf[ks] = *reinterpret_cast<const bf16x8 *>(p + o + 64 * ks);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const uint32_t ov = 2u * ((uint32_t)min(16 * w + 4 * q4 + r, last_row(c)) * (uint32_t)a.sv_t + n16);
#pragma unroll
            for (int x = 0; x < NC; ++x) vf[x][r] = *reinterpret_cast<const unsigned short *>(v + ov + 32 * x);
        }
    };
    const int f0 = tri_frag(w, 0) * 1024;
    const uint32_t l16 = 16 * lane;
    auto fetch_t = [&](const char *p) {
#pragma unroll
        for (int pl = 0; pl < RAG_TP; ++pl) t0[pl] = *reinterpret_cast<const bf16x8 *>(p + f0 + pl * RAG_FRAGS * 1024 + l16);
        if (two) {
#pragma unroll
            for (int pl = 0; pl < RAG_TP; ++pl)
                t1[pl] = *reinterpret_cast<const bf16x8 *>(p + f0 + (pl * RAG_FRAGS + 1) * 1024 + l16);
        }
    };
    const uint32_t r16 = 1024 * (q4 >> 1) + 512 * (q4 & 1) + 16 * n16;
    auto fetch_r = [&](const char *p) {
        p += RAG_R + 2 * f0;
#pragma unroll
        for (int m = 0; m < 2; ++m) rf[0][m] = *reinterpret_cast<const f32x4 *>(p + r16 + 256 * m);
        if (two) {
#pragma unroll
            for (int m = 0; m < 2; ++m) rf[1][m] = *reinterpret_cast<const f32x4 *>(p + 2048 + r16 + 256 * m);
        }
    };
    auto fetch_gates = [&](const char *p) {
        p += RAG_GATES + 64 * w;
        eb = *reinterpret_cast<const f32x4 *>(p + 16 * q4);
        ee = *reinterpret_cast<const f32x4 *>(p + 256 + 16 * q4);
        be = *reinterpret_cast<const f32x4 *>(p + 512 + 16 * q4);
        et = *reinterpret_cast<const float *>(p + 4 * n16);
        gam = *reinterpret_cast<const float *>(p - 64 * w + 4 * 63);
    };
    const bf16x8 zero8 = __builtin_bit_cast(bf16x8, u32x4{0u, 0u, 0u, 0u});
#pragma unroll
    for (int pl = 0; pl < RAG_TP; ++pl) t1[pl] = zero8;
    rf[1][0] = rf[1][1] = f32x4{0.f, 0.f, 0.f, 0.f};
    fetch_k(0);
    fetch_qv(0);
    fetch_t(sys);
    fetch_r(sys);
    fetch_gates(sys);
    const LaneOff tr = tr_off<__bf16, L::LD, SW>(lane);
    bf16x4 out[NC];
    const char *next = sys;
    unsigned ahead = 0u;
    for (int64_t c = 0; c < n; c += 64) {
        next += sys_step;
        const bool more = c + 64 < n;
        if (ALIAS && c > 0) __syncthreads();  // the last chunk is done with K and U
        // S's pieces, [piece][column][key row]
#pragma unroll
        for (int x = 0; x < NC; ++x)
#pragma unroll
            for (int t = 0; t < NS; ++t) {
                bf16x4 f[3];
                split3(S[t][x], f[0], f[1], f[2]);
#pragma unroll
                for (int p = 0; p < 3; ++p)
                    *reinterpret_cast<bf16x4 *>(sS + (p * CW + 16 * x + n16) * L::LS + 16 * (NS * w + t) + 4 * q4) = f[p];
            }
        vm_wait_all();
        asm volatile("" ::"v"(ahead));  // the line has come; nothing uses it
        if (c > 0) {
#pragma unroll
            for (int x = 0; x < NC; ++x) *reinterpret_cast<bf16x4 *>(O + (c - 64) * a.so_t + 16 * x) = out[x];
        }
        __syncthreads();
        // The system after next, a line a lane shared out over the head's column blocks:
        // its fragments then come from this XCD's L2 when they are fetched.
        if (reach && c + 128 < n && lane % ncb == cb)
            ahead = *reinterpret_cast<const unsigned *>(next + sys_step + 128 * min(64 * w + lane, RAG_SYS / 128 - 1));
        // Operand fragments are read a step ahead of their products, and the fences keep it
        // so: left alone, the compiler may read each pair just before its use, and then
        // every two matrix instructions wait for LDS.
        bf16x8 rp[2][3];     // R's pieces
        f32x4 X[NC], Y[NC];  // K S (rows: tokens 16 w + 4 q4 + r), (Q S)^T (columns: tokens 16 w + n16)
        {
            bf16x8 f[2][NK];
            auto read = [&](int step) {  // column tile step / 3, piece 2 - step % 3
#pragma unroll
                for (int ks = 0; ks < NK; ++ks)
                    f[step & 1][ks] = *reinterpret_cast<const bf16x8 *>(
                        sS + ((2 - step % 3) * CW + 16 * (step / 3) + n16) * L::LS + 32 * ks + 8 * q4);
            };
            read(0);
#pragma unroll
            for (int step = 0; step < 3 * NC; ++step) {
                const int x = step / 3;
                if (step + 1 < 3 * NC) read(step + 1);
                sched_fence();
                if (step % 3 == 0) X[x] = Y[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < NK; ++ks) {
                    mma(X[x], kf[ks], f[step & 1][ks]);
                    mma(Y[x], f[step & 1][ks], qf[ks]);
                }
                if (step == 0) split3(rf[0][0], rf[0][1], rp[0][0], rp[0][1], rp[0][2]);
                if (step == 1) split3(rf[1][0], rf[1][1], rp[1][0], rp[1][1], rp[1][2]);
                sched_fence();
            }
        }
#pragma unroll
        for (int x = 0; x < NC; ++x) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                X[x][r] = be[r] * (__uint_as_float((unsigned)vf[x][r] << 16) - eb[r] * X[x][r]);
            bf16x4 f[3];
            split3(X[x], f[0], f[1], f[2]);
#pragma unroll
            for (int p = 0; p < 3; ++p)
                *reinterpret_cast<bf16x4 *>(sX + (p * CW + 16 * x + n16) * L::LT + 16 * w + 4 * q4) = f[p];
        }
        if (more) fetch_qv(c + 64);
        __syncthreads();
        bf16x8 xf[NC][3][2];
#pragma unroll
        for (int x = 0; x < NC; ++x)
#pragma unroll
            for (int p = 0; p < 3; ++p)
#pragma unroll
                for (int ks = 0; ks < 2; ++ks)
                    xf[x][p][ks] = *reinterpret_cast<const bf16x8 *>(sX + (p * CW + 16 * x + n16) * L::LT + 32 * ks + 8 * q4);
        sched_fence();
        // K's tile, for the transposed reads (S's pieces have had their last read)
#pragma unroll
        for (int ks = 0; ks < NK; ++ks)
            *reinterpret_cast<bf16x8 *>(sK + tok * L::LD + swz_col(tok, 32 * ks + 8 * q4, SW)) = kf[ks];
        if (more) fetch_k(c + 64);
        // O^T = e^b (Q S)^T + X^T R^T; the last tile's while the next phase's operands come from LDS
        auto out_products = [&](int x) {
            Y[x] *= et;
            f32x4 Y1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                if (ks == 1 && !two) continue;
                mma(Y1, xf[x][0][ks], rp[ks][2]);
                mma(Y[x], xf[x][1][ks], rp[ks][1]);
                mma(Y1, xf[x][2][ks], rp[ks][0]);
                mma(Y[x], xf[x][1][ks], rp[ks][0]);
                mma(Y1, xf[x][0][ks], rp[ks][1]);
                mma(Y[x], xf[x][0][ks], rp[ks][0]);
            }
            Y[x] += Y1;
        };
        f32x4 U[NC];
#pragma unroll
        for (int x = 0; x < NC; ++x) {
            U[x] = f32x4{0.f, 0.f, 0.f, 0.f};
            f32x4 U1 = U[x];
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                if (ks == 1 && !two) continue;
                const bf16x8(&t)[RAG_TP] = ks ? t1 : t0;
                mma(U1, t[2], xf[x][0][ks]);
                mma(U[x], t[1], xf[x][1][ks]);
                mma(U1, t[0], xf[x][2][ks]);
                mma(U[x], t[1], xf[x][0][ks]);
                mma(U1, t[0], xf[x][1][ks]);
                mma(U[x], t[0], xf[x][0][ks]);
            }
            U[x] += U1;
            if (x + 1 < NC) out_products(x);
            bf16x4 f[3];
            const f32x4 ue = U[x] * ee;
            split3(ue, f[0], f[1], f[2]);
#pragma unroll
            for (int p = 0; p < 3; ++p)
                *reinterpret_cast<bf16x4 *>(sU + (p * CW + 16 * x + n16) * L::LT + 16 * w + 4 * q4) = f[p];
        }
        if (more) fetch_t(next);
        __syncthreads();
        auto u_piece = [&](int x, int p, int ks) {
            return *reinterpret_cast<const bf16x8 *>(sU + (p * CW + 16 * x + n16) * L::LT + 32 * ks + 8 * q4);
        };
        bf16x8 uf[2][3][2], kt[NS][2];  // U's pieces, K^T
        auto read_pieces = [&](int x) {
#pragma unroll
            for (int p = 0; p < 3; ++p)
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) uf[x & 1][p][ks] = u_piece(x, p, ks);
        };
        read_pieces(0);
        sched_fence();
        out_products(NC - 1);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int t = 0; t < NS; ++t) kt[t][ks] = ldfragTR<__bf16, L::LD, SW>(sK, tr, 32 * ks, 16 * (NS * w + t));
        if (more) fetch_r(next);
        // S = e^(b_63) S + K^T e^(b_63 - b) U
#pragma unroll
        for (int x = 0; x < NC; ++x) {
            if (x + 1 < NC) read_pieces(x + 1);
            sched_fence();
#pragma unroll
            for (int t = 0; t < NS; ++t) S[t][x] *= gam;
            if (x + 1 == NC && more) fetch_gates(next);
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int p = 2; p >= 0; --p)
#pragma unroll
                    for (int t = 0; t < NS; ++t) mma(S[t][x], kt[t][ks], uf[x & 1][p][ks]);
            sched_fence();
        }
#pragma unroll
        for (int x = 0; x < NC; ++x)
#pragma unroll
            for (int r = 0; r < 4; ++r) out[x][r] = (__bf16)Y[x][r];
    }
    const int64_t last = (n - 1) / 64 * 64;
    if (last + tok < n) {
#pragma unroll
        for (int x = 0; x < NC; ++x) *reinterpret_cast<bf16x4 *>(O + last * a.so_t + 16 * x) = out[x];
    }
#pragma unroll
    for (int t = 0; t < NS; ++t)
#pragma unroll
        for (int x = 0; x < NC; ++x)
#pragma unroll
            for (int r = 0; r < 4; ++r) st[(int64_t)(16 * t + r) * a.Dv + 16 * x] = S[t][x][r];
}

// Items of the walk over the planned sequences from..to, numbered from `first` on, in
// steps of the launch's workgroups: pairs of a sequence and a value head eight at a time,
// their column blocks eight apart, so that the blocks of a pair run on one XCD, whose L2
// then holds what they share.
template <int DK, int NC>
__device__ __forceinline__ void rag_walk_items(const GdnRaggedArgs &a, __bf16 *mem, int from, int to, int64_t first,
                                               int groups, bool reach) {
    const int ncb = a.Dv / (16 * NC);
    const int64_t items = gdn_walk_items(a, to - from, NC);
    int64_t id = (int64_t)blockIdx.x - first % groups;
    if (id < 0) id += groups;
    for (; id < items; id += groups) {
        const int64_t pair = id / (8 * ncb) * 8 + id % 8;
        const int rank = from + (int)(pair / a.Hv);
        if (rank >= to) continue;
        __syncthreads();  // the last item is done with the LDS
        rag_walk<DK, NC>(a, mem, __builtin_amdgcn_readfirstlane(a.plan[2 + rank]), (int)(pair % a.Hv), (int)(id / 8 % ncb), reach);
    }
}

// The long sequences' walk, and beside it, behind its workgroups, the tokens of the
// short ones: the walk waits for its own chain, the tokens for memory.
template <int DK>
__global__ void __launch_bounds__(256, 2) k_rag_walk(GdnRaggedArgs a, int groups) {
    constexpr int S1 = WalkLds<DK, 1>::SIZE, S2 = WalkLds<DK, 2>::SIZE;
    __shared__ __attribute__((aligned(16))) __bf16 mem[S1 > S2 ? S1 : S2];
    if ((int)blockIdx.x >= groups) {
        gdn_tokens<__bf16, DK, TOK_CL>(a, (int64_t)(blockIdx.x - groups) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
        return;
    }
    const int count = __builtin_amdgcn_readfirstlane(a.plan[0]), single = __builtin_amdgcn_readfirstlane(a.plan[1]);
    // lines are fetched two chunks ahead while all items run at once (16384 tokens of 40
    // heads: 992 us against 1009; but 32 prompts of 1024 of 20 heads, five items to a place:
    // 584 against 577)
    const int64_t one = gdn_walk_items(a, single, 1), pairs = gdn_walk_items(a, count - single, 2);
    const bool reach = one + pairs <= 2 * (int64_t)a.n_cu;
    rag_walk_items<DK, 1>(a, mem, 0, single, 0, groups, reach);
    rag_walk_items<DK, 2>(a, mem, single, count, one, groups, reach);
}

}  // namespace

hipError_t launch_gdn_chunk_prep(const GdnRaggedArgs &a, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
    const dim3 grid((unsigned)(a.n_chunks * a.Hk + 1));
    if (a.Dk == 128) hipExtLaunchKernelGGL((k_rag_prep<128>), grid, dim3(256), 0, s, e0, e1, 0, a);
    else hipExtLaunchKernelGGL((k_rag_prep<64>), grid, dim3(256), 0, s, e0, e1, 0, a);
    return hipGetLastError();
}

hipError_t launch_gdn_chunk_walk(const GdnRaggedArgs &a, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
    const int groups = (int)gdn_walk_groups(a);
    const dim3 grid((unsigned)(groups + (gdn_token_waves(a) + 3) / 4)), block(256);
    if (a.Dk == 128) hipExtLaunchKernelGGL((k_rag_walk<128>), grid, block, 0, s, e0, e1, 0, a, groups);
    else hipExtLaunchKernelGGL((k_rag_walk<64>), grid, block, 0, s, e0, e1, 0, a, groups);
    return hipGetLastError();
}

}  // namespace sf
