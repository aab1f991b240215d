// sf_launch.hpp -- argument block shared by the host driver and the kernels.
#pragma once
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "stateflow.h"

namespace sf {

// segments of a chain that one set of launches can cover: their table travels in the
// kernel arguments; longer chains run segment by segment (H 16, 512 tokens each: 41.8 us
// a segment, forward and backward, for 32 of them, 60.9 for 33)
constexpr int MAX_MERGED = 32;

// One segment (or one superchunk-parallel launch over a segment).  Token
// tensors point at the segment's first token; strides are in elements.
struct SegArgs {
    const void *q, *k, *v, *dO;
    void *o, *dq, *dk, *dv;
    const float *g;
    float *dg;
    int64_t sx_b, sx_l, sx_h;
    int64_t sg_b, sg_l, sg_h;
    int32_t B, H;
    int32_t vec;      // 1: per-key-channel gate (g, dg are [B][L][H][D])
    int32_t n_cu;     // compute units of the device
    int64_t L;        // tokens in the segment
    int32_t ts;       // superchunk length (multiple of 64)
    int32_t n_super;  // ceil(L / ts)
    const float *S_in;
    float *S_out;
    const float *dS_out;
    float *dS_in;
    float *wsS;    // [B][H][n_super][D][D]: D_J, replaced by S_J by the scan
    float *wsE;    // [B][H][n_super][D][D]: E_J, replaced by G_{J+1} (backward only)
    float *wsLg;   // [B][H][n_super] (vector gate: [..][D]): log2 of the superchunk decay
    float *wsDot;  // [B][H][n_super][D]: <G_{J+1}, S_{J+1}> per key row (scalar
                   // gate, one superchunk: D partials of it)
    float *wsSn;   // [B][H][D][D] or NULL: the state leaving the segment, kept
                   // beside the superchunk states when the forward keeps them
    int32_t ckpt;  // backward: 1 when wsS, wsLg and wsSn already hold the
                   // forward's superchunk states, decays and final state
    // a chain run as one segment: n_seg > 1 segments, segment i holding the
    // superchunks seg_sc[i] .. seg_sc[i + 1] - 1 of seg_m[i] chunks from chunk seg_ck[i]
    // on (the last superchunk of each may be short); the forward scan writes the state
    // entering segment i >= 1 to S_bnd + i B H D D, the backward's replay starts from it
    int32_t n_seg;
    int32_t seg_sc[MAX_MERGED + 1], seg_ck[MAX_MERGED + 1], seg_m[MAX_MERGED];
    float *S_bnd;
};

// kind is an sf_kernel_id; io an sf_dtype.  The scan runs its backward form
// when wsE is set.  Non-null e0/e1 take the begin timestamp of the first
// kernel the kind launches and the end timestamp of its last (the timing
// rides on the dispatch packets, no marker packets are added).
hipError_t launch_kernel(int kind, int io, int D, const SegArgs &a, hipStream_t s, hipEvent_t e0 = nullptr,
                         hipEvent_t e1 = nullptr);
hipError_t launch_kernel_vg(int kind, int io, int D, const SegArgs &a, hipStream_t s, hipEvent_t e0, hipEvent_t e1);
hipError_t launch_state_copy(const float *src, float *dst, int64_t n, hipStream_t s);

// Short convolution (sf_conv.hip).  Token blocks of T; nTB blocks per batch;
// ws holds B * nTB dw partials of C * W floats.
struct ConvArgs {
    const void *x;
    const float *w;
    const float *tail_in;
    void *y;
    float *tail_out;
    const void *dy;
    const float *dtail_out;
    void *dx;
    float *dw;
    float *dtail_in;
    float *ws;
    int32_t B, C, W, act, io;
    int32_t nTB, n_cu;  // token blocks; compute units of the device
    int64_t L, T, sx_b, sx_l;
};
int conv_channels_per_thread();
constexpr int CONV_E = 8, CONV_G = 8;  // channels per thread, tokens per load group
// Threads per CU that fill the chip, below which runs are shortened.  Forward: six
// waves (256 CUs, bf16, 101248 threads: whole runs 214 us, halves 226).  Backward: the
// split runs cost halos, so the line lies where they stop paying (256 CUs, whole
// blocks / runs, us): bf16 122880 threads 350/384, 101248 340/343, 50624 253/199; fp32
// 61440 threads 318/352, 50624 309/346, 25312 253/200.
constexpr int64_t CONV_FILL = 384, CONV_FILL_BWD16 = 384, CONV_FILL_BWD32 = 160;
// tokens per thread of the forward: 256, halved until the launch fills the chip
inline int64_t conv_fwd_run(int64_t B, int64_t C, int64_t L, int n_cu) {
    int64_t T = 256;
    while (T > CONV_G && B * (C / CONV_E) * ((L + T - 1) / T) < CONV_FILL * n_cu) T /= 2;
    return T;
}
// runs per block of the backward: doubled until the launch fills the chip, at most
// one per load group of the shortest block
inline int conv_bwd_runs(int64_t threads, bool b16, int n_cu) {
    int sub = 1;
    while (sub < 32 && threads * sub < (b16 ? CONV_FILL_BWD16 : CONV_FILL_BWD32) * n_cu) sub *= 2;
    return sub;
}

// Gated delta rule (sf_gdn.hip).  n_super superchunks of ts tokens per
// (batch, head); with n_super > 1 the workspace holds the boundary states
// wsS [B*H][n_super][D][D] and the superchunk maps wsM, wsN
// [B*H][n_prep][D][D] (these fp32; n_prep = n_super - 1 for the forward,
// n_super for the backward, which also needs M of the last superchunk).
struct GdnArgs {
    const void *q, *k, *v;
    const float *g, *beta, *S_in;
    void *o, *v_new;
    float *S_out;
    float *wsS, *wsM, *wsN;  // boundary states; superchunk maps (n_prep per head)
    float *wsSc;             // backward: the state entering every chunk [B*H][L/64], as two D x D planes of
                             // bf16 (hi, lo), transposed: the bytes of an fp32 state
    // backward
    const void *dO;
    const float *dS_out;
    void *dq, *dk, *dv;
    float *dg, *dbeta, *dS_in;
    float *wsE, *wsDe;  // superchunk dS offsets E_J [B*H][n_super-1], dS_end(J) [B*H][n_super]
    float *wsDc;        // dS' of every chunk, as wsSc
    int32_t B, H, n_super, ts, n_prep, n_x;  // n_x: workgroups of the per-chunk gradient kernel
    int32_t scan_out;  // forward chains: maps of every superchunk, the scan writes S_out
    int32_t n_cu;      // compute units of the device
    void *tw;          // D = 128: the output (o or dq) whose rows hold T until it is written;
                       // NULL: the output walk forms T (calls of one chunk)
    int64_t L, sx_b, sx_l, sx_h, sg_b, sg_l, sg_h;
};
// One kernel of the delta-rule pipeline: T of every chunk (D = 128); forward prep
// (the superchunks' maps M and N), scan (S_J), output walk; backward state-storing walk, dS prep
// (E_J), dS scan (dS_end(J)), dS walk, per-chunk gradients.
enum GdnPhase { GDN_PREP, GDN_SCAN, GDN_OUT, GDN_STORE, GDN_DPREP, GDN_DSCAN, GDN_DWALK, GDN_DCHUNK, GDN_TPREP };
hipError_t launch_gdn_phase(int phase, const GdnArgs &a, int D, hipStream_t s, hipEvent_t e0, hipEvent_t e1);
hipError_t launch_conv(bool bwd, const ConvArgs &a, hipStream_t s, hipEvent_t e0, hipEvent_t e1);


// Ragged batches (sf_ragged.hip): see sf_ragged in stateflow.h for cu, slot, fresh.
struct RaggedArgs {
    const int32_t *cu, *slot;
    const uint8_t *fresh;
    int32_t N, n_slots;
    int64_t T;
};
struct GdnRaggedArgs {
    RaggedArgs r;
    const void *q, *k, *v;
    const float *g, *beta;
    float *state;
    void *o;
    int32_t Hk, Hv, Dk, Dv, io, n_cu;
    int64_t sq_t, sq_h, sv_t, sv_h, so_t, so_h, sg_t, sg_h, ss;
    int32_t longer;    // sequences of more tokens are taken in chunks (0: none are)
    int32_t sys_div, sys_add;  // see gdn_first_system
    int64_t n_chunks;  // numbers of chunk systems
    char *ws;          // chunk systems: [n_chunks][Hv] of RAG_SYS bytes
    int32_t *plan;     // [2 + N], see gdn_plan_at
};
// waves of the token-by-token kernel: one for each sequence, value head and tile of 4 cl
// columns.  TOK_CL column lanes take whole 128-byte lines of the state; half of them make
// a token cheaper for a wave, and pay while there is a SIMD for each (16 tokens of 20
// heads of 128, us with 8 / 4 lanes: one sequence 17.8 / 15.4, 8 sequences 19.7 / 22.1,
// 64 71 / 96): launches of at most TOK_FEW full waves a CU.
constexpr int TOK_CL = 8, TOK_FEW = 2;
inline int64_t gdn_token_waves(const GdnRaggedArgs &a, int cl = TOK_CL) { return (int64_t)a.r.N * a.Hv * (a.Dv / (4 * cl)); }
// A chunk's triangular system: T = (I + A)^-1 as operand fragments in three bf16 planes
// (exact), six of 1 KB a plane, R = P T as it is in 12 tiles of 16 x 16, then the chunk's
// e^b, e^(b_63 - b) and beta (sf_ragged_chunk.hip)
constexpr int RAG_FRAGS = 6, RAG_TP = 3, RAG_R = RAG_TP * RAG_FRAGS * 1024, RAG_GATES = RAG_R + 12 * 1024, RAG_SYS = RAG_GATES + 1024;
// Sequences up to so many tokens are taken token by token: a chunk costs the same
// whatever its tokens, a token what the CUs' other waves leave it (20 heads of 128, us in
// chunks / token by token: one sequence of 8 tokens 13.4 / 9.2, of 12 13.3 / 12.0, of 16
// 13.4 / 15.1; 64 sequences of 16 tokens 101 / 72, of 24 99 / 98, of 32 99 / 122; 256 of 24
// with 40 heads 697 / 632, of 32 720 / 856).
constexpr int RAG_LONG = 24, RAG_LONG_FEW = 12;
static_assert(RAG_LONG < 32 && RAG_LONG_FEW < 32, "n / (longer + 1) >= ceil(n / 64) from longer + 1 tokens on");
inline int gdn_long(const GdnRaggedArgs &a) { return gdn_token_waves(a) <= a.n_cu ? RAG_LONG_FEW : RAG_LONG; }
// Chunk systems are numbered without a table: those of sequence i, if it is taken in chunks,
// begin at cu[i] / sys_div + sys_add i.  Either 64 and 1, T / 64 + N numbers: a sequence
// has room for its last, short chunk.  Or longer + 1 and 0, T / (longer + 1) numbers: one of n
// tokens, n > longer, has n / (longer + 1) >= ceil(n / 64) of them, and short sequences,
// however many, none.  The fewer are taken (gdn_number).
__host__ __device__ inline int64_t gdn_first_system(const GdnRaggedArgs &a, int64_t begin, int64_t i) {
    return (int64_t)((uint32_t)begin / (uint32_t)a.sys_div) + a.sys_add * i;  // rows fit 31 bits
}
inline void gdn_number(GdnRaggedArgs &a) {
    const int64_t all = a.r.T / 64 + a.r.N, few = a.longer ? a.r.T / (a.longer + 1) : all;
    a.sys_div = few < all ? a.longer + 1 : 64;
    a.sys_add = few < all ? 0 : 1;
    a.n_chunks = few < all ? few : all;
}
// items of the walk with nc 16-column tiles each, for n sequences: (sequence, value
// head) pairs in eights, their column blocks
__host__ __device__ inline int64_t gdn_walk_items(const GdnRaggedArgs &a, int64_t n, int nc) {
    return (n * a.Hv + 7) / 8 * 8 * (a.Dv / (16 * nc));
}
// workgroups of the walk: an item each while there are fewer than eight a CU
inline int64_t gdn_walk_groups(const GdnRaggedArgs &a) {
    const int64_t n = gdn_walk_items(a, a.r.N, 1), most = 8 * (int64_t)a.n_cu;
    return n < most ? n : most;
}
// behind the chunk systems: how many sequences are taken in chunks, how many of them in
// single column tiles, then their numbers, longest first
inline size_t gdn_plan_at(const GdnRaggedArgs &a) { return (size_t)a.n_chunks * (size_t)a.Hv * RAG_SYS; }
inline size_t gdn_chunk_ws_bytes(const GdnRaggedArgs &a) { return gdn_plan_at(a) + 4 * ((size_t)a.r.N + 2); }
// T and R of every chunk and the plan; then the walk, with the other sequences' tokens
hipError_t launch_gdn_chunk_prep(const GdnRaggedArgs &a, hipStream_t s, hipEvent_t e0, hipEvent_t e1);
hipError_t launch_gdn_chunk_walk(const GdnRaggedArgs &a, hipStream_t s, hipEvent_t e0, hipEvent_t e1);
hipError_t launch_gdn_tokens(const GdnRaggedArgs &a, hipStream_t s, hipEvent_t e0, hipEvent_t e1);
struct ConvRaggedArgs {
    RaggedArgs r;
    const void *x;
    const float *w;
    float *tails;
    void *y;
    int32_t C, W, act, io;
    int32_t run;     // tokens of one sequence that a thread takes
    int64_t n_runs;  // upper bound of the runs: T / run + N
    int64_t sx_t, sy_t, ss;
};
// Tokens of a run: 32 keep the halo rows, read twice, under a tenth (8259 tokens of
// 15360 channels: runs of 8 118 us, 16 99, 32 101, 64 113), 8 (one load group) where
// longer ones would leave the chip short of threads (CONV_FILL).
inline int conv_ragged_run(int64_t T, int64_t N, int64_t C, int n_cu) {
    int run = 32;
    while (run > CONV_G && (T / run + N) * (C / CONV_E) < CONV_FILL * n_cu) run /= 2;
    return run;
}
hipError_t launch_conv_ragged(const ConvRaggedArgs &a, hipStream_t s, hipEvent_t e0, hipEvent_t e1);

// Norms and rotation of queries and keys (sf_qk.hip).
struct QkArgs {
    const void *q, *k, *dyq, *dyk;  // dyq, dyk: backward
    void *yq, *yk;                  // backward: dq, dk
    const float *wq, *wk;
    const double *inv_freq;
    const int64_t *pos;
    float *dwq, *dwk, *ws;
    int32_t B, Hq, Hk, D, io, norm, R, inter;
    float eps, q_scale;
    int32_t n_tok;   // B * L
    int32_t parts;   // waves that share one token's heads
    int32_t blocks;  // workgroups
    int64_t L, pos0, sp_b, sp_l;
    sf_strides sq, sk, syq, syk, sdyq, sdyk;
};
constexpr int QK_W = 4;  // waves of a workgroup
// workgroups that share a CU (the weights' gradients take registers)
constexpr int qk_resident(bool bwd, bool weights) { return bwd && weights ? 3 : 4; }
// row groups a wave has in flight, twice over: 64 bytes a lane, which fits the registers
constexpr int qk_groups(bool bwd, size_t elem) { return (int)((bwd ? 4 : 8) / elem); }
// parts and blocks of a launch, from the shape
inline void qk_plan(QkArgs &a, bool bwd, bool weights, int n_cu) {
    int lpr = 2;  // lanes of a row
    while (8 * lpr < a.D) lpr *= 2;
    const int rows = 64 / lpr * qk_groups(bwd, a.io == SF_BF16 ? 2 : 4);
    const int groups = (a.Hq + rows - 1) / rows + (a.Hk + rows - 1) / rows;
    // a token's row groups are shared between waves until the launch has eight a CU
    a.parts = 1;
    while (a.parts < groups && (int64_t)a.n_tok * a.parts < 8 * (int64_t)n_cu) ++a.parts;
    // no more workgroups than the CUs hold, each wave with the same number of tokens, or one less
    const int64_t units = (int64_t)a.n_tok * a.parts, most = qk_resident(bwd, weights) * (int64_t)n_cu * QK_W;
    const int64_t each = (units + most - 1) / most;
    a.blocks = each ? (int32_t)(((units + each - 1) / each + QK_W - 1) / QK_W) : 0;
}
hipError_t launch_qk(bool bwd, const QkArgs &a, hipStream_t s, hipEvent_t e0, hipEvent_t e1);

}  // namespace sf
