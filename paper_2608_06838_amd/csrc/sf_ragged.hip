// sf_ragged.hip -- gfx950 kernels over ragged batches: sequences of any lengths
// packed along the token axis, each with a state of its own in a pool of slots,
// updated in place.
//
// Gated delta rule: sequences taken token by token (gdn_tokens, sf_ragged.hpp); long
// ones are taken in chunks by sf_ragged_chunk.hip.  Short convolution: below.
#include "sf_ragged.hpp"

#include <type_traits>

namespace sf {

namespace {

// ------------------------------------------------- gated delta rule, token by token
template <typename T, int DK, int CL>
__global__ void __launch_bounds__(TOK_NT) k_gdn_tokens(GdnRaggedArgs a) {
    gdn_tokens<T, DK, CL>(a, (int64_t)blockIdx.x * (TOK_NT / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
}

template <typename T, int CL>
hipError_t gdn_tokens_t(const GdnRaggedArgs &a, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
    const dim3 grid((unsigned)((gdn_token_waves(a, CL) + TOK_NT / 64 - 1) / (TOK_NT / 64)));
    if (a.Dk == 128) hipExtLaunchKernelGGL((k_gdn_tokens<T, 128, CL>), grid, dim3(TOK_NT), 0, s, e0, e1, 0, a);
    else hipExtLaunchKernelGGL((k_gdn_tokens<T, 64, CL>), grid, dim3(TOK_NT), 0, s, e0, e1, 0, a);
    return hipGetLastError();
}

// ------------------------------------------------------------------ short convolution
// u_t = sum_j w_j xh_{t-W+1+j}, y_t = act(u_t), each sequence preceded by its slot's
// tail.  Streaming work like the training form: a thread takes 8 consecutive channels
// and a run of tokens of one sequence (find_seq).  The sequence's first run alone reads the old tail, and it writes the new one, after
// that read, from the sequence's last rows, so the pool is updated in place with no
// order between workgroups.  8259 tokens of 15360 channels: 100 us, 5.1 TB/s.
constexpr int CR_NT = 256, CR_G = 8;  // threads; tokens loaded together

// u sigmoid(u) by the hardware exp2 and reciprocal, one unit in the last place each
// (an exact division is ten instructions an element, more than the window's)
template <bool SILU>
__device__ __forceinline__ float conv_act(float u) {
    if constexpr (SILU) return u * __builtin_amdgcn_rcpf(1.f + fexp2(-u * LOG2E));
    else return u;
}

template <typename T>
__device__ __forceinline__ void ld8(const T *p, float (&f)[8]) {
    const f32x4 lo = ld4f(p), hi = ld4f(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        f[e] = lo[e];
        f[4 + e] = hi[e];
    }
}

// a row's 8 channels as they lie in memory, read and written past the caches (the packed
// prompts above: 108 us through them)
template <typename T>
struct Row {
    static constexpr int NV = 8 * (int)sizeof(T) / 16;
    typedef unsigned u4 __attribute__((ext_vector_type(4)));
    u4 v[NV];
    __device__ __forceinline__ void load(const T *p) {
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = __builtin_nontemporal_load(reinterpret_cast<const u4 *>(p) + i);
    }
    __device__ __forceinline__ void f32(float (&f)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (sizeof(T) == 2) f[e] = __uint_as_float((e & 1) ? v[0][e / 2] & 0xffff0000u : v[0][e / 2] << 16);
            else f[e] = __uint_as_float(v[e / 4][e % 4]);
        }
    }
};

template <typename T, int W, bool SILU>
__global__ void __launch_bounds__(CR_NT) k_conv_ragged(ConvRaggedArgs a) {
    const int nb = (a.C / 8 + (int)blockDim.x - 1) / (int)blockDim.x;  // workgroups of a run
    const int c0 = 8 * ((int)(blockIdx.x % nb) * (int)blockDim.x + (int)threadIdx.x);
    const int64_t id = blockIdx.x / nb;
    const int i = find_seq(a.r, a.run, id);
    const Seq sq = seq_of(a.r, i);
    const int64_t t0 = (id - first_run(sq, a.run, i)) * a.run, n = sq.end - sq.begin;
    if (t0 < 0 || t0 >= n || sq.slot < 0 || c0 >= a.C) return;
    const int64_t t1 = t0 + a.run < n ? t0 + a.run : n;
    const T *x = (const T *)a.x + sq.begin * a.sx_t + c0;
    T *y = (T *)a.y + sq.begin * a.sy_t + c0;
    float wt[W][8], h[W][8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int j = 0; j < W; ++j) wt[j][e] = a.w[(int64_t)(c0 + e) * W + j];
    float *const tail = a.tails + sq.slot * a.ss + c0;
    if (t0 == 0) {
        const bool fresh = a.r.fresh && a.r.fresh[i];
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
#pragma unroll
            for (int e = 0; e < 8; ++e) h[j][e] = 0.f;
            if (!fresh) ld8<float>(tail + (int64_t)j * a.C, h[j]);
        }
        float nt[W][8];  // the new tail: entries W - 1 + n - (W - 1) + j of the old one, then x
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            const int64_t s = n - (W - 1) + j;
            if (s >= 0) {
                ld8<T>(x + s * a.sx_t, nt[j]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float v = 0.f;
#pragma unroll
                    for (int o = 0; o < W - 1; ++o) v = s + W - 1 == o ? h[o][e] : v;
                    nt[j][e] = v;
                }
            }
        }
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            st4(tail + (int64_t)j * a.C, nt[j][0], nt[j][1], nt[j][2], nt[j][3]);
            st4(tail + (int64_t)j * a.C + 4, nt[j][4], nt[j][5], nt[j][6], nt[j][7]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < W - 1; ++j) ld8<T>(x + (t0 - (W - 1) + j) * a.sx_t, h[j]);
    }
    for (int64_t tg = t0; tg < t1; tg += CR_G) {
        Row<T> rows[CR_G];
#pragma unroll
        for (int g = 0; g < CR_G; ++g)
            if (tg + g < t1) rows[g].load(x + (tg + g) * a.sx_t);
#pragma unroll
        for (int g = 0; g < CR_G; ++g) {
            if (tg + g >= t1) continue;
            rows[g].f32(h[W - 1]);
            float o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float u = 0.f;
#pragma unroll
                for (int j = 0; j < W; ++j) u = fmaf(wt[j][e], h[j][e], u);
                o[e] = conv_act<SILU>(u);
            }
            T *p = y + (tg + g) * a.sy_t;
            if constexpr (sizeof(T) == 2) {
                bf16x8 v = {};
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = (__bf16)o[e];
                __builtin_nontemporal_store(v, reinterpret_cast<bf16x8 *>(p));
            } else {
                __builtin_nontemporal_store(f32x4{o[0], o[1], o[2], o[3]}, reinterpret_cast<f32x4 *>(p));
                __builtin_nontemporal_store(f32x4{o[4], o[5], o[6], o[7]}, reinterpret_cast<f32x4 *>(p) + 1);
            }
#pragma unroll
            for (int j = 0; j < W - 1; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) h[j][e] = h[j + 1][e];
        }
    }
}

template <typename T, bool SILU>
hipError_t conv_ragged_t(const ConvRaggedArgs &a, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
    const int ncg = a.C / 8, nt = std::min(CR_NT, (ncg + 63) / 64 * 64);
    const dim3 grid((unsigned)((ncg + nt - 1) / nt * a.n_runs)), block((unsigned)nt);
    switch (a.W) {
    case 1: hipExtLaunchKernelGGL((k_conv_ragged<T, 1, SILU>), grid, block, 0, s, e0, e1, 0, a); break;
    case 2: hipExtLaunchKernelGGL((k_conv_ragged<T, 2, SILU>), grid, block, 0, s, e0, e1, 0, a); break;
    case 3: hipExtLaunchKernelGGL((k_conv_ragged<T, 3, SILU>), grid, block, 0, s, e0, e1, 0, a); break;
    default: hipExtLaunchKernelGGL((k_conv_ragged<T, 4, SILU>), grid, block, 0, s, e0, e1, 0, a); break;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_gdn_tokens(const GdnRaggedArgs &a, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
    if (gdn_token_waves(a, TOK_CL) <= TOK_FEW * (int64_t)a.n_cu)
        return a.io == SF_BF16 ? gdn_tokens_t<__bf16, TOK_CL / 2>(a, s, e0, e1) : gdn_tokens_t<float, TOK_CL / 2>(a, s, e0, e1);
    return a.io == SF_BF16 ? gdn_tokens_t<__bf16, TOK_CL>(a, s, e0, e1) : gdn_tokens_t<float, TOK_CL>(a, s, e0, e1);
}

hipError_t launch_conv_ragged(const ConvRaggedArgs &a, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
    if (a.io == SF_BF16) return a.act ? conv_ragged_t<__bf16, true>(a, s, e0, e1) : conv_ragged_t<__bf16, false>(a, s, e0, e1);
    return a.act ? conv_ragged_t<float, true>(a, s, e0, e1) : conv_ragged_t<float, false>(a, s, e0, e1);
}

}  // namespace sf
