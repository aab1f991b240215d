// sf_qk.hip -- gfx950 kernels of the norms of queries and keys for each head with
// the position rotation in the same pass, forward and backward.  Per row x of D
// channels (one token, one head), with w the norm's weights and s a scale:
//
//   r = (c sum x^2 + eps)^-1/2,   z = w o (r x),   y = s Rot z
//   dz = s Rot^T dy,   dw += dz o (r x),   h = w o dz,   dx = r h - c r^3 (h . x) x
//
// Rot turns pairs of channels by p_t inv_freq[i]; Rot^T is the turn by the negative
// angle.  A few operations for each element moved: the roofline is HBM, x and y
// once each (backward: x, dy and dx).
//
// A lane holds 8 consecutive channels of a row (16 bytes in bf16, two times 16 in
// fp32), LPR lanes a row and 64 / LPR rows a wave, so a row's sums stay inside a
// few lanes (DPP and lane swaps) and the loads of a wave are whole rows.  A wave
// takes all heads of one token, qk_groups row groups at a time: the angles, their
// 64-bit reduction and the sines are formed once for a token and serve its
// queries and keys alike.  A pair's other channel is in another lane (halves) or
// in the same one (interleaved); where it is in another, the raw 16-bit values
// cross over, half the traffic of finished ones, and cos and sin come with the
// weights of both channels multiplied in.  Calls with few tokens share a token's
// heads between waves (qk_plan).  32K tokens of 80 heads of 128, bf16: 249 us forward,
// 371 backward, 5.4 TB/s where a copy reaches 4.9.
#include "sf_device.hpp"
#include "sf_launch.hpp"

#include <type_traits>

namespace sf {

namespace {

constexpr int QK_NT = 64 * QK_W;

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// 8 consecutive channels as they lie in memory.  Loads and stores are non-temporal:
// nothing is read twice (32K tokens of 80 heads of 128, bf16: forward 262 us with plain
// ones, 254 with stores alone, 249 with both; backward 391, 390, 371).
template <typename T>
struct Oct {
    static constexpr int NV = 8 * (int)sizeof(T) / 16;
    u32x4 v[NV];
    __device__ __forceinline__ void load(const T *p) {
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p) + i);
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = u32x4{0u, 0u, 0u, 0u};
    }
    __device__ __forceinline__ void f32(float (&f)[8]) const {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f[2 * i] = __uint_as_float(v[0][i] << 16);
                f[2 * i + 1] = __uint_as_float(v[0][i] & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(v[i / 4][i % 4]);
        }
    }
    // the piece of another lane (byte address 4 * lane)
    __device__ __forceinline__ Oct from(int addr) const {
        Oct o;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o.v[i][e] = (unsigned)__builtin_amdgcn_ds_bpermute(addr, (int)v[i][e]);
        return o;
    }
};
template <typename T>
__device__ __forceinline__ void store8(T *p, const float (&f)[8]) {
    if constexpr (sizeof(T) == 2) {
        bf16x8 o = {};
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = (__bf16)f[e];
        __builtin_nontemporal_store(o, reinterpret_cast<bf16x8 *>(p));
    } else {
        __builtin_nontemporal_store(f32x4{f[0], f[1], f[2], f[3]}, reinterpret_cast<f32x4 *>(p));
        __builtin_nontemporal_store(f32x4{f[4], f[5], f[6], f[7]}, reinterpret_cast<f32x4 *>(p) + 1);
    }
}

template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
    const int y = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true);
    return x + __builtin_bit_cast(float, y);
}
// sum over the LPR lanes of a row, in each of them: neighbours, pairs of pairs, then
// mirrored halves, which hold equal sums by then
template <int LPR>
__device__ __forceinline__ float row_sum(float x) {
    if constexpr (LPR >= 2) x = dpp_add<0xB1>(x);   // quad_perm [1,0,3,2]
    if constexpr (LPR >= 4) x = dpp_add<0x4E>(x);   // quad_perm [2,3,0,1]
    if constexpr (LPR >= 8) x = dpp_add<0x141>(x);  // row_half_mirror
    if constexpr (LPR >= 16) x = dpp_add<0x140>(x); // row_mirror
    if constexpr (LPR >= 32) {
        const unsigned u = __builtin_bit_cast(unsigned, x);
        const auto s = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        x = __builtin_bit_cast(float, (unsigned)s[0]) + __builtin_bit_cast(float, (unsigned)s[1]);
    }
    return x;
}

// What a lane knows of its 8 channels: where their partners are, the rotation.
struct Turn {
    int addr;          // ds_bpermute address of the lane with the partners (halves)
    float c[8], s[8];  // y_e = z_e c_e + z_partner s_e
    const double *f;   // LDS: inv_freq / 2 pi of the channels' pairs, in their order
};

// cos and sin of token position p; channels past R keep c = 1, s = 0 (R and 8 j are
// multiples of 8: a lane's channels are all rotated or none is)
__device__ __forceinline__ void turn_at(Turn &t, const QkArgs &a, int ch, int64_t p) {
    if (ch >= a.R) return;
    auto sincos = [&](double f, float &sn, float &cs) {
        double rev = (double)p * f;  // revolutions
        rev = 2.0 * (rev - rint(rev));
        const float hi = (float)rev, lo = 3.14159265358979f * (float)(rev - hi);
        float s0, c0;
        sincospif(hi, &s0, &c0);
        sn = fmaf(c0, lo, s0);  // what the float leaves of the angle, up to pi 2^-25, in first order
        cs = fmaf(-s0, lo, c0);
    };
    if (a.inter) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            float sn, cs;
            sincos(t.f[e >> 1], sn, cs);
            t.c[e] = t.c[e + 1] = cs;
            t.s[e] = -sn;
            t.s[e + 1] = sn;
        }
    } else {
        const bool first = 2 * ch < a.R;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float sn;
            sincos(t.f[e], sn, t.c[e]);
            t.s[e] = first ? -sn : sn;
        }
    }
}

__device__ __forceinline__ void turn_init(Turn &t, const QkArgs &a, const double *freq, int lane, int j) {
    const int hp = a.R >> 4, ch = 8 * j;  // hp: pieces of half the rotated channels
    t.addr = 4 * lane;
    if (!a.inter && ch < a.R) t.addr = 4 * (j < hp ? lane + hp : lane - hp);
    t.f = freq + (ch >= a.R ? 0 : a.inter ? ch >> 1 : 2 * ch < a.R ? ch : ch - (a.R >> 1));
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        t.c[e] = 1.f;
        t.s[e] = 0.f;
    }
}
// first channel of the lane's partners
__device__ __forceinline__ int partner_ch(const QkArgs &a, int j) {
    const int hp = a.R >> 4;
    if (a.inter || 8 * j >= a.R) return 8 * j;
    return 8 * (j < hp ? j + hp : j - hp);
}

// the partners of a piece: another lane's, or the neighbours; zero behind the rotated
// channels, where an infinity times sin = 0 would be NaN
template <typename T>
__device__ __forceinline__ void partners(const QkArgs &a, const Turn &t, const Oct<T> &x, const float (&f)[8],
                                         float (&p)[8], int ch) {
    if (a.inter) {
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = f[e ^ 1];
    } else {
        x.from(t.addr).f32(p);
    }
    if (a.R < a.D) {
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = ch < a.R ? p[e] : 0.f;
    }
}

__device__ __forceinline__ float norm_factor(const QkArgs &a, float ss) {
    if (a.norm == SF_NORM_NONE) return 1.f;
    const float c = a.norm == SF_NORM_L2 ? 1.f : 1.f / (float)a.D;
    return 1.f / sqrtf(fmaf(c, ss, a.eps));
}

// Heads of one token as groups of U RPW rows, the queries' first, then the keys';
// group g belongs to part g % parts.  A group is loaded while the one before it is
// computed, the token's first one before its angles are formed.
template <typename T, int LPR, bool BWD, bool WGT>
__global__ void __launch_bounds__(QK_NT, qk_resident(BWD, WGT)) k_qk(QkArgs a) {
    constexpr int RPW = 64 / LPR, U = qk_groups(BWD, sizeof(T));
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane / LPR, j = lane % LPR, ch = 8 * j;
    const bool live = ch < a.D;
    __shared__ __attribute__((aligned(16))) float swt[WGT ? 2 : 1][256];  // the weights
    if constexpr (WGT) {
        for (int i = threadIdx.x; i < a.D; i += QK_NT) {
            swt[0][i] = a.wq[i];
            swt[1][i] = a.wk[i];
        }
    }
    __shared__ double freq[128];
    for (int i = threadIdx.x; i < a.R >> 1; i += QK_NT) freq[i] = a.inv_freq[i] * 0.15915494309189533577;
    __syncthreads();
    const int pch = partner_ch(a, j);
    Turn t = {};
    turn_init(t, a, freq, lane, j);
    float dwq[8], dwk[8];  // BWD && WGT: this lane's part of dwq, dwk
#pragma unroll
    for (int e = 0; e < 8; ++e) dwq[e] = dwk[e] = 0.f;
    const int nq = (a.Hq + RPW * U - 1) / (RPW * U), nk = (a.Hk + RPW * U - 1) / (RPW * U);
    const int64_t units = (int64_t)a.n_tok * a.parts;
    for (int64_t unit = (int64_t)blockIdx.x * QK_W + w; unit < units; unit += (int64_t)gridDim.x * QK_W) {
        const int tok = (int)(unit / a.parts), part = (int)(unit % a.parts);
        const int64_t b = tok / (int)a.L, l = tok % (int)a.L;
        const T *const xq = (const T *)a.q + b * a.sq.b + l * a.sq.l + ch, *const xk = (const T *)a.k + b * a.sk.b + l * a.sk.l + ch;
        const T *const dq = BWD ? (const T *)a.dyq + b * a.sdyq.b + l * a.sdyq.l + ch : nullptr;
        const T *const dk = BWD ? (const T *)a.dyk + b * a.sdyk.b + l * a.sdyk.l + ch : nullptr;
        T *const yq = (T *)a.yq + b * a.syq.b + l * a.syq.l + ch, *const yk = (T *)a.yk + b * a.syk.b + l * a.syk.l + ch;
        Oct<T> x[U], d[U];
        auto load = [&](int g, Oct<T>(&x)[U], Oct<T>(&d)[U]) {
            const bool key = g >= nq;
            const int H = key ? a.Hk : a.Hq, h0 = (key ? g - nq : g) * U * RPW + r;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = h0 + u * RPW;
                x[u].zero();
                if constexpr (BWD) d[u].zero();
                if (live && h < H) {
                    x[u].load(key ? xk + h * a.sk.h : xq + h * a.sq.h);
                    if constexpr (BWD) d[u].load(key ? dk + h * a.sdyk.h : dq + h * a.sdyq.h);
                }
            }
        };
        load(part, x, d);
        if (a.R) turn_at(t, a, ch, a.pos ? a.pos[b * a.sp_b + l * a.sp_l] : a.pos0 + l);
        for (int g = part; g < nq + nk; g += a.parts) {
            const bool key = g >= nq;
            const int H = key ? a.Hk : a.Hq, h0 = (key ? g - nq : g) * U * RPW + r;
            const float scale = key ? 1.f : a.q_scale;
            Oct<T> xn[U], dn[U];
            if (g + a.parts < nq + nk) load(g + a.parts, xn, dn);
            float wt[8], wp[8];  // the channels' weights; cos and sin with weights
            if constexpr (WGT) {
                const f32x4 *p = reinterpret_cast<const f32x4 *>(&swt[key ? 1 : 0][live ? ch : 0]);
                const f32x4 *pp = reinterpret_cast<const f32x4 *>(&swt[key ? 1 : 0][live ? pch : 0]);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int ep = a.inter ? e ^ 1 : e;
                    wt[e] = p[e >> 2][e & 3];
                    wp[e] = a.inter ? p[ep >> 2][ep & 3] : pp[e >> 2][e & 3];
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) wt[e] = wp[e] = 1.f;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = h0 + u * RPW;
                float f[8], o[8], ss = 0.f;
                x[u].f32(f);
#pragma unroll
                for (int e = 0; e < 8; ++e) ss = fmaf(f[e], f[e], ss);
                const float rn = norm_factor(a, row_sum<LPR>(ss));
                if constexpr (!BWD) {
                    const float m = rn * scale;
                    if (a.R) {
                        float p[8];
                        partners<T>(a, t, x[u], f, p, ch);
#pragma unroll
                        for (int e = 0; e < 8; ++e) o[e] = m * fmaf(f[e], wt[e] * t.c[e], p[e] * (wp[e] * t.s[e]));
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) o[e] = f[e] * (m * wt[e]);
                    }
                } else {
                    float dz[8], dot = 0.f;
                    d[u].f32(dz);
                    if (a.R) {  // the transposed turn: sin changes its sign
                        float p[8];
                        partners<T>(a, t, d[u], dz, p, ch);
#pragma unroll
                        for (int e = 0; e < 8; ++e) dz[e] = fmaf(dz[e], t.c[e], -(p[e] * t.s[e]));
                    }
                    if constexpr (WGT) {
                        const float m = scale * rn;
                        if (key) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) dwk[e] = fmaf(dz[e], f[e] * m, dwk[e]);
                        } else {
#pragma unroll
                            for (int e = 0; e < 8; ++e) dwq[e] = fmaf(dz[e], f[e] * m, dwq[e]);
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] = dz[e] * (scale * wt[e]);
                    if (a.norm != SF_NORM_NONE) {  // without a norm x has no part in dx, whatever it holds
#pragma unroll
                        for (int e = 0; e < 8; ++e) dot = fmaf(o[e], f[e], dot);
                        const float c = a.norm == SF_NORM_L2 ? 1.f : 1.f / (float)a.D;
                        const float m = c * rn * rn * row_sum<LPR>(dot);
#pragma unroll
                        for (int e = 0; e < 8; ++e) o[e] = rn * (o[e] - m * f[e]);
                    }
                }
                if (live && h < H) store8<T>(key ? yk + h * a.syk.h : yq + h * a.syq.h, o);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                x[u] = xn[u];
                if constexpr (BWD) d[u] = dn[u];
            }
        }
    }
    if constexpr (BWD && WGT) {  // the workgroup's part: ws[block][which][channel]
        __shared__ float sw[QK_W][2][256];
#pragma unroll
        for (int which = 0; which < 2; ++which)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float v = which ? dwk[e] : dwq[e];
#pragma unroll
                for (int m = LPR; m < 64; m <<= 1) v += __shfl_xor(v, m, 64);
                if (r == 0 && live) sw[w][which][ch + e] = v;
            }
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * a.D; i += QK_NT) {
            const int which = i / a.D, c = i % a.D;
            float v = 0.f;
#pragma unroll
            for (int k = 0; k < QK_W; ++k) v += sw[k][which][c];
            a.ws[(int64_t)blockIdx.x * 2 * a.D + i] = v;
        }
    }
}

// dwq, dwk: the workgroups' parts, added in a fixed order (64 interleaved runs of
// parts for each channel, then the runs): no atomics, bitwise reproducible
constexpr int QS_C = 16, QS_S = 64;
__global__ void __launch_bounds__(QS_C *QS_S) k_qk_dw_sum(const float *ws, float *dwq, float *dwk, int D, int parts) {
    __shared__ float part[QS_S][QS_C + 1];
    const int c = threadIdx.x % QS_C, sl = threadIdx.x / QS_C, i = blockIdx.x * QS_C + c;
    float v = 0.f;
    for (int p = sl; p < parts; p += QS_S) v += ws[(int64_t)p * 2 * D + i];
    part[sl][c] = v;
    __syncthreads();
    if (sl == 0) {
        float s = 0.f;
        for (int k = 0; k < QS_S; ++k) s += part[k][c];
        (i < D ? dwq : dwk)[i < D ? i : i - D] = s;
    }
}

template <typename T, int LPR>
hipError_t qk_tl(bool bwd, const QkArgs &a, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
    const dim3 grid((unsigned)a.blocks), nt(QK_NT);
    const bool wgt = a.wq != nullptr;
    if (a.blocks == 0) {  // no rows: the weights' gradients alone, zero
        hipExtLaunchKernelGGL(k_qk_dw_sum, dim3((unsigned)(2 * a.D / QS_C)), dim3(QS_C * QS_S), 0, s, e0, e1, 0,
                              (const float *)a.ws, a.dwq, a.dwk, (int)a.D, 0);
    } else if (!bwd && wgt) hipExtLaunchKernelGGL((k_qk<T, LPR, false, true>), grid, nt, 0, s, e0, e1, 0, a);
    else if (!bwd) hipExtLaunchKernelGGL((k_qk<T, LPR, false, false>), grid, nt, 0, s, e0, e1, 0, a);
    else if (!wgt) hipExtLaunchKernelGGL((k_qk<T, LPR, true, false>), grid, nt, 0, s, e0, e1, 0, a);
    else {
        hipExtLaunchKernelGGL((k_qk<T, LPR, true, true>), grid, nt, 0, s, e0, nullptr, 0, a);
        hipExtLaunchKernelGGL(k_qk_dw_sum, dim3((unsigned)(2 * a.D / QS_C)), dim3(QS_C * QS_S), 0, s, nullptr, e1, 0,
                              (const float *)a.ws, a.dwq, a.dwk, (int)a.D, (int)a.blocks);
    }
    return hipGetLastError();
}
template <typename T>
hipError_t qk_t(bool bwd, const QkArgs &a, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
    if (a.D <= 16) return qk_tl<T, 2>(bwd, a, s, e0, e1);
    if (a.D <= 32) return qk_tl<T, 4>(bwd, a, s, e0, e1);
    if (a.D <= 64) return qk_tl<T, 8>(bwd, a, s, e0, e1);
    if (a.D <= 128) return qk_tl<T, 16>(bwd, a, s, e0, e1);
    return qk_tl<T, 32>(bwd, a, s, e0, e1);
}

}  // namespace

hipError_t launch_qk(bool bwd, const QkArgs &a, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
    return a.io == SF_BF16 ? qk_t<__bf16>(bwd, a, s, e0, e1) : qk_t<float>(bwd, a, s, e0, e1);
}

}  // namespace sf
