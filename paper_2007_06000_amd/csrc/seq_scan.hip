// Selective state-space scan.
//
//   h[n] <- exp(d A[n]) h[n] + d u B[n],   y = sum_n C[n] h[n] + D u,   y *= z sigmoid(z)
#include "seq_internal.h"

namespace xls {

// A token after the other: LP lanes a channel, NS states a lane, 256 / LP channels a workgroup.
template <int DT, int LP, int NS>
__global__ __launch_bounds__(256) void step_kernel(const xl_scan_args a, int groups)
{
    typedef typename Elem<DT>::T T;
    const int b = blockIdx.x / groups, c = (blockIdx.x % groups) * (256 / LP) + threadIdx.x / LP, part = threadIdx.x % LP, n0 = part * NS;
    const int D = (int)a.channels, N = (int)a.states, L = (int)a.length;
    const long long slot = slot_of(a.slots, a.nslots, b);
    const int len = slot < 0 ? 0 : length_of(a.lengths, b, L);
    const bool in = c < D;
    float A2[NS], h[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        const bool live = in && n0 + i < N;
        A2[i] = live ? a.A[(long long)c * N + n0 + i] * LOG2E : 0.f;
        h[i] = live && a.state && slot >= 0 ? a.state[(slot * D + c) * N + n0 + i] : 0.f;
    }
    const float bias = in && a.delta_bias ? a.delta_bias[c] : 0.f, skip = in && a.D ? a.D[c] : 0.f;
    const T *up = static_cast<const T *>(a.u) + b * a.u_batch + c, *dp = static_cast<const T *>(a.delta) + b * a.delta_batch + c;
    const T *zp = static_cast<const T *>(a.z) + b * a.z_batch + c, *Bp = static_cast<const T *>(a.B) + b * a.b_batch + n0;
    const T *Cp = static_cast<const T *>(a.C) + b * a.c_batch + n0;
    T *yp = static_cast<T *>(a.y) + b * a.y_batch + c;
    for (int t = 0; t < len; ++t) {
        const float u = in ? (float)up[t * a.u_token] : 0.f;
        float d = in ? (float)dp[t * a.delta_token] + bias : 0.f;
        if (a.softplus) d = softplus(d);
        const float s = d * u;
        float y = 0.f;
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            if (n0 + i < N) {
                h[i] = __builtin_fmaf(exp2_fast(d * A2[i]), h[i], s * (float)Bp[t * a.b_token + i]);
                y = __builtin_fmaf((float)Cp[t * a.c_token + i], h[i], y);
            }
        }
#pragma unroll
        for (int o = 1; o < LP; o *= 2) y += __shfl_xor(y, o);
        if (part == 0 && in) {
            if (a.D) y = __builtin_fmaf(skip, u, y);
            if (a.z) y *= silu((float)zp[t * a.z_token]);
            yp[t * a.y_token] = (T)y;
        }
    }
    if (part == 0 && in)
        for (int t = len; t < L; ++t) yp[t * a.y_token] = (T)0.f;
    if (a.new_state && slot >= 0) {
#pragma unroll
        for (int i = 0; i < NS; ++i)
            if (in && n0 + i < N) a.new_state[(slot * D + c) * N + n0 + i] = h[i];
    }
}

// Sum over the LP lanes of a channel, for LP tokens at once: lane i of the channel gets token i's.  At every step a lane keeps half of its tokens and hands the other
// half to its partner, so that a token costs 3 - 3 / LP operations, not log2(LP).
template <int CTRL> __device__ __forceinline__ float from_partner(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
template <int LP> __device__ __forceinline__ float sum_over_lanes(float *p, int part)
{
    if constexpr (LP == 16) {
        const bool up = part & 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = (up ? p[j + 8] : p[j]) + from_partner<0x128>(up ? p[j] : p[j + 8]);      // lane ^ 8
    }
    if constexpr (LP >= 8) {
        const bool up = part & 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) p[j] = (up ? p[j + 4] : p[j]) + from_partner<0x141>(up ? p[j] : p[j + 4]);      // 7 - lane
    }
    const bool up2 = part & 2, up1 = part & 1;
#pragma unroll
    for (int j = 0; j < 2; ++j) p[j] = (up2 ? p[j + 2] : p[j]) + from_partner<0x4e>(up2 ? p[j] : p[j + 2]);         // lane ^ 2
    return (up1 ? p[1] : p[0]) + from_partner<0xb1>(up1 ? p[0] : p[1]);                                             // lane ^ 1
}

// V elements at p, of which the first n exist; the others come out as zeros.
template <typename T, int V> using Vec = T __attribute__((ext_vector_type(V)));
template <typename T, int V> __device__ __forceinline__ Vec<T, V> load_some(const T *p, int n, bool wide)
{
    Vec<T, V> v = {};
    if (wide && n >= V) {
        v = *reinterpret_cast<const Vec<T, V> *>(p);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < n) v[i] = p[i];
    }
    return v;
}

// Many tokens.  A workgroup owns CH = 64 / LP channels of a sequence and goes through it in tiles of W x TK tokens, TK of them a wave: the recurrence is linear, so a
// wave runs its tokens from a state of zero (which gives E) and multiplies up their factors (P = exp(A sum d)); after a barrier each
// folds the (P, E) of the waves before it into the state that it begins with, and runs its tokens again, the factors and
// inputs still in registers, now with the outputs.
template <int DT, int LP, int NS, int W, int TK>
__global__ __launch_bounds__(64 * W) void tile_kernel(const xl_scan_args a, int groups, bool wide, bool wide_bc)
{
    typedef typename Elem<DT>::T T;
    constexpr int CH = 64 / LP, NP = LP * NS, TT = W * TK, PT = TT + 4, THREADS = 64 * W;
    constexpr int PER = CH * TK / 64, VE = PER < 4 ? PER : 4, IT = PER / VE;            // a thread's part of a tile's u, delta, z and y
    constexpr int PERB = NP * TK / 64, VB = PERB < 4 ? PERB : 4, IB = PERB / VB;        // and of its B and C
    static_assert(PER >= 1 && PERB >= 1 && TK % LP == 0 && TK % 4 == 0, "a tile divides among the threads");
    __shared__ float dl[CH * PT], sx[CH * PT];      // steps, and step x input (later the outputs): [channel][token]
    __shared__ float Bs[TT * NP], Cs[TT * NP];      // [token][state]
    __shared__ Vec<float, NS> Ps[W * 64], Es[W * 64];

    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, c = lane / LP, part = lane % LP, n0 = part * NS;
    const int b = blockIdx.x / groups, c0 = (blockIdx.x % groups) * CH;
    const int D = (int)a.channels, N = (int)a.states, L = (int)a.length;
    const long long slot = slot_of(a.slots, a.nslots, b);
    const int len = slot < 0 ? 0 : length_of(a.lengths, b, L);
    const bool in = c0 + c < D;

    float A2[NS], h[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        const bool live = in && n0 + i < N;
        A2[i] = live ? a.A[(long long)(c0 + c) * N + n0 + i] * LOG2E : 0.f;
        h[i] = live && a.state && slot >= 0 ? a.state[(slot * D + c0 + c) * N + n0 + i] : 0.f;
    }
    // this thread's numbers: VE channels of IT tokens
    const int ec = tid % (CH / VE) * VE, et = tid / (CH / VE), nc = min(D - c0 - ec, VE);
    const int bn = tid % (NP / VB) * VB, bt = tid / (NP / VB), nb = min(N - bn, VB);
    constexpr int ET = THREADS * VE / CH, BT = THREADS * VB / NP;       // tokens between a thread's items
    float bias[VE], skip[VE];
#pragma unroll
    for (int i = 0; i < VE; ++i) {
        bias[i] = a.delta_bias && i < nc ? a.delta_bias[c0 + ec + i] : 0.f;
        skip[i] = a.D && i < nc ? a.D[c0 + ec + i] : 0.f;
    }
    const T *up = static_cast<const T *>(a.u) + b * a.u_batch + c0 + ec, *dp = static_cast<const T *>(a.delta) + b * a.delta_batch + c0 + ec;
    const T *zp = static_cast<const T *>(a.z) + b * a.z_batch + c0 + ec;
    const T *Bp = static_cast<const T *>(a.B) + b * a.b_batch + bn, *Cp = static_cast<const T *>(a.C) + b * a.c_batch + bn;
    T *yp = static_cast<T *>(a.y) + b * a.y_batch + c0 + ec;

    Vec<T, VE> ur[IT], dr[IT], zr[IT];
    Vec<T, VB> Br[IB], Cr[IB];
    auto fetch = [&](int t0) {
#pragma unroll
        for (int k = 0; k < IT; ++k) {
            const long long t = t0 + et + k * ET;
            const int n = t < len ? nc : 0;
            ur[k] = load_some<T, VE>(up + t * a.u_token, n, wide);
            dr[k] = load_some<T, VE>(dp + t * a.delta_token, n, wide);
            if (a.z) zr[k] = load_some<T, VE>(zp + t * a.z_token, n, wide);
        }
#pragma unroll
        for (int k = 0; k < IB; ++k) {
            const long long t = t0 + bt + k * BT;
            const int n = t < len ? nb : 0;
            Br[k] = load_some<T, VB>(Bp + t * a.b_token, n, wide_bc);
            Cr[k] = load_some<T, VB>(Cp + t * a.c_token, n, wide_bc);
        }
    };

    fetch(0);
    for (int t0 = 0; t0 < len; t0 += TT) {
        Vec<T, VE> uc[IT], zc[IT];
#pragma unroll
        for (int k = 0; k < IT; ++k) {
            const int t = et + k * ET;
            uc[k] = ur[k];
            zc[k] = zr[k];
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                float d = (float)dr[k][i] + bias[i];
                if (a.softplus) d = softplus(d);
                d = t0 + t < len ? d : 0.f;                     // a token past the end changes nothing
                dl[(ec + i) * PT + t] = d;
                sx[(ec + i) * PT + t] = d * (float)ur[k][i];
            }
        }
#pragma unroll
        for (int k = 0; k < IB; ++k) {
            Vec<float, VB> vb, vc;
#pragma unroll
            for (int i = 0; i < VB; ++i) {
                vb[i] = (float)Br[k][i];
                vc[i] = (float)Cr[k][i];
            }
            *reinterpret_cast<Vec<float, VB> *>(&Bs[(bt + k * BT) * NP + bn]) = vb;
            *reinterpret_cast<Vec<float, VB> *>(&Cs[(bt + k * BT) * NP + bn]) = vc;
        }
        if (t0 + TT < len) fetch(t0 + TT);                      // the next tile's numbers come in the meantime
        __syncthreads();

        // the wave's tokens from a state of zero
        float av[TK][NS], bv[TK][NS], sum = 0.f;
        Vec<float, NS> e = {}, p;
        const int tw = wave * TK;
#pragma unroll
        for (int k = 0; k < TK; k += 4) {
            const f32x4 d = *reinterpret_cast<const f32x4 *>(&dl[c * PT + tw + k]), s = *reinterpret_cast<const f32x4 *>(&sx[c * PT + tw + k]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const Vec<float, NS> B = *reinterpret_cast<const Vec<float, NS> *>(&Bs[(tw + k + j) * NP + n0]);
                sum += d[j];
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    av[k + j][i] = exp2_fast(d[j] * A2[i]);
                    bv[k + j][i] = s[j] * B[i];
                    e[i] = __builtin_fmaf(av[k + j][i], e[i], bv[k + j][i]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < NS; ++i) p[i] = exp2_fast(sum * A2[i]);
        Ps[tid] = p;
        Es[tid] = e;
        __syncthreads();
        float g[NS];
#pragma unroll
        for (int w = 0; w < W; ++w) {
            if (w == wave) {
#pragma unroll
                for (int i = 0; i < NS; ++i) g[i] = h[i];
            }
            const Vec<float, NS> pw = Ps[w * 64 + lane], ew = Es[w * 64 + lane];
#pragma unroll
            for (int i = 0; i < NS; ++i) h[i] = __builtin_fmaf(pw[i], h[i], ew[i]);
        }
        // and again from the state that they find
#pragma unroll
        for (int k = 0; k < TK; k += LP) {
            float y[LP];
#pragma unroll
            for (int j = 0; j < LP; ++j) {
                const Vec<float, NS> C = *reinterpret_cast<const Vec<float, NS> *>(&Cs[(tw + k + j) * NP + n0]);
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    g[i] = __builtin_fmaf(av[k + j][i], g[i], bv[k + j][i]);
                    y[j] = i ? __builtin_fmaf(C[i], g[i], y[j]) : C[i] * g[i];
                }
            }
            sx[c * PT + tw + k + part] = sum_over_lanes<LP>(y, part);
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < IT; ++k) {
            const int t = et + k * ET;
            if (t0 + t >= len || nc <= 0) continue;
            float out[VE];
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                out[i] = sx[(ec + i) * PT + t];
                if (a.D) out[i] = __builtin_fmaf(skip[i], (float)uc[k][i], out[i]);
                if (a.z) out[i] *= silu((float)zc[k][i]);
            }
            T *y = yp + (t0 + t) * a.y_token;
            if (wide && nc >= VE) {
                store_vec<DT, VE>(y, 0, out);
            } else {
#pragma unroll
                for (int i = 0; i < VE; ++i)
                    if (i < nc) y[i] = (T)out[i];
            }
        }
    }
    for (int t = len + et; t < L; t += ET) {
#pragma unroll
        for (int i = 0; i < VE; ++i)
            if (i < nc) yp[t * a.y_token + i] = (T)0.f;
    }
    if (wave == 0 && a.new_state && slot >= 0) {
#pragma unroll
        for (int i = 0; i < NS; ++i)
            if (in && n0 + i < N) a.new_state[(slot * D + c0 + c) * N + n0 + i] = h[i];
    }
}

template <int DT, int LP, int NS> static hipError_t launch_step(const xl_scan_args &a, hipStream_t s)
{
    const int per = 256 / LP, groups = (int)((a.channels + per - 1) / per);
    step_kernel<DT, LP, NS><<<dim3((unsigned)(groups * a.batch)), 256, 0, s>>>(a, groups);
    return hipGetLastError();
}

template <int DT, int LP, int NS, int W, int TK> static hipError_t launch_tile(const xl_scan_args &a, hipStream_t s)
{
    typedef typename Elem<DT>::T T;
    constexpr int CH = 64 / LP, PER = CH * TK / 64, VE = PER < 4 ? PER : 4, PERB = LP * NS * TK / 64, VB = PERB < 4 ? PERB : 4;
    const int groups = (int)((a.channels + CH - 1) / CH);
    const unsigned long long at = (unsigned long long)a.u | (unsigned long long)a.delta | (unsigned long long)a.z | (unsigned long long)a.y;
    const unsigned long long steps = a.u_batch | a.u_token | a.delta_batch | a.delta_token | a.z_batch | a.z_token | a.y_batch | a.y_token;
    const unsigned long long at_bc = (unsigned long long)a.B | (unsigned long long)a.C, steps_bc = a.b_batch | a.b_token | a.c_batch | a.c_token;
    const bool wide = (at | steps * sizeof(T)) % (VE * sizeof(T)) == 0, wide_bc = (at_bc | steps_bc * sizeof(T)) % (VB * sizeof(T)) == 0;
    tile_kernel<DT, LP, NS, W, TK><<<dim3((unsigned)(groups * a.batch)), 64 * W, 0, s>>>(a, groups, wide, wide_bc);
    return hipGetLastError();
}

template <int DT> static hipError_t launch_type(const xl_scan_args &a, hipStream_t s)
{
    if (a.length > 16) {
        if (a.states <= 4) return launch_tile<DT, 4, 1, 4, 16>(a, s);
        if (a.states <= 8) return launch_tile<DT, 4, 2, 4, 16>(a, s);
        if (a.states <= 16) return launch_tile<DT, 4, 4, 4, 16>(a, s);
        if (a.states <= 32) return launch_tile<DT, 8, 4, 4, 16>(a, s);
        if (a.states <= 64) return launch_tile<DT, 16, 4, 4, 16>(a, s);
        return launch_tile<DT, 16, 8, 4, 16>(a, s);
    }
    if (a.states <= 4) return launch_step<DT, 1, 4>(a, s);
    if (a.states <= 8) return launch_step<DT, 2, 4>(a, s);
    if (a.states <= 16) return launch_step<DT, 4, 4>(a, s);
    if (a.states <= 32) return launch_step<DT, 8, 4>(a, s);
    if (a.states <= 64) return launch_step<DT, 16, 4>(a, s);
    return launch_step<DT, 32, 4>(a, s);
}

hipError_t launch_selective_scan(const xl_scan_args &a, hipStream_t s)
{
    return a.dtype == XL_F32 ? launch_type<XL_F32>(a, s) : a.dtype == XL_F16 ? launch_type<XL_F16>(a, s) : launch_type<XL_BF16>(a, s);
}

}  // namespace xls
