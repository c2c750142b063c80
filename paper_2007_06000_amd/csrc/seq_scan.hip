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

template <int DT, int LP, int NS> static hipError_t launch_step(const xl_scan_args &a, hipStream_t s)
{
    const int per = 256 / LP, groups = (int)((a.channels + per - 1) / per);
    step_kernel<DT, LP, NS><<<dim3((unsigned)(groups * a.batch)), 256, 0, s>>>(a, groups);
    return hipGetLastError();
}

template <int DT> static hipError_t launch_type(const xl_scan_args &a, hipStream_t s)
{
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
