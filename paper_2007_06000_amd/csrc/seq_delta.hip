// The gated delta rule.
//
//   S <- e^g S,  S <- S + beta k (v - S^T k)^T,  y = scale S^T q
//
// Columns of S do not meet: each is a recurrence of its own, with the same keys, queries, decays and steps.
#include "seq_internal.h"

namespace xls {

static constexpr float NORM_EPS = 1e-6f;

// e^g is 0 in fp32 long before g reaches -128, and the differences of sums of g stay numbers where g is minus infinity.
__device__ __forceinline__ float clamped(float g)
{
    g = g < -128.f ? -128.f : g;
    return g > 0.f ? 0.f : g;       // a NaN stays
}

// A wave has 32 columns of a head's states in registers, eight of them rows' parts: lane % 8 names four columns, lane / 8 a run of R = rows / 8 rows.
// One pass over them gives both S^T k and S^T q, from which y follows without the new states:  S'^T q = S^T q + (k.q) beta (v - S^T k).
static constexpr int COLS = 32;

__device__ __forceinline__ float over_rows(float s)
{
#pragma unroll
    for (int o = 8; o < 64; o *= 2) s += __shfl_xor(s, o);
    return s;
}

template <int DT, int R>
__global__ __launch_bounds__(256) void token_kernel(const xl_delta_args a, int tiles)
{
    typedef typename Elem<DT>::T T;
    const int lane = threadIdx.x % 64, DK = (int)a.dk, DV = (int)a.dv, H = (int)a.heads, length = (int)a.length, first = lane / 8 * R;
    const long long units = a.batch * a.heads * tiles;
    for (long long unit = (long long)blockIdx.x * 4 + threadIdx.x / 64; unit < units; unit += (long long)gridDim.x * 4) {
        const int tile = (int)(unit % tiles), h = (int)(unit / tiles % H), b = (int)(unit / tiles / H), hk = h / (int)(a.heads / a.key_heads);
        const int j = tile * COLS + lane % 8 * 4, live = DV - j;
        const long long slot = slot_of(a.slots, a.nslots, b);
        const int n = slot < 0 ? 0 : length_of(a.lengths, b, length);
        T *y = static_cast<T *>(a.y) + b * a.y_batch + h * a.y_head + j;
        if (lane < 8 && live > 0)
            for (int t = n; t < length; ++t) store_some<T, 4>(y + t * a.y_token, live, Vec<T, 4>{});
        if (slot < 0) continue;
        const long long at = (slot * H + h) * DK * DV + j;
        f32x4 S[R];
#pragma unroll
        for (int r = 0; r < R; ++r) S[r] = a.state && first + r < DK ? load_some<float, 4>(a.state + at + (long long)(first + r) * DV, live) : f32x4{};
        for (int t = 0; t < n; ++t) {
            const T *kp = static_cast<const T *>(a.k) + b * a.k_batch + t * a.k_token + hk * a.k_head + first;
            const T *qp = static_cast<const T *>(a.q) + b * a.q_batch + t * a.q_token + hk * a.q_head + first;
            float k[R], q[R];
#pragma unroll
            for (int r = 0; r < R; r += 8) {
                const Vec<T, 8> kv = load_some<T, 8>(kp + r, DK - first - r), qv = load_some<T, 8>(qp + r, DK - first - r);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    k[r + i] = (float)kv[i];
                    q[r + i] = (float)qv[i];
                }
            }
            const float decay = exp_fast(clamped(a.g[b * a.g_batch + t * a.g_token + h])), beta = a.beta[b * a.beta_batch + t * a.beta_token + h];
            const Vec<T, 4> v = load_some<T, 4>(static_cast<const T *>(a.v) + b * a.v_batch + t * a.v_token + h * a.v_head + j, live);
            float kk = 0.f, qq = 0.f, kq = 0.f;
            f32x4 kS = {}, qS = {};
#pragma unroll
            for (int r = 0; r < R; ++r) {
                kk = __builtin_fmaf(k[r], k[r], kk);
                qq = __builtin_fmaf(q[r], q[r], qq);
                kq = __builtin_fmaf(k[r], q[r], kq);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    S[r][c] *= decay;
                    kS[c] = __builtin_fmaf(k[r], S[r][c], kS[c]);
                    qS[c] = __builtin_fmaf(q[r], S[r][c], qS[c]);
                }
            }
            kq = over_rows(kq);
            float nk = 1.f, nq = (float)a.scale;
            if (a.normalize) {
                nk = __builtin_amdgcn_rsqf(over_rows(kk) + NORM_EPS);
                nq *= __builtin_amdgcn_rsqf(over_rows(qq) + NORM_EPS);
            }
            f32x4 add;
            Vec<T, 4> out;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                add[c] = beta * ((float)v[c] - nk * over_rows(kS[c])) * nk;
                out[c] = (T)(nq * __builtin_fmaf(kq, add[c], over_rows(qS[c])));
            }
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int c = 0; c < 4; ++c) S[r][c] = __builtin_fmaf(k[r], add[c], S[r][c]);
            if (lane < 8 && live > 0) store_some<T, 4>(y + t * a.y_token, live, out);
        }
        if (a.new_state && live > 0)
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (first + r < DK) store_some<float, 4>(a.new_state + at + (long long)(first + r) * DV, live, S[r]);
    }
}

template <int DT> static hipError_t launch_type(const xl_delta_args &a, hipStream_t s)
{
    const int tiles = (int)((a.dv + COLS - 1) / COLS);
    const long long groups = (a.batch * a.heads * tiles + 3) / 4;
    const dim3 grid((unsigned)(groups < 1 << 20 ? groups : 1 << 20));
    return a.dk <= 64 ? launch_kernel(token_kernel<DT, 8>, grid, 256, s, a, tiles)
         : a.dk <= 128 ? launch_kernel(token_kernel<DT, 16>, grid, 256, s, a, tiles) : launch_kernel(token_kernel<DT, 32>, grid, 256, s, a, tiles);
}

long long delta_workspace(const xl_delta_args &) { return 0; }

hipError_t launch_gated_delta_rule(const xl_delta_args &a, hipStream_t s)
{
    return a.dtype == XL_F32 ? launch_type<XL_F32>(a, s) : a.dtype == XL_F16 ? launch_type<XL_F16>(a, s) : launch_type<XL_BF16>(a, s);
}

}  // namespace xls
