// Causal depthwise convolution over time.
//
//   y[t,c] = act(bias[c] + sum_j w[c,j] x[t-(K-1)+j, c])
//
// Bound by memory: 2 K + 4 operations for a number read and one written.  A thread owns V channels (16 bytes of a row) and `run`
// tokens in a row, with the last K - 1 inputs and the filter in registers, so a number is read once, but for the K - 1 tokens
// before each run (an L2 hit: the run before them is a neighbour's).
#include "seq_internal.h"

namespace xls {

template <int DT, int K, int V>
__global__ __launch_bounds__(256) void conv_kernel(const xl_causal_conv_args a, int run, int runs)
{
    typedef typename Elem<DT>::T T;
    const int C = (int)a.channels, L = (int)a.length, vecs = (C + V - 1) / V;
    const long long item = (long long)blockIdx.x * 256 + threadIdx.x;
    const int c = (int)(item % vecs) * V;
    const long long rest = item / vecs;
    const int b = (int)(rest / runs), t0 = (int)(rest % runs) * run;
    if (b >= a.batch) return;
    const T *x = static_cast<const T *>(a.x) + b * a.x_batch + c;
    T *y = static_cast<T *>(a.y) + b * a.y_batch + c;
    const long long slot = (a.state || a.new_state) || a.slots ? slot_of(a.slots, a.nslots, b) : 0;
    const int len = slot < 0 ? 0 : length_of(a.lengths, b, L);
    const long long srow = (slot * (K - 1)) * C + c;

    float w[K][V], bias[V], h[K][V];       // h: the inputs that the next token sees, oldest first
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
        for (int j = 0; j < K; ++j) w[j][i] = a.weight[(c + i) * K + j];
        bias[i] = a.bias ? a.bias[c + i] : 0.f;
    }
    float old[K - 1][V];
#pragma unroll
    for (int j = 0; j < K - 1; ++j) {
#pragma unroll
        for (int i = 0; i < V; ++i) old[j][i] = 0.f;
        const int t = t0 - (K - 1) + j;
        if (t < 0) {
            if (a.state && slot >= 0) load_vec<DT, V>(a.state, srow + (long long)(t + K - 1) * C, old[j]);
        } else if (t < len) {
            load_vec<DT, V>(x, t * a.x_token, old[j]);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) h[j][i] = old[j][i];
    }
    const int end = min(t0 + run, L), live = min(end, len);
    int t = t0;
    auto step = [&](const float *v, int at) {
        float s[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            h[K - 1][i] = v[i];
            s[i] = bias[i];
#pragma unroll
            for (int j = 0; j < K; ++j) s[i] = __builtin_fmaf(w[j][i], h[j][i], s[i]);
            if (a.silu) s[i] = silu(s[i]);
#pragma unroll
            for (int j = 0; j < K - 1; ++j) h[j][i] = h[j + 1][i];
        }
        store_vec<DT, V>(y, at * a.y_token, s);
    };
    for (; t + 4 <= live; t += 4) {     // four loads on their way at once
        float v[4][V];
#pragma unroll
        for (int k = 0; k < 4; ++k) load_vec<DT, V>(x, (t + k) * a.x_token, v[k]);
#pragma unroll
        for (int k = 0; k < 4; ++k) step(v[k], t + k);
    }
    for (; t < live; ++t) {
        float v[V];
        load_vec<DT, V>(x, t * a.x_token, v);
        step(v, t);
    }
    const float zero[V] = {};
    for (t = max(t, t0); t < end; ++t) store_vec<DT, V>(y, t * a.y_token, zero);
    // The thread of the first tokens, the only one that reads the old state, writes the new one (both may be the same memory).
    if (t0 == 0 && a.new_state && slot >= 0) {
#pragma unroll
        for (int j = 0; j < K - 1; ++j) {
            const int at = len - (K - 1) + j;
            float v[V] = {};
            if (at >= 0) {
                load_vec<DT, V>(x, at * a.x_token, v);
            } else {
#pragma unroll
                for (int o = 0; o < K - 1; ++o)
                    if (o == at + K - 1) {
#pragma unroll
                        for (int i = 0; i < V; ++i) v[i] = old[o][i];
                    }
            }
            store_vec<DT, V>(a.new_state, srow + (long long)j * C, v);
        }
    }
}

template <int DT, int K> static hipError_t launch_taps(const xl_causal_conv_args &a, hipStream_t s)
{
    typedef typename Elem<DT>::T T;
    constexpr int V = 16 / sizeof(T);
    const unsigned long long at = (unsigned long long)a.x | (unsigned long long)a.y | (unsigned long long)a.state | (unsigned long long)a.new_state |
                                  (unsigned long long)(a.x_batch * sizeof(T)) | (a.x_token * sizeof(T)) | (a.y_batch * sizeof(T)) | (a.y_token * sizeof(T));
    const bool wide = at % 16 == 0 && a.channels % V == 0;
    const long long vecs = wide ? a.channels / V : a.channels;
    // Runs of 32 tokens read an input 1.1 times; shorter ones where there would be fewer than 2048 threads a compute unit.
    long long run = 32;
    while (run > 4 && a.batch * vecs * ((a.length + run - 1) / run) < 256ll * 2048) run /= 2;
    const long long runs = a.length > 0 ? (a.length + run - 1) / run : 1, blocks = (a.batch * vecs * runs + 255) / 256;
    if (wide) conv_kernel<DT, K, V><<<dim3((unsigned)blocks), 256, 0, s>>>(a, (int)run, (int)runs);
    else conv_kernel<DT, K, 1><<<dim3((unsigned)blocks), 256, 0, s>>>(a, (int)run, (int)runs);
    return hipGetLastError();
}

template <int DT> static hipError_t launch_type(const xl_causal_conv_args &a, hipStream_t s)
{
    return a.taps == 2 ? launch_taps<DT, 2>(a, s) : a.taps == 3 ? launch_taps<DT, 3>(a, s) : launch_taps<DT, 4>(a, s);
}

hipError_t launch_causal_conv(const xl_causal_conv_args &a, hipStream_t s)
{
    return a.dtype == XL_F32 ? launch_type<XL_F32>(a, s) : a.dtype == XL_F16 ? launch_type<XL_F16>(a, s) : launch_type<XL_BF16>(a, s);
}

}  // namespace xls
