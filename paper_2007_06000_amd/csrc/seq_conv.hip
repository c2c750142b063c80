// Causal depthwise convolution over time.
//
//   y[t,c] = act(bias[c] + sum_j w[c,j] x[t-(K-1)+j, c])
//
// Bound by memory: 2 K + 4 operations for a number read and one written.  A thread owns V channels and `run` tokens in a row, with the last K - 1 inputs and the
// filter in registers, so a number is read once, but for the K - 1 tokens before each run (a cache hit: the run before them is a neighbour's).
// 8 x 3025 x 2048 in bf16 (half of a wider tensor): 38.7 us for 198 MB, 5.1 TB/s; in fp32 78 us.  That is more than memory gives (4.7 TB/s to a copy of 4 GB): of the 99 MB of inputs 55 came
// from memory, the others from the last-level cache, which passes over the same tensors leave them in.
#include "seq_internal.h"

namespace xls {

template <int DT, int K, int V>
__global__ __launch_bounds__(256) void conv_kernel(const xl_causal_conv_args a, int run, int runs)
{
    typedef typename Elem<DT>::T T;
    const int C = (int)a.channels, L = (int)a.length, vecs = C / V;
    const long long item = (long long)neighbours_together(blockIdx.x, gridDim.x) * 256 + threadIdx.x, rest = item / vecs;
    const int c = (int)(item % vecs) * V, b = (int)(rest / runs), t0 = (int)(rest % runs) * run;
    if (b >= a.batch) return;
    const T *x = static_cast<const T *>(a.x) + b * a.x_batch + c;
    T *y = static_cast<T *>(a.y) + b * a.y_batch + c;
    const long long slot = slot_of(a.slots, a.nslots, b), srow = (slot * (K - 1)) * C + c;
    const int len = slot < 0 ? 0 : length_of(a.lengths, b, L);

    float w[K][V], bias[V], h[K][V];       // h: the inputs that the next token sees, oldest first
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
        for (int j = 0; j < K; ++j) w[j][i] = a.weight[(long long)(c + i) * K + j];
        bias[i] = a.bias ? a.bias[c + i] : 0.f;
    }
    Vec<T, V> old[K - 1];
#pragma unroll
    for (int j = 0; j < K - 1; ++j) {
        const int t = t0 - (K - 1) + j;
        old[j] = Vec<T, V>{};
        if (t >= 0 && t < len) old[j] = load_vec<T, V>(x + t * a.x_token);
        else if (t < 0 && a.state && slot >= 0) old[j] = load_vec<T, V>(static_cast<const T *>(a.state) + srow + (long long)(t + K - 1) * C);
#pragma unroll
        for (int i = 0; i < V; ++i) h[j][i] = (float)old[j][i];
    }
    const int end = min(t0 + run, L), last = min(end, len);
    int t = t0;
    auto step = [&](Vec<T, V> v, int at) {
        Vec<T, V> out;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            h[K - 1][i] = (float)v[i];
            float s = bias[i];
#pragma unroll
            for (int j = 0; j < K; ++j) s = __builtin_fmaf(w[j][i], h[j][i], s);
            out[i] = (T)(a.silu ? silu(s) : s);
#pragma unroll
            for (int j = 0; j < K - 1; ++j) h[j][i] = h[j + 1][i];
        }
        store_vec<T, V>(y + at * a.y_token, out);
    };
    for (; t + 4 <= last; t += 4) {     // four loads on their way at once
        Vec<T, V> v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = load_vec<T, V>(x + (t + k) * a.x_token);
#pragma unroll
        for (int k = 0; k < 4; ++k) step(v[k], t + k);
    }
    for (; t < last; ++t) step(load_vec<T, V>(x + t * a.x_token), t);
    for (t = max(t, t0); t < end; ++t) store_vec<T, V>(y + t * a.y_token, Vec<T, V>{});
    // The thread of the first tokens, the only one that reads the old state, writes the new one (both may be the same memory).
    if (t0 == 0 && a.new_state && slot >= 0) {
#pragma unroll
        for (int j = 0; j < K - 1; ++j) {
            const int at = len - (K - 1) + j;
            Vec<T, V> v = {};
            if (at >= 0) {
                v = load_vec<T, V>(x + at * a.x_token);
            } else {
#pragma unroll
                for (int o = 0; o < K - 1; ++o)
                    if (o == at + K - 1) v = old[o];
            }
            store_vec<T, V>(static_cast<T *>(a.new_state) + srow + (long long)j * C, v);
        }
    }
}

static xl_causal_conv_args piece_of(const xl_causal_conv_args &a, long long first, long long count)
{
    const int size = a.dtype == XL_F32 ? 4 : 2;
    xl_causal_conv_args p = piece_of_states(a, first, count, (a.taps - 1) * a.channels, size);
    p.x = behind(a.x, first * a.x_batch, size);
    p.y = behind(a.y, first * a.y_batch, size);
    return p;
}

template <int DT, int K, int V> static hipError_t launch(const xl_causal_conv_args &a, hipStream_t s)
{
    const long long vecs = a.channels / V;
    // Runs of 32 tokens read an input 1.1 times (of 8, 16, 32 tokens: 42.7, 39.1, 38.7 us; 2047 channels 70, 56, 51); shorter ones where there would be fewer than 2048 threads a compute unit.
    long long run = 32;
    while (run > 4 && a.batch * vecs * ((a.length + run - 1) / run) < 256ll * 2048) run /= 2;
    const long long runs = a.length > 0 ? (a.length + run - 1) / run : 1;
    return in_pieces(a, vecs * runs, piece_of, [&](const xl_causal_conv_args &p) {
        return launch_kernel(conv_kernel<DT, K, V>, dim3((unsigned)((p.batch * vecs * runs + 255) / 256)), 256, s, p, (int)run, (int)runs);
    });
}

template <int DT, int K> static hipError_t launch_taps(const xl_causal_conv_args &a, hipStream_t s)
{
    // 4 bytes of a row a thread (8 x 3025 x 2048 in bf16, us with 4, 8: 38.6, 42; 3025 x 1024 5.6, 6.5 and with 16 9.2), one number where those do not divide
    // a row (8 x 3025 x 2047: 51)
    constexpr int V = 4 / sizeof(typename Elem<DT>::T);
    if (V == 1 || a.channels % V) return launch<DT, K, 1>(a, s);
    return launch<DT, K, V>(a, s);
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
