// Low-rank adapters of many sequences beside a shared product.
//
//   out[b,t] = y[b,t] + scales[e] * up[e] (down[e] x[b,t]),  e = index[b]
#include "seq_internal.h"

namespace xls {

// The adapter of sequence b, or -1.
__device__ __forceinline__ long long adapter_of(const xl_adapters_args &a, int b)
{
    const int e = a.index[b];
    return e >= 0 && e < a.adapters ? e : -1;
}

// A token a workgroup: its waves take the rows of down in turn, then each thread columns of up.
template <int DT>
__global__ __launch_bounds__(256) void token_kernel(const xl_adapters_args a)
{
    typedef typename Elem<DT>::T T;
    __shared__ float inner[XL_MAX_RANK];
    const int K = (int)a.k, N = (int)a.n, R = (int)a.rank, length = (int)a.length;
    for (long long token = blockIdx.x; token < a.batch * a.length; token += gridDim.x) {
        const int b = (int)(token / length), t = (int)(token % length);
        T *out = static_cast<T *>(a.out) + b * a.out_batch + t * a.out_token;
        if (t >= length_of(a.lengths, b, length)) {
            for (int j = threadIdx.x; j < N; j += 256) out[j] = (T)0.f;
            continue;
        }
        const T *x = static_cast<const T *>(a.x) + b * a.x_batch + t * a.x_token, *y = static_cast<const T *>(a.y) + b * a.y_batch + t * a.y_token;
        const long long e = adapter_of(a, b);
        __syncthreads();        // what the token before has left is no longer read
        if (e >= 0) {
            const T *down = static_cast<const T *>(a.down) + e * a.rank * a.k;
            for (int r = threadIdx.x / 64; r < R; r += 4) {
                float s = 0.f;
                for (int k = threadIdx.x % 64; k < K; k += 64) s = __builtin_fmaf((float)x[k], (float)down[(long long)r * K + k], s);
#pragma unroll
                for (int o = 1; o < 64; o *= 2) s += __shfl_xor(s, o);
                if (threadIdx.x % 64 == 0) inner[r] = s * (a.scales ? a.scales[e] : 1.f);
            }
        }
        __syncthreads();
        const T *up = static_cast<const T *>(a.up) + (e >= 0 ? e : 0) * a.rank * a.n;
        for (int j = threadIdx.x; j < N; j += 256) {
            float s = (float)y[j];
            if (e >= 0)
                for (int r = 0; r < R; ++r) s = __builtin_fmaf(inner[r], (float)up[(long long)j * R + r], s);
            out[j] = (T)s;
        }
    }
}

template <int DT> static hipError_t launch_type(const xl_adapters_args &a, hipStream_t s)
{
    const long long tokens = a.batch * a.length;
    return launch_kernel(token_kernel<DT>, dim3((unsigned)(tokens < 1 << 20 ? tokens : 1 << 20)), 256, s, a);
}

long long adapters_workspace(const xl_adapters_args &) { return 0; }

hipError_t launch_add_adapters(const xl_adapters_args &a, hipStream_t s)
{
    return a.dtype == XL_F32 ? launch_type<XL_F32>(a, s) : a.dtype == XL_F16 ? launch_type<XL_F16>(a, s) : launch_type<XL_BF16>(a, s);
}

}  // namespace xls
