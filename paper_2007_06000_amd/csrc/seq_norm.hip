// Root-mean-square norm of rows, with the residual's addition in front and eight-bit numbers behind.
//
//   r = x + residual,  y = r / sqrt(mean(r^2) + eps) * weight,  and with 8 bits  scale = max(max|y| / 448, 2^-126), q = e4m3(y / scale)
//
// Bound by memory.  A row's numbers stay in the registers of the lanes that have loaded them until its sum is known: eight neighbours a lane and load, so that sixteen
// lanes hold a block of 128 with its scale.  24642 x 4096 in bf16 with a residual, to 8 bits: 141 us for 710 MB, 5.0 TB/s (a copy of 4 GB: 4.9); 3645 x 1001 in fp32 12.8 us, 4.6 TB/s;
// 16 x 2048 3.5 us, of which a launch is 1.6 to 1.9.
#include "seq_e4m3.h"
#include "seq_internal.h"

namespace xls {

struct Row {
    const char *x, *residual;
    char *kept, *y;
    float *scales;
};

template <int DT> __device__ __forceinline__ void load8f(const void *row, int k, int K, float *v)
{
    typedef typename Elem<DT>::T T;
    const Vec<T, 8> w = load_some<T, 8>(static_cast<const T *>(row) + k, K - k);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)w[i];
}
template <int DT> __device__ __forceinline__ void store8f(void *row, int k, int K, const float *v)
{
    typedef typename Elem<DT>::T T;
    Vec<T, 8> w;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = (T)v[i];
    store_some<T, 8>(static_cast<T *>(row) + k, K - k, w);
}

// r of eight neighbours from column k on; zeros past the end
template <int DT> __device__ __forceinline__ void load_sum(const xl_rms_norm_args &a, const Row &row, int k, int K, float *r)
{
    load8f<DT>(row.x, k, K, r);
    if (!row.residual) return;
    float more[8];
    if (a.residual_dtype == XL_F32) load8f<XL_F32>(row.residual, k, K, more);
    else load8f<DT>(row.residual, k, K, more);
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] += more[i];
}
template <int DT> __device__ __forceinline__ void keep(const xl_rms_norm_args &a, const Row &row, int k, int K, const float *r)
{
    if (!row.kept || k >= K) return;
    if (a.residual_dtype == XL_F32) store8f<XL_F32>(row.kept, k, K, r);
    else store8f<DT>(row.kept, k, K, r);
}

template <int W, typename S> __device__ __forceinline__ S sum_of_row(S s, S *shared)
{
#pragma unroll
    for (int o = 1; o < 64; o *= 2) s += __shfl_xor(s, o);
    if constexpr (W > 1) {
        __syncthreads();        // the sums before have been read
        if (threadIdx.x % 64 == 0) shared[threadIdx.x / 64] = s;
        __syncthreads();
        s = 0;
#pragma unroll
        for (int i = 0; i < W; ++i) s += shared[i];
    }
    return s;
}

// Squares of numbers above 2^64 leave fp32, and so may a mean and eps together.  Then both are taken scaled down: numbers whose squares vanish do not count beside them.
static constexpr float DOWN = 0x1p-80f;

// y, or q and a scale, of eight neighbours: r is multiplied with the root's inverse, `down` (behind it: small numbers must not leave fp32 on the way) and the weight
template <int DT, bool Q> __device__ __forceinline__ void finish(const xl_rms_norm_args &a, const Row &row, int k, int K, float *v, float down, float inverse)
{
    float w[8];
    load8f<XL_F32>(a.weight, k, K, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = v[i] * inverse * down * w[i];
    if constexpr (Q) {
        unsigned most = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) most = max(most, magnitude(v[i]));
#pragma unroll
        for (int o = 1; o < 16; o *= 2) most = max(most, (unsigned)__shfl_xor((int)most, o));
        const float scale = scale_of(most);
        if (threadIdx.x % 16 == 0 && k < K) row.scales[k / XL_SCALE_BLOCK * a.scale_block] = scale;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = v[i] / scale;
        if (k < (K + 15) / 16 * 16) *reinterpret_cast<unsigned long long *>(row.y + k) = e4m3x8(v, K - k);
    } else if (k < K) {
        store8f<DT>(row.y, k, K, v);
    }
}

template <int DT, bool Q> __device__ __forceinline__ Row row_of(const xl_rms_norm_args &a, long long i)
{
    const int size = sizeof(typename Elem<DT>::T), kept = a.residual_dtype == XL_F32 ? 4 : size;
    return {static_cast<const char *>(a.x) + i * a.x_row * size, a.residual ? static_cast<const char *>(a.residual) + i * a.residual_row * kept : nullptr,
            a.new_residual ? static_cast<char *>(a.new_residual) + i * a.new_residual_row * kept : nullptr, static_cast<char *>(a.y) + i * a.y_row * (Q ? 1 : size),
            Q ? a.scales + i * a.scale_row : nullptr};
}

// W waves a row, N times eight numbers a lane: rows of up to 512 W N numbers.  One wave up to 1024, whose sum needs no other; four up to what their registers hold, so that a row's loads are all on their
// way at once.
template <int DT, bool Q, int W, int N>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void norm_kernel(const xl_rms_norm_args a)
{
    constexpr int ROWS = W == 1 ? 4 : 1;
    __shared__ float shared[W];
    const int lane = threadIdx.x % (64 * W), K = (int)a.k;
    const float k_inverse = 1.f / (float)K, eps = (float)a.eps;
    for (long long i = (long long)blockIdx.x * ROWS + threadIdx.x / (64 * W); i < a.rows; i += (long long)gridDim.x * ROWS) {
        const Row row = row_of<DT, Q>(a, i);
        float r[N][8], s = 0.f;
#pragma unroll
        for (int n = 0; n < N; ++n) load_sum<DT>(a, row, (n * 64 * W + lane) * 8, K, r[n]);
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int j = 0; j < 8; ++j) s = __builtin_fmaf(r[n][j], r[n][j], s);
        s = sum_of_row<W>(s, shared);
        const float mean = s * k_inverse + eps;
        float down = 1.f, inverse = __builtin_amdgcn_rsqf(mean);
        if (!(mean < __builtin_inff())) {
            s = 0.f;
            down = DOWN;
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int j = 0; j < 8; ++j) s = __builtin_fmaf(r[n][j] * DOWN, r[n][j] * DOWN, s);
            inverse = __builtin_amdgcn_rsqf(sum_of_row<W>(s, shared) * k_inverse + eps * DOWN * DOWN);
        }
#pragma unroll
        for (int n = 0; n < N; ++n) keep<DT>(a, row, (n * 64 * W + lane) * 8, K, r[n]);
#pragma unroll
        for (int n = 0; n < N; ++n) finish<DT, Q>(a, row, (n * 64 * W + lane) * 8, K, r[n], down, inverse);
    }
}

// Longer rows are read twice.  Their sums are in 64 bits, which hold every square: a lane adds one square in 1024 of the row's, and equal ones are rounded the same way.  (In 32 bits a row of 2^24 numbers 0.95
// came out 6e-5 off.  512 x 65536 in bf16 take 39 us either way, 2048 x 40000 95.)
template <int DT, bool Q>
__global__ __launch_bounds__(1024) void long_norm_kernel(const xl_rms_norm_args a)
{
    __shared__ double shared[16];
    const int K = (int)a.k, last = (K + 127) / 128 * 128;        // all lanes of a block of 128 take part in its scale
    // k in 64 bits: a turn is longer than what is left of 32 behind the longest row
    for (long long i = blockIdx.x; i < a.rows; i += gridDim.x) {
        const Row row = row_of<DT, Q>(a, i);
        float r[8];
        double s = 0.;
        for (long long k = threadIdx.x * 8; k < K; k += 8192) {
            load_sum<DT>(a, row, k, K, r);
#pragma unroll
            for (int j = 0; j < 8; ++j) s = __builtin_fma((double)r[j], (double)r[j], s);
        }
        const double mean = sum_of_row<16>(s, shared) / K + a.eps;
        const bool large = !((float)mean < __builtin_inff());
        const float inverse = __builtin_amdgcn_rsqf((float)(large ? mean * DOWN * DOWN : mean));
        for (long long k = threadIdx.x * 8; k < last; k += 8192) {
            load_sum<DT>(a, row, k, K, r);
            keep<DT>(a, row, k, K, r);
            finish<DT, Q>(a, row, k, K, r, large ? DOWN : 1.f, inverse);
        }
    }
}

template <int DT, bool Q, int W, int N> static hipError_t launch_rows(const xl_rms_norm_args &a, hipStream_t s)
{
    const long long groups = W == 1 ? (a.rows + 3) / 4 : a.rows;
    return launch_kernel(norm_kernel<DT, Q, W, N>, dim3((unsigned)(groups < 1 << 20 ? groups : 1 << 20)), W == 1 ? 256 : 64 * W, s, a);
}

template <int DT, bool Q> static hipError_t launch_type(const xl_rms_norm_args &a, hipStream_t s)
{
    if (a.k <= 512) return launch_rows<DT, Q, 1, 1>(a, s);
    if (a.k <= 1024) return launch_rows<DT, Q, 1, 2>(a, s);
    if (a.k <= 2048) return launch_rows<DT, Q, 4, 1>(a, s);
    if (a.k <= 4096) return launch_rows<DT, Q, 4, 2>(a, s);
    if (a.k <= 8192) return launch_rows<DT, Q, 4, 4>(a, s);
    if (a.k <= 16384) return launch_rows<DT, Q, 4, 8>(a, s);
    if (a.k <= 32768) return launch_rows<DT, Q, 16, 4>(a, s);
    return launch_kernel(long_norm_kernel<DT, Q>, dim3((unsigned)(a.rows < 1 << 20 ? a.rows : 1 << 20)), 1024, s, a);
}

template <int DT> static hipError_t launch_result(const xl_rms_norm_args &a, hipStream_t s) { return a.quantized ? launch_type<DT, true>(a, s) : launch_type<DT, false>(a, s); }

hipError_t launch_rms_norm(const xl_rms_norm_args &a, hipStream_t s)
{
    return a.dtype == XL_F32 ? launch_result<XL_F32>(a, s) : a.dtype == XL_F16 ? launch_result<XL_F16>(a, s) : launch_result<XL_BF16>(a, s);
}

}  // namespace xls
