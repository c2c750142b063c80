// Blocks of numbers to e4m3 with a scale each.
//
//   scale = max(max|x| / 448, 2^-126),  q = e4m3(x / scale)
//
// Bound by memory.  The division is a true one (about ten operations a number, hidden behind the loads): a product with the reciprocal lands on the
// other side of a tie now and then, and q would depend on how it was computed.
#include "seq_internal.h"

namespace xls {

static constexpr float E4M3_MAX = 448.f, MIN_SCALE = 1.17549435e-38f;

// The largest |x| as the bits of a float: the order of the bits is the order of the numbers, infinity and then NaN above them.
__device__ __forceinline__ unsigned magnitude(float x) { return __builtin_bit_cast(unsigned, x) & 0x7fffffffu; }
__device__ __forceinline__ float scale_of(unsigned most)
{
    const float s = __builtin_bit_cast(float, most) / E4M3_MAX;
    return s < MIN_SCALE ? MIN_SCALE : s;      // a NaN stays
}

__device__ __forceinline__ unsigned e4m3x4(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// Eight numbers of a row from column k on; those past its end are zeros.
template <int DT> __device__ __forceinline__ void load8(const typename Elem<DT>::T *x, long long at, int k, int K, float *v)
{
    if (k + 8 <= K) {
        const Vec<typename Elem<DT>::T, 8> w = load_vec<typename Elem<DT>::T, 8>(x + at + k);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)w[i];
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = k + i < K ? (float)x[at + k + i] : 0.f;
}

// Rows beyond 65535 groups go on in z.
static constexpr unsigned GRID_Y = 65535;
static dim3 grid_of(long long blocks, long long groups)
{
    return dim3((unsigned)blocks, (unsigned)(groups < GRID_Y ? groups : GRID_Y), (unsigned)((groups + GRID_Y - 1) / GRID_Y));
}
__device__ __forceinline__ long long group_of_rows() { return (long long)blockIdx.z * GRID_Y + blockIdx.y; }

// 16 lanes a block, 8 numbers a lane, PER neighbouring blocks of 16 / PER rows a workgroup; workgroups next to each other go on along the rows.
// With four blocks a wave reads a kilobyte of a row in one go; 24642 x 4096 in bf16 takes 65 us for 303 MB (4.7 TB/s, as a copy of 4 GB; a copy of 300 MB whose source the
// last-level cache holds 55), in fp32 (x 4000) 88.  One block of sixteen rows, workgroups going down the rows: 70 and 123.  Fewer blocks where a row has no four.
template <int DT, int PER>
__global__ __launch_bounds__(256) void rows_kernel(const xl_quantize_args a)
{
    typedef typename Elem<DT>::T T;
    const int lane = threadIdx.x % 16, K = (int)a.k, at = threadIdx.x / 16, kb = blockIdx.x * PER + at % PER, k = kb * XL_SCALE_BLOCK + lane * 8;
    const long long row = group_of_rows() * (16 / PER) + at / PER;
    if (row >= a.rows || kb * XL_SCALE_BLOCK >= K) return;
    float v[8];
    load8<DT>(static_cast<const T *>(a.x), row * a.x_row, k, K, v);
    unsigned most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max(most, magnitude(v[i]));
#pragma unroll
    for (int o = 1; o < 16; o *= 2) most = max(most, (unsigned)__shfl_xor((int)most, o));
    const float scale = scale_of(most);
    if (lane == 0) a.scales[row * a.scale_row + kb * a.scale_block] = scale;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = v[i] / scale;
    if (k < (K + 15) / 16 * 16)
        *reinterpret_cast<u32x2 *>(static_cast<char *>(a.q) + row * a.q_row + k) = u32x2{e4m3x4(v[0], v[1], v[2], v[3]), e4m3x4(v[4], v[5], v[6], v[7])};
}

// A block of 128 rows by 128 columns a workgroup; a thread has 8 columns of every sixteenth row.  Weights are quantised once.
template <int DT>
__global__ __launch_bounds__(256) void blocks_kernel(const xl_quantize_args a)
{
    typedef typename Elem<DT>::T T;
    __shared__ unsigned shared_most[4];
    const int K = (int)a.k, kb = blockIdx.x, k = kb * XL_SCALE_BLOCK + (threadIdx.x % 16) * 8;
    const long long group = group_of_rows(), row0 = group * XL_SCALE_BLOCK + threadIdx.x / 16;
    if (row0 - threadIdx.x / 16 >= a.rows) return;      // all of the workgroup
    float v[8][8];
    unsigned most = 0;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        const long long row = row0 + r * 16;
        if (row < a.rows) {
            load8<DT>(static_cast<const T *>(a.x), row * a.x_row, k, K, v[r]);
#pragma unroll
            for (int i = 0; i < 8; ++i) most = max(most, magnitude(v[r][i]));
        }
    }
#pragma unroll
    for (int o = 1; o < 64; o *= 2) most = max(most, (unsigned)__shfl_xor((int)most, o));
    if (threadIdx.x % 64 == 0) shared_most[threadIdx.x / 64] = most;
    __syncthreads();
    most = max(max(shared_most[0], shared_most[1]), max(shared_most[2], shared_most[3]));
    const float scale = scale_of(most);
    if (threadIdx.x == 0) a.scales[group * a.scale_row + kb * a.scale_block] = scale;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        const long long row = row0 + r * 16;
        if (row < a.rows && k < (K + 15) / 16 * 16) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[r][i] = v[r][i] / scale;
            *reinterpret_cast<u32x2 *>(static_cast<char *>(a.q) + row * a.q_row + k) =
                u32x2{e4m3x4(v[r][0], v[r][1], v[r][2], v[r][3]), e4m3x4(v[r][4], v[r][5], v[r][6], v[r][7])};
        }
    }
}

template <int DT, int PER> static hipError_t launch_rows(const xl_quantize_args &a, hipStream_t s)
{
    const long long blocks = (a.k + XL_SCALE_BLOCK - 1) / XL_SCALE_BLOCK, under = 16 / PER;
    return launch_kernel(rows_kernel<DT, PER>, grid_of((blocks + PER - 1) / PER, (a.rows + under - 1) / under), 256, s, a);
}

template <int DT> static hipError_t launch_type(const xl_quantize_args &a, hipStream_t s)
{
    const long long blocks = (a.k + XL_SCALE_BLOCK - 1) / XL_SCALE_BLOCK;
    if (a.block_rows != 1) return launch_kernel(blocks_kernel<DT>, grid_of(blocks, (a.rows + XL_SCALE_BLOCK - 1) / XL_SCALE_BLOCK), 256, s, a);
    return blocks == 1 ? launch_rows<DT, 1>(a, s) : blocks == 2 ? launch_rows<DT, 2>(a, s) : launch_rows<DT, 4>(a, s);
}

hipError_t launch_quantize(const xl_quantize_args &a, hipStream_t s)
{
    return a.dtype == XL_F32 ? launch_type<XL_F32>(a, s) : a.dtype == XL_F16 ? launch_type<XL_F16>(a, s) : launch_type<XL_BF16>(a, s);
}

}  // namespace xls
