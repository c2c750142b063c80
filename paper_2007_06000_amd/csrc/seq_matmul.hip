// Product of two e4m3 operands with a scale for each block of 128 numbers.
//
//   y[i,j] = bias[j] + sum_b sa[i,b] sb[j/128,b] (sum over k of block b of a[i,k] b[j,k])
//
// A block's sum is one matrix operation 16 x 16 x 128 (or four of 16 x 16 x 32, below); it starts at zero, and its result is scaled into the fp32 sums by one
// multiply-add for each of a lane's four.  The rows of b are the operation's rows and those of a its columns: a lane's four results are then neighbours in a row of
// y, and share one scale of a (the lane's column) and one of b (its 16 rows lie in one block of 128).
#include "seq_internal.h"

namespace xls {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// A lane's 32 of a row's 128 numbers.  Which of the 128 does not matter, as long as both operands agree.
union Part {
    u32x4 q[2];
    i32x8 v;
};

// The sum of one block.  The 8-bit operation adds its 128 products with fewer bits than fp32 has: measured on normal numbers its result
// is 1.3e-5 off (at most 9e-6 of the sum of the products' magnitudes), which a result of 16 bits (2e-4 to 2e-3) hides.  A result of 32 bits does not, so it is
// computed on bf16 operations instead, whose products and sums are fp32: e4m3 is exact in bf16.  They take twice the time.
template <bool EXACT> struct BlockProduct;
template <> struct BlockProduct<false> {
    typedef Part Operand;
    static __device__ __forceinline__ Operand operand(const Part &p) { return p; }
    static __device__ __forceinline__ f32x4 run(const Operand &rows, const Operand &cols)
    {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(rows.v, cols.v, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
    }
};
template <> struct BlockProduct<true> {
    struct Operand {
        bf16x8 part[4];
    };
    static __device__ __forceinline__ Operand operand(const Part &p)
    {
        Operand o;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(p.v[i], 1.f, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(p.v[i], 1.f, true);
            o.part[i / 2][i % 2 * 4] = lo[0];
            o.part[i / 2][i % 2 * 4 + 1] = lo[1];
            o.part[i / 2][i % 2 * 4 + 2] = hi[0];
            o.part[i / 2][i % 2 * 4 + 3] = hi[1];
        }
        return o;
    }
    static __device__ __forceinline__ f32x4 run(const Operand &rows, const Operand &cols)
    {
        f32x4 s = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(rows.part[i], cols.part[i], s, 0, 0, 0);
        return s;
    }
};

// 16 numbers of a row from column k on; those at K and past it are zeros.
__device__ __forceinline__ u32x4 load16(const char *row, int k, int K)
{
    u32x4 v = {};
    if (k < K) {
        v = *reinterpret_cast<const u32x4 *>(row + k);
        const int live = K - k;
        if (live < 16) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int bytes = live - 4 * i;
                v[i] &= bytes >= 4 ? 0xffffffffu : bytes <= 0 ? 0u : (1u << (8 * bytes)) - 1;
            }
        }
    }
    return v;
}

template <int DT> __device__ __forceinline__ void store4(const xl_block_matmul_args &a, long long i, int j, f32x4 v, bool wide)
{
    typedef typename Elem<DT>::T T;
    if (i >= a.m || j >= a.n) return;
    float out[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) out[k] = v[k] + (a.bias && j + k < a.n ? a.bias[j + k] : 0.f);
    T *y = static_cast<T *>(a.y) + i * a.y_row;
    if (wide && j + 4 <= a.n) {
        store_vec<DT, 4>(y, j, out);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (j + k < a.n) y[j + k] = (T)out[k];
    }
}

// 16 rows of b by 16 rows of a; the waves of the workgroup divide the reduction.
template <int DT, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void thin_kernel(const xl_block_matmul_args a, int tiles_n, bool wide)
{
    __shared__ f32x4 part[WAVES][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, col = lane % 16, quad = lane / 16, K = (int)a.k;
    const int n0 = (blockIdx.x % tiles_n) * 16, blocks = (K + XL_SCALE_BLOCK - 1) / XL_SCALE_BLOCK;
    const long long m0 = (long long)(blockIdx.x / tiles_n) * 16;
    const char *brow = static_cast<const char *>(a.b) + min((long long)n0 + col, a.n - 1) * a.b_row;
    const long long ai = min(m0 + col, a.m - 1);
    const char *arow = static_cast<const char *>(a.a) + ai * a.a_row;
    const float *sa = a.a_scales + ai * a.a_scale_row, *sb = a.b_scales + (n0 / XL_SCALE_BLOCK) * a.b_scale_row;
    f32x4 acc = {};
    for (int kb = wave; kb < blocks; kb += WAVES) {
        const int k = kb * XL_SCALE_BLOCK + quad * 32;
        Part r, c;
        r.q[0] = load16(brow, k, K);
        r.q[1] = load16(brow, k + 16, K);
        c.q[0] = load16(arow, k, K);
        c.q[1] = load16(arow, k + 16, K);
        typedef BlockProduct<DT == XL_F32> P;
        const f32x4 p = P::run(P::operand(r), P::operand(c));
        const float s = sa[kb * a.a_scale_block] * sb[kb * a.b_scale_block];
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = __builtin_fmaf(s, p[i], acc[i]);
    }
    part[wave][lane] = acc;
    __syncthreads();
    if (wave == 0) {
#pragma unroll
        for (int w = 1; w < WAVES; ++w) acc += part[w][lane];
        store4<DT>(a, m0 + col, n0 + quad * 4, acc, wide);
    }
}

template <int DT> static hipError_t launch_type(const xl_block_matmul_args &a, hipStream_t s)
{
    typedef typename Elem<DT>::T T;
    const bool wide = ((unsigned long long)a.y | (unsigned long long)a.y_row * sizeof(T)) % (4 * sizeof(T)) == 0;
    const long long tiles_n = (a.n + 15) / 16, tiles = tiles_n * ((a.m + 15) / 16);
    thin_kernel<DT, 4><<<dim3((unsigned)tiles), 256, 0, s>>>(a, (int)tiles_n, wide);
    return hipGetLastError();
}

hipError_t launch_block_matmul(const xl_block_matmul_args &a, hipStream_t s)
{
    return a.dtype == XL_F32 ? launch_type<XL_F32>(a, s) : a.dtype == XL_F16 ? launch_type<XL_F16>(a, s) : launch_type<XL_BF16>(a, s);
}

}  // namespace xls
