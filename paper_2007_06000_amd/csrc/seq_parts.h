// Numbers of more than 8 bits on the bf16 matrix operations: as sums of bf16 parts, whose products are exact and are added in fp32.
#pragma once
#include "seq_internal.h"

namespace xls {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

// Parts that hold an element exactly: fp16 has 11 bits, fp32 24.
template <int DT> constexpr int parts_of() { return DT == XL_BF16 ? 1 : DT == XL_F16 ? 2 : 3; }

template <int N> struct Parts {
    bf16x8 p[N];
};

// Each part is what is left, rounded to nearest: after two of them at most 2^-16 of a number is missing, after three nothing.
template <int N> __device__ __forceinline__ Parts<N> split(f32x8 v)
{
    Parts<N> out;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        out.p[n] = __builtin_convertvector(v, bf16x8);
        if (n + 1 < N) v -= __builtin_convertvector(out.p[n], f32x8);
    }
    return out;
}
template <int DT> __device__ __forceinline__ Parts<parts_of<DT>()> parts(Vec<typename Elem<DT>::T, 8> v)
{
    if constexpr (DT == XL_BF16) return {{v}};
    else return split<parts_of<DT>()>(__builtin_convertvector(v, f32x8));
}

// acc += rows x columns, 16 x 16 x 32: the pairs of parts whose product counts beside the last place of an fp32 number.
template <int A, int B> __device__ __forceinline__ f32x4 product(const Parts<A> &rows, const Parts<B> &cols, f32x4 acc)
{
#pragma unroll
    for (int i = A + B - 2; i >= 0; --i)        // small ones first
#pragma unroll
        for (int j = 0; j < A; ++j)
            if (i - j >= 0 && i - j < B && i < 3) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(rows.p[j], cols.p[i - j], acc, 0, 0, 0);
    return acc;
}

}  // namespace xls
