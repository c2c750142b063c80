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

// Each part is what is left, rounded to nearest: after two of them at most 2^-16 of a number is missing, after three nothing.  Four numbers, two to a register:
template <int N> struct Parts4 {
    u32x2 p[N];
};
template <int N> __device__ __forceinline__ Parts4<N> split4(f32x4 v)
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    Parts4<N> out;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const unsigned both = __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2{v[2 * i], v[2 * i + 1]}), bf16x2));
            out.p[n][i] = both;
            if (n + 1 < N) {
                v[2 * i] -= __builtin_bit_cast(float, both << 16);
                v[2 * i + 1] -= __builtin_bit_cast(float, both & 0xffff0000u);
            }
        }
    return out;
}
template <int N> __device__ __forceinline__ Parts<N> split(f32x8 v)
{
    const Parts4<N> lo = split4<N>(f32x4{v[0], v[1], v[2], v[3]}), hi = split4<N>(f32x4{v[4], v[5], v[6], v[7]});
    Parts<N> out;
#pragma unroll
    for (int n = 0; n < N; ++n) out.p[n] = __builtin_bit_cast(bf16x8, u32x4{lo.p[n][0], lo.p[n][1], hi.p[n][0], hi.p[n][1]});
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
