// What the kernels of the sequence operators share: element types, accesses, elementary functions.
#pragma once
#include <hip/hip_runtime.h>

#include "seq_launch.h"

namespace xls {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// A kernel's launch and its own status.  (The runtime's last error may be one that somebody else's call has left.)
template <typename T> struct Same {
    typedef T Type;
};
template <typename... P> static hipError_t launch_kernel(void (*kernel)(P...), dim3 grid, unsigned threads, hipStream_t s, typename Same<P>::Type... args)
{
    void *list[] = {&args...};
    return hipLaunchKernel(reinterpret_cast<const void *>(kernel), grid, dim3(threads), list, 0, s);
}

// A launch has fewer than 2^32 threads along x.  A batch that needs more goes in pieces of sequences, each of `threads` threads, rounded up to a workgroup's.
static constexpr long long MAX_THREADS = (1ll << 32) - 1024;
template <typename A, typename F> static hipError_t in_pieces(const A &a, long long threads, A (*piece_of)(const A &, long long, long long), F launch)
{
    if (threads > MAX_THREADS) return hipErrorInvalidConfiguration;         // one sequence by itself
    const long long most = threads > 0 ? MAX_THREADS / threads : a.batch;
    if (a.batch <= most) return launch(a);
    for (long long b = 0; b < a.batch; b += most) {
        const hipError_t e = launch(piece_of(a, b, a.batch - b < most ? a.batch - b : most));
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
// `count` elements of `size` bytes behind p, or still nothing
template <typename T> static T *behind(T *p, long long count, long long size)
{
    return p ? reinterpret_cast<T *>(reinterpret_cast<unsigned long long>(p) + (unsigned long long)(count * size)) : p;
}
// What all batches have: their own lengths and slots, or the next rows of the states.
template <typename A> static A piece_of_states(A a, long long first, long long count, long long row, long long size)
{
    a.batch = count;
    a.lengths = behind(a.lengths, first, sizeof(int));
    if (a.slots) {
        a.slots += first;
    } else {
        a.nslots -= first;
        a.state = behind(a.state, first * row, size);
        a.new_state = behind(a.new_state, first * row, size);
    }
    return a;
}

static constexpr float LOG2E = 1.44269504088896340736f;

// Activations in memory <-> fp32.  Conversions to 16 bits round to nearest, ties to even.
template <int DT> struct Elem;
template <> struct Elem<XL_F32> {
    typedef float T;
};
template <> struct Elem<XL_F16> {
    typedef _Float16 T;
};
template <> struct Elem<XL_BF16> {
    typedef __bf16 T;
};

template <typename T, int V> using Vec = T __attribute__((ext_vector_type(V)));

// V elements at p, of any alignment, as one access.
template <typename T, int V> __device__ __forceinline__ Vec<T, V> load_vec(const T *p)
{
    Vec<T, V> v;
    __builtin_memcpy(&v, p, V * sizeof(T));
    return v;
}
template <typename T, int V> __device__ __forceinline__ void store_vec(T *p, Vec<T, V> v) { __builtin_memcpy(p, &v, V * sizeof(T)); }

// V elements at p, of any alignment, of which the first n exist; the others come out as zeros.
template <typename T, int V> __device__ __forceinline__ Vec<T, V> load_some(const T *p, int n)
{
    Vec<T, V> v = {};
    if (n >= V) {
        v = load_vec<T, V>(p);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < n) v[i] = p[i];
    }
    return v;
}
template <typename T, int V> __device__ __forceinline__ void store_some(T *p, int n, Vec<T, V> v)
{
    if (n >= V) {
        store_vec<T, V>(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < n) p[i] = v[i];
    }
}

// One hardware exponential (about one unit in the last place; results below the normal range are zero).
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float exp_fast(float x) { return exp2_fast(x * LOG2E); }

// v * sigmoid(v)
__device__ __forceinline__ float silu(float v) { return v * __builtin_amdgcn_rcpf(1.f + exp_fast(-v)); }

// log(1 + exp(x)) = max(x, 0) + log(1 + e), e = exp(-|x|) in (0, 1].  log(1 + e) = 2 artanh(r), r = e / (2 + e) <= 1/3, with artanh(r) / r a polynomial in
// r^2 fitted to within 8e-9.  (The hardware logarithm of 1 + e would lose the digits of a small e, and small steps are the usual
// ones.)  NaN and infinities come through.
__device__ __forceinline__ float softplus(float x)
{
    const float e = exp_fast(-fabsf(x));
    const float r = e * __builtin_amdgcn_rcpf(2.f + e), q = r * r;
    float s = 2 * 0.14087329f;
    s = __builtin_fmaf(s, q, 2 * 0.13980709f);
    s = __builtin_fmaf(s, q, 2 * 0.20012427f);
    s = __builtin_fmaf(s, q, 2 * 0.33333158f);
    s = __builtin_fmaf(s, q, 2.f);
    // max(x, 0) on the bits: what is negative as a float is so as an integer (and a NaN has come through e)
    const float m = __builtin_bit_cast(float, max(__builtin_bit_cast(int, x), 0));
    return __builtin_fmaf(r, s, m);
}

// The row of the states that belongs to sequence b, or -1 if it is absent.
__device__ __forceinline__ long long slot_of(const int *slots, long long nslots, int b)
{
    const long long s = slots ? slots[b] : b;
    return s >= 0 && s < nslots ? s : -1;
}
__device__ __forceinline__ int length_of(const int *lengths, int b, int length)
{
    return lengths ? min(max(lengths[b], 0), length) : length;
}

// What lanes of this wave have put into LDS can be read by the others.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Workgroups go round the eight XCDs, each with a cache of its own; this numbers them so that neighbours are on the same one.
__device__ __forceinline__ int neighbours_together(int block, int blocks)
{
    const int xcd = block % 8, per = blocks / 8, more = blocks % 8;
    return xcd * per + min(xcd, more) + block / 8;
}

}  // namespace xls
