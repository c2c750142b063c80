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

// BM rows of a by BN rows of b, WM x WN waves, each with BM / WM by BN / WN of them: TM x TN matrix operations a block.  Both operands' blocks go straight to LDS, two
// stages in turn: the next block comes while this one is multiplied.  A row's block is 128 bytes, 8 chunks of 16; chunk c of row r lies at chunk c ^ (r & 7),
// so that the 16 rows that an operation reads at once, 128 bytes apart, fall on different banks.
template <int BM, int BN> struct Stage {
    char a[BM * 128], b[BN * 128];
    float scale[BM];
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void *p, long long begin, long long size)
{
    const unsigned long long at = (unsigned long long)p + begin;
    const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)at), hi = __builtin_amdgcn_readfirstlane((unsigned)(at >> 32)), bytes = (unsigned)size;
    return __builtin_amdgcn_make_buffer_rsrc((void *)(((unsigned long long)hi << 32) | lo), (short)0, (int)__builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}

// A wave's 64 times 16 (or 4) bytes from memory into LDS, lane after lane from `to` on.
__device__ __forceinline__ void to_lds16(__amdgpu_buffer_rsrc_t from, void *to, unsigned at, unsigned begin)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void *)to, 16, at, begin, 0, 0);
}
__device__ __forceinline__ void to_lds4(__amdgpu_buffer_rsrc_t from, void *to, unsigned at, unsigned begin)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void *)to, 4, at, begin, 0, 0);
}

template <int DT, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void tile_kernel(const xl_block_matmul_args p, int tiles_m, int tiles_n, bool wide)
{
    constexpr int WAVES = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16, LA = BM / 8 / WAVES, LB = BN / 8 / WAVES;
    static_assert(LA >= 1 && LB >= 1 && TN * 16 <= XL_SCALE_BLOCK && BM % 64 == 0 && BM / 64 <= WAVES, "the waves share the loads");
    typedef BlockProduct<DT == XL_F32> P;
    __shared__ Stage<BM, BN> even, odd;

    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), col = lane % 16, quad = lane / 16;
    // Workgroups go to the 8 XCDs in turn; each XCD gets a contiguous part of an order in which 8 x 4 neighbours share rows of a and of b in its L2.
    const int tiles = tiles_m * tiles_n, per = tiles / 8, more = tiles % 8, xcd = blockIdx.x % 8;
    const int order = xcd * per + min(xcd, more) + blockIdx.x / 8;
    const int group = order / (8 * tiles_n), in_group = order % (8 * tiles_n), high = min(8, tiles_m - group * 8);
    const long long m0 = (long long)(group * 8 + in_group % high) * BM;
    const int n0 = in_group / high * BN;
    const int K = (int)p.k, blocks = (K + XL_SCALE_BLOCK - 1) / XL_SCALE_BLOCK;
    const int rows_a = (int)min((long long)BM, p.m - m0), rows_b = (int)min((long long)BN, p.n - n0);

    const int row = (K + 15) / 16 * 16;
    const __amdgpu_buffer_rsrc_t ra = buffer(p.a, m0 * p.a_row, (rows_a - 1) * p.a_row + row), rb = buffer(p.b, n0 * p.b_row, (rows_b - 1) * p.b_row + row);
    const __amdgpu_buffer_rsrc_t rs = buffer(p.a_scales, m0 * p.a_scale_row * 4, ((rows_a - 1) * p.a_scale_row + (blocks - 1) * p.a_scale_block + 1) * 4);
    // A wave's load brings 8 rows; rows past the end are the last one's, and their results are not kept.
    const int chunk = (lane % 8) ^ (lane / 8);
    // in a last block that K does not fill, chunks past the end are the last one's: `clear` removes them
    const unsigned last_chunk = (unsigned)min(chunk * 16, (K - 1 - (blocks - 1) * XL_SCALE_BLOCK) / 16 * 16);
    unsigned a_at[LA], b_at[LB];
#pragma unroll
    for (int i = 0; i < LA; ++i) a_at[i] = (unsigned)min((wave + i * WAVES) * 8 + lane / 8, rows_a - 1) * (unsigned)p.a_row;
#pragma unroll
    for (int i = 0; i < LB; ++i) b_at[i] = (unsigned)min((wave + i * WAVES) * 8 + lane / 8, rows_b - 1) * (unsigned)p.b_row;
    const unsigned s_at = (unsigned)min(wave % (BM / 64) * 64 + lane, rows_a - 1) * (unsigned)p.a_scale_row * 4;
    const int wm = wave % WM, wn = wave / WM;
    const float *sb = p.b_scales + ((n0 + min(wn * TN * 16, rows_b - 1)) / XL_SCALE_BLOCK) * p.b_scale_row;

    auto fetch = [&](Stage<BM, BN> &st, int kb) __attribute__((always_inline)) {
        const unsigned c = kb == blocks - 1 ? last_chunk : chunk * 16;
#pragma unroll
        for (int i = 0; i < LA; ++i) to_lds16(ra, st.a + (wave + i * WAVES) * 1024, a_at[i] + c, kb * XL_SCALE_BLOCK);
#pragma unroll
        for (int i = 0; i < LB; ++i) to_lds16(rb, st.b + (wave + i * WAVES) * 1024, b_at[i] + c, kb * XL_SCALE_BLOCK);
        to_lds4(rs, st.scale + wave % (BM / 64) * 64, s_at, kb * (unsigned)p.a_scale_block * 4);
    };
    auto clear = [&](Stage<BM, BN> &st) __attribute__((always_inline)) {       // numbers from K on become zeros
        const int live = K % XL_SCALE_BLOCK;
        for (int i = threadIdx.x; i < (BM + BN) * 8; i += 64 * WAVES) {
            char *at = st.a + i * 16;           // b follows a
            const int c = (i % 8) ^ (i / 8 % 8), bytes = live - c * 16;
            if (bytes >= 16) continue;
            u32x4 v = *reinterpret_cast<u32x4 *>(at);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int n = bytes - 4 * j;
                v[j] &= n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << (8 * n)) - 1;
            }
            *reinterpret_cast<u32x4 *>(at) = v;
        }
    };
    auto part = [&](const char *rows16, int quad_) __attribute__((always_inline)) {
        Part q;
        q.q[0] = *reinterpret_cast<const u32x4 *>(rows16 + col * 128 + ((quad_ ^ (col & 7)) * 16));
        q.q[1] = *reinterpret_cast<const u32x4 *>(rows16 + col * 128 + (((quad_ + 4) ^ (col & 7)) * 16));
        return q;
    };

    f32x4 acc[TM][TN] = {};
    // The operations of one row of tiles run while the results of the row before are scaled in.
    auto multiply = [&](const Stage<BM, BN> &st, float s_b) __attribute__((always_inline)) {
        typename P::Operand b[TN];
#pragma unroll
        for (int j = 0; j < TN; ++j) b[j] = P::operand(part(st.b + (wn * TN + j) * 2048, quad));
        f32x4 v[2][TN];
        float s = 0.f;
#pragma unroll
        for (int i = 0; i <= TM; ++i) {
            if (i < TM) {
                const typename P::Operand a = P::operand(part(st.a + (wm * TM + i) * 2048, quad));
#pragma unroll
                for (int j = 0; j < TN; ++j) v[i % 2][j] = P::run(b[j], a);
            }
            if (i > 0) {
#pragma unroll
                for (int j = 0; j < TN; ++j) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[i - 1][j][k] = __builtin_fmaf(s, v[(i - 1) % 2][j][k], acc[i - 1][j][k]);
                    asm volatile("" : "+v"(acc[i - 1][j]));     // here, and not put off until all of a block's results wait in registers
                }
            }
            if (i < TM) s = st.scale[(wm * TM + i) * 16 + col] * s_b;
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto arrived = [&]() __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };
    auto last_arrived = [&](Stage<BM, BN> &st) __attribute__((always_inline)) {
        arrived();
        if (K % XL_SCALE_BLOCK) {
            clear(st);
            __syncthreads();
        }
    };
    // The next block is on its way to `to` while the one in `from` is multiplied.  (Without the promise that the two are apart the compiler waits for the one before it
    // reads the other.)
    auto step = [&](Stage<BM, BN> *__restrict__ to, const Stage<BM, BN> *__restrict__ from, int kb, float s_b) __attribute__((always_inline)) {
        fetch(*to, kb);
        multiply(*from, s_b);
    };
    auto scale_b = [&](int kb) __attribute__((always_inline)) { return sb[min(kb, blocks - 1) * p.b_scale_block]; };

    if (blocks > 0) {
        float se = scale_b(0), so = scale_b(1);
        fetch(even, 0);
        int kb = 0;
        for (; kb + 2 < blocks; kb += 2) {
            arrived();
            step(&odd, &even, kb + 1, se);
            se = scale_b(kb + 2);
            arrived();
            step(&even, &odd, kb + 2, so);
            so = scale_b(kb + 3);
        }
        if (kb + 1 < blocks) {
            arrived();
            step(&odd, &even, kb + 1, se);
            last_arrived(odd);
            multiply(odd, so);
        } else {
            last_arrived(even);
            multiply(even, se);
        }
    }
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) store4<DT>(p, m0 + (wm * TM + i) * 16 + col, n0 + (wn * TN + j) * 16 + quad * 4, acc[i][j], wide);
}

template <int DT, int BM, int BN, int WM, int WN> static hipError_t launch_tile(const xl_block_matmul_args &a, bool wide, hipStream_t s)
{
    const long long tm = (a.m + BM - 1) / BM, tn = (a.n + BN - 1) / BN;
    tile_kernel<DT, BM, BN, WM, WN><<<dim3((unsigned)(tm * tn)), 64 * WM * WN, 0, s>>>(a, (int)tm, (int)tn, wide);
    return hipGetLastError();
}

template <int DT> static hipError_t launch_type(const xl_block_matmul_args &a, hipStream_t s)
{
    typedef typename Elem<DT>::T T;
    const bool wide = ((unsigned long long)a.y | (unsigned long long)a.y_row * sizeof(T)) % (4 * sizeof(T)) == 0;
    // a tile of the tile kernel lies within 31 bits, and so do its scales
    const long long limit = 1ll << 22, blocks = (a.k + XL_SCALE_BLOCK - 1) / XL_SCALE_BLOCK;
    if (a.m > 32 && a.a_row < limit && a.b_row < limit && a.a_scale_row < limit / 16 && a.a_scale_block < (1ll << 28) / (blocks + 1)) {
        if (DT != XL_F32 && a.m * a.n >= 256ll * 256 * 128) return launch_tile<DT, 256, 256, 2, 4>(a, wide, s);
        return launch_tile<DT, 128, 128, 2, 2>(a, wide, s);
    }
    const long long tiles_n = (a.n + 15) / 16, tiles = tiles_n * ((a.m + 15) / 16);
    thin_kernel<DT, 4><<<dim3((unsigned)tiles), 256, 0, s>>>(a, (int)tiles_n, wide);
    return hipGetLastError();
}

hipError_t launch_block_matmul(const xl_block_matmul_args &a, hipStream_t s)
{
    return a.dtype == XL_F32 ? launch_type<XL_F32>(a, s) : a.dtype == XL_F16 ? launch_type<XL_F16>(a, s) : launch_type<XL_BF16>(a, s);
}

}  // namespace xls
