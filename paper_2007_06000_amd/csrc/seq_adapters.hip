// Low-rank adapters of many sequences beside a shared product.
//
//   out[b,t] = y[b,t] + scales[e] * up[e] (down[e] x[b,t]),  e = index[b]
//
// Bound by memory: x and y are read and out is written once, the adapter's matrices come from the caches.  One kernel does both products, so that the numbers between them stay in LDS: a workgroup takes
// MT x 16 tokens of a sequence and a slice of out's columns.  Where the tiles of tokens alone do not fill the chip out is cut into slices, and each slice's workgroup makes down x again: reading x and
// down from the cache once more on a compute unit that would have had nothing to do costs less than a second launch.
#include "seq_parts.h"

namespace xls {

// The adapter of sequence b, or -1.
__device__ __forceinline__ long long adapter_of(const xl_adapters_args &a, int b)
{
    const int e = a.index[b];
    return e >= 0 && e < a.adapters ? e : -1;
}

// The rows of the first product are RT x 16 ranks, its columns tokens: a lane (token, quad) gets four ranks.  Its operands are read as runs of eight numbers a lane, eight lanes' runs
// of 64 numbers of a row behind each other: which of them meet in which operation does not matter, as long as both operands agree.
// The second product's rows are columns of out, its columns the same tokens.  Its four row tiles of a strip of 64 are dealt so that a lane's results are 16 neighbours of a row.
template <int DT, int MT, int RT, int W>
__global__ __launch_bounds__(64 * W) void adapters_kernel(const xl_adapters_args a, int tiles, int slices, int strips)
{
    typedef typename Elem<DT>::T T;
    typedef Vec<T, 8> T8;
    constexpr int NP = parts_of<DT>(), NT = DT == XL_F32 ? 3 : 2, R = RT * 16, RK = (RT + 1) / 2, PITCH = R + 4;
    __shared__ float part[W][MT * 16][PITCH];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), col = lane % 16, quad = lane / 16;
    const int K = (int)a.k, N = (int)a.n, rank = (int)a.rank, length = (int)a.length;
    const long long units = a.batch * tiles * slices;
    for (long long u = blockIdx.x; u < units; u += gridDim.x) {
        const int slice = (int)(u % slices), b = (int)(u / slices / tiles), t0 = (int)(u / slices % tiles) * (MT * 16);
        const int live = length_of(a.lengths, b, length);
        const long long e = adapter_of(a, b);
        Parts<NT> inner[MT][RK];
        if (e >= 0 && t0 < live) {
            const T *x = static_cast<const T *>(a.x) + b * a.x_batch, *down = static_cast<const T *>(a.down) + e * a.rank * a.k;
            const T *xrow[MT], *drow[RT];
#pragma unroll
            for (int m = 0; m < MT; ++m) xrow[m] = x + min(t0 + m * 16 + col, live - 1) * a.x_token;
#pragma unroll
            for (int r = 0; r < RT; ++r) drow[r] = down + (long long)min(r * 16 + col, rank - 1) * K;
            f32x4 acc[MT][RT] = {};
            const auto step = [&](auto load) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    Parts<NP> xs[MT];
#pragma unroll
                    for (int m = 0; m < MT; ++m) xs[m] = parts<DT>(load(xrow[m], half));
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        const Parts<NP> d = parts<DT>(load(drow[r], half));
#pragma unroll
                        for (int m = 0; m < MT; ++m) acc[m][r] = product(d, xs[m], acc[m][r]);
                    }
                }
            };
            int k = wave * 64;
            for (; k + 64 <= K; k += W * 64) step([&](const T *row, int half) { return load_vec<T, 8>(row + k + quad * 16 + half * 8); });
            if (k < K) step([&](const T *row, int half) { return load_some<T, 8>(row + k + quad * 16 + half * 8, K - (k + quad * 16 + half * 8)); });
            __syncthreads();        // the unit before has been read
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int r = 0; r < RT; ++r) *reinterpret_cast<f32x4 *>(&part[wave][m * 16 + col][r * 16 + quad * 4]) = acc[m][r];
            __syncthreads();
            const float scale = a.scales ? a.scales[e] : 1.f;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int r = 0; r < RK; ++r) {
                    const int at = r * 32 + quad * 8;
                    f32x8 s = {};
                    if (at < R)
#pragma unroll
                        for (int w = 0; w < W; ++w) {
                            const f32x4 *p = reinterpret_cast<const f32x4 *>(&part[w][m * 16 + col][at]);
                            s += __builtin_shufflevector(p[0], p[1], 0, 1, 2, 3, 4, 5, 6, 7);
                        }
#pragma unroll
                    for (int i = 0; i < 8; ++i) s[i] = at + i < rank ? s[i] * scale : 0.f;
                    inner[m][r] = split<NT>(s);
                }
        }
        const T *up = static_cast<const T *>(a.up) + (e >= 0 ? e : 0) * a.rank * a.n;
        for (int strip = slice * strips + wave; strip < min((slice + 1) * strips, (N + 63) / 64); strip += W) {
            const int j = strip * 64 + quad * 16;
            f32x4 acc[MT][4] = {};
            T8 y[MT][2];
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const int t = t0 + m * 16 + col;
                const T *row = static_cast<const T *>(a.y) + b * a.y_batch + t * a.y_token;
                y[m][0] = t < live ? load_some<T, 8>(row + j, N - j) : T8{};
                y[m][1] = t < live ? load_some<T, 8>(row + j + 8, N - j - 8) : T8{};
            }
            if (e >= 0 && t0 < live) {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    // row i of tile c is column 16 (i / 4) + 4 c + i % 4 of the strip
                    const T *row = up + (long long)min(strip * 64 + col / 4 * 16 + c * 4 + col % 4, N - 1) * rank;
#pragma unroll
                    for (int r = 0; r < RK; ++r) {
                        const Parts<NP> w = parts<DT>(load_some<T, 8>(row + r * 32 + quad * 8, rank - (r * 32 + quad * 8)));
#pragma unroll
                        for (int m = 0; m < MT; ++m) acc[m][c] = product(w, inner[m][r], acc[m][c]);
                    }
                }
            }
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const int t = t0 + m * 16 + col;
                if (t >= length) continue;
                T *row = static_cast<T *>(a.out) + b * a.out_batch + t * a.out_token;
                if (e >= 0 && t < live)
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i) y[m][c / 2][c % 2 * 4 + i] = (T)((float)y[m][c / 2][c % 2 * 4 + i] + acc[m][c][i]);
                store_some<T, 8>(row + j, N - j, y[m][0]);
                store_some<T, 8>(row + j + 8, N - j - 8, y[m][1]);
            }
        }
    }
}

template <int DT, int MT, int RT, int W> static hipError_t launch_tile(const xl_adapters_args &a, hipStream_t s)
{
    const long long tiles = (a.length + MT * 16 - 1) / (MT * 16), all = (a.n + 63) / 64, most = (all + W - 1) / W;
    long long slices = 512 / (a.batch * tiles);
    slices = slices < 1 ? 1 : slices > most ? most : slices;
    const long long strips = (all + slices - 1) / slices;
    slices = (all + strips - 1) / strips;
    const long long units = a.batch * tiles * slices;
    return launch_kernel(adapters_kernel<DT, MT, RT, W>, dim3((unsigned)(units < 1 << 20 ? units : 1 << 20)), 64 * W, s, a, (int)tiles, (int)slices, (int)strips);
}

template <int DT, int RT> static hipError_t launch_rank(const xl_adapters_args &a, hipStream_t s)
{
    return a.length <= 16 ? launch_tile<DT, 1, RT, 8>(a, s) : launch_tile<DT, RT == 8 ? 2 : 4, RT, 4>(a, s);
}

template <int DT> static hipError_t launch_type(const xl_adapters_args &a, hipStream_t s)
{
    return a.rank <= 16 ? launch_rank<DT, 1>(a, s) : a.rank <= 32 ? launch_rank<DT, 2>(a, s) : a.rank <= 64 ? launch_rank<DT, 4>(a, s) : launch_rank<DT, 8>(a, s);
}

long long adapters_workspace(const xl_adapters_args &) { return 0; }

hipError_t launch_add_adapters(const xl_adapters_args &a, hipStream_t s)
{
    return a.dtype == XL_F32 ? launch_type<XL_F32>(a, s) : a.dtype == XL_F16 ? launch_type<XL_F16>(a, s) : launch_type<XL_BF16>(a, s);
}

}  // namespace xls
