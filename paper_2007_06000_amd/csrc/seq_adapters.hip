// Low-rank adapters of many sequences beside a shared product.
//
//   out[b,t] = y[b,t] + scales[e] * up[e] (down[e] x[b,t]),  e = index[b]
//
// Bound by memory: x and y are read and out is written once, the adapter's matrices come from the caches.  Few tokens go through one kernel, where the numbers between the products stay in LDS: out
// is cut into slices until they fill the chip, and each slice's workgroup makes down x again, which costs less than a second launch.  More tokens take two kernels, so that both can be cut into as many parts
// as the chip wants: of k, and of out's columns.  (In one, 2 x 12321 tokens were 386 tiles of 64 for 256 compute units, the second round of them half empty: 176 us instead of 168 (170 with other inputs each time), of
// which the second kernel, y to out, is 98 at 4.1 TB/s.)  Up read as runs of memory and dealt through LDS measured 174 us, and 33 instead of 35 for 3136 tokens in one kernel.
#include "seq_parts.h"

namespace xls {

// The adapter of sequence b, or -1.
__device__ __forceinline__ long long adapter_of(const xl_adapters_args &a, int b)
{
    const int e = a.index[b];
    return e >= 0 && e < a.adapters ? e : -1;
}

// Which tokens a workgroup has: MT x 16 of sequence b from t0 on, of which the first `live` of the sequence count; and their adapter, or -1.
struct Tile {
    int b, t0, live;
    long long adapter;
    bool adapted;
    __device__ __forceinline__ Tile(const xl_adapters_args &a, long long at, int tiles, int tokens) : b((int)divided(at, tiles))
    {
        t0 = (int)(at - (long long)b * tiles) * tokens;
        live = length_of(a.lengths, b, (int)a.length);
        adapter = adapter_of(a, b);
        adapted = adapter >= 0 && t0 < live;
    }
};

// The rows of the first product are RT x 16 ranks, its columns tokens: a lane (token, quad) gets four ranks.  Waves take runs of 64 numbers of k in turn; their sums meet in LDS.
template <int DT, int MT, int RT, int W> struct First {
    typedef typename Elem<DT>::T T;
    typedef Vec<T, 8> T8;
    static constexpr int NP = parts_of<DT>(), PITCH = RT * 16 + 4;
    float part[W][MT * 16][PITCH];

    __device__ __forceinline__ void run(const xl_adapters_args &a, const Tile &tile, int begin, int end)
    {
        const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), col = lane % 16, quad = lane / 16, rank = (int)a.rank;
        const T *x = static_cast<const T *>(a.x) + tile.b * a.x_batch, *down = static_cast<const T *>(a.down) + tile.adapter * a.rank * a.k;
        const T *xrow[MT], *drow[RT];
#pragma unroll
        for (int m = 0; m < MT; ++m) xrow[m] = x + min(tile.t0 + m * 16 + col, tile.live - 1) * a.x_token;
#pragma unroll
        for (int r = 0; r < RT; ++r) drow[r] = down + min(r * 16 + col, rank - 1) * a.k;
        f32x4 acc[MT][RT] = {};
        // Each half of a run is asked for again as soon as it has been used: one half's products hide the other's loads.
        T8 xs[2][MT], ds[2][RT];
        const auto ask = [&](int k, int half) {
            const int at = k + half * 32 + quad * 8;
            if (k + 64 <= end) {
#pragma unroll
                for (int m = 0; m < MT; ++m) xs[half][m] = load_vec<T, 8>(xrow[m] + at);
#pragma unroll
                for (int r = 0; r < RT; ++r) ds[half][r] = load_vec<T, 8>(drow[r] + at);
            } else {
#pragma unroll
                for (int m = 0; m < MT; ++m) xs[half][m] = load_some<T, 8>(xrow[m] + at, end - at);
#pragma unroll
                for (int r = 0; r < RT; ++r) ds[half][r] = load_some<T, 8>(drow[r] + at, end - at);
            }
        };
        const int first = begin + wave * 64;
        if (first < end) {
            ask(first, 0);
            ask(first, 1);
        }
        for (int k = first; k < end; k += W * 64) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                Parts<NP> x[MT];
#pragma unroll
                for (int m = 0; m < MT; ++m) x[m] = parts<DT>(xs[half][m]);
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    const Parts<NP> d = parts<DT>(ds[half][r]);
#pragma unroll
                    for (int m = 0; m < MT; ++m) acc[m][r] = product(d, x[m], acc[m][r]);
                }
                __builtin_amdgcn_sched_barrier(0);
                if (k + W * 64 < end) ask(k + W * 64, half);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __syncthreads();        // what was there has been read
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int r = 0; r < RT; ++r) *reinterpret_cast<f32x4 *>(&part[wave][m * 16 + col][r * 16 + quad * 4]) = acc[m][r];
        __syncthreads();
    }
    __device__ __forceinline__ f32x4 sum(int token, int at) const
    {
        f32x4 s = {};
#pragma unroll
        for (int w = 0; w < W; ++w) s += *reinterpret_cast<const f32x4 *>(&part[w][token][at]);
        return s;
    }
};

// The second product's rows are columns of out, its columns the tokens.  Its four row tiles of a strip of 64 are dealt so that a lane's results are twice eight neighbours of a row, behind those of the quad before.
template <int DT, int MT, int RT, int W> struct Second {
    typedef typename Elem<DT>::T T;
    typedef Vec<T, 8> T8;
    static constexpr int NP = parts_of<DT>(), RK = (RT + 1) / 2;
    Parts<3> inner[MT][RK];

    // The sum over `parts` of of(part, token, rank): four neighbours of down x.  The numbers of a part are asked for together.
    template <typename F> __device__ __forceinline__ void take(const xl_adapters_args &a, const Tile &tile, int parts, F of)
    {
        const int lane = threadIdx.x % 64, col = lane % 16, quad = lane / 16;
        const float scale = a.scales ? a.scales[tile.adapter] : 1.f;
        f32x8 s[MT][RK] = {};
        for (int p = 0; p < parts; ++p)
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int r = 0; r < RK; ++r)
                    if (RT > 1 || quad < 2) s[m][r] += __builtin_shufflevector(of(p, m * 16 + col, r * 32 + quad * 8), of(p, m * 16 + col, r * 32 + quad * 8 + 4), 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int r = 0; r < RK; ++r) {
#pragma unroll
                for (int i = 0; i < 8; ++i) s[m][r][i] = r * 32 + quad * 8 + i < a.rank ? s[m][r][i] * scale : 0.f;
                inner[m][r] = split<3>(s[m][r]);
            }
    }

    // Strips begin to end.  `first` makes what `inner` is made of: their first numbers are on their way meanwhile.
    template <typename F> __device__ __forceinline__ void run(const xl_adapters_args &a, const Tile &tile, int begin, int end, F first)
    {
        const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), col = lane % 16, quad = lane / 16;
        const int N = (int)a.n, rank = (int)a.rank, length = (int)a.length, t0 = tile.t0, live = tile.live;
        const T *up = static_cast<const T *>(a.up) + (tile.adapted ? tile.adapter : 0) * a.rank * a.n;
        // Each strip is asked for while the one before is worked on.
        T8 ys[MT][2], us[4][RK];
        const auto inside = [&](int strip) { return (strip + 1) * 64 <= N; };
        const auto ask_y = [&](int strip) {
            const int j = strip * 64 + quad * 8;
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const T *row = static_cast<const T *>(a.y) + tile.b * a.y_batch + min(t0 + m * 16 + col, live - 1) * a.y_token + j;
                if (inside(strip)) {
                    ys[m][0] = load_vec<T, 8>(row);
                    ys[m][1] = load_vec<T, 8>(row + 32);
                } else {
                    ys[m][0] = load_some<T, 8>(row, N - j);
                    ys[m][1] = load_some<T, 8>(row + 32, N - j - 32);
                }
            }
        };
        const auto ask_up = [&](int strip) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                // row i of tiles 2 s and 2 s + 1 is column 32 s + 8 (i / 4) + i % 4 (+ 4 in the second) of the strip
                const T *row = up + (long long)min(strip * 64 + c / 2 * 32 + col / 4 * 8 + c % 2 * 4 + col % 4, N - 1) * rank;
                if (rank == RK * 32) {
#pragma unroll
                    for (int r = 0; r < RK; ++r) us[c][r] = load_vec<T, 8>(row + r * 32 + quad * 8);
                } else if (RT == 1 && rank == 16) {
                    us[c][0] = load_vec<T, 8>(row + quad % 2 * 8);      // the upper quads' numbers meet zeros ...
                    if (quad >= 2) us[c][0] = T8{};                     // ... and may not be infinite
                } else {
#pragma unroll
                    for (int r = 0; r < RK; ++r) us[c][r] = load_some<T, 8>(row + r * 32 + quad * 8, rank - (r * 32 + quad * 8));
                }
            }
        };
        int strip = begin + wave;
        if (strip < end && live > 0) {
            ask_y(strip);
            if (tile.adapted) ask_up(strip);
        }
        if (tile.adapted) first();
        for (; strip < end; strip += W) {
            const int j = strip * 64 + quad * 8, next = strip + W;
            f32x4 acc[MT][4] = {};
            if (tile.adapted) {
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int r = 0; r < RK; ++r) {
                        const Parts<NP> w = parts<DT>(us[c][r]);
#pragma unroll
                        for (int m = 0; m < MT; ++m) acc[m][c] = product(w, inner[m][r], acc[m][c]);
                    }
                __builtin_amdgcn_sched_barrier(0);
                if (next < end) ask_up(next);
                __builtin_amdgcn_sched_barrier(0);
            }
            T8 out[MT][2];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const T y = ys[m][c / 2][c % 2 * 4 + i];
                        out[m][c / 2][c % 2 * 4 + i] = t0 + m * 16 + col >= live ? (T)0.f : tile.adapted ? (T)((float)y + acc[m][c][i]) : y;
                    }
            if (next < end && live > 0) ask_y(next);        // of other columns: out may be y
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const int t = t0 + m * 16 + col;
                if (t >= length) continue;
                T *row = static_cast<T *>(a.out) + tile.b * a.out_batch + t * a.out_token + j;
                if (inside(strip)) {
                    store_vec<T, 8>(row, out[m][0]);
                    store_vec<T, 8>(row + 32, out[m][1]);
                } else {
                    store_some<T, 8>(row, N - j, out[m][0]);
                    store_some<T, 8>(row + 32, N - j - 32, out[m][1]);
                }
            }
        }
    }
};

// Few tokens: both products, for `strips` strips of out.
template <int DT, int RT, int W>
__global__ __launch_bounds__(64 * W) void both_kernel(const xl_adapters_args a, int tiles, int slices, int strips)
{
    __shared__ First<DT, 1, RT, W> first;
    for (long long u = blockIdx.x; u < a.batch * tiles * slices; u += gridDim.x) {
        const long long at = divided(u, slices);
        const Tile tile(a, at, tiles, 16);
        const int begin = (int)(u - at * slices) * strips;
        Second<DT, 1, RT, W> second;
        second.run(a, tile, begin, min(begin + strips, ((int)a.n + 63) / 64), [&] {
            first.run(a, tile, 0, (int)a.k);
            second.take(a, tile, 1, [&](int, int token, int at) { return first.sum(token, at); });
        });
    }
}

// More: the sums over `run` numbers of k of every token into the workspace [parts of k][token][rank], ...
template <int DT, int MT, int RT, int W>
__global__ __launch_bounds__(64 * W) void first_kernel(const xl_adapters_args a, int tiles, int parts, int run)
{
    __shared__ First<DT, MT, RT, W> first;
    const int length = (int)a.length;
    for (long long u = blockIdx.x; u < a.batch * tiles * parts; u += gridDim.x) {
        const long long at = divided(u, parts);
        const Tile tile(a, at, tiles, MT * 16);
        const int p = (int)(u - at * parts);
        if (!tile.adapted) continue;
        first.run(a, tile, p * run, min((p + 1) * run, (int)a.k));
        float *out = static_cast<float *>(a.workspace) + (p * a.batch * length + (long long)tile.b * length + tile.t0) * (RT * 16);
        for (int i = threadIdx.x; i < MT * 16 * RT * 4; i += 64 * W)
            if (tile.t0 + i / (RT * 4) < length) *reinterpret_cast<f32x4 *>(out + i * 4) = first.sum(i / (RT * 4), i % (RT * 4) * 4);
    }
}

// ... and the second product of what is there.
template <int DT, int MT, int RT, int W>
__global__ __launch_bounds__(64 * W) void second_kernel(const xl_adapters_args a, int tiles, int parts, int slices, int strips)
{
    const int length = (int)a.length;
    for (long long u = blockIdx.x; u < a.batch * tiles * slices; u += gridDim.x) {
        const long long at = divided(u, slices);
        const Tile tile(a, at, tiles, MT * 16);
        const int begin = (int)(u - at * slices) * strips;
        Second<DT, MT, RT, W> second;
        second.run(a, tile, begin, min(begin + strips, ((int)a.n + 63) / 64), [&] {
            second.take(a, tile, parts, [&](int p, int token, int at) {
                return *reinterpret_cast<const f32x4 *>(static_cast<const float *>(a.workspace) + (p * a.batch * length + (long long)tile.b * length + min(tile.t0 + token, tile.live - 1)) * (RT * 16) + at);
            });
        });
    }
}

static unsigned grid_of(long long units) { return (unsigned)(units < 1 << 20 ? units : 1 << 20); }
static long long up_to(long long most, long long v) { return v < 1 ? 1 : v > most ? most : v; }

// Tiles of 64 and 32 tokens, or of what the registers hold; k and out's columns in as many parts as give the chip some 1000 and 4000 workgroups, with two turns at least for each wave (four along out's columns in
// 16 bits: each workgroup begins with the sums of its tokens).
template <int DT, int RT> struct Many {
    static constexpr int W = 4, MT1 = DT == XL_F32 ? 1 : RT == 8 ? 2 : 4, MT2 = DT == XL_F32 || RT == 8 ? 1 : 2;
    long long tiles1, tiles2, parts, run, slices, strips;
    explicit Many(const xl_adapters_args &a)
    {
        tiles1 = (a.length + MT1 * 16 - 1) / (MT1 * 16);
        tiles2 = (a.length + MT2 * 16 - 1) / (MT2 * 16);
        const long long turn = W * 64, all = (a.n + 63) / 64;
        parts = up_to(up_to(16, a.k / (2 * turn)), 1024 / (a.batch * tiles1));
        run = (a.k + parts * turn - 1) / (parts * turn) * turn;
        parts = run > 0 ? (a.k + run - 1) / run : 0;
        slices = up_to(up_to(all, all / ((DT == XL_F32 ? 2 : 4) * W)), 4096 / (a.batch * tiles2));
        strips = (all + slices - 1) / slices;
        slices = (all + strips - 1) / strips;
    }
    static long long bytes(const xl_adapters_args &a) { return Many(a).parts * a.batch * a.length * RT * 16 * 4; }
    static hipError_t launch(const xl_adapters_args &a, hipStream_t s)
    {
        const Many m(a);
        if (m.parts > 0) {
            const hipError_t e = launch_kernel(first_kernel<DT, MT1, RT, W>, dim3(grid_of(a.batch * m.tiles1 * m.parts)), 64 * W, s, a, (int)m.tiles1, (int)m.parts, (int)m.run);
            if (e != hipSuccess) return e;
        }
        return launch_kernel(second_kernel<DT, MT2, RT, W>, dim3(grid_of(a.batch * m.tiles2 * m.slices)), 64 * W, s, a, (int)m.tiles2, (int)m.parts, (int)m.slices, (int)m.strips);
    }
};

// One kernel where tiles of 16 tokens do not fill the chip, and for sequences of no more: 5 x up to 729 tokens, 520 to 1000, rank 13 in fp32 take 13 us in one and 17 in two (the same inputs each time; with others 16 in one), 3136 tokens, 1024 to 4096, rank 64 in fp16
// 35 and 38.
static bool in_one(const xl_adapters_args &a) { return a.length <= 16 || a.batch * ((a.length + 15) / 16) <= 256; }

template <int DT, int RT> static hipError_t launch_rank(const xl_adapters_args &a, hipStream_t s)
{
    if (!in_one(a)) return Many<DT, RT>::launch(a, s);
    constexpr int W = DT == XL_F32 && RT >= 4 ? 4 : 8;         // fp32's registers
    const long long all = (a.n + 63) / 64, tiles = (a.length + 15) / 16;
    long long slices = up_to((all + W - 1) / W, 256 / (a.batch * tiles));
    const long long strips = (all + slices - 1) / slices;
    slices = (all + strips - 1) / strips;
    return launch_kernel(both_kernel<DT, RT, W>, dim3(grid_of(a.batch * tiles * slices)), 64 * W, s, a, (int)tiles, (int)slices, (int)strips);
}

template <int DT> static hipError_t launch_type(const xl_adapters_args &a, hipStream_t s)
{
    return a.rank <= 16 ? launch_rank<DT, 1>(a, s) : a.rank <= 32 ? launch_rank<DT, 2>(a, s) : a.rank <= 64 ? launch_rank<DT, 4>(a, s) : launch_rank<DT, 8>(a, s);
}

template <int DT> static long long workspace_of(const xl_adapters_args &a)
{
    return a.rank <= 16 ? Many<DT, 1>::bytes(a) : a.rank <= 32 ? Many<DT, 2>::bytes(a) : a.rank <= 64 ? Many<DT, 4>::bytes(a) : Many<DT, 8>::bytes(a);
}
long long adapters_workspace(const xl_adapters_args &a)
{
    return in_one(a) ? 0 : a.dtype == XL_F32 ? workspace_of<XL_F32>(a) : a.dtype == XL_F16 ? workspace_of<XL_F16>(a) : workspace_of<XL_BF16>(a);
}

hipError_t launch_add_adapters(const xl_adapters_args &a, hipStream_t s)
{
    return a.dtype == XL_F32 ? launch_type<XL_F32>(a, s) : a.dtype == XL_F16 ? launch_type<XL_F16>(a, s) : launch_type<XL_BF16>(a, s);
}

}  // namespace xls
