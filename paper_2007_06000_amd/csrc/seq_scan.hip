// Selective state-space scan.
//
//   h[n] <- exp(d A[n]) h[n] + d u B[n],   y = sum_n C[n] h[n] + D u,   y *= z sigmoid(z)
//
// exp(d A) is taken as 2^(d A log2 e), one hardware exponential.  Many tokens are bound by the issue of vector instructions: a state and token take an exponential, which takes two
// issue slots, and five others (four are the least: two runs), a channel and token some fifty more (softplus, gate, layouts), 10.7 slots for each of 16 states in all.  2 x 12321 x 2048
// with 16 states in bf16: 259 us, 3.1e12 states a second, the vector units issuing for 83 % of it (steps without softplus 274 us); its 404 MB alone would take 86 us.  Single tokens are bound
// by the states' bytes.
#include <algorithm>
#include <climits>
#include <initializer_list>

#include "seq_internal.h"

namespace xls {

// A sequence's rows of one tensor: element [t][i] lies t * step + i elements behind `base`.  Where rows do not overlap and a sequence lies within 2 GB a buffer covers exactly the
// tokens that the sequence has, so that one past its end reads as zeros and its store goes nowhere, without a comparison.
struct Rows {
    __amdgpu_buffer_rsrc_t rsrc;
    __device__ __forceinline__ Rows(const void *base, long long step, int rows, int width, int size)
    {
        const unsigned bytes = rows > 0 ? ((rows - 1) * (unsigned)step + width) * size : 0u;
        const unsigned long long p = (unsigned long long)base;
        const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)p), hi = __builtin_amdgcn_readfirstlane((unsigned)(p >> 32));
        rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)(((unsigned long long)hi << 32) | lo), (short)0, (int)__builtin_amdgcn_readfirstlane(bytes), 0x00020000);
    }
    // `tile`: where the tile's first row begins (inside the buffer), `at`: this thread's place behind it, both in bytes
    template <typename V> __device__ __forceinline__ V load(unsigned at, unsigned tile) const
    {
        if constexpr (sizeof(V) == 2) return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b16(rsrc, at, tile, 0));
        else if constexpr (sizeof(V) == 4) return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b32(rsrc, at, tile, 0));
        else if constexpr (sizeof(V) == 8) return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b64(rsrc, at, tile, 0));
        else return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, tile, 0));
    }
    template <typename V> __device__ __forceinline__ void store(unsigned at, unsigned tile, V v) const
    {
        if constexpr (sizeof(V) == 2) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, v), rsrc, at, tile, 0);
        else if constexpr (sizeof(V) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, v), rsrc, at, tile, 0);
        else if constexpr (sizeof(V) == 8) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, v), rsrc, at, tile, 0);
        else __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), rsrc, at, tile, 0);
    }
};
static constexpr unsigned NOWHERE = 0x80000000u;       // past the end of every such buffer

// How a lane reads its part of a tile: up to four numbers of a token at once, where rows are aligned and of whole vectors; one number of as many tokens; and
// the same with comparisons and 64-bit addresses, where there are no such buffers.
enum Access { VECTORS, SINGLES, SCATTERED };

// A token after the other: LP lanes a channel, four states (a 16-byte load) a lane, 256 / LP channels a workgroup.  One token of 64 sequences of 2048 channels and 16
// states: 5.9 us for 17.8 MB, of which a launch is 1.9; of 256 sequences 15 us for 71 MB (4.7 TB/s).
template <int DT, int LP>
__global__ __launch_bounds__(256) void step_kernel(const xl_scan_args a, int groups)
{
    typedef typename Elem<DT>::T T;
    constexpr int NS = 4;
    const int b = blockIdx.x / groups, c = (blockIdx.x % groups) * (256 / LP) + threadIdx.x / LP, part = threadIdx.x % LP, n0 = part * NS;
    const int D = (int)a.channels, N = (int)a.states, L = (int)a.length;
    const long long slot = slot_of(a.slots, a.nslots, b);
    const int len = slot < 0 ? 0 : length_of(a.lengths, b, L);
    const bool in = c < D;
    const int live = in ? N - n0 : 0;
    const long long at = (slot * D + c) * N + n0;
    const f32x4 A2 = load_some<float, NS>(a.A + (long long)c * N + n0, live) * LOG2E;
    f32x4 h = load_some<float, NS>(a.state + at, a.state && slot >= 0 ? live : 0);
    const float bias = in && a.delta_bias ? a.delta_bias[c] : 0.f, skip = in && a.D ? a.D[c] : 0.f;
    const T *up = static_cast<const T *>(a.u) + b * a.u_batch + c, *dp = static_cast<const T *>(a.delta) + b * a.delta_batch + c;
    const T *zp = static_cast<const T *>(a.z) + b * a.z_batch + c, *Bp = static_cast<const T *>(a.B) + b * a.b_batch + n0;
    const T *Cp = static_cast<const T *>(a.C) + b * a.c_batch + n0;
    T *yp = static_cast<T *>(a.y) + b * a.y_batch + c;
    // a token's numbers are read while the one before it is worked on, the first one's together with the states
    struct Token {
        T u, d, z;
        Vec<T, NS> B, C;
    };
    auto read = [&](int t) {
        Token k = {};
        if (in) {
            k.u = up[t * a.u_token];
            k.d = dp[t * a.delta_token];
            if (a.z) k.z = zp[t * a.z_token];
        }
        k.B = load_some<T, NS>(Bp + t * a.b_token, N - n0);
        k.C = load_some<T, NS>(Cp + t * a.c_token, N - n0);
        return k;
    };
    Token next = {};
    if (len > 0) next = read(0);
    for (int t = 0; t < len; ++t) {
        const Token k = next;
        if (t + 1 < len) next = read(t + 1);
        const float u = (float)k.u;
        float d = in ? (float)k.d + bias : 0.f;
        if (a.softplus) d = softplus(d);
        const float s = d * u;
        float y = 0.f;
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            h[i] = __builtin_fmaf(exp2_fast(d * A2[i]), h[i], s * (float)k.B[i]);
            y = __builtin_fmaf((float)k.C[i], h[i], y);
        }
#pragma unroll
        for (int o = 1; o < LP; o *= 2) y += __shfl_xor(y, o);
        if (part == 0 && in) {
            if (a.D) y = __builtin_fmaf(skip, u, y);
            if (a.z) y *= silu((float)k.z);
            yp[t * a.y_token] = (T)y;
        }
    }
    if (part == 0 && in)
        for (int t = len; t < L; ++t) yp[t * a.y_token] = (T)0.f;
    if (a.new_state && slot >= 0 && live > 0) store_some<float, NS>(a.new_state + at, live, h);
}

// Sum over the LP lanes of a channel, for LP tokens at once: lane i of the channel gets token i's.  At every step a lane keeps half of its tokens and hands the other
// half to its partner, so that a token costs 3 - 3 / LP operations, not log2(LP).
template <int CTRL> __device__ __forceinline__ float from_partner(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
template <int LP> __device__ __forceinline__ float sum_over_lanes(float *p, int part)
{
    if constexpr (LP == 16) {
        const bool up = part & 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = (up ? p[j + 8] : p[j]) + from_partner<0x128>(up ? p[j] : p[j + 8]);      // lane ^ 8
    }
    if constexpr (LP >= 8) {
        const bool up = part & 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) p[j] = (up ? p[j + 4] : p[j]) + from_partner<0x141>(up ? p[j] : p[j + 4]);      // 7 - lane
    }
    const bool up2 = part & 2, up1 = part & 1;
#pragma unroll
    for (int j = 0; j < 2; ++j) p[j] = (up2 ? p[j + 2] : p[j]) + from_partner<0x4e>(up2 ? p[j] : p[j + 2]);         // lane ^ 2
    return (up1 ? p[1] : p[0]) + from_partner<0xb1>(up1 ? p[0] : p[1]);                                             // lane ^ 1
}

// A run of tokens makes P h + E of a state h, with E what a state of zero becomes and P = 2^x, x the sum of its tokens' exponents.  P may lie outside fp32 where P h does not, and
// 0 x inf would be NaN.  So a P that underflows is the smallest number (an infinite state stays infinite), and one that overflows the largest (a state that is still zero stays zero).
// Steps that may be negative let states grow by any amount: there (ROOT) P is kept as its square root, between 2^-126 and 2^127, and applied twice, which is right up to a growth of
// 2^254, behind which every normal number is infinite; what shrinks by more than 2^-252 is below 1e-37.  With steps out of softplus states grow where A is positive, which is not what
// such models learn: there one that is not zero is followed up to a growth of 2^128 within a wave's 16 tokens.  (Roots for them too: 2 x 12321 x 2048 with 16 states 282 us, not 258; a
// test of the signs in front of the loop 266.)
template <bool ROOT> __device__ __forceinline__ float factor(float x)
{
    return ROOT ? exp2_fast(__builtin_amdgcn_fmed3f(0.5f * x, -126.f, 127.f)) : __builtin_amdgcn_fmed3f(exp2_fast(x), 0x1p-149f, 0x1.fffffep127f);
}
template <bool ROOT> __device__ __forceinline__ float past(float p, float h, float e) { return __builtin_fmaf(p, ROOT ? p * h : h, e); }

// Where there are not enough channels for the chip a sequence is worked on in `count` parts of `tokens` each.  For every part but the first there is what the one
// before it makes of a state, E and then, behind all E, the root of P, [batch][part][channel][state]; for the first the state that it begins with.
struct Parts {
    float *results;
    int count, tokens;
    __device__ __forceinline__ float *at(int b, int part, int c, int D, int N) const { return results + (((long long)b * count + part) * D + c) * N; }
    __device__ __forceinline__ long long factors(long long batch, int D, int N) const { return batch * count * D * N; }
};

// Many tokens.  A workgroup owns CH = 64 / LP channels of a sequence and goes through it in tiles of W x TK tokens, TK of them a wave: the recurrence is linear, so a
// wave runs its tokens from a state of zero (which gives E) and multiplies up their factors (P = exp(A sum d)); then the waves exchange (P, E), each
// takes the state that its last tokens ended with past those of the others in between, and runs its tokens again, the factors and inputs
// still in registers, now with the outputs.  The exchange is all that waves have to do with each other: what they read through LDS otherwise (steps, inputs, B, C, outputs of their own
// tokens, transposed there between a layout for memory and one for the recurrence) is theirs alone, so a tile has one barrier.
template <int DT, int LP, int NS, int W, int TK, Access ACCESS, bool ROOT>
__global__ __launch_bounds__(64 * W) void tile_kernel(const xl_scan_args a, int groups, const Parts parts)
{
    typedef typename Elem<DT>::T T;
    constexpr int CH = 64 / LP, NP = LP * NS, TT = W * TK, PT = TK + 4;
    constexpr int PER = CH * TK / 64, VE = ACCESS != VECTORS ? 1 : PER < 4 ? PER : 4, IT = PER / VE;    // a thread's part of a tile's u, delta, z and y
    constexpr int PERB = NP * TK / 64, VB = ACCESS != VECTORS ? 1 : PERB < 4 ? PERB : 4, IB = PERB / VB; // and of its B and C
    static_assert(PER >= 1 && PERB >= 1 && TK % LP == 0, "a wave's tokens divide among its lanes");
    constexpr int ACROSS = NP > 64 * VB ? NP / (64 * VB) : 1;   // a lane's items in a row of B and C, 64 VB apart: more than one where a row has more items than there are lanes
    __shared__ float dl_all[W][CH * PT], sx_all[W][CH * PT];    // steps, and step x input (later the outputs): [channel][token]
    __shared__ float Bs_all[W][TK * NP], Cs_all[W][TK * NP];    // [token][state]
    __shared__ Vec<float, NS> Ps[3][W * 64], Es[3][W * 64];

    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), c = lane / LP, part = lane % LP, n0 = part * NS;
    float *dl = dl_all[wave], *sx = sx_all[wave], *Bs = Bs_all[wave], *Cs = Cs_all[wave];
    const int block = neighbours_together(blockIdx.x, gridDim.x), b = block / groups, c0 = (block % groups) * CH;
    const int D = (int)a.channels, N = (int)a.states, L = (int)a.length;
    const long long slot = slot_of(a.slots, a.nslots, b);
    const int whole = slot < 0 ? 0 : length_of(a.lengths, b, L);
    const bool in = c0 + c < D;
    // this workgroup's tokens: from `first` to `len`, and up to `last` zeros
    const int first = blockIdx.y * parts.tokens, last = min(L - first, parts.tokens) + first, len = min(whole, last);

    float A2[NS], h[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        const bool live = in && n0 + i < N;
        A2[i] = live ? a.A[(long long)(c0 + c) * N + n0 + i] * LOG2E : 0.f;
        h[i] = live && a.state && slot >= 0 && parts.count == 1 ? a.state[(slot * D + c0 + c) * N + n0 + i] : 0.f;
    }
    if (parts.count > 1 && (first < len || first == 0)) {       // what part 0 begins with, or part 0's end and the parts behind it
        const float *E = parts.at(b, first ? 1 : 0, c0 + c, D, N) + n0, *P = E + parts.factors(a.batch, D, N);
        const long long step = (long long)D * N;
        const int live = in ? N - n0 : 0;
        Vec<float, NS> v = load_some<float, NS>(E, live);
        for (int k = 2; k <= (int)blockIdx.y; ++k) {
            E += step;
            P += step;
            const Vec<float, NS> p = load_some<float, NS>(P, live), e = load_some<float, NS>(E, live);
#pragma unroll
            for (int i = 0; i < NS; ++i) v[i] = past<true>(p[i], v[i], e[i]);
        }
#pragma unroll
        for (int i = 0; i < NS; ++i) h[i] = v[i];
    }
    // this lane's numbers of its wave's tokens: VE channels of IT tokens
    const int ec = lane % (CH / VE) * VE, et = lane / (CH / VE), nc = min(D - c0 - ec, VE), tw = wave * TK;
    const int bn = lane % (NP / VB) * VB, bt = lane / (NP / VB), nb = N - bn;
    constexpr int ET = 64 * VE / CH, BT = 64 * VB * ACROSS / NP;        // tokens between a lane's items (its rows of items)
    static_assert(BT >= 1 && BT * (IB / ACROSS) == TK, "the items cover the tile");
    float bias[VE], skip[VE];
#pragma unroll
    for (int i = 0; i < VE; ++i) {
        bias[i] = a.delta_bias && i < nc ? a.delta_bias[c0 + ec + i] : 0.f;
        skip[i] = a.D && i < nc ? a.D[c0 + ec + i] : 0.f;
    }
    // the workgroup's first token of each tensor, and this lane's place in a tile
    const T *up = static_cast<const T *>(a.u) + b * a.u_batch + c0, *dp = static_cast<const T *>(a.delta) + b * a.delta_batch + c0;
    const T *zp = static_cast<const T *>(a.z) + b * a.z_batch + c0, *Bp = static_cast<const T *>(a.B) + b * a.b_batch, *Cp = static_cast<const T *>(a.C) + b * a.c_batch;
    T *yp = static_cast<T *>(a.y) + b * a.y_batch + c0;
    constexpr unsigned S = sizeof(T);
    const unsigned u_at = nc > 0 ? ((tw + et) * (unsigned)a.u_token + ec) * S : NOWHERE, d_at = nc > 0 ? ((tw + et) * (unsigned)a.delta_token + ec) * S : NOWHERE, z_at = nc > 0 ? ((tw + et) * (unsigned)a.z_token + ec) * S : NOWHERE;
    const unsigned y_at = nc > 0 ? ((tw + et) * (unsigned)a.y_token + ec) * S : NOWHERE, b_at = nb > 0 ? ((tw + bt) * (unsigned)a.b_token + bn) * S : NOWHERE, c_at = nb > 0 ? ((tw + bt) * (unsigned)a.c_token + bn) * S : NOWHERE;

    const int tokens = ACCESS != SCATTERED ? len : 0;
    const int width = min(CH, D - c0);
    const Rows urows(up, a.u_token, tokens, width, S), drows(dp, a.delta_token, tokens, width, S), zrows(zp, a.z_token, a.z ? tokens : 0, width, S);
    const Rows yrows(yp, a.y_token, tokens, width, S), Brows(Bp, a.b_token, tokens, N, S), Crows(Cp, a.c_token, tokens, N, S);
    const unsigned u_row = (unsigned)a.u_token * S, d_row = (unsigned)a.delta_token * S, z_row = a.z ? (unsigned)a.z_token * S : 0, y_row = (unsigned)a.y_token * S;
    const unsigned b_row = (unsigned)a.b_token * S, c_row = (unsigned)a.c_token * S;

    Vec<T, VE> ur[IT], dr[IT], zr[IT];
    Vec<T, VB> Br[IB], Cr[IB];
    auto fetch = [&](int t0) {
        if constexpr (ACCESS != SCATTERED) {
#pragma unroll
            for (int k = 0; k < IT; ++k) {
                ur[k] = urows.template load<Vec<T, VE>>(u_at + k * ET * u_row, t0 * u_row);
                dr[k] = drows.template load<Vec<T, VE>>(d_at + k * ET * d_row, t0 * d_row);
                zr[k] = zrows.template load<Vec<T, VE>>(z_at + k * ET * z_row, t0 * z_row);
            }
#pragma unroll
            for (int k = 0; k < IB; ++k) {
                const unsigned side = k % ACROSS * 64 * VB * S;      // past the end of the row: nowhere
                Br[k] = Brows.template load<Vec<T, VB>>(side && k % ACROSS * 64 * VB >= nb ? NOWHERE : b_at + k / ACROSS * BT * b_row + side, t0 * b_row);
                Cr[k] = Crows.template load<Vec<T, VB>>(side && k % ACROSS * 64 * VB >= nb ? NOWHERE : c_at + k / ACROSS * BT * c_row + side, t0 * c_row);
            }
        } else {
#pragma unroll
            for (int k = 0; k < IT; ++k) {
                const long long t = t0 + tw + et + k * ET;
                const int n = t < len ? nc : 0;
                ur[k] = load_some<T, VE>(up + t * a.u_token + ec, n);
                dr[k] = load_some<T, VE>(dp + t * a.delta_token + ec, n);
                zr[k] = load_some<T, VE>(zp + t * a.z_token + ec, a.z ? n : 0);
            }
#pragma unroll
            for (int k = 0; k < IB; ++k) {
                const long long t = t0 + tw + bt + k / ACROSS * BT;
                const int side = k % ACROSS * 64 * VB, n = t < len ? nb - side : 0;
                Br[k] = load_some<T, VB>(Bp + t * a.b_token + bn + side, n);
                Cr[k] = load_some<T, VB>(Cp + t * a.c_token + bn + side, n);
            }
        }
    };

    if (first < len) fetch(first);
    Ps[2][threadIdx.x] = Vec<float, NS>{} + 1.f;        // before the first tile: nothing
    Es[2][threadIdx.x] = Vec<float, NS>{};
    int before = 2, set = 0;
    for (int t0 = first; t0 < len; t0 += TT) {
        Vec<T, VE> uc[IT], zc[IT];
#pragma unroll
        for (int k = 0; k < IT; ++k) {
            const int t = et + k * ET;
            uc[k] = ur[k];
            zc[k] = zr[k];
            float d[VE];
#pragma unroll
            for (int i = 0; i < VE; ++i) d[i] = (float)dr[k][i] + bias[i];
            if (a.softplus) {
#pragma unroll
                for (int i = 0; i < VE; ++i) d[i] = softplus(d[i]);
            }
            if (t0 + TT > len) {
                asm volatile("");       // a branch: only the last tile has such tokens
#pragma unroll
                for (int i = 0; i < VE; ++i) d[i] = t0 + tw + t < len ? d[i] : 0.f;      // a token past the end changes nothing
            }
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                dl[(ec + i) * PT + t] = d[i];
                sx[(ec + i) * PT + t] = d[i] * (float)ur[k][i];
            }
        }
#pragma unroll
        for (int k = 0; k < IB; ++k) {
            Vec<float, VB> vb, vc;
#pragma unroll
            for (int i = 0; i < VB; ++i) {
                vb[i] = (float)Br[k][i];
                vc[i] = (float)Cr[k][i];
            }
            *reinterpret_cast<Vec<float, VB> *>(&Bs[(bt + k / ACROSS * BT) * NP + bn + k % ACROSS * 64 * VB]) = vb;
            *reinterpret_cast<Vec<float, VB> *>(&Cs[(bt + k / ACROSS * BT) * NP + bn + k % ACROSS * 64 * VB]) = vc;
        }
        if (t0 + TT < len) fetch(t0 + TT);                      // the next tile's numbers come in the meantime
        wave_sync();

        // the wave's tokens from a state of zero
        constexpr bool KEEP = TK * NS <= 64;     // the inputs too; with eight states a lane there is no room, and they are computed twice
        float av[TK][NS], bv[KEEP ? TK : 1][NS], sum = 0.f;
        Vec<float, NS> e = {}, p;
#pragma unroll
        for (int k = 0; k < TK; k += 4) {
            const f32x4 d = *reinterpret_cast<const f32x4 *>(&dl[c * PT + k]), s = *reinterpret_cast<const f32x4 *>(&sx[c * PT + k]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const Vec<float, NS> B = *reinterpret_cast<const Vec<float, NS> *>(&Bs[(k + j) * NP + n0]);
                sum += d[j];
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    av[k + j][i] = exp2_fast(d[j] * A2[i]);
                    const float put = s[j] * B[i];
                    if (KEEP) bv[KEEP ? k + j : 0][i] = put;
                    e[i] = __builtin_fmaf(av[k + j][i], e[i], put);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < NS; ++i) p[i] = factor<ROOT>(sum * A2[i]);
        // Three sets in turn: a wave that writes one again has passed the second barrier behind it, and every reader of it the first.
        Ps[set][threadIdx.x] = p;
        Es[set][threadIdx.x] = e;
        __syncthreads();
        // from where this wave's tokens of the tile before ended, past the other waves': those behind it there, those before it here
#pragma unroll
        for (int j = 1; j < W; ++j) {
            const int from = wave + j < W ? before * W + wave + j : set * W + wave + j - W;
            const Vec<float, NS> pw = Ps[0][from * 64 + lane], ew = Es[0][from * 64 + lane];
#pragma unroll
            for (int i = 0; i < NS; ++i) h[i] = past<ROOT>(pw[i], h[i], ew[i]);
        }
        // and again from the state that they find
#pragma unroll
        for (int k = 0; k < TK; k += LP) {
            float y[LP], s[LP];
            if (!KEEP) {
#pragma unroll
                for (int j = 0; j < LP; ++j) s[j] = sx[c * PT + k + j];
            }
#pragma unroll
            for (int j = 0; j < LP; ++j) {
                const Vec<float, NS> C = *reinterpret_cast<const Vec<float, NS> *>(&Cs[(k + j) * NP + n0]);
                const Vec<float, NS> B = KEEP ? Vec<float, NS>{} : *reinterpret_cast<const Vec<float, NS> *>(&Bs[(k + j) * NP + n0]);
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    h[i] = __builtin_fmaf(av[k + j][i], h[i], KEEP ? bv[KEEP ? k + j : 0][i] : s[j] * B[i]);
                    y[j] = i ? __builtin_fmaf(C[i], h[i], y[j]) : C[i] * h[i];
                }
            }
            sx[c * PT + k + part] = sum_over_lanes<LP>(y, part);
        }
        before = set;
        set = set == 2 ? 0 : set + 1;
        wave_sync();
#pragma unroll
        for (int k = 0; k < IT; ++k) {
            const int t = et + k * ET;
            float out[VE];
#pragma unroll
            for (int i = 0; i < VE; ++i) out[i] = __builtin_fmaf(skip[i], (float)uc[k][i], sx[(ec + i) * PT + t]);
            if (a.z) {
#pragma unroll
                for (int i = 0; i < VE; ++i) out[i] *= silu((float)zc[k][i]);
            }
            Vec<T, VE> v;
#pragma unroll
            for (int i = 0; i < VE; ++i) v[i] = (T)out[i];
            if constexpr (ACCESS != SCATTERED) yrows.store(y_at + k * ET * y_row, t0 * y_row, v);
            else if (t0 + tw + t < len) store_some<T, VE>(yp + (t0 + tw + t) * a.y_token + ec, nc, v);
        }
    }
    for (int t = max(len, first) + wave * ET + et; t < last; t += W * ET) {
#pragma unroll
        for (int i = 0; i < VE; ++i)
            if (i < nc) yp[t * a.y_token + ec + i] = (T)0.f;
    }
    if (wave == 0 && a.new_state && slot >= 0 && (first < len || first == 0) && len == whole) {     // the sequence ends here
        if (first < len) {
#pragma unroll
            for (int w = 1; w < W; ++w) {
                const Vec<float, NS> pw = Ps[before][w * 64 + lane], ew = Es[before][w * 64 + lane];
#pragma unroll
                for (int i = 0; i < NS; ++i) h[i] = past<ROOT>(pw[i], h[i], ew[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < NS; ++i)
            if (in && n0 + i < N) a.new_state[(slot * D + c0 + c) * N + n0 + i] = h[i];
    }
}

// The first of two kernels where a sequence is worked on in parts: what each part but the last makes of a state, h -> P h + E; part 0 of the state it begins with.
// A wave goes through its share of the part by itself, as above but for the outputs; the waves' results are joined at the end.
template <int DT, int LP, int NS, int W, int TK, Access ACCESS>
__global__ __launch_bounds__(64 * W) void part_kernel(const xl_scan_args a, int groups, const Parts parts)
{
    typedef typename Elem<DT>::T T;
    constexpr int CH = 64 / LP, NP = LP * NS, PT = TK + 4;
    constexpr int PER = CH * TK / 64, VE = ACCESS != VECTORS ? 1 : PER < 4 ? PER : 4, IT = PER / VE;
    constexpr int PERB = NP * TK / 64, VB = ACCESS != VECTORS ? 1 : PERB < 4 ? PERB : 4, IB = PERB / VB;
    static_assert(NP <= 64 * VB, "a row of B has no more items than there are lanes");
    __shared__ float dl_all[W][CH * PT], sx_all[W][CH * PT], Bs_all[W][TK * NP];
    __shared__ Vec<float, NS> Es[W * 64];
    __shared__ float totals[W * 64];

    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), c = lane / LP, part = lane % LP, n0 = part * NS;
    float *dl = dl_all[wave], *sx = sx_all[wave], *Bs = Bs_all[wave];
    const int block = neighbours_together(blockIdx.x, gridDim.x), b = block / groups, c0 = (block % groups) * CH;
    const int D = (int)a.channels, N = (int)a.states, L = (int)a.length;
    const long long slot = slot_of(a.slots, a.nslots, b);
    const int len = slot < 0 ? 0 : length_of(a.lengths, b, L), first = blockIdx.y * parts.tokens;
    const bool in = c0 + c < D;
    const int live = in ? N - n0 : 0;
    float *out = parts.at(b, blockIdx.y, c0 + c, D, N) + n0;
    const long long step = (long long)D * N;
    Vec<float, NS> begin = {};
    if (first == 0) {
        if (a.state && slot >= 0) begin = load_some<float, NS>(a.state + (slot * D + c0 + c) * N + n0, live);
        if (wave == 0 && live > 0) store_some<float, NS>(out, live, begin);
    }
    if (len <= first + parts.tokens) return;        // all of the workgroup: no part behind this one

    float A2[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) A2[i] = i < live ? a.A[(long long)(c0 + c) * N + n0 + i] * LOG2E : 0.f;
    const int ec = lane % (CH / VE) * VE, et = lane / (CH / VE), nc = min(D - c0 - ec, VE);
    const int bn = lane % (NP / VB) * VB, bt = lane / (NP / VB), nb = min(N - bn, VB);
    constexpr int ET = 64 * VE / CH, BT = 64 * VB / NP;
    float bias[VE];
#pragma unroll
    for (int i = 0; i < VE; ++i) bias[i] = a.delta_bias && i < nc ? a.delta_bias[c0 + ec + i] : 0.f;
    constexpr unsigned S = sizeof(T);
    const unsigned u_row = (unsigned)a.u_token * S, d_row = (unsigned)a.delta_token * S, b_row = (unsigned)a.b_token * S;
    const unsigned u_at = nc > 0 ? et * u_row + ec * S : NOWHERE, d_at = nc > 0 ? et * d_row + ec * S : NOWHERE, b_at = nb > 0 ? bt * b_row + bn * S : NOWHERE;
    const int width = min(CH, D - c0);
    const Rows urows(static_cast<const T *>(a.u) + b * a.u_batch + c0, a.u_token, len, width, S), drows(static_cast<const T *>(a.delta) + b * a.delta_batch + c0, a.delta_token, len, width, S);
    const Rows Brows(static_cast<const T *>(a.B) + b * a.b_batch, a.b_token, len, N, S);
    Vec<T, VE> ur[IT], dr[IT];
    Vec<T, VB> Br[IB];
    auto fetch = [&](int t0) {
#pragma unroll
        for (int k = 0; k < IT; ++k) {
            ur[k] = urows.template load<Vec<T, VE>>(u_at + k * ET * u_row, t0 * u_row);
            dr[k] = drows.template load<Vec<T, VE>>(d_at + k * ET * d_row, t0 * d_row);
        }
#pragma unroll
        for (int k = 0; k < IB; ++k) Br[k] = Brows.template load<Vec<T, VB>>(b_at + k * BT * b_row, t0 * b_row);
    };
    const int share = parts.tokens / W, t1 = first + wave * share, end = t1 + share;
    Vec<float, NS> e = {}, p;
    float total = 0.f;
    fetch(t1);
    for (int t0 = t1; t0 < end; t0 += TK) {
#pragma unroll
        for (int k = 0; k < IT; ++k) {
            float d[VE];
#pragma unroll
            for (int i = 0; i < VE; ++i) d[i] = (float)dr[k][i] + bias[i];
            if (a.softplus) {
#pragma unroll
                for (int i = 0; i < VE; ++i) d[i] = softplus(d[i]);
            }
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                dl[(ec + i) * PT + et + k * ET] = d[i];
                sx[(ec + i) * PT + et + k * ET] = d[i] * (float)ur[k][i];
            }
        }
#pragma unroll
        for (int k = 0; k < IB; ++k) {
            Vec<float, VB> v;
#pragma unroll
            for (int i = 0; i < VB; ++i) v[i] = (float)Br[k][i];
            *reinterpret_cast<Vec<float, VB> *>(&Bs[(bt + k * BT) * NP + bn]) = v;
        }
        if (t0 + TK < end) fetch(t0 + TK);
        wave_sync();
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < TK; k += 4) {
            const f32x4 d = *reinterpret_cast<const f32x4 *>(&dl[c * PT + k]), s = *reinterpret_cast<const f32x4 *>(&sx[c * PT + k]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const Vec<float, NS> B = *reinterpret_cast<const Vec<float, NS> *>(&Bs[(k + j) * NP + n0]);
                sum += d[j];
#pragma unroll
                for (int i = 0; i < NS; ++i) e[i] = __builtin_fmaf(exp2_fast(d[j] * A2[i]), e[i], s[j] * B[i]);
            }
        }
        total += sum;
        wave_sync();
    }
    totals[threadIdx.x] = total;
    Es[threadIdx.x] = e;
    __syncthreads();
    if (wave != 0 || live <= 0) return;
    e = begin;
    total = 0.f;
    for (int w = 0; w < W; ++w) {
        const float t = totals[w * 64 + lane];
        const Vec<float, NS> ew = Es[w * 64 + lane];
#pragma unroll
        for (int i = 0; i < NS; ++i) e[i] = past<true>(factor<true>(t * A2[i]), e[i], ew[i]);
        total += t;
    }
#pragma unroll
    for (int i = 0; i < NS; ++i) p[i] = factor<true>(total * A2[i]);
    store_some<float, NS>(out + step, live, e);
    store_some<float, NS>(out + step + parts.factors(a.batch, D, N), live, p);
}

static xl_scan_args piece_of(const xl_scan_args &a, long long first, long long count)
{
    const int size = a.dtype == XL_F32 ? 4 : 2;
    xl_scan_args p = piece_of_states(a, first, count, a.channels * a.states, 4);
    p.u = behind(a.u, first * a.u_batch, size);
    p.delta = behind(a.delta, first * a.delta_batch, size);
    p.B = behind(a.B, first * a.b_batch, size);
    p.C = behind(a.C, first * a.c_batch, size);
    p.z = behind(a.z, first * a.z_batch, size);
    p.y = behind(a.y, first * a.y_batch, size);
    return p;
}

template <int DT, int LP> static hipError_t launch_step(const xl_scan_args &a, hipStream_t s)
{
    const int per = 256 / LP, groups = (int)((a.channels + per - 1) / per);
    return in_pieces(a, groups * 256ll, piece_of, [&](const xl_scan_args &p) { return launch_kernel(step_kernel<DT, LP>, dim3((unsigned)(groups * p.batch)), 256, s, p, groups); });
}

template <int DT, int LP, int NS, int W, int TK, bool SPLIT, bool ROOT> static hipError_t launch_tile_as(const xl_scan_args &a, hipStream_t s, const Parts &parts)
{
    typedef typename Elem<DT>::T T;
    constexpr int CH = 64 / LP, PER = CH * TK / 64, VE = PER < 4 ? PER : 4, PERB = LP * NS * TK / 64, VB = PERB < 4 ? PERB : 4;
    const int groups = (int)((a.channels + CH - 1) / CH);
    const unsigned long long at = (unsigned long long)a.u | (unsigned long long)a.delta | (unsigned long long)a.z | (unsigned long long)a.y;
    const unsigned long long steps = a.u_batch | a.u_token | a.delta_batch | a.delta_token | a.z_batch | a.z_token | a.y_batch | a.y_token;
    const unsigned long long at_bc = (unsigned long long)a.B | (unsigned long long)a.C, steps_bc = a.b_batch | a.b_token | a.c_batch | a.c_token;
    const bool vectors = (at | steps * sizeof(T)) % (VE * sizeof(T)) == 0 && a.channels % VE == 0 && (at_bc | steps_bc * sizeof(T)) % (VB * sizeof(T)) == 0 && a.states % VB == 0;
    // a sequence's rows in one buffer: not overlapping (what follows the last token stays outside), offsets within 31 bits also a tile past the end
    auto rows = [&](long long width, std::initializer_list<long long> tokens) {
        for (long long t : tokens)
            if (t < width || t > INT_MAX / (long long)sizeof(T) / (a.length + 2 * W * TK)) return false;
        return true;
    };
    const bool buffers = rows(a.channels, {a.u_token, a.delta_token, a.y_token}) && (!a.z || rows(a.channels, {a.z_token})) && rows(a.states, {a.b_token, a.c_token});
    // 2 x 12321 x 2048 with 16 states in bf16: 258 us as vectors, 303 one by one, 560 scattered (these with four waves in every case)
    const Parts whole = {nullptr, 1, INT_MAX};
    if (!buffers)
        return in_pieces(a, groups * 64 * 4ll, piece_of, [&](const xl_scan_args &p) { return launch_kernel(tile_kernel<DT, LP, NS, 4, TK, SCATTERED, ROOT>, dim3((unsigned)(groups * p.batch)), 64 * 4, s, p, groups, whole); });
    const auto tiles = vectors ? tile_kernel<DT, LP, NS, W, TK, VECTORS, ROOT> : tile_kernel<DT, LP, NS, W, TK, SINGLES, ROOT>;
    if constexpr (SPLIT) {          // few workgroups
        const unsigned wide = (unsigned)(groups * a.batch);
        const dim3 grid(wide, (unsigned)parts.count - 1);
        const hipError_t e = launch_kernel(vectors ? part_kernel<DT, LP, NS, W, TK, VECTORS> : part_kernel<DT, LP, NS, W, TK, SINGLES>, grid, 64 * W, s, a, groups, parts);
        return e != hipSuccess ? e : launch_kernel(tiles, dim3(wide, (unsigned)parts.count), 64 * W, s, a, groups, parts);
    } else {
        return in_pieces(a, groups * 64ll * W, piece_of, [&](const xl_scan_args &p) { return launch_kernel(tiles, dim3((unsigned)(groups * p.batch)), 64 * W, s, p, groups, whole); });
    }
}

template <int DT, int LP, int NS, int W, int TK, bool SPLIT = false> static hipError_t launch_tile(const xl_scan_args &a, hipStream_t s, const Parts &parts = {nullptr, 1, INT_MAX})
{
    return a.softplus ? launch_tile_as<DT, LP, NS, W, TK, SPLIT, false>(a, s, parts) : launch_tile_as<DT, LP, NS, W, TK, SPLIT, true>(a, s, parts);
}

static constexpr long long CUS = 256;

// Workgroups of 64 / LP channels each.
static long long groups_of(const xl_scan_args &a, int lp) { return a.batch * ((a.channels * lp + 63) / 64); }

// Lanes of a channel that leave each four states (fewer where there are no more).
static int lanes_of(const xl_scan_args &a) { return a.states <= 16 ? 4 : a.states <= 32 ? 8 : 16; }

// Parts of a sequence: as many as it takes to give every compute unit a workgroup of eight waves, of at least 256 tokens, and whole tiles.  A second kernel and
// the tokens' first run twice cost what eight parts bring (1 sequence, 16 states, us whole and in parts: 2048 tokens x 256 channels 20, 16; 12321 x 256 107,
// 41; 12321 x 512 108, 64; 4096 x 1024, four parts, 39, 42), or four with up to eight states, which spread over fewer workgroups when whole
// (3025 x 1001, 3 states 50, 23; 7 states 38, 29).
static constexpr long long TILE = 128, MIN_PART = 256, MAX_PARTS = 32;
static Parts parts_of(const xl_scan_args &a)
{
    const long long groups = groups_of(a, lanes_of(a)), most = groups > 0 ? std::min({CUS / groups, a.length / MIN_PART, MAX_PARTS}) : 0;
    if (most < (a.states <= 8 ? 4 : 8) || a.states > 64 || a.length < 1536) return {nullptr, 1, INT_MAX};
    const long long tokens = (a.length + most * TILE - 1) / (most * TILE) * TILE;
    return {static_cast<float *>(a.workspace), (int)((a.length + tokens - 1) / tokens), (int)tokens};
}
long long scan_workspace(const xl_scan_args &a)
{
    const Parts p = parts_of(a);
    return p.count > 1 ? (2ll * p.count * a.batch * a.channels * a.states * 4 + 15) / 16 * 16 : 0;
}

// Waves of a workgroup.  One that has a compute unit to itself (its registers leave room for two waves a SIMD) takes eight, four where two fit, and where there are four and more
// to overlap two, or four if they stay long (us with 2, 4, 8 waves: 16 states, 3025 tokens, 256 workgroups 183, 96, 70, 512 workgroups 243, 134, 140; with 2, 4: 2048
// workgroups of 3025 tokens 536, 488, 4096 of 200 164, 190, 4096 of 50 114, 153; 64 states, whose registers are short with four, 904, 974).
template <int DT, int LP, int NS> static hipError_t launch_waves(const xl_scan_args &a, hipStream_t s)
{
    const long long groups = groups_of(a, LP);
    if (groups <= CUS && a.length > 64) return launch_tile<DT, LP, NS, 8, 16>(a, s);
    if (a.length > (groups < 4 * CUS ? 32 : LP < 16 ? 512 : INT_MAX)) return launch_tile<DT, LP, NS, 4, 16>(a, s);
    return launch_tile<DT, LP, NS, 2, 16>(a, s);
}

// The same where channels are spread over more lanes, so that workgroups have a compute unit each: as many waves as there are tokens for, MOST at most (1024
// channels, 16 states, us with 4, 8, 16 waves: 64 tokens 3.4, 4.0, 5.8; 128 tokens 4.4, 4.0, 5.8; 400 tokens 9.1, 7.6, 7.9; 3136 tokens -, 34.7, 32.3).
template <int DT, int LP, int NS, int MOST> static hipError_t launch_spread(const xl_scan_args &a, hipStream_t s)
{
    if (a.length <= 64) return launch_tile<DT, LP, NS, 4, 16>(a, s);
    if (MOST == 8 || a.length <= 512) return launch_tile<DT, LP, NS, 8, 16>(a, s);
    return launch_tile<DT, LP, NS, MOST, 16>(a, s);
}

template <int DT> static hipError_t launch_type(const xl_scan_args &a, hipStream_t s)
{
    // A token after the other costs 0.45 us and more each behind the launch, a tile the same for up to 32 (2048 channels, 16 states, us with 2, 4, 8, 24 tokens: 1 sequence
    // 2.9, 3.8, 5.6, 12.6, tile 4.1; 8 sequences 3.1, 4.0, 5.8, 12.9, tile 6.5; 32 sequences 4.4, 5.7, 8.3, 20.3, tile 22).
    const long long fours = groups_of(a, 4);
    if (a.length <= (fours <= CUS ? 3 : fours <= 4 * CUS ? 8 : 24)) {
        if (a.states <= 4) return launch_step<DT, 1>(a, s);
        if (a.states <= 8) return launch_step<DT, 2>(a, s);
        if (a.states <= 16) return launch_step<DT, 4>(a, s);
        if (a.states <= 32) return launch_step<DT, 8>(a, s);
        if (a.states <= 64) return launch_step<DT, 16>(a, s);
        return launch_step<DT, 32>(a, s);
    }
    const long long bytes = scan_workspace(a);
    if (bytes > 0 && a.workspace && a.workspace_bytes >= bytes) {
        const Parts parts = parts_of(a);
        if (a.states <= 4) return launch_tile<DT, 4, 1, 8, 16, true>(a, s, parts);
        if (a.states <= 8) return launch_tile<DT, 4, 2, 8, 16, true>(a, s, parts);
        if (a.states <= 16) return launch_tile<DT, 4, 4, 8, 16, true>(a, s, parts);
        if (a.states <= 32) return launch_tile<DT, 8, 4, 8, 16, true>(a, s, parts);
        return launch_tile<DT, 16, 4, 8, 16, true>(a, s, parts);
    }
    // Four states a lane cost the fewest operations.  With fewer the channels spread over more workgroups, which pays while each still has a compute unit to itself
    // (16 states, 3025 tokens, us with 4, 2, 1 states a lane: 1024 channels 69, 45, 30; 2048 channels 69, 46, 57; 4096 channels 69, 73, 112; 7 states, 1900 tokens,
    // with 2, 1: 1024 channels 38, 25; 4096 channels 39, 36).
    if (a.states <= 4) return launch_waves<DT, 4, 1>(a, s);
    if (a.states <= 8) {
        if (groups_of(a, 8) <= 2 * CUS) return launch_spread<DT, 8, 1, 8>(a, s);
        return launch_waves<DT, 4, 2>(a, s);
    }
    if (a.states <= 16) {
        if (groups_of(a, 16) <= CUS) return launch_spread<DT, 16, 1, 16>(a, s);
        if (groups_of(a, 8) <= CUS) return launch_spread<DT, 8, 2, 8>(a, s);
        return launch_waves<DT, 4, 4>(a, s);
    }
    if (a.states <= 32) {
        if (groups_of(a, 16) <= CUS) return launch_spread<DT, 16, 2, 8>(a, s);
        return launch_waves<DT, 8, 4>(a, s);
    }
    if (a.states <= 64) return launch_waves<DT, 16, 4>(a, s);
    return launch_tile<DT, 16, 8, 4, 16>(a, s);
}

hipError_t launch_selective_scan(const xl_scan_args &a, hipStream_t s)
{
    return a.dtype == XL_F32 ? launch_type<XL_F32>(a, s) : a.dtype == XL_F16 ? launch_type<XL_F16>(a, s) : launch_type<XL_BF16>(a, s);
}

}  // namespace xls
