// The gated delta rule.
//
//   S <- e^g S,  S <- S + beta k (v - S^T k)^T,  y = scale S^T q
//
// Columns of S do not meet: each is a recurrence of its own, with the same keys, queries, decays and steps.
//
// Single tokens and a few go one after the other.  Longer runs go in chunks of 64 tokens.  With G_i the sum of g up to token i of a chunk, and S0 the states before it, the corrections
// d_i = beta_i (v_i - S_i^T k_i) of its tokens solve a triangular system:
//   (I + A) D = diag(beta) (V - diag(e^G) K S0),     A[i,j] = beta_i (k_i.k_j) e^(G_i - G_j) for j < i
//   Y = scale (diag(e^G) Q S0 + P D),                P[i,j] = (q_i.k_j) e^(G_i - G_j) for j <= i
//   S = e^G_64 S0 + K^T diag(e^(G_64 - G)) D
// A first kernel makes T = (I + A)^-1 and P of all chunks at once, a second one goes through the chunks of a sequence with the states in registers.
#include "seq_parts.h"

namespace xls {

static constexpr float NORM_EPS = 1e-6f;

// e^g is 0 in fp32 long before g reaches -128, and the differences of sums of g stay numbers where g is minus infinity.
__device__ __forceinline__ float clamped(float g)
{
    g = g < -128.f ? -128.f : g;
    return g > 0.f ? 0.f : g;       // a NaN stays
}

// A wave has 32 columns of a head's states in registers, eight of them rows' parts: lane % 8 names four columns, lane / 8 a run of R = rows / 8 rows.
// One pass over them gives both S^T k and S^T q, from which y follows without the new states:  S'^T q = S^T q + (k.q) beta (v - S^T k).
// A token is bound by reading and writing the states: 64 sequences of 16 heads of 128 x 128 take 27.3 us for 135 MB (4.9 TB/s, as a copy), 16 of 8 heads of 64 x 64 4.1 us.  (With the same states
// each time, out of the last-level cache, 23.4 and 3.9; then sums over lanes through LDS and numbers asked for when they are needed took 26.5 and 5.6 us, and 1.4 instead of 0.5 to 1 us for each further token.)
static constexpr int COLS = 32;

// The sum over lanes whose number is the same modulo 8, without a way through LDS.
__device__ __forceinline__ float over_rows(float s)
{
    s += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, s), 0x128, 0xf, 0xf, true));      // eight lanes round, of sixteen
    unsigned at = __builtin_bit_cast(unsigned, s);
    const auto rows = __builtin_amdgcn_permlane16_swap(at, at, false, false);
    const unsigned r0 = rows[0], r1 = rows[1];
    at = __builtin_bit_cast(unsigned, __builtin_bit_cast(float, r0) + __builtin_bit_cast(float, r1));
    const auto halves = __builtin_amdgcn_permlane32_swap(at, at, false, false);
    const unsigned h0 = halves[0], h1 = halves[1];
    return __builtin_bit_cast(float, h0) + __builtin_bit_cast(float, h1);
}

// FULL: the states fill their registers, and nothing is compared.
template <int DT, int R, bool FULL> __device__ __forceinline__ void step_through(const xl_delta_args &a, int tile, int b, int h)
{
    typedef typename Elem<DT>::T T;
    typedef Vec<T, 8> T8;
    typedef Vec<T, 4> T4;
    const int lane = threadIdx.x % 64, DK = (int)a.dk, DV = (int)a.dv, H = (int)a.heads, length = (int)a.length, first = lane / 8 * R, hk = h / (int)(a.heads / a.key_heads);
    const int j = tile * COLS + lane % 8 * 4, live = FULL ? 4 : DV - j;
    const long long slot = slot_of(a.slots, a.nslots, b);
    const int n = slot < 0 ? 0 : length_of(a.lengths, b, length);
    T *y = static_cast<T *>(a.y) + b * a.y_batch + h * a.y_head + j;
    if (lane < 8 && live > 0)
        for (int t = n; t < length; ++t) store_some<T, 4>(y + t * a.y_token, live, T4{});
    if (slot < 0) return;
    const long long at = (slot * H + h) * DK * DV + j + (long long)first * DV;
    const T *kp = static_cast<const T *>(a.k) + b * a.k_batch + hk * a.k_head + first, *qp = static_cast<const T *>(a.q) + b * a.q_batch + hk * a.q_head + first;
    const T *vp = static_cast<const T *>(a.v) + b * a.v_batch + h * a.v_head + j;
    // a token's numbers are asked for a token ahead
    T8 k8[R / 8], q8[R / 8];
    T4 v4;
    float g, beta;
    const auto ask = [&](int t) {
#pragma unroll
        for (int r = 0; r < R / 8; ++r) {
            k8[r] = FULL ? load_vec<T, 8>(kp + t * a.k_token + r * 8) : load_some<T, 8>(kp + t * a.k_token + r * 8, DK - first - r * 8);
            q8[r] = FULL ? load_vec<T, 8>(qp + t * a.q_token + r * 8) : load_some<T, 8>(qp + t * a.q_token + r * 8, DK - first - r * 8);
        }
        v4 = FULL ? load_vec<T, 4>(vp + t * a.v_token) : load_some<T, 4>(vp + t * a.v_token, live);
        g = a.g[b * a.g_batch + t * a.g_token + h];
        beta = a.beta[b * a.beta_batch + t * a.beta_token + h];
    };
    if (n > 0) ask(0);
    f32x4 S[R] = {};
    if (a.state) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (FULL) S[r] = load_vec<float, 4>(a.state + at + (long long)r * DV);
            else if (first + r < DK) S[r] = load_some<float, 4>(a.state + at + (long long)r * DV, live);
        }
    }
    for (int t = 0; t < n; ++t) {
        float k[R], q[R], v[4];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            k[r] = (float)k8[r / 8][r % 8];
            q[r] = (float)q8[r / 8][r % 8];
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) v[c] = (float)v4[c];
        const float decay = exp_fast(clamped(g)), step = beta;
        if (t + 1 < n) ask(t + 1);
        float kk = 0.f, qq = 0.f, kq = 0.f;
        f32x4 kS = {}, qS = {};
#pragma unroll
        for (int r = 0; r < R; ++r) {
            kk = __builtin_fmaf(k[r], k[r], kk);
            qq = __builtin_fmaf(q[r], q[r], qq);
            kq = __builtin_fmaf(k[r], q[r], kq);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                S[r][c] *= decay;
                kS[c] = __builtin_fmaf(k[r], S[r][c], kS[c]);
                qS[c] = __builtin_fmaf(q[r], S[r][c], qS[c]);
            }
        }
        kq = over_rows(kq);
        float nk = 1.f, nq = (float)a.scale;
        if (a.normalize) {
            nk = __builtin_amdgcn_rsqf(over_rows(kk) + NORM_EPS);
            nq *= __builtin_amdgcn_rsqf(over_rows(qq) + NORM_EPS);
        }
        f32x4 add;
        T4 out;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            add[c] = step * (v[c] - nk * over_rows(kS[c])) * nk;
            out[c] = (T)(nq * __builtin_fmaf(kq, add[c], over_rows(qS[c])));
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < 4; ++c) S[r][c] = __builtin_fmaf(k[r], add[c], S[r][c]);
        if (lane < 8 && live > 0) store_some<T, 4>(y + t * a.y_token, live, out);
    }
    if (a.new_state && live > 0) {
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (FULL || first + r < DK) store_some<float, 4>(a.new_state + at + (long long)r * DV, live, S[r]);
    }
}

template <int DT, int R>
__global__ __launch_bounds__(256) void token_kernel(const xl_delta_args a, int tiles)
{
    const int waves = blockDim.x / 64;
    const long long units = a.batch * a.heads * tiles;
    for (long long unit = (long long)blockIdx.x * waves + threadIdx.x / 64; unit < units; unit += (long long)gridDim.x * waves) {
        const long long head = divided(unit, tiles);
        const int tile = (int)(unit - head * tiles), b = (int)divided(head, a.heads), h = (int)(head - b * a.heads);
        if (a.dk == 8 * R && (tile + 1) * COLS <= a.dv) step_through<DT, R, true>(a, tile, b, h);
        else step_through<DT, R, false>(a, tile, b, h);
    }
}

// The chunks.  All products are operations of 16 x 16 x 32 on bf16 parts.  An operation's result has in a lane (col = lane % 16, quad = lane / 16) rows 4 quad ... 4 quad + 3 of column col, and its operands
// eight numbers from 8 quad on of row (column) col.  If row m of the tiles 2 s and 2 s + 1 stands for number 32 s + 8 (m / 4) + m % 4 (+ 4 in the second), a lane has eight neighbours of
// a column in the two results, which is an operand of the next product: results turn into operands without crossing lanes.
static constexpr int CHUNK = 64;
__device__ __forceinline__ int dealt(int tile, int m) { return tile / 2 * 32 + m / 4 * 8 + tile % 2 * 4 + m % 4; }

// What the first kernel leaves of a chunk: operands as the second one's lanes read them, one after the other, so that each load is one run of memory (read where they lie, sixteen rows at a time, the
// second kernel took 433 us of 2 x 12321 tokens and 16 heads instead of 368).  Keys and queries are filled up with zeros to DK, and as they came: heads that share a key head share them.
template <int DT, int DK> struct KeyChunk {
    Vec<typename Elem<DT>::T, 8> rows[2][4][DK / 32][64];               // keys and queries, by token tiles
    bf16x8 columns[DK / 16][2][parts_of<DT>()][64];                     // keys, by tiles of their numbers
};
// T and P: tiles 0 and 1 have numbers for tokens 0 to 31, tiles 2 and 3 for all.
struct HeadChunk {
    bf16x8 T[6][3][64], P[6][3][64];
    float factors[5][64];       // of each token: e^G / |k|, beta, e^(G_64 - G) / |k|, scale e^G / |q|; and e^G_64
};
__device__ __forceinline__ int piece(int tile, int s) { return tile < 2 ? tile : 2 * tile - 2 + s; }

struct Delta {
    xl_delta_args a;
    int first, chunks;          // of every sequence in this launch
    const float *carried;       // states between launches [batch, heads, dk, dv], or NULL
    float *carry;
    void *keys, *heads;         // chunks [batch, key heads, chunks] and [batch, heads, chunks]
};

// A row's numbers from quad * 8 on, eight of every 32.  Keys that fill their place are read without comparisons: all loads are on their way at once.
template <int DK, typename T> __device__ __forceinline__ void load_keys(const T *row, int dk, int quad, Vec<T, 8> (&out)[DK / 32])
{
    if (dk == DK) {
#pragma unroll
        for (int s = 0; s < DK / 32; ++s) out[s] = load_vec<T, 8>(row + s * 32 + quad * 8);
    } else {
#pragma unroll
        for (int s = 0; s < DK / 32; ++s) out[s] = load_some<T, 8>(row + s * 32 + quad * 8, dk - (s * 32 + quad * 8));
    }
}

template <typename V> __device__ __forceinline__ float squares(V v)
{
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s = __builtin_fmaf((float)v[i], (float)v[i], s);
    return s;
}

__device__ __forceinline__ f32x4 four(const float *p) { return *reinterpret_cast<const f32x4 *>(p); }
__device__ __forceinline__ bool finite(float v) { return fabsf(v) < __builtin_inff(); }

// A chunk of a head.  2 x 12321 tokens of 16 heads of 128 x 128 (8 of keys) take 130 us for 514 MB, 387 of them written; a workgroup's chain of loads, products and the inverse is some 8 us, three of them a compute
// unit.  (One round of workgroups by itself takes 18 us, 1 x 3136 tokens of 8 heads; what the rest of it goes into has not been measured.)  Wave w makes row tile w of A and P.  Their columns' tokens are the operation's rows, so that a lane has eight neighbours of a row.
// Rows from the first on that has an infinity or a NaN are left out of A, and T's diagonal says so with NaN: tokens before it get their right results.  (A token whose own key is not finite has such a
// right side, whatever its row.  k.k is no part of A: it may leave fp32.)
template <int DT, int DK>
__global__ __launch_bounds__(256, parts_of<DT>() * DK <= 192 ? 3 : parts_of<DT>() * DK < 512 ? 2 : 1) void prepare_kernel(const Delta d)
{
    typedef typename Elem<DT>::T T;
    constexpr int KS = DK / 32, PITCH = CHUNK + 4, NP = parts_of<DT>();
    constexpr int KEYS_PITCH = DK + 16 / sizeof(T);
    __shared__ __align__(16) float A[CHUNK][PITCH];
    __shared__ __align__(16) union {            // T is made when the keys have been used
        T keys[CHUNK][KEYS_PITCH];
        float X[CHUNK][PITCH];
    } room;
    auto &keys = room.keys;
    auto &X = room.X;
    __shared__ double G[CHUNK];
    __shared__ float beta[CHUNK], inverse_k[CHUNK], inverse_q[CHUNK];
    __shared__ int first_bad;
    const xl_delta_args &a = d.a;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), col = lane % 16, quad = lane / 16, H = (int)a.heads;
    const long long units = a.batch * a.heads * d.chunks;
    for (long long u = blockIdx.x; u < units; u += gridDim.x) {
        const long long head = divided(u, d.chunks);
        const int c = (int)(u - head * d.chunks), b = (int)divided(head, H), h = (int)(head - (long long)b * H), hk = h / (int)(a.heads / a.key_heads), t0 = (d.first + c) * CHUNK;
        const int n = (slot_of(a.slots, a.nslots, b) < 0 ? 0 : length_of(a.lengths, b, (int)a.length)) - t0;        // tokens from here on
        if (n <= 0) continue;
        const T *k = static_cast<const T *>(a.k) + b * a.k_batch + hk * a.k_head + t0 * a.k_token, *q = static_cast<const T *>(a.q) + b * a.q_batch + hk * a.q_head + t0 * a.q_token;
        HeadChunk &out = static_cast<HeadChunk *>(d.heads)[u];
        const int group = (int)(a.heads / a.key_heads);
        KeyChunk<DT, DK> &shared = static_cast<KeyChunk<DT, DK> *>(d.keys)[((long long)b * a.key_heads + hk) * d.chunks + c];       // by the first of the heads that share them
        __syncthreads();        // the unit before is done with
        const int token = dealt(wave, col);
        float gate = 0.f, step = 0.f;       // in front of the longer loads: the sums over them take longest
        if (wave == 0 && lane < n) {
            gate = a.g[b * a.g_batch + (t0 + lane) * a.g_token + h];
            step = a.beta[b * a.beta_batch + (t0 + lane) * a.beta_token + h];
        }
        Vec<T, 8> mine[KS], query[KS];
        load_keys<DK>(k + min(token, n - 1) * a.k_token, (int)a.dk, quad, mine);
        load_keys<DK>(q + min(token, n - 1) * a.q_token, (int)a.dk, quad, query);
        if (wave == 0) {
            double g = (double)clamped(gate);
#pragma unroll
            for (int o = 1; o < 64; o *= 2) {
                const double more = __shfl_up(g, o);
                g += lane >= o ? more : 0.;
            }
            G[lane] = g;
            beta[lane] = step;
            if (lane == 0) first_bad = CHUNK;
        }
        float kk = 0.f, qq = 0.f;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            if (h % group == 0) {
                shared.rows[0][wave][s][lane] = mine[s];
                shared.rows[1][wave][s][lane] = query[s];
            }
            kk += squares(mine[s]);
            qq += squares(query[s]);
            *reinterpret_cast<Vec<T, 8> *>(&keys[token][s * 32 + quad * 8]) = mine[s];
        }
        kk += __shfl_xor(kk, 16);
        qq += __shfl_xor(qq, 16);
        kk += __shfl_xor(kk, 32);
        qq += __shfl_xor(qq, 32);
        if (quad == 0) {
            inverse_k[token] = a.normalize ? __builtin_amdgcn_rsqf(kk + NORM_EPS) : 1.f;
            inverse_q[token] = (a.normalize ? __builtin_amdgcn_rsqf(qq + NORM_EPS) : 1.f) * (float)a.scale;
        }
        __syncthreads();
        // dot products of this tile's tokens with those of tile j
        f32x4 with_k[4] = {}, with_q[4] = {};
        Parts<NP> mine_parts[KS], query_parts[KS];
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            mine_parts[s] = parts<DT>(mine[s]);
            query_parts[s] = parts<DT>(query[s]);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (j > (wave | 1)) continue;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const Parts<NP> o = parts<DT>(*reinterpret_cast<const Vec<T, 8> *>(&keys[dealt(j, col)][s * 32 + quad * 8]));
                with_k[j] = product(o, mine_parts[s], with_k[j]);
                with_q[j] = product(o, query_parts[s], with_q[j]);
            }
        }
        const int before = token < n ? token : 0;       // numbers of the row: behind the last token it would be 0 beta, of products that may be infinite
        const double Gi = G[token];
        const float ki = inverse_k[token] * beta[token], qi = inverse_q[token];
        float none = 0.f;       // a NaN if a number of the row is not finite
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            if (s > wave / 2) continue;
            f32x8 p;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int j0 = s * 32 + quad * 8 + half * 4;
                f32x4 row;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int j = j0 + i;
                    const float e = exp_fast((float)(Gi - G[j])) * inverse_k[j], v = with_k[2 * s + half][i] * e * ki;
                    row[i] = j < before ? v : 0.f;
                    none = __builtin_fmaf(row[i], 0.f, none);
                    p[half * 4 + i] = j <= token ? with_q[2 * s + half][i] * e * qi : 0.f;
                }
                *reinterpret_cast<f32x4 *>(&A[token][j0]) = row;
            }
            const Parts<3> split_p = split<3>(p);
#pragma unroll
            for (int i = 0; i < 3; ++i) out.P[piece(wave, s)][i][lane] = split_p.p[i];
        }
        if (none != 0.f) atomicMin(&first_bad, token);
        if (wave == 0) {
            out.factors[0][lane] = exp_fast((float)G[lane]) * inverse_k[lane];
            out.factors[1][lane] = beta[lane];
            out.factors[2][lane] = exp_fast((float)(G[CHUNK - 1] - G[lane])) * inverse_k[lane];
            out.factors[3][lane] = exp_fast((float)G[lane]) * inverse_q[lane];
            out.factors[4][lane] = exp_fast((float)G[CHUNK - 1]);
        }
        // the keys' columns, eight tokens a lane
        for (int i = wave; i < (h % group == 0 ? DK / 16 * 2 : 0); i += 4) {
            Vec<T, 8> v;
            const int at = dealt(i / 2, col), t = i % 2 * 32 + quad * 8;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = keys[t + e][at];
            const Parts<NP> kp = parts<DT>(v);
#pragma unroll
            for (int e = 0; e < NP; ++e) shared.columns[i / 2][i % 2][e][lane] = kp.p[e];
        }
        __syncthreads();
        const int good = first_bad;
        // T = (I + A)^-1 by blocks of 16 tokens.  On the diagonal: column col of block `wave`, one number after the other.
        const int base = wave * 16;
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float s = i == col ? 1.f : 0.f;
#pragma unroll
            for (int j = 0; j < i; j += 4) {
                const f32x4 r = four(&A[base + i][base + j]);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (j + e < i) s = __builtin_fmaf(base + i < good ? -r[e] : 0.f, x[j + e], s);
            }
            x[i] = s;
        }
        f32x4 t[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            t[0][e] = quad == 0 ? x[e] : quad == 1 ? x[4 + e] : quad == 2 ? x[8 + e] : x[12 + e];
            X[base + quad * 4 + e][base + col] = t[0][e];
        }
        __syncthreads();
        // Below it, column of blocks `wave`: T_ij = -T_ii sum over m of A_im T_mj
#pragma unroll
        for (int i = 1; i < 4; ++i) {
            const int row = (wave + i) * 16;
            if (row >= CHUNK) break;
            f32x4 sum = {};
#pragma unroll
            for (int m = 0; m < i; ++m) {
                f32x4 r = four(&A[row + col][(wave + m) * 16 + quad * 4]);
                if (row + col >= good) r = f32x4{};
#pragma unroll
                for (int e = 0; e < 4; ++e) sum = __builtin_amdgcn_mfma_f32_16x16x4f32(r[e], t[m][e], sum, 0, 0, 0);
            }
            const f32x4 diagonal = four(&X[row + col][row + quad * 4]);
            t[i] = f32x4{};
#pragma unroll
            for (int e = 0; e < 4; ++e) t[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(-diagonal[e], sum[e], t[i], 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) X[row + quad * 4 + e][base + col] = t[i][e];
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            if (s > wave / 2) continue;
            const int j0 = s * 32 + quad * 8;
            const f32x4 lo = four(&X[token][j0]), hi = four(&X[token][j0 + 4]);
            f32x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = j0 + e <= token ? v[e] : 0.f;        // blocks above the diagonal were never written
                if (token >= good && j0 + e == token) v[e] = __builtin_nanf("");
            }
            const Parts<3> p = split<3>(v);
#pragma unroll
            for (int e = 0; e < 3; ++e) out.T[piece(wave, s)][e][lane] = p.p[e];
        }
    }
}

// What is written before this is done before what is written after it: loads from LDS all at once ahead of the products, not each in front of its own.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }
// v is there now: what it was made of may be loaded anew into the same registers.
__device__ __forceinline__ void settle(f32x4 &v)
{
    asm volatile("" : "+v"(v));
    __builtin_amdgcn_sched_barrier(0);
}

// The rows of a chunk that exist, as a buffer: what lies past the last one's end comes out as zeros and is not written.  (Rows that overlap go on behind the last one in the same memory.)
struct Tokens {
    __amdgpu_buffer_rsrc_t rsrc;
    __device__ __forceinline__ Tokens(const void *base, long long first, int rows, long long step, int width)      // in bytes
    {
        const unsigned long long p = (unsigned long long)base + first * step;
        const int lo = __builtin_amdgcn_readfirstlane((int)p), hi = __builtin_amdgcn_readfirstlane((int)(p >> 32));
        const int bytes = (int)(min(rows, CHUNK) - 1) * (int)step + width;
        rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)(((unsigned long long)(unsigned)hi << 32) | (unsigned)lo), (short)0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
    }
    template <typename V> __device__ __forceinline__ V load(int at) const
    {
        if constexpr (sizeof(V) == 2) return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b16(rsrc, at, 0, 0));
        else if constexpr (sizeof(V) == 4) return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b32(rsrc, at, 0, 0));
        else if constexpr (sizeof(V) == 8) return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b64(rsrc, at, 0, 0));
        else return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, 0, 0));
    }
    template <typename V> __device__ __forceinline__ void store(int at, V v) const
    {
        if constexpr (sizeof(V) == 2) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, v), rsrc, at, 0, 0);
        else if constexpr (sizeof(V) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, v), rsrc, at, 0, 0);
        else if constexpr (sizeof(V) == 8) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, v), rsrc, at, 0, 0);
        else __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), rsrc, at, 0, 0);
    }
};
static constexpr int NOWHERE = (int)0x80000000u;        // past the end of every such buffer

// What the waves of a workgroup need of each other.
template <int DK, typename T> struct Meeting {
    static constexpr int PITCH = 20;        // numbers between tokens of 16: the quads' tokens lie in other banks
    bf16x8 states[DK / 32][3][64], right[2][3][64], wrote[2][3][64];
    f32x4 corrections[2][4][64];
    __align__(16) T values[CHUNK][PITCH], results[CHUNK][PITCH];
    __align__(16) float factors[5][64];
    int first_bad[2][16];
    // A wave's result as half of an operand of the next product.
    static __device__ __forceinline__ void put(bf16x8 (*to)[64], int half, int lane, f32x4 v)
    {
        const Parts4<3> parts = split4<3>(v);
#pragma unroll
        for (int p = 0; p < 3; ++p) reinterpret_cast<u32x2 *>(&to[p][lane])[half] = parts.p[p];
    }
};

// 16 columns of a head's states through the chunks of a sequence: twelve waves, a third of them for each part.  SOLVE: for D, wave w the rows of token tile w.  FETCH: tokens' values and factors, on their way into LDS.
// Both also have parts of the states' rows in their registers (FETCH alone where DK is 64).  RESULT: y, a step behind.  What the waves need of each other meets in LDS three times a chunk: S0, the right side of
// the system, and D.
// Where a token's correction is not finite, zero stands for it, and its column is not finite from that token on: no product spreads it to tokens before.
// Bound by the chain of chunks: 1 x 3136 tokens of 8 heads of 128 x 128 take 67 us, 1.4 us a chunk, of which K S0 and the right side are some 950 of 2900 cycles, T and D 600, the states 400, what they wait for each other
// 900.  With a workgroup on each compute unit (2 x 12321 tokens, 16 heads: 384 us, 2.0 us a chunk) what is read, 85 KB a chunk and tile of 16 columns, comes out of the XCD's cache more slowly than the
// products need it.  These were measured with two parts in what makes y instead of three, 63 and 354 us: the cycles; 272 us with one chunk read again and again; four waves that do all of it 123 and 528 us, four with two
// token tiles each 130 and 594, eight (four that solve) 73 and 366.
// What a chunk is made of is asked for a chunk ahead, each part behind the product that has used the registers: all at once the loads would hold up the wave that issues them (16 cycles of
// a compute unit's address unit for 16 bytes a lane).
enum { SOLVE, FETCH, RESULT };
template <int DT, int DK, int ROLE> __device__ __forceinline__ void go_through(const Delta &d, Meeting<DK, typename Elem<DT>::T> &m, int tile, int b, int h, int wave)
{
    typedef typename Elem<DT>::T T;
    typedef Vec<T, 4> T4;
    constexpr bool HOLDS = ROLE == FETCH || (ROLE == SOLVE && DK > 64), READS = ROLE != FETCH;      // a tile of 16 rows of the states, or more; the states
    constexpr bool AHEAD = parts_of<DT>() * DK < 384, COLUMNS_AHEAD = parts_of<DT>() * DK < 768;       // there are registers for the next chunk's rows, columns
    constexpr int KS = DK / 32, TW = DK <= 128 ? 1 : DK / 128, NP = parts_of<DT>(), SIZE = sizeof(T);
    const xl_delta_args &a = d.a;
    const int lane = threadIdx.x % 64, col = lane % 16, quad = lane / 16, H = (int)a.heads, DV = (int)a.dv, hk = h / (int)(a.heads / a.key_heads);
    const int j = tile * 16 + col, at_column = min(j, DV - 1), w4 = wave % 4, held = DK > 64 ? wave * TW : w4;
    const long long slot = slot_of(a.slots, a.nslots, b);
    const int n = length_of(a.lengths, b, (int)a.length), end = min((n + CHUNK - 1) / CHUNK, d.first + d.chunks);
    const long long here = ((long long)b * H + h) * a.dk * DV + at_column, there = (slot * H + h) * a.dk * DV + at_column;
    const float *from = d.first > 0 ? d.carried + here : a.state ? a.state + there : nullptr;
    float *to = d.carry ? d.carry + here : a.new_state ? a.new_state + there : nullptr;
    f32x4 S[TW] = {};
    if constexpr (HOLDS) {
#pragma unroll
        for (int i = 0; i < TW; ++i) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int row = dealt(held + i, quad * 4 + e);
                if (from && row < a.dk) S[i][e] = from[(long long)row * DV];
            }
        }
#pragma unroll
        for (int i = 0; i < TW; ++i) settle(S[i]);
    }
    const HeadChunk *heads = static_cast<const HeadChunk *>(d.heads) + ((long long)b * H + h) * d.chunks - d.first;
    const KeyChunk<DT, DK> *shared = static_cast<const KeyChunk<DT, DK> *>(d.keys) + ((long long)b * a.key_heads + hk) * d.chunks - d.first;
    const int rows = dealt(w4, quad * 4);       // the four tokens of a lane's results
    Vec<T, 8> row[KS];          // of keys, or of queries
    Parts<3> triangle[2];       // T, or P
    Parts<NP> columns[TW][2];
    const auto ask_row = [&](int c, int s) { row[s] = shared[c].rows[ROLE == RESULT][w4][s][lane]; };
    const auto ask_triangle = [&](int c, int s) {
#pragma unroll
        for (int p = 0; p < 3; ++p) triangle[s].p[p] = ROLE == SOLVE ? heads[c].T[piece(w4, s)][p][lane] : heads[c].P[piece(w4, s)][p][lane];
    };
    const auto ask_columns = [&](int c, int i, int s) {
#pragma unroll
        for (int p = 0; p < NP; ++p) columns[i][s].p[p] = shared[c].columns[held + i][s][p][lane];
    };
    // Values and results go four neighbours of a token a lane where their places allow it (one by one, in the lanes that compute with them, four loads and four stores took a third of a
    // chunk's time).
    const T *v_base = static_cast<const T *>(a.v) + b * a.v_batch + h * a.v_head + tile * 16;
    T *y_base = static_cast<T *>(a.y) + b * a.y_batch + h * a.y_head + tile * 16;
    const long long v_step = a.v_token * SIZE, y_step = a.y_token * SIZE;
    const int width = (DV - tile * 16) * SIZE, four_at = lane % 4 * 4, one_token = dealt(w4, lane / 4);
    const bool wide_v = (((unsigned long long)v_base | (unsigned long long)v_step) & (4 * SIZE - 1)) == 0 && DV % 4 == 0;
    const bool wide_y = (((unsigned long long)y_base | (unsigned long long)y_step) & (4 * SIZE - 1)) == 0 && DV % 4 == 0;
    T4 value;
    float factor, last_factor;
    const auto ask_values = [&](int c) {
        const int left = n - c * CHUNK;
        const Tokens tokens(v_base, (long long)c * CHUNK, left, v_step, width);
        if (wide_v) {
            value = tokens.template load<T4>(four_at * SIZE < width && one_token < left ? one_token * (int)v_step + four_at * SIZE : NOWHERE);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) value[e] = tokens.template load<T>(j < DV && rows + e < left ? (rows + e) * (int)v_step + col * SIZE : NOWHERE);
        }
        factor = heads[c].factors[w4][lane];
        last_factor = heads[c].factors[4][lane];
    };
    const auto hand_over = [&] {
        if (wide_v) {
            *reinterpret_cast<T4 *>(&m.values[one_token][four_at]) = value;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) m.values[rows + e][col] = value[e];
        }
        m.factors[w4][lane] = factor;
        if (w4 == 0) m.factors[4][lane] = last_factor;
    };
    // y of a chunk, from Q S0
    const auto result = [&](int c, f32x4 out) {
        Parts<3> D[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const f32x4 lo = m.corrections[c % 2][2 * s][lane], hi = m.corrections[c % 2][2 * s + 1][lane];
            D[s] = split<3>(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
#pragma unroll
        for (int s = 0; s < 2; ++s)
            if (s <= w4 / 2) {
                out = product(triangle[s], D[s], out);
                in_order();
                ask_triangle(min(c + 1, end - 1), s);
            }
        settle(out);
        return out;
    };
    const auto store = [&](int c, f32x4 out, int lost) {
        const Tokens tokens(y_base, (long long)c * CHUNK, n - c * CHUNK, y_step, width);
        T4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = (T)(rows + e < lost ? out[e] : __builtin_nanf(""));
        if (wide_y) {
#pragma unroll
            for (int e = 0; e < 4; ++e) m.results[rows + e][col] = y[e];
            wave_sync();
            tokens.store(four_at * SIZE < width ? one_token * (int)y_step + four_at * SIZE : NOWHERE, *reinterpret_cast<const T4 *>(&m.results[one_token][four_at]));
            wave_sync();
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) tokens.store(j < DV ? (rows + e) * (int)y_step + col * SIZE : NOWHERE, y[e]);
        }
    };
    if (d.first < end) {
        if constexpr (ROLE == FETCH) {
            ask_values(d.first);
            hand_over();
            ask_values(min(d.first + 1, end - 1));
        }
        if constexpr (READS) {
#pragma unroll
            for (int s = 0; s < (AHEAD ? KS : 0); ++s) ask_row(d.first, s);
            ask_triangle(d.first, 0);
            if (w4 >= 2) ask_triangle(d.first, 1);
        }
        if constexpr (HOLDS && COLUMNS_AHEAD) {
#pragma unroll
            for (int i = 0; i < TW; ++i) {
                ask_columns(d.first, i, 0);
                ask_columns(d.first, i, 1);
            }
        }
    }
    f32x4 y_before = {};        // of the chunk before: Q S0, then y
    int lost = CHUNK;
    for (int c = d.first; c < end; ++c) {
        const int odd = c % 2, next = min(c + 1, end - 1);
        // numbers that are not finite: noted for their column, and zero from here on
        const auto clean = [&](f32x4 &v) {
            float none = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) none = __builtin_fmaf(v[e], 0.f, none);
            if (__any(none != 0.f)) {       // a NaN
#pragma unroll
                for (int e = 3; e >= 0; --e)
                    if (!finite(v[e])) {
                        atomicMin(&m.first_bad[odd][col], rows + e);
                        v[e] = 0.f;
                    }
            }
        };
        if constexpr (HOLDS) {
#pragma unroll
            for (int i = 0; i < TW; ++i) m.put(m.states[(held + i) / 2], (held + i) % 2, lane, S[i]);
        }
        __syncthreads();
        f32x4 acc = {};         // K S0, or Q S0
        const float decay = m.factors[4][lane];
        const f32x4 write_factor = four(&m.factors[2][rows]);
        if constexpr (READS) {
            const f32x4 row_factor = four(&m.factors[ROLE == SOLVE ? 0 : 3][rows]), beta = four(&m.factors[1][rows]);
            const f32x4 values = {(float)m.values[rows][col], (float)m.values[rows + 1][col], (float)m.values[rows + 2][col], (float)m.values[rows + 3][col]};
            constexpr int AT_ONCE = DK == 256 || NP == 3 ? 2 : KS;
#pragma unroll
            for (int s0 = 0; s0 < KS; s0 += AT_ONCE) {
                Parts<3> S0[AT_ONCE];
#pragma unroll
                for (int s = 0; s < AT_ONCE; ++s) {
#pragma unroll
                    for (int p = 0; p < 3; ++p) S0[s].p[p] = m.states[s0 + s][p][lane];
                    if (!AHEAD) ask_row(c, s0 + s);
                }
                in_order();
#pragma unroll
                for (int s = 0; s < AT_ONCE; ++s) {
                    acc = product(parts<DT>(row[s0 + s]), S0[s], acc);
                    in_order();
                    if (AHEAD) ask_row(next, s0 + s);
                    in_order();
                }
            }
            acc *= row_factor;
            if constexpr (ROLE == SOLVE) {
                f32x4 side = beta * (values - acc);
                if (threadIdx.x < 16) m.first_bad[!odd][col] = CHUNK;
                clean(side);
                m.put(m.right[w4 / 2], w4 % 2, lane, side);
            } else {
                settle(acc);
            }
        }
        __syncthreads();
        if constexpr (ROLE == SOLVE) {
            Parts<3> right[2];
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int p = 0; p < 3; ++p) right[s].p[p] = m.right[s][p][lane];
            in_order();
            f32x4 D = product(triangle[0], right[0], f32x4{});
            in_order();
            ask_triangle(next, 0);
            if (w4 >= 2) {
                D = product(triangle[1], right[1], D);
                in_order();
                ask_triangle(next, 1);
            }
            clean(D);
            m.put(m.wrote[w4 / 2], w4 % 2, lane, write_factor * D);
            m.corrections[odd][w4][lane] = D;
        } else if constexpr (ROLE == FETCH) {
            hand_over();
            ask_values(min(c + 2, end - 1));
        } else if (c > d.first) {
            y_before = result(c - 1, y_before);
        }
        __syncthreads();
        if constexpr (ROLE == RESULT) {
            if (c > d.first) store(c - 1, y_before, lost);
            y_before = acc;
        }
        lost = m.first_bad[odd][col];
        if constexpr (HOLDS) {
            Parts<3> wrote[2];
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int p = 0; p < 3; ++p) wrote[s].p[p] = m.wrote[s][p][lane];
#pragma unroll
            for (int i = 0; i < TW; ++i) S[i] *= decay;
            in_order();
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int i = 0; i < TW; ++i) {
                    if (!COLUMNS_AHEAD) ask_columns(c, i, s);
                    S[i] = product(columns[i][s], wrote[s], S[i]);
                    in_order();
                    if (COLUMNS_AHEAD) ask_columns(next, i, s);
                    in_order();
                }
            if (lost < CHUNK) {
#pragma unroll
                for (int i = 0; i < TW; ++i) S[i] = f32x4{__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
            }
#pragma unroll
            for (int i = 0; i < TW; ++i) settle(S[i]);
        }
    }
    if constexpr (ROLE == RESULT) {
        if (d.first < end) store(end - 1, result(end - 1, y_before), lost);
    }
    if constexpr (HOLDS) {
        if (to && j < DV) {
#pragma unroll
            for (int i = 0; i < TW; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int row = dealt(held + i, quad * 4 + e);
                    if (row < a.dk) to[(long long)row * DV] = S[i][e];
                }
        }
    }
}

template <int DT, int DK>
__global__ __launch_bounds__(768) void chunks_kernel(const Delta d, int tiles)
{
    typedef typename Elem<DT>::T T;
    __shared__ Meeting<DK, T> m;
    const xl_delta_args &a = d.a;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), H = (int)a.heads, length = (int)a.length;
    const int u = neighbours_together(blockIdx.x, gridDim.x), tile = u % tiles, h = u / tiles % H, b = u / tiles / H, j = tile * 16 + threadIdx.x % 16;
    const bool absent = slot_of(a.slots, a.nslots, b) < 0;
    if (d.first == 0 && j < a.dv)
        for (int t = (absent ? 0 : length_of(a.lengths, b, length)) + threadIdx.x / 16; t < length; t += 48) static_cast<T *>(a.y)[b * a.y_batch + t * a.y_token + h * a.y_head + j] = (T)0.f;
    if (absent) return;
    if (threadIdx.x < 32) m.first_bad[threadIdx.x / 16][threadIdx.x % 16] = CHUNK;
    // the thirds meet at the same three barriers a chunk, each from a loop of its own: registers and loads on their way are its own too
    if (wave < 4) go_through<DT, DK, SOLVE>(d, m, tile, b, h, wave);
    else if (wave < 8) go_through<DT, DK, FETCH>(d, m, tile, b, h, wave);
    else go_through<DT, DK, RESULT>(d, m, tile, b, h, wave);
}

// How many tokens go one by one.  us of 16 / 24 / 48 / 64 / 128 tokens, keys and values of 128, bf16, one by one | in chunks:
//   8 heads 19 / 26 / 49 / 64 / 125 | 16 / 16 / 16 / 16 / 18          128 heads 22 / 29 / 53 / 68 / 132 | 34 / 34 / 34 / 34 / 41
//   512 heads 36 / 48 / 83 / 105 / 196 | 82 / 82 / 83 / 85 / 120      1024 heads 63 / 85 / 150 / 194 / 371 | 152 / 153 / 158 / 161 / 294
// The ways meet at 16, 25, 52 and 61 tokens with keys and values of 64, at 13, 20, 37 and 42 with keys of 256.  In fp32 a chunk takes twice as many operations, and from 1024 heads on it is never the faster way:
// 128 tokens of 4096 heads take 506 one by one, 848 in chunks (64 x 64), 1642 and 2105 (128 x 128).
static long long few_tokens(const xl_delta_args &a)
{
    const long long heads = a.batch * a.heads;
    return heads >= 1024 && a.dtype == XL_F32 ? a.length : heads >= 512 ? 48 : heads >= 128 ? 24 : 14;
}
static constexpr long long MOST_BYTES = 1ll << 29;         // of chunks that are prepared at once

// The sequences [first, first + count) of a call by themselves.
template <int DT> static xl_delta_args piece_of(const xl_delta_args &a, long long first, long long count)
{
    const long long size = sizeof(typename Elem<DT>::T);
    xl_delta_args p = piece_of_states(a, first, count, a.heads * a.dk * a.dv, sizeof(float));
    p.q = behind(a.q, first * a.q_batch, size);
    p.k = behind(a.k, first * a.k_batch, size);
    p.v = behind(a.v, first * a.v_batch, size);
    p.y = behind(a.y, first * a.y_batch, size);
    p.g = behind(a.g, first * a.g_batch, sizeof(float));
    p.beta = behind(a.beta, first * a.beta_batch, sizeof(float));
    return p;
}

// Sequences in pieces, and their chunks so many at once, that these take no more than MOST_BYTES.
template <int DT, int DK> struct Chunked {
    long long sequences, chunks, at_once, of_keys, of_heads, carried;     // of a piece; of a sequence, in one launch; bytes of a launch's chunks, of states between launches
    Chunked() {}
    explicit Chunked(const xl_delta_args &a)
    {
        sequences = MOST_BYTES / bytes_of_a_sequence(a);
        sequences = sequences < 1 ? 1 : sequences > a.batch ? a.batch : sequences;
        chunks = (a.length + CHUNK - 1) / CHUNK;
        at_once = MOST_BYTES / (sequences * bytes_of_a_sequence(a));
        at_once = at_once < 1 ? 1 : at_once > chunks ? chunks : at_once;
        of_keys = at_once * sequences * a.key_heads * (long long)sizeof(KeyChunk<DT, DK>);
        of_heads = at_once * sequences * a.heads * (long long)sizeof(HeadChunk);
        carried = at_once < chunks ? (sequences * a.heads * a.dk * a.dv * 4 + 15) / 16 * 16 : 0;
    }
    static long long bytes_of_a_sequence(const xl_delta_args &a)      // of one chunk of all its heads
    {
        return a.key_heads * (long long)sizeof(KeyChunk<DT, DK>) + a.heads * (long long)sizeof(HeadChunk);
    }
    static long long bytes(const xl_delta_args &a)
    {
        const Chunked plan(a);
        return plan.of_keys + plan.of_heads + plan.carried;
    }
    static hipError_t launch(const xl_delta_args &all, hipStream_t s)
    {
        const Chunked plan(all);
        for (long long b = 0; b < all.batch; b += plan.sequences) {
            const hipError_t e = plan.launch_piece(piece_of<DT>(all, b, all.batch - b < plan.sequences ? all.batch - b : plan.sequences), s);
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    }
    hipError_t launch_piece(const xl_delta_args &a, hipStream_t s) const
    {
        const int tiles = (int)((a.dv + 15) / 16);
        char *w = static_cast<char *>(a.workspace);
        float *between = carried ? reinterpret_cast<float *>(w + of_keys + of_heads) : nullptr;
        for (long long first = 0; first < chunks; first += at_once) {
            const long long some = chunks - first < at_once ? chunks - first : at_once, units = a.batch * a.heads * some;
            const Delta d = {a, (int)first, (int)some, between, first + some < chunks ? between : nullptr, w, w + of_keys};
            hipError_t e = launch_kernel(prepare_kernel<DT, DK>, dim3((unsigned)(units < 1 << 20 ? units : 1 << 20)), 256, s, d);
            if (e == hipSuccess) e = launch_kernel(chunks_kernel<DT, DK>, dim3((unsigned)(a.batch * a.heads * tiles)), 768, s, d, tiles);
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    }
};

// Rows of a chunk lie within 2 GB of each other.
static constexpr long long FURTHEST = 1ll << 22;

// f with the chunks of these arguments
template <int DT, typename F> static auto with_keys(const xl_delta_args &a, F f)
{
    return a.dk <= 64 ? f(Chunked<DT, 64>()) : a.dk <= 128 ? f(Chunked<DT, 128>()) : f(Chunked<DT, 256>());
}

// Tens of thousands of heads go token by token (64 tokens of 65536 heads of 64 x 64 in bf16 take 3.8 ms, of 65520 in chunks 5.1), and so do thousands of one sequence, whose chunk alone would take more than MOST_BYTES.
template <int DT> static bool in_chunks(const xl_delta_args &a)
{
    if (a.batch * a.heads >= 1 << 16 || with_keys<DT>(a, [&](auto chunked) { return chunked.bytes_of_a_sequence(a); }) > MOST_BYTES) return false;
    return a.length > few_tokens(a) && a.batch * a.heads * ((a.dv + 15) / 16) < 1 << 22 && a.v_token <= FURTHEST && a.y_token <= FURTHEST && a.dv <= FURTHEST;
}

template <int DT> static hipError_t launch_type(const xl_delta_args &a, hipStream_t s)
{
    if (in_chunks<DT>(a)) return with_keys<DT>(a, [&](auto chunked) { return chunked.launch(a, s); });
    const int tiles = (int)((a.dv + COLS - 1) / COLS);
    // few waves have a compute unit each
    const long long units = a.batch * a.heads * tiles, waves = units <= 1024 ? 1 : 4, groups = (units + waves - 1) / waves;
    const dim3 grid((unsigned)(groups < 1 << 20 ? groups : 1 << 20));
    const unsigned threads = (unsigned)waves * 64;
    return a.dk <= 64 ? launch_kernel(token_kernel<DT, 8>, grid, threads, s, a, tiles)
         : a.dk <= 128 ? launch_kernel(token_kernel<DT, 16>, grid, threads, s, a, tiles) : launch_kernel(token_kernel<DT, 32>, grid, threads, s, a, tiles);
}

template <int DT> static long long workspace_of(const xl_delta_args &a)
{
    return in_chunks<DT>(a) ? with_keys<DT>(a, [&](auto chunked) { return chunked.bytes(a); }) : 0;
}
long long delta_workspace(const xl_delta_args &a)
{
    return a.dtype == XL_F32 ? workspace_of<XL_F32>(a) : a.dtype == XL_F16 ? workspace_of<XL_F16>(a) : workspace_of<XL_BF16>(a);
}

hipError_t launch_gated_delta_rule(const xl_delta_args &a, hipStream_t s)
{
    return a.dtype == XL_F32 ? launch_type<XL_F32>(a, s) : a.dtype == XL_F16 ? launch_type<XL_F16>(a, s) : launch_type<XL_BF16>(a, s);
}

}  // namespace xls
