/* Host side of the operators around a projection under -fsanitize=address,undefined, as seq_asan.cpp does for the others: argument structs of exactly their size
 * on the heap, with fields drawn from the ends of their ranges, go through the C ABI; the launchers are stubs that check what the kernels take for granted. */
#include <cfloat>
#include <climits>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>

#include "seq_launch.h"

static long long launched, failures;
#define CHECK(c) do { if (!(c)) { ++failures; fprintf(stderr, "line %d: %s\n", __LINE__, #c); } } while (0)

static bool size(long long v) { return v >= 0 && v <= INT_MAX - 4096; }
static bool rows_ok(const void *p, long long batch_step, long long token_step, long long batch, long long length, long long least)
{
    return length == 0 || (p && (batch <= 1 || batch_step >= least) && (length <= 1 || token_step >= least));
}
static const __int128 ITEMS = (__int128)1 << 38;

namespace xls {
hipError_t launch_causal_conv(const xl_causal_conv_args &, hipStream_t) { return hipSuccess; }
hipError_t launch_selective_scan(const xl_scan_args &, hipStream_t) { return hipSuccess; }
long long scan_workspace(const xl_scan_args &) { return 0; }
hipError_t launch_quantize(const xl_quantize_args &, hipStream_t) { return hipSuccess; }
hipError_t launch_block_matmul(const xl_block_matmul_args &, hipStream_t) { return hipSuccess; }
hipError_t launch_rms_norm(const xl_rms_norm_args &a, hipStream_t)
{
    ++launched;
    CHECK(a.rows > 0 && a.k > 0 && size(a.rows) && size(a.k) && (__int128)a.rows * a.k <= ITEMS && a.x && a.weight && a.y && (!a.quantized || a.scales));
    CHECK(a.dtype >= 0 && a.dtype <= 2 && ((!a.residual && !a.new_residual) || a.residual_dtype == a.dtype || a.residual_dtype == XL_F32));
    CHECK(a.rows == 1 || (a.x_row >= 0 && a.y_row >= a.k && (!a.residual || a.residual_row >= 0) && (!a.new_residual || a.new_residual_row >= a.k)));
    CHECK(!a.quantized || (a.y_row % 16 == 0 && a.scale_row >= 0 && a.scale_block >= 0));
    CHECK(a.eps >= FLT_MIN && a.eps <= FLT_MAX);
    return hipSuccess;
}
static void adapters_ok(const xl_adapters_args &a)
{
    CHECK(a.batch > 0 && a.length > 0 && a.n > 0 && size(a.batch) && size(a.length) && size(a.k) && size(a.n) && size(a.adapters) && a.rank >= 1 && a.rank <= XL_MAX_RANK);
    CHECK((__int128)a.batch * (a.length + 1) * a.k <= ITEMS && (__int128)a.batch * (a.length + 1) * a.n <= ITEMS && (__int128)a.batch * a.length * XL_MAX_RANK <= ITEMS);
    CHECK((__int128)a.adapters * a.k * a.rank <= ITEMS && (__int128)a.adapters * a.n * a.rank <= ITEMS);
}
long long adapters_workspace(const xl_adapters_args &a)
{
    adapters_ok(a);
    return a.batch % 3 == 0 ? 48 : 0;
}
hipError_t launch_add_adapters(const xl_adapters_args &a, hipStream_t)
{
    ++launched;
    adapters_ok(a);
    CHECK(rows_ok(a.x, a.x_batch, a.x_token, a.batch, a.k ? a.length : 0, 0) && rows_ok(a.y, a.y_batch, a.y_token, a.batch, a.length, 0) && rows_ok(a.out, a.out_batch, a.out_token, a.batch, a.length, a.n));
    CHECK(a.index && (a.adapters == 0 || (a.up && (a.k == 0 || a.down))) && (a.batch % 3 || (a.workspace && a.workspace_bytes >= 48)));
    return hipSuccess;
}
static void delta_ok(const xl_delta_args &a)
{
    CHECK(a.batch > 0 && a.heads > 0 && a.dv > 0 && size(a.batch) && size(a.length) && size(a.heads) && size(a.dv) && a.dk >= 1 && a.dk <= XL_MAX_KEY && a.key_heads > 0 && a.heads % a.key_heads == 0);
    CHECK((__int128)a.batch * a.heads * (a.length + 1) * a.dv <= ITEMS && (__int128)a.batch * a.heads * a.dv * XL_MAX_KEY <= ITEMS && (__int128)a.batch * a.heads * (a.length + 64) * XL_MAX_KEY <= ITEMS);
}
long long delta_workspace(const xl_delta_args &a)
{
    delta_ok(a);
    return a.batch % 3 == 0 ? 48 : 0;
}
hipError_t launch_gated_delta_rule(const xl_delta_args &a, hipStream_t)
{
    ++launched;
    delta_ok(a);
    CHECK(rows_ok(a.q, a.q_batch, a.q_token, a.batch, a.length, 0) && rows_ok(a.k, a.k_batch, a.k_token, a.batch, a.length, 0) && rows_ok(a.v, a.v_batch, a.v_token, a.batch, a.length, 0));
    CHECK(rows_ok(a.g, a.g_batch, a.g_token, a.batch, a.length, 0) && rows_ok(a.beta, a.beta_batch, a.beta_token, a.batch, a.length, 0) && rows_ok(a.y, a.y_batch, a.y_token, a.batch, a.length, a.dv));
    CHECK(a.length == 0 || ((a.key_heads == 1 || (a.q_head >= 0 && a.k_head >= 0)) && (a.heads == 1 || (a.v_head >= 0 && a.y_head >= a.dv))));
    CHECK((!a.state && !a.new_state) || a.slots || a.nslots >= a.batch);
    CHECK(a.scale >= -FLT_MAX && a.scale <= FLT_MAX && (a.batch % 3 || (a.workspace && a.workspace_bytes >= 48)));
    return hipSuccess;
}
}  // namespace xls

extern "C" {
hipError_t hipGetDevicePropertiesR0600(hipDeviceProp_tR0600 *p, int) { memset(p, 0, sizeof *p); strcpy(p->gcnArchName, "gfx950:sramecc+:xnack-"); return hipSuccess; }
hipError_t hipGetDevice(int *d) { *d = 0; return hipSuccess; }
const char *hipGetErrorString(hipError_t) { return "an error"; }
}

static std::mt19937_64 rng(1);

static void ask(const xl_adapters_args *a) { CHECK(xl_add_adapters_workspace(a) >= 0); }
static void ask(const xl_delta_args *a) { CHECK(xl_gated_delta_rule_workspace(a) >= 0); }
static void ask(const void *) {}
/* Whole numbers, perhaps a double, then pointers; most of them ordinary, so that a call gets past its first checks. */
template <typename A> static void run(xl_status (*f)(const A *, void *), int numbers, bool real)
{
    static const long long ends[] = {-1, LLONG_MIN, LLONG_MAX, INT_MAX, INT_MAX - 4096ll, 1ll << 32, 1ll << 38, 1ll << 62, 0, 128};
    static const long long usual[] = {1, 2, 3, 4, 16, 48, 64, 128, 1, 2};
    static const double reals[] = {1e-6, 1, 0.5, -1, 0, 1e300, -1e300, 1e-40, __builtin_nan(""), __builtin_inf()};
    const int fields = sizeof(A) / 8;
    A *a = static_cast<A *>(malloc(sizeof(A)));
    long long v[64];
    for (long long i = 0; i < 400000; ++i) {
        const unsigned wild = rng() % 8;        /* of 64 */
        for (int j = 0; j < fields; ++j) {
            const bool odd = rng() % 64 < wild;
            if (j < numbers) v[j] = odd ? ends[rng() % 10] : usual[rng() % 10];
            else if (real && j == numbers) memcpy(&v[j], &reals[odd ? rng() % 10 : rng() % 3], 8);
            else v[j] = odd ? (long long)(rng() % 3) : 1 << 20;
        }
        memcpy(a, v, sizeof(A));
        const xl_status st = f(a, nullptr);
        ask(a);
        CHECK(st == XL_OK || strlen(xl_seq_last_error()) > 10);
    }
    free(a);
}

int main()
{
    long long before = 0;
    const auto some = [&] { CHECK(launched - before > 300); before = launched; };
    run(xl_rms_norm, 11, true);
    some();
    run(xl_add_adapters, 14, false);
    some();
    run(xl_gated_delta_rule, 26, true);
    some();
    printf("%lld launches, %lld failures\n", launched, failures);
    return failures != 0;
}
