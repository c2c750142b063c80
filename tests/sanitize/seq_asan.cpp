/* Host side of the sequence operators under -fsanitize=address,undefined: argument structs of exactly their size on the heap, with
 * fields drawn from the ends of their ranges, go through the C ABI; the launchers are stubs that check what the kernels take for granted. */
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

namespace xls {
hipError_t launch_causal_conv(const xl_causal_conv_args &a, hipStream_t)
{
    ++launched;
    CHECK(a.batch > 0 && a.channels > 0 && size(a.batch) && size(a.length) && size(a.channels) && a.taps >= 2 && a.taps <= XL_MAX_TAPS && a.weight);
    CHECK((__int128)a.batch * (a.length + 1) * a.channels <= (__int128)1 << 38);
    CHECK(rows_ok(a.x, a.x_batch, a.x_token, a.batch, a.length, 0) && rows_ok(a.y, a.y_batch, a.y_token, a.batch, a.length, a.channels));
    CHECK((!a.state && !a.new_state) || a.slots || a.nslots >= a.batch);
    return hipSuccess;
}
hipError_t launch_selective_scan(const xl_scan_args &a, hipStream_t)
{
    ++launched;
    CHECK(a.batch > 0 && a.channels > 0 && size(a.batch) && size(a.length) && size(a.channels) && a.states >= 1 && a.states <= XL_MAX_STATES && a.A);
    CHECK((__int128)a.batch * (a.length + 1) * a.channels <= (__int128)1 << 38 && (__int128)a.batch * a.channels <= 1 << 30);
    CHECK(rows_ok(a.u, a.u_batch, a.u_token, a.batch, a.length, 0) && rows_ok(a.delta, a.delta_batch, a.delta_token, a.batch, a.length, 0));
    CHECK(rows_ok(a.B, a.b_batch, a.b_token, a.batch, a.length, 0) && rows_ok(a.C, a.c_batch, a.c_token, a.batch, a.length, 0));
    CHECK((!a.z || rows_ok(a.z, a.z_batch, a.z_token, a.batch, a.length, 0)) && rows_ok(a.y, a.y_batch, a.y_token, a.batch, a.length, a.channels));
    CHECK((!a.state && !a.new_state) || a.slots || a.nslots >= a.batch);
    return hipSuccess;
}
long long scan_workspace(const xl_scan_args &a)
{
    CHECK(size(a.batch) && size(a.length) && size(a.channels) && a.states >= 1 && a.states <= XL_MAX_STATES && (__int128)a.batch * a.channels <= 1 << 30);
    return 0;
}
hipError_t launch_quantize(const xl_quantize_args &a, hipStream_t)
{
    ++launched;
    CHECK(a.rows > 0 && a.k > 0 && size(a.rows) && size(a.k) && (a.block_rows == 1 || a.block_rows == XL_SCALE_BLOCK) && a.x && a.q && a.scales);
    CHECK(a.q_row % 16 == 0 && (a.rows == 1 || (a.q_row >= a.k && a.x_row >= 0)) && a.scale_row >= 0 && a.scale_block >= 0);
    return hipSuccess;
}
hipError_t launch_block_matmul(const xl_block_matmul_args &a, hipStream_t)
{
    ++launched;
    CHECK(a.m > 0 && a.n > 0 && size(a.m) && size(a.n) && size(a.k) && (__int128)a.m * a.n <= (__int128)1 << 38 && a.y);
    CHECK(a.k == 0 || (a.a && a.b && a.a_scales && a.b_scales && (a.m == 1 || (a.a_row >= a.k && a.a_row % 16 == 0)) && (a.n == 1 || (a.b_row >= a.k && a.b_row % 16 == 0))));
    CHECK(a.m == 1 || a.y_row >= a.n);
    return hipSuccess;
}
}  // namespace xls

extern "C" {
hipError_t hipGetDevicePropertiesR0600(hipDeviceProp_tR0600 *p, int) { memset(p, 0, sizeof *p); strcpy(p->gcnArchName, "gfx950:sramecc+:xnack-"); return hipSuccess; }
hipError_t hipGetDevice(int *d) { *d = 0; return hipSuccess; }
const char *hipGetErrorString(hipError_t) { return "an error"; }
}

static std::mt19937_64 rng(1);

/* Numbers, then pointers; most of them ordinary, so that a call gets past its first checks. */
static void ask(const xl_scan_args *a) { CHECK(xl_selective_scan_workspace(a) == 0); }
static void ask(const void *) {}
template <typename A> static void run(xl_status (*f)(const A *, void *), int numbers)
{
    static const long long ends[] = {-1, LLONG_MIN, LLONG_MAX, INT_MAX, INT_MAX - 4096ll, 1ll << 32, 1ll << 38, 1ll << 62, 0, 128};
    static const long long usual[] = {1, 2, 3, 4, 16, 48, 64, 128, 1, 2};
    const int fields = sizeof(A) / 8;
    A *a = static_cast<A *>(malloc(sizeof(A)));
    long long v[64];
    for (long long i = 0; i < 400000; ++i) {
        const unsigned wild = rng() % 8;        /* of 64 */
        for (int j = 0; j < fields; ++j) {
            const bool odd = rng() % 64 < wild;
            if (j < numbers) v[j] = odd ? ends[rng() % 10] : usual[rng() % 10];
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
    run(xl_causal_conv, 11);
    run(xl_selective_scan, 20);
    run(xl_quantize_blocks, 8);
    run(xl_block_matmul, 11);
    printf("%lld launches, %lld failures\n", launched, failures);
    return failures != 0 || launched < 1000;
}
