// C ABI of libxl_seq (see include/xl_seq.h): checks of the arguments, then one launch.
#include <atomic>
#include <climits>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <cstring>

#include "seq_launch.h"

static thread_local char g_error[256] = "";

static xl_status fail(xl_status st, const char *format, ...)
{
    va_list args;
    va_start(args, format);
    vsnprintf(g_error, sizeof g_error, format, args);
    va_end(args);
    return st;
}

// The current device is asked about once: 0 unknown, 1 a gfx950, 2 something else.
static xl_status check_device()
{
    static std::atomic<int> known[64];
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return fail(XL_E_DEVICE, "no current HIP device");
    int k = known[dev].load(std::memory_order_relaxed);
    if (!k) {
        hipDeviceProp_t prop;
        if (hipGetDeviceProperties(&prop, dev) != hipSuccess) return fail(XL_E_DEVICE, "device %d cannot be queried", dev);
        k = strncmp(prop.gcnArchName, "gfx950", 6) == 0 ? 1 : 2;
        known[dev].store(k, std::memory_order_relaxed);
    }
    return k == 1 ? XL_OK : fail(XL_E_DEVICE, "device %d is not a gfx950 GPU", dev);
}

static xl_status launched(const char *what, hipError_t e)
{
    if (e == hipErrorInvalidConfiguration) return fail(XL_E_SHAPE, "%s: the sizes take a larger launch than the device has", what);
    return e == hipSuccess ? XL_OK : fail(XL_E_LAUNCH, "%s: kernel launch failed: %s", what, hipGetErrorString(e));
}

static int size_of(long long dtype) { return dtype == XL_F32 ? 4 : dtype == XL_F16 || dtype == XL_BF16 ? 2 : 0; }
static bool aligned(const void *p, unsigned n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
// Sizes are indexes of 32 bits in the kernels; offsets in memory are 64 bits wide.
static bool is_size(long long v) { return v >= 0 && v <= INT_MAX - 4096; }
// a * b * c <= limit, for numbers that are not negative
static bool product_fits(long long a, long long b, long long c, long long limit)
{
    long long p;
    return !__builtin_mul_overflow(a, b, &p) && !__builtin_mul_overflow(p, c, &p) && p <= limit;
}
static constexpr long long MAX_ITEMS = 1ll << 38;      // numbers of an activation or a result: more than a device has memory for

static xl_status check_sequences(const char *what, long long batch, long long length, long long channels, long long dtype, long long &nslots,
                                 const void *state, const void *new_state, const int *slots, const int *lengths)
{
    if (!size_of(dtype)) return fail(XL_E_UNSUPPORTED, "%s: unknown element type %lld", what, dtype);
    if (!is_size(batch) || !is_size(length) || !is_size(channels) || !product_fits(batch, length + 1, channels, MAX_ITEMS))
        return fail(XL_E_SHAPE, "%s: batch %lld, length %lld or channels %lld out of range", what, batch, length, channels);
    if (!aligned(slots, 4) || !aligned(lengths, 4)) return fail(XL_E_ALIGN, "%s: slots and lengths are 32-bit numbers", what);
    if (state || new_state) {
        if (nslots < 0 || (!slots && nslots < batch))
            return fail(XL_E_SHAPE, "%s: %lld rows of states for a batch of %lld", what, nslots, batch);
    } else if (!slots) {
        nslots = batch;
    }
    if (nslots < 0) return fail(XL_E_SHAPE, "%s: a negative number of slots", what);
    return XL_OK;
}

// One activation: present, aligned to its elements, steps not negative; a written one's rows do not overlap.
static xl_status check_rows(const char *what, const char *name, const void *p, long long batch_step, long long token_step, long long batch, long long length,
                            long long width, int size, bool written)
{
    if (batch == 0 || length == 0 || width == 0) return XL_OK;
    if (!p) return fail(XL_E_NULL, "%s: %s is NULL", what, name);
    if (!aligned(p, size)) return fail(XL_E_ALIGN, "%s: %s is not aligned to its elements", what, name);
    if ((length > 1 && token_step < (written ? width : 0)) || (batch > 1 && batch_step < (written ? width : 0)))
        return fail(XL_E_SHAPE, "%s: steps %lld, %lld of %s do not fit rows of %lld", what, batch_step, token_step, name, width);
    return XL_OK;
}

extern "C" {

const char *xl_seq_last_error(void) { return g_error; }

xl_status xl_causal_conv(const xl_causal_conv_args *args, void *stream)
{
    if (!args) return fail(XL_E_NULL, "causal_conv: no arguments");
    xl_causal_conv_args a = *args;
    const char *w = "causal_conv";
    xl_status st = check_sequences(w, a.batch, a.length, a.channels, a.dtype, a.nslots, a.state, a.new_state, a.slots, a.lengths);
    if (st != XL_OK) return st;
    if (a.taps < 2 || a.taps > XL_MAX_TAPS) return fail(XL_E_UNSUPPORTED, "%s: %lld taps (2 to %d are covered)", w, a.taps, XL_MAX_TAPS);
    if (a.batch == 0 || a.channels == 0) return XL_OK;
    const int size = size_of(a.dtype);
    if ((st = check_rows(w, "x", a.x, a.x_batch, a.x_token, a.batch, a.length, a.channels, size, false)) != XL_OK) return st;
    if ((st = check_rows(w, "y", a.y, a.y_batch, a.y_token, a.batch, a.length, a.channels, size, true)) != XL_OK) return st;
    if (!a.weight) return fail(XL_E_NULL, "%s: weight is NULL", w);
    if (!aligned(a.weight, 4) || !aligned(a.bias, 4) || !aligned(a.state, size) || !aligned(a.new_state, size))
        return fail(XL_E_ALIGN, "%s: a filter, bias or state is not aligned to its elements", w);
    if (a.length == 0 && !a.new_state) return XL_OK;
    if ((st = check_device()) != XL_OK) return st;
    return launched(w, xls::launch_causal_conv(a, static_cast<hipStream_t>(stream)));
}

xl_status xl_selective_scan(const xl_scan_args *args, void *stream)
{
    if (!args) return fail(XL_E_NULL, "selective_scan: no arguments");
    xl_scan_args a = *args;
    const char *w = "selective_scan";
    xl_status st = check_sequences(w, a.batch, a.length, a.channels, a.dtype, a.nslots, a.state, a.new_state, a.slots, a.lengths);
    if (st != XL_OK) return st;
    if (a.states < 1 || a.states > XL_MAX_STATES) return fail(XL_E_UNSUPPORTED, "%s: %lld states (1 to %d are covered)", w, a.states, XL_MAX_STATES);
    if (!product_fits(a.batch, a.channels, 1, 1 << 30)) return fail(XL_E_SHAPE, "%s: batch %lld x channels %lld out of range", w, a.batch, a.channels);
    if (a.batch == 0 || a.channels == 0) return XL_OK;
    const int size = size_of(a.dtype);
    const struct { const char *name; const void *p; long long batch, token, width; bool written; } rows[] = {
        {"u", a.u, a.u_batch, a.u_token, a.channels, false},     {"delta", a.delta, a.delta_batch, a.delta_token, a.channels, false},
        {"B", a.B, a.b_batch, a.b_token, a.states, false},       {"C", a.C, a.c_batch, a.c_token, a.states, false},
        {"z", a.z, a.z_batch, a.z_token, a.channels, false},     {"y", a.y, a.y_batch, a.y_token, a.channels, true}};
    for (const auto &r : rows)
        if ((r.p || r.name[0] != 'z') && (st = check_rows(w, r.name, r.p, r.batch, r.token, a.batch, a.length, r.width, size, r.written)) != XL_OK) return st;
    if (!a.A) return fail(XL_E_NULL, "%s: A is NULL", w);
    if (!aligned(a.A, 4) || !aligned(a.D, 4) || !aligned(a.delta_bias, 4) || !aligned(a.state, 4) || !aligned(a.new_state, 4))
        return fail(XL_E_ALIGN, "%s: A, D, delta_bias or a state is not aligned to its elements", w);
    if (!aligned(a.workspace, 16)) return fail(XL_E_ALIGN, "%s: the workspace is not aligned to 16 bytes", w);
    if (a.length == 0 && !a.new_state) return XL_OK;
    if ((st = check_device()) != XL_OK) return st;
    return launched(w, xls::launch_selective_scan(a, static_cast<hipStream_t>(stream)));
}

long long xl_selective_scan_workspace(const xl_scan_args *args)
{
    if (!args || !is_size(args->batch) || !is_size(args->length) || !is_size(args->channels) || args->states < 1 || args->states > XL_MAX_STATES ||
        !product_fits(args->batch, args->channels, 1, 1 << 30))
        return 0;
    return xls::scan_workspace(*args);
}

xl_status xl_quantize_blocks(const xl_quantize_args *args, void *stream)
{
    if (!args) return fail(XL_E_NULL, "quantize_blocks: no arguments");
    const xl_quantize_args &a = *args;
    const char *w = "quantize_blocks";
    const int size = size_of(a.dtype);
    if (!size) return fail(XL_E_UNSUPPORTED, "%s: unknown element type %lld", w, a.dtype);
    if (a.block_rows != 1 && a.block_rows != XL_SCALE_BLOCK) return fail(XL_E_UNSUPPORTED, "%s: blocks of %lld rows (1 or %d)", w, a.block_rows, XL_SCALE_BLOCK);
    if (!is_size(a.rows) || !is_size(a.k)) return fail(XL_E_SHAPE, "%s: %lld rows of %lld out of range", w, a.rows, a.k);
    if (a.rows == 0 || a.k == 0) return XL_OK;
    if (!a.x || !a.q || !a.scales) return fail(XL_E_NULL, "%s: x, q or scales is NULL", w);
    if (!aligned(a.x, size) || !aligned(a.scales, 4)) return fail(XL_E_ALIGN, "%s: x or scales is not aligned to its elements", w);
    if (!aligned(a.q, 16) || a.q_row % 16) return fail(XL_E_ALIGN, "%s: rows of q begin at multiples of 16 bytes", w);
    if ((a.rows > 1 && (a.x_row < 0 || a.q_row < a.k)) || a.scale_row < 0 || a.scale_block < 0)
        return fail(XL_E_SHAPE, "%s: steps %lld (x), %lld (q), %lld, %lld (scales) do not fit rows of %lld", w, a.x_row, a.q_row, a.scale_row, a.scale_block, a.k);
    const xl_status st = check_device();
    if (st != XL_OK) return st;
    return launched(w, xls::launch_quantize(a, static_cast<hipStream_t>(stream)));
}

xl_status xl_block_matmul(const xl_block_matmul_args *args, void *stream)
{
    if (!args) return fail(XL_E_NULL, "block_matmul: no arguments");
    const xl_block_matmul_args &a = *args;
    const char *w = "block_matmul";
    const int size = size_of(a.dtype);
    if (!size) return fail(XL_E_UNSUPPORTED, "%s: unknown element type %lld", w, a.dtype);
    if (!is_size(a.m) || !is_size(a.n) || !is_size(a.k) || !product_fits(a.m + 15, a.n + 15, 1, MAX_ITEMS))
        return fail(XL_E_SHAPE, "%s: m %lld, n %lld or k %lld out of range", w, a.m, a.n, a.k);
    if (a.m == 0 || a.n == 0) return XL_OK;
    if (!a.y || (a.k > 0 && (!a.a || !a.b || !a.a_scales || !a.b_scales))) return fail(XL_E_NULL, "%s: an operand, its scales or y is NULL", w);
    if (a.k > 0 && (!aligned(a.a, 16) || !aligned(a.b, 16) || (a.m > 1 && a.a_row % 16) || (a.n > 1 && a.b_row % 16)))
        return fail(XL_E_ALIGN, "%s: rows of a and b begin at multiples of 16 bytes", w);
    if (!aligned(a.y, size) || !aligned(a.a_scales, 4) || !aligned(a.b_scales, 4) || !aligned(a.bias, 4))
        return fail(XL_E_ALIGN, "%s: y, bias or scales are not aligned to their elements", w);
    if ((a.m > 1 && (a.a_row < a.k || a.y_row < a.n)) || (a.n > 1 && a.b_row < a.k) || a.a_scale_row < 0 || a.a_scale_block < 0 || a.b_scale_row < 0 || a.b_scale_block < 0)
        return fail(XL_E_SHAPE, "%s: steps %lld (a), %lld (b), %lld (y) do not fit %lld x %lld x %lld", w, a.a_row, a.b_row, a.y_row, a.m, a.n, a.k);
    const xl_status st = check_device();
    if (st != XL_OK) return st;
    return launched(w, xls::launch_block_matmul(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
