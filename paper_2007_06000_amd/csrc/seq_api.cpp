// C ABI of libxl_seq (see include/xl_seq.h): checks of the arguments, then one launch.
#include "seq_checks.h"

using namespace xls;

thread_local char xls::g_error[256] = "";

extern "C" {

const char *xl_seq_last_error(void) { return xls::g_error; }

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
