// C ABI of libxl_seq, the operators around a projection (see include/xl_seq.h): checks of the arguments, then the launches.
#include <cfloat>

#include "seq_checks.h"

using namespace xls;

extern "C" {

xl_status xl_rms_norm(const xl_rms_norm_args *args, void *stream)
{
    if (!args) return fail(XL_E_NULL, "rms_norm: no arguments");
    const xl_rms_norm_args &a = *args;
    const char *w = "rms_norm";
    const int size = size_of(a.dtype), kept = size_of(a.residual_dtype);
    if (!size) return fail(XL_E_UNSUPPORTED, "%s: unknown element type %lld", w, a.dtype);
    if ((a.residual || a.new_residual) && a.residual_dtype != a.dtype && a.residual_dtype != XL_F32)
        return fail(XL_E_UNSUPPORTED, "%s: residual of type %lld beside numbers of type %lld (the same, or fp32)", w, a.residual_dtype, a.dtype);
    if (!is_size(a.rows) || !is_size(a.k) || !product_fits(a.rows, a.k, 1, MAX_ITEMS)) return fail(XL_E_SHAPE, "%s: %lld rows of %lld out of range", w, a.rows, a.k);
    if (!(a.eps >= FLT_MIN && a.eps <= FLT_MAX)) return fail(XL_E_SHAPE, "%s: eps %g is not a positive fp32 number", w, a.eps);
    if (a.rows == 0 || a.k == 0) return XL_OK;
    if (!a.x || !a.weight || !a.y || (a.quantized && !a.scales)) return fail(XL_E_NULL, "%s: x, weight, y or scales is NULL", w);
    if (!aligned(a.x, size) || !aligned(a.weight, 4) || !aligned(a.scales, 4) || (a.residual && !aligned(a.residual, kept)) || (a.new_residual && !aligned(a.new_residual, kept)))
        return fail(XL_E_ALIGN, "%s: x, weight, scales or a residual is not aligned to its elements", w);
    if (a.quantized ? !aligned(a.y, 16) || a.y_row % 16 : !aligned(a.y, size))
        return fail(XL_E_ALIGN, "%s: y is not aligned (rows of 8-bit numbers begin at multiples of 16 bytes)", w);
    if (a.rows > 1 && (a.x_row < 0 || (a.residual && a.residual_row < 0) || (a.new_residual && a.new_residual_row < a.k) || a.y_row < a.k))
        return fail(XL_E_SHAPE, "%s: steps %lld (x), %lld, %lld (residuals), %lld (y) do not fit rows of %lld", w, a.x_row, a.residual_row, a.new_residual_row, a.y_row, a.k);
    if (a.quantized && (a.scale_row < 0 || a.scale_block < 0)) return fail(XL_E_SHAPE, "%s: steps %lld, %lld of the scales are negative", w, a.scale_row, a.scale_block);
    const xl_status st = check_device();
    if (st != XL_OK) return st;
    return launched(w, launch_rms_norm(a, static_cast<hipStream_t>(stream)));
}

static bool adapters_sizes(const xl_adapters_args &a)
{
    return is_size(a.batch) && is_size(a.length) && is_size(a.k) && is_size(a.n) && is_size(a.adapters) && product_fits(a.batch, a.length + 1, a.k, MAX_ITEMS) &&
           product_fits(a.batch, a.length + 1, a.n, MAX_ITEMS) && a.rank >= 1 && a.rank <= XL_MAX_RANK && product_fits(a.adapters, a.k, XL_MAX_RANK, MAX_ITEMS) &&
           product_fits(a.adapters, a.n, XL_MAX_RANK, MAX_ITEMS) && product_fits(a.batch, a.length + 1, XL_MAX_RANK, MAX_ITEMS);
}

xl_status xl_add_adapters(const xl_adapters_args *args, void *stream)
{
    if (!args) return fail(XL_E_NULL, "add_adapters: no arguments");
    const xl_adapters_args &a = *args;
    const char *w = "add_adapters";
    const int size = size_of(a.dtype);
    if (!size) return fail(XL_E_UNSUPPORTED, "%s: unknown element type %lld", w, a.dtype);
    if (a.rank < 1 || a.rank > XL_MAX_RANK) return fail(XL_E_UNSUPPORTED, "%s: a rank of %lld (1 to %d are covered)", w, a.rank, XL_MAX_RANK);
    if (!adapters_sizes(a)) return fail(XL_E_SHAPE, "%s: batch %lld, length %lld, k %lld, n %lld or %lld adapters out of range", w, a.batch, a.length, a.k, a.n, a.adapters);
    if (a.batch == 0 || a.length == 0 || a.n == 0) return XL_OK;
    xl_status st;
    if ((st = check_rows(w, "x", a.x, a.x_batch, a.x_token, a.batch, a.length, a.k, size, false)) != XL_OK) return st;
    if ((st = check_rows(w, "y", a.y, a.y_batch, a.y_token, a.batch, a.length, a.n, size, false)) != XL_OK) return st;
    if ((st = check_rows(w, "out", a.out, a.out_batch, a.out_token, a.batch, a.length, a.n, size, true)) != XL_OK) return st;
    if (!a.index || (a.adapters > 0 && (!a.up || (a.k > 0 && !a.down)))) return fail(XL_E_NULL, "%s: index, down or up is NULL", w);
    if (!aligned(a.down, size) || !aligned(a.up, size) || !aligned(a.index, 4) || !aligned(a.scales, 4) || !aligned(a.lengths, 4))
        return fail(XL_E_ALIGN, "%s: down, up, index, scales or lengths are not aligned to their elements", w);
    const long long need = adapters_workspace(a);
    if (need > 0 && (!a.workspace || a.workspace_bytes < need)) return fail(XL_E_NULL, "%s: a workspace of %lld bytes is needed, %lld are there", w, need, a.workspace ? a.workspace_bytes : 0ll);
    if (!aligned(a.workspace, 16)) return fail(XL_E_ALIGN, "%s: the workspace is not aligned to 16 bytes", w);
    if ((st = check_device()) != XL_OK) return st;
    return launched(w, launch_add_adapters(a, static_cast<hipStream_t>(stream)));
}

long long xl_add_adapters_workspace(const xl_adapters_args *args)
{
    return args && size_of(args->dtype) && adapters_sizes(*args) && args->batch > 0 && args->length > 0 && args->n > 0 ? adapters_workspace(*args) : 0;
}

static bool delta_sizes(const xl_delta_args &a)
{
    return is_size(a.batch) && is_size(a.length) && is_size(a.key_heads) && is_size(a.heads) && is_size(a.dv) && a.dk >= 1 && a.dk <= XL_MAX_KEY && a.key_heads > 0 &&
           a.heads % a.key_heads == 0 && product_fits(a.heads, a.dv, XL_MAX_KEY, MAX_ITEMS) && product_fits(a.batch, a.length + 64, a.heads, MAX_ITEMS / XL_MAX_KEY) &&
           product_fits(a.batch * a.heads, a.length + 1, a.dv, MAX_ITEMS) && product_fits(a.batch * a.heads, XL_MAX_KEY, a.dv, MAX_ITEMS);
}

xl_status xl_gated_delta_rule(const xl_delta_args *args, void *stream)
{
    if (!args) return fail(XL_E_NULL, "gated_delta_rule: no arguments");
    xl_delta_args a = *args;
    const char *w = "gated_delta_rule";
    if (a.dk < 1 || a.dk > XL_MAX_KEY) return fail(XL_E_UNSUPPORTED, "%s: keys of %lld (1 to %d are covered)", w, a.dk, XL_MAX_KEY);
    xl_status st = check_sequences(w, a.batch, a.length, 1, a.dtype, a.nslots, a.state, a.new_state, a.slots, a.lengths);
    if (st != XL_OK) return st;
    if (a.heads == 0 && a.key_heads >= 0) return XL_OK;
    if (!delta_sizes(a)) return fail(XL_E_SHAPE, "%s: %lld heads of %lld, %lld of keys or a length of %lld out of range", w, a.heads, a.dv, a.key_heads, a.length);
    if (!(a.scale >= -FLT_MAX && a.scale <= FLT_MAX)) return fail(XL_E_SHAPE, "%s: scale %g is not an fp32 number", w, a.scale);
    if (a.batch == 0 || a.dv == 0) return XL_OK;
    const int size = size_of(a.dtype);
    const struct { const char *name; const void *p; long long batch, token, head, heads, width; int size; bool written; } rows[] = {
        {"q", a.q, a.q_batch, a.q_token, a.q_head, a.key_heads, a.dk, size, false}, {"k", a.k, a.k_batch, a.k_token, a.k_head, a.key_heads, a.dk, size, false},
        {"v", a.v, a.v_batch, a.v_token, a.v_head, a.heads, a.dv, size, false},     {"g", a.g, a.g_batch, a.g_token, 1, a.heads, 1, 4, false},
        {"beta", a.beta, a.beta_batch, a.beta_token, 1, a.heads, 1, 4, false},      {"y", a.y, a.y_batch, a.y_token, a.y_head, a.heads, a.dv, size, true}};
    for (const auto &r : rows) {
        if ((st = check_rows(w, r.name, r.p, r.batch, r.token, a.batch, a.length, r.width, r.size, r.written)) != XL_OK) return st;
        if (a.length > 0 && r.heads > 1 && r.head < (r.written ? r.width : 0)) return fail(XL_E_SHAPE, "%s: a step of %lld between heads of %s does not fit %lld", w, r.head, r.name, r.width);
    }
    if (!aligned(a.state, 4) || !aligned(a.new_state, 4)) return fail(XL_E_ALIGN, "%s: a state is not aligned to its elements", w);
    if (a.length == 0 && !a.new_state) return XL_OK;
    const long long need = delta_workspace(a);
    if (need > 0 && (!a.workspace || a.workspace_bytes < need)) return fail(XL_E_NULL, "%s: a workspace of %lld bytes is needed, %lld are there", w, need, a.workspace ? a.workspace_bytes : 0ll);
    if (!aligned(a.workspace, 16)) return fail(XL_E_ALIGN, "%s: the workspace is not aligned to 16 bytes", w);
    if ((st = check_device()) != XL_OK) return st;
    return launched(w, launch_gated_delta_rule(a, static_cast<hipStream_t>(stream)));
}

long long xl_gated_delta_rule_workspace(const xl_delta_args *args)
{
    return args && size_of(args->dtype) && delta_sizes(*args) && args->batch > 0 && args->dv > 0 && args->heads > 0 ? delta_workspace(*args) : 0;
}

}  // extern "C"
