// Checks that the entry points of the C ABI share (see include/xl_seq.h).  Host code.
#pragma once
#include <atomic>
#include <climits>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <cstring>

#include "seq_launch.h"

namespace xls {

extern thread_local char g_error[256];      // the calling thread's last failure; of seq_api.cpp

inline xl_status fail(xl_status st, const char *format, ...)
{
    va_list args;
    va_start(args, format);
    vsnprintf(g_error, sizeof g_error, format, args);
    va_end(args);
    return st;
}

// The current device is asked about once: 0 unknown, 1 a gfx950, 2 something else.
inline xl_status check_device()
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

inline xl_status launched(const char *what, hipError_t e)
{
    if (e == hipErrorInvalidConfiguration) return fail(XL_E_SHAPE, "%s: the sizes take a larger launch than the device has", what);
    return e == hipSuccess ? XL_OK : fail(XL_E_LAUNCH, "%s: kernel launch failed: %s", what, hipGetErrorString(e));
}

inline int size_of(long long dtype) { return dtype == XL_F32 ? 4 : dtype == XL_F16 || dtype == XL_BF16 ? 2 : 0; }
inline bool aligned(const void *p, unsigned n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
// Sizes are indexes of 32 bits in the kernels; offsets in memory are 64 bits wide.
inline bool is_size(long long v) { return v >= 0 && v <= INT_MAX - 4096; }
// a * b * c <= limit, for numbers that are not negative
inline bool product_fits(long long a, long long b, long long c, long long limit)
{
    long long p;
    return !__builtin_mul_overflow(a, b, &p) && !__builtin_mul_overflow(p, c, &p) && p <= limit;
}
constexpr long long MAX_ITEMS = 1ll << 38;      // numbers of an activation or a result: more than a device has memory for

inline xl_status check_sequences(const char *what, long long batch, long long length, long long channels, long long dtype, long long &nslots,
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
inline xl_status check_rows(const char *what, const char *name, const void *p, long long batch_step, long long token_step, long long batch, long long length,
                            long long width, int size, bool written)
{
    if (batch == 0 || length == 0 || width == 0) return XL_OK;
    if (!p) return fail(XL_E_NULL, "%s: %s is NULL", what, name);
    if (!aligned(p, size)) return fail(XL_E_ALIGN, "%s: %s is not aligned to its elements", what, name);
    if ((length > 1 && token_step < (written ? width : 0)) || (batch > 1 && batch_step < (written ? width : 0)))
        return fail(XL_E_SHAPE, "%s: steps %lld, %lld of %s do not fit rows of %lld", what, batch_step, token_step, name, width);
    return XL_OK;
}

}  // namespace xls
