// The launchers of the sequence operators' kernels: arguments that the C ABI has checked, one or two launches on the stream.
#pragma once
#include <hip/hip_runtime.h>

#include "xl_seq.h"

namespace xls {

hipError_t launch_causal_conv(const xl_causal_conv_args &a, hipStream_t s);
hipError_t launch_selective_scan(const xl_scan_args &a, hipStream_t s);
long long scan_workspace(const xl_scan_args &a);       // of arguments whose sizes have been checked
hipError_t launch_quantize(const xl_quantize_args &a, hipStream_t s);
hipError_t launch_block_matmul(const xl_block_matmul_args &a, hipStream_t s);
hipError_t launch_rms_norm(const xl_rms_norm_args &a, hipStream_t s);
hipError_t launch_add_adapters(const xl_adapters_args &a, hipStream_t s);
long long adapters_workspace(const xl_adapters_args &a);
hipError_t launch_gated_delta_rule(const xl_delta_args &a, hipStream_t s);
long long delta_workspace(const xl_delta_args &a);

}  // namespace xls
