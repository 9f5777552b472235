// Status, messages and event timing shared by the files of the C ABI.
#include "api_common.h"

namespace dtst {

std::string& last_error() {
  thread_local std::string s;
  return s;
}

dtst_status fail(dtst_status s, const std::string& msg) {
  last_error() = msg;
  return s;
}

dtst_status ok() {
  last_error().clear();
  return DTST_OK;
}

dtst_status device_status(int e, const char* what) {
  if (e == hipSuccess) return ok();
  return fail(DTST_ERR_DEVICE, std::string(what) + ": " + hipGetErrorString(static_cast<hipError_t>(e)));
}

dtst_status check_ptr(const void* ptr, const char* name) {
  if (ptr == nullptr) return fail(DTST_ERR_INVALID_ARG, std::string(name) + " is null");
  if (!aligned16(ptr)) return fail(DTST_ERR_INVALID_ARG, std::string(name) + " is not 16-byte aligned");
  return DTST_OK;
}

const char* const kRoleNames[K_COUNT] = {"stream_fwd_tz", "axis_fwd_y", "axis_fwd_x", "axis_inv_x", "axis_inv_y",
                                         "stream_inv_zt", "mix", "mix_h", "wgrad", "block_epilogue",
                                         "stream_fwd_tzy", "stream_inv_yzt", "pointwise", "stream_inv_zt_block",
                                         "rms_norm", "rms_norm_adj", "quantise", "product", "recurrence",
                                         "recurrence_adj", "layer_norm", "layer_norm_adj", "global_norm", "clip", "conv",
                                         "conv_adj", "scan", "scan_adj"};

Profiler& prof() {
  static Profiler p;
  return p;
}

}  // namespace dtst
