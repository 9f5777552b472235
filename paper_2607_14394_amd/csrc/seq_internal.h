// Launchers of the latent-sequence operators.  Arguments are checked by the
// callers (api_seq.cpp); every launcher returns a HIP error code.
#pragma once

#include <cstddef>
#include <cstdint>

#include "dtst.h"

namespace dtst {

constexpr int64_t kNormMaxCols = 32768;

// Workgroups of the norm, and the threads of each.
struct NormGrid {
  int64_t groups;
  int threads;
};
NormGrid norm_grid(int64_t rows, int64_t cols);
int launch_rms_norm(const dtst_norm_desc& d, const void* x, const void* res, const float* weight, void* sum_out,
                    void* y, void* scale, float* rstd, void* stream);
size_t rms_norm_adj_workspace(int64_t rows, int64_t cols);
int launch_rms_norm_adj(const dtst_norm_adj_desc& d, const void* g_y, const void* u, const float* weight,
                        const float* rstd, const void* g_sum, void* g_u, void* g_x, float* g_weight, void* workspace,
                        void* stream);
int launch_layer_norm(const dtst_norm_desc& d, const void* x, const void* res, const float* weight, const float* bias,
                      void* sum_out, void* y, void* scale, float* mean, float* rstd, void* stream);
size_t layer_norm_adj_workspace(int64_t rows, int64_t cols);
int launch_layer_norm_adj(const dtst_norm_adj_desc& d, const void* g_y, const void* u, const float* weight,
                          const float* mean, const float* rstd, const void* g_sum, void* g_u, void* g_x,
                          float* g_weight, float* g_bias, void* workspace, void* stream);
// first (cols) and second (the columns from there to width) as the sum, or (accumulate)
// with the sum, of `parts` rows of part.  In a fixed order.
int launch_sum_parts(const float* part, int64_t parts, int64_t pitch, int64_t cols, int64_t width, int accumulate,
                     float* first, float* second, void* stream);
int launch_quantise(const dtst_quantise_desc& d, const void* x, void* q, void* scale, void* qt, void* scale_t,
                    void* stream);
int launch_product(const dtst_product_desc& d, const void* a, const void* a_scale, const void* b, const void* b_scale,
                   const float* bias, void* c, void* stream);
size_t recurrence_workspace(int64_t batch, int64_t steps, int64_t features, int type);
int launch_recurrence(const dtst_recurrence_desc& d, const void* z, const void* v, const void* o, const float* h_zero,
                      const int32_t* lengths, void* y, float* h_out, float* states, void* workspace, void* stream);
int launch_recurrence_adj(const dtst_recurrence_desc& d, const void* z, const void* v, const void* o,
                          const int32_t* lengths, const float* states, const void* g_y, const float* g_h, void* g_z,
                          void* g_v, void* g_o, float* g_hzero, void* workspace, void* stream);
constexpr int64_t kConvMaxTaps = 8;
int64_t conv_groups(const dtst_conv_desc& d, bool adj);  // workgroups of 256
int launch_conv(const dtst_conv_desc& d, const void* x, const float* w, const float* bias, const void* state,
                const int32_t* lengths, void* y, void* state_out, void* stream);
size_t conv_adj_workspace(const dtst_conv_desc& d);
int launch_conv_adj(const dtst_conv_desc& d, const void* x, const float* w, const float* bias, const void* state,
                    const int32_t* lengths, const void* g_y, const void* g_state_out, void* g_x, float* g_weight,
                    float* g_bias, void* g_state, void* workspace, void* stream);

constexpr int64_t kScanMaxStates = 64;
int scan_segments(int64_t batch, int64_t steps, int64_t features, int64_t states, bool adj);
size_t scan_carry_bytes(const dtst_scan_desc& d, bool adj);
int launch_scan(const dtst_scan_desc& d, const void* x, const void* delta, const float* a, const void* b, const void* c,
                const float* skip, const void* o, const float* h_zero, const int32_t* lengths, void* y, float* h_out,
                float* states, void* workspace, void* stream);
size_t scan_adj_workspace(const dtst_scan_desc& d);
int launch_scan_adj(const dtst_scan_desc& d, const void* x, const void* delta, const float* a, const void* b,
                    const void* c, const float* skip, const void* o, const int32_t* lengths, const float* states,
                    const void* g_y, const float* g_h, void* g_x, void* g_delta, float* g_a, void* g_b, void* g_c,
                    float* g_skip, void* g_o, float* g_hzero, void* workspace, void* stream);

// n tensors: pointers, counts of values, types.  out: where the scaled ones go,
// null for in place.
struct TensorList {
  int64_t n;
  void* const* p;
  void* const* out;
  const int64_t* counts;
  const int32_t* types;
};
int64_t clip_chunks(int64_t count);  // a launch holds fewer than 2^31 of them
size_t global_norm_workspace(const TensorList& l);
int launch_global_norm(const TensorList& l, float* norm, void* workspace, void* stream);
int launch_clip(const TensorList& l, const float* norm, float most, void* stream);

}  // namespace dtst
