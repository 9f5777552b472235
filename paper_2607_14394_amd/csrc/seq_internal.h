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
NormGrid rms_norm_grid(int64_t rows, int64_t cols);
int launch_rms_norm(const dtst_norm_desc& d, const void* x, const void* res, const float* weight, void* sum_out,
                    void* y, void* scale, float* rstd, void* stream);
size_t rms_norm_adj_workspace(int64_t rows, int64_t cols);
int launch_rms_norm_adj(const dtst_norm_adj_desc& d, const void* g_y, const void* u, const float* weight,
                        const float* rstd, const void* g_sum, void* g_u, void* g_x, float* g_weight, void* workspace,
                        void* stream);
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

}  // namespace dtst
