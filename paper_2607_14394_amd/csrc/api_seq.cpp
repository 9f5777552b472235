// C ABI of the latent-sequence operators: argument checks and dispatch.
//
// As in api.cpp, everything is checked on the host first; on any error
// nothing is launched, the outputs are untouched and dtst_last_error() says
// why.  No exception leaves an entry point.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdlib>
#include <new>
#include <string>
#include <utility>

#include "api_common.h"
#include "seq_checks.h"
#include "seq_internal.h"

namespace {

using namespace dtst;

dtst_status check_norm_types(int x_type, int res_type) {
  if (!is_float_type(x_type)) return bad("x_type must be DTST_F32, DTST_BF16 or DTST_F16");
  if (res_type != x_type && res_type != DTST_F32) return bad("res_type must be x_type or DTST_F32");
  return DTST_OK;
}

dtst_status check_rows_cols(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 1) return bad("need rows >= 0 and cols >= 1");
  return DTST_OK;
}

// RMS norm, and layer norm with `layer` (bias and mean are null without).
dtst_status norm(bool layer, const dtst_norm_desc* d, const void* x, const void* res, const float* weight,
                 const float* bias, void* sum_out, void* y, void* scale, float* mean, float* rstd, void* stream) {
  if (d == nullptr) return bad("descriptor is null");
  DTST_TRY(check_rows_cols(d->rows, d->cols));
  DTST_TRY(check_norm_types(d->x_type, d->res_type));
  const bool q8 = d->y_type == DTST_E4M3;
  if (!q8 && d->y_type != d->x_type) return bad("y_type must be x_type or DTST_E4M3");
  if (q8 != (scale != nullptr)) return bad("scale goes with y of DTST_E4M3, and only with it");
  if (!(d->eps >= 0.f) || std::isinf(d->eps)) return bad("need a finite eps >= 0");
  if (d->cols > kNormMaxCols) return fail(DTST_ERR_UNSUPPORTED, "cols above " + std::to_string(kNormMaxCols));
  if (d->rows == 0) return ok();
  const int sx = type_size(d->x_type), sr = type_size(d->res_type);
  const Array ax{x, d->rows, d->cols, d->ld_x, sx, "x"}, ar{res, d->rows, d->cols, d->ld_res, sr, "res"};
  const Array as{sum_out, d->rows, d->cols, d->ld_sum, sr, "sum_out"};
  const Array ay = q8 ? codes_of(y, d->rows, d->cols, d->ld_y, "y") : Array{y, d->rows, d->cols, d->ld_y, sx, "y"};
  const Array asc = scales_of(scale, d->rows, d->cols, d->ld_scale, "scale");
  const Array aw{weight, 1, d->cols, d->cols, 4, "weight"}, art{rstd, 1, d->rows, d->rows, 4, "rstd"};
  const Array ab{bias, 1, d->cols, d->cols, 4, "bias"}, am{mean, 1, d->rows, d->rows, 4, "mean"};
  DTST_TRY(check_array(ax, sx));
  DTST_TRY(check_align(weight, 4, "weight"));
  if (bias) DTST_TRY(check_align(bias, 4, "bias"));
  if (mean) DTST_TRY(check_align(mean, 4, "mean"));
  if (res) DTST_TRY(check_array(ar, sr));
  if (sum_out) DTST_TRY(check_array(as, sr));
  if (rstd) DTST_TRY(check_align(rstd, 4, "rstd"));
  DTST_TRY(q8 ? check_codes(ay, asc) : check_array(ay, sx));
  const NormGrid grid = norm_grid(d->rows, d->cols);
  DTST_TRY(check_grid(grid.groups, grid.threads));
  DTST_TRY(check_apart(as, ar, true));
  DTST_TRY(check_apart(as, ax, res == nullptr));
  DTST_TRY(check_apart(ay, ax, !q8));
  for (const Array* out : {&as, &ay, &asc, &art, &am}) {
    DTST_TRY(check_apart(*out, aw, false));
    DTST_TRY(check_apart(*out, ab, false));
  }
  for (const Array* in : {&ax, &ar})
    for (const Array* out : {&asc, &art, &am}) DTST_TRY(check_apart(*out, *in, false));
  DTST_TRY(check_apart(ay, ar, false));
  DTST_TRY(check_apart(ay, as, false));
  DTST_TRY(check_apart(asc, ay, false));
  DTST_TRY(check_apart(asc, as, false));
  for (const Array* out : {&as, &ay, &asc, &am}) DTST_TRY(check_apart(art, *out, false));
  for (const Array* out : {&as, &ay, &asc}) DTST_TRY(check_apart(am, *out, false));
  const int e = timed(layer ? K_LAYER_NORM : K_NORM, stream, [&] {
    return layer ? launch_layer_norm(*d, x, res, weight, bias, sum_out, y, scale, mean, rstd, stream)
                 : launch_rms_norm(*d, x, res, weight, sum_out, y, scale, rstd, stream);
  });
  return device_status(e, "norm launch");
}

dtst_status norm_adj(bool layer, const dtst_norm_adj_desc* d, const void* g_y, const void* u, const float* weight,
                     const float* mean, const float* rstd, const void* g_sum, void* g_u, void* g_x, float* g_weight,
                     float* g_bias, void* workspace, size_t workspace_bytes, void* stream) {
  if (d == nullptr) return bad("descriptor is null");
  DTST_TRY(check_rows_cols(d->rows, d->cols));
  DTST_TRY(check_norm_types(d->x_type, d->res_type));
  if (d->accumulate != 0 && d->accumulate != 1) return bad("accumulate must be 0 or 1");
  if (d->cols > kNormMaxCols) return fail(DTST_ERR_UNSUPPORTED, "cols above " + std::to_string(kNormMaxCols));
  const int sx = type_size(d->x_type), sr = type_size(d->res_type);
  const Array ag{g_y, d->rows, d->cols, d->ld_g_y, sx, "g_y"}, au{u, d->rows, d->cols, d->ld_u, sr, "u"};
  const Array as{g_sum, d->rows, d->cols, d->ld_g_sum, sr, "g_sum"};
  const Array agu{g_u, d->rows, d->cols, d->ld_g_u, sr, "g_u"}, agx{g_x, d->rows, d->cols, d->ld_g_x, sx, "g_x"};
  const Array aw{weight, 1, d->cols, d->cols, 4, "weight"}, art{rstd, 1, d->rows, d->rows, 4, "rstd"};
  const Array agw{g_weight, 1, d->cols, d->cols, 4, "g_weight"}, agb{g_bias, 1, d->cols, d->cols, 4, "g_bias"};
  const Array am{mean, 1, d->rows, d->rows, 4, "mean"};
  const size_t need = layer ? layer_norm_adj_workspace(d->rows, d->cols) : rms_norm_adj_workspace(d->rows, d->cols);
  const Array aws{workspace, 1, int64_t(need), int64_t(need), 1, "workspace"};
  DTST_TRY(check_align(g_weight, 4, "g_weight"));
  if (layer) DTST_TRY(check_align(g_bias, 4, "g_bias"));
  DTST_TRY(check_workspace(workspace, workspace_bytes, need));
  if (d->rows > 0) {
    DTST_TRY(check_array(ag, sx));
    DTST_TRY(check_array(au, sr));
    DTST_TRY(check_align(weight, 4, "weight"));
    if (layer) DTST_TRY(check_align(mean, 4, "mean"));
    DTST_TRY(check_align(rstd, 4, "rstd"));
    if (g_sum) DTST_TRY(check_array(as, sr));
    DTST_TRY(check_array(agu, sr));
    if (g_x) DTST_TRY(check_array(agx, sx));
    DTST_TRY(check_apart(agu, as, true));
    for (const Array* in : {&ag, &au, &aw, &am, &art}) DTST_TRY(check_apart(agu, *in, false));
    for (const Array* in : {&ag, &au, &as, &aw, &am, &art, &agu}) DTST_TRY(check_apart(agx, *in, false));
    for (const Array* in : {&ag, &au, &as, &aw, &am, &art, &agu, &agx})
      for (const Array* out : {&agw, &agb, &aws}) DTST_TRY(check_apart(*out, *in, false));
  }
  DTST_TRY(check_apart(aws, agw, false));
  DTST_TRY(check_apart(aws, agb, false));
  DTST_TRY(check_apart(agw, agb, false));
  const int e = timed(layer ? K_LAYER_NORM_ADJ : K_NORM_ADJ, stream, [&] {
    return layer ? launch_layer_norm_adj(*d, g_y, u, weight, mean, rstd, g_sum, g_u, g_x, g_weight, g_bias, workspace,
                                         stream)
                 : launch_rms_norm_adj(*d, g_y, u, weight, rstd, g_sum, g_u, g_x, g_weight, workspace, stream);
  });
  return device_status(e, "norm backward launch");
}

dtst_status norm_adj_workspace(bool layer, int64_t rows, int64_t cols, size_t* bytes) {
  if (bytes == nullptr) return bad("bytes is null");
  DTST_TRY(check_rows_cols(rows, cols));
  if (cols > kNormMaxCols) return fail(DTST_ERR_UNSUPPORTED, "cols above " + std::to_string(kNormMaxCols));
  *bytes = layer ? layer_norm_adj_workspace(rows, cols) : rms_norm_adj_workspace(rows, cols);
  return ok();
}

dtst_status quantise(const dtst_quantise_desc* d, const void* x, void* q, void* scale, void* qt, void* scale_t,
                     void* stream) {
  if (d == nullptr) return bad("descriptor is null");
  DTST_TRY(check_rows_cols(d->rows, d->cols));
  if (!is_float_type(d->type)) return bad("type must be DTST_F32, DTST_BF16 or DTST_F16");
  if ((q != nullptr) != (scale != nullptr) || (qt != nullptr) != (scale_t != nullptr))
    return bad("codes and scales go together");
  if (q == nullptr && qt == nullptr) return bad("q and qt are null");
  if (d->rows == 0) return ok();
  const int sx = type_size(d->type);
  const Array ax{x, d->rows, d->cols, d->ld_x, sx, "x"};
  const Array aq = codes_of(q, d->rows, d->cols, d->ld_q, "q"), as = scales_of(scale, d->rows, d->cols, d->ld_scale, "scale");
  const Array at = codes_of(qt, d->cols, d->rows, d->ld_qt, "qt");
  const Array ast = scales_of(scale_t, d->cols, d->rows, d->ld_scale_t, "scale_t");
  DTST_TRY(check_array(ax, sx));
  if (q) DTST_TRY(check_codes(aq, as));
  if (qt) DTST_TRY(check_codes(at, ast));
  DTST_TRY(check_extent(d->rows, (d->cols + 127) / 128, "x"));
  DTST_TRY(check_grid((d->rows + 15) * ((d->cols + 127) / 128) / 16 + 1, 256));
  const Array* all[] = {&ax, &aq, &as, &at, &ast};
  for (int i = 1; i < 5; ++i)
    for (int j = 0; j < i; ++j) DTST_TRY(check_apart(*all[i], *all[j], false));
  const int e = timed(K_QUANTISE, stream, [&] { return launch_quantise(*d, x, q, scale, qt, scale_t, stream); });
  return device_status(e, "quantise launch");
}

dtst_status product(const dtst_product_desc* d, const void* a, const void* a_scale, const void* b, const void* b_scale,
                    const float* bias, void* c, void* stream) {
  if (d == nullptr) return bad("descriptor is null");
  if (d->m < 0 || d->n < 0 || d->k < 1) return bad("need m >= 0, n >= 0 and k >= 1");
  if (!is_float_type(d->c_type)) return bad("c_type must be DTST_F32, DTST_BF16 or DTST_F16");
  if (d->accumulate != 0 && d->accumulate != 1) return bad("accumulate must be 0 or 1");
  if (d->short_sums != 0 && d->short_sums != 1) return bad("short_sums must be 0 or 1");
  if (d->m == 0 || d->n == 0) return ok();
  const Array aa = codes_of(a, d->m, d->k, d->ld_a, "a"), asa = scales_of(a_scale, d->m, d->k, d->ld_a_scale, "a_scale");
  const Array ab = codes_of(b, d->n, d->k, d->ld_b, "b"), asb = scales_of(b_scale, d->n, d->k, d->ld_b_scale, "b_scale");
  const int sc = type_size(d->c_type);
  const Array ac{c, d->m, d->n, d->ld_c, sc, "c"}, abi{bias, 1, d->n, d->n, 4, "bias"};
  DTST_TRY(check_codes(aa, asa));
  DTST_TRY(check_codes(ab, asb));
  DTST_TRY(check_array(ac, sc));
  if (bias) DTST_TRY(check_align(bias, 4, "bias"));
  if (d->k > (1 << 23) || d->ld_a > (1 << 23) || d->ld_b > (1 << 23))
    return fail(DTST_ERR_UNSUPPORTED, "k or a stride of a or b above 2^23");
  if (d->m > (int64_t(1) << 31) || d->n > (int64_t(1) << 31))
    return fail(DTST_ERR_UNSUPPORTED, "m or n above 2^31");
  DTST_TRY(check_grid(((d->m + 127) / 128) * ((d->n + 127) / 128), 512));
  for (const Array* in : {&aa, &asa, &ab, &asb, &abi}) DTST_TRY(check_apart(ac, *in, false));
  const int e = timed(K_PRODUCT, stream, [&] { return launch_product(*d, a, a_scale, b, b_scale, bias, c, stream); });
  return device_status(e, "product launch");
}

dtst_status check_sequence_sizes(const dtst_recurrence_desc* d) {
  if (d == nullptr) return bad("descriptor is null");
  if (d->batch < 0 || d->steps < 0 || d->features < 0) return bad("need batch, steps and features >= 0");
  if (!is_float_type(d->type)) return bad("type must be DTST_F32, DTST_BF16 or DTST_F16");
  if (d->features > (int64_t(1) << 28)) return fail(DTST_ERR_UNSUPPORTED, "features above 2^28");
  int64_t n = 0;
  if (__builtin_mul_overflow(d->batch, d->steps, &n) || __builtin_mul_overflow(n, d->features, &n) || n > kMost ||
      __builtin_mul_overflow(d->batch, d->features, &n) || n > kMost)
    return bad("problem size overflows the supported element counts");
  for (const int64_t(*s)[2] : {&d->z_stride, &d->v_stride, &d->o_stride, &d->y_stride, &d->g_z_stride, &d->g_v_stride,
                               &d->g_o_stride})
    if ((*s)[0] > kMost || (*s)[1] > kMost || (*s)[0] < -kMost || (*s)[1] < -kMost) return bad("a stride is too large");
  return DTST_OK;
}

// (one workgroup of 64 lanes a step's features, or of 512 for each 128 steps)
dtst_status check_recurrence_grid(const dtst_recurrence_desc* d) {
  const int64_t tiles = d->batch * ((d->features + 63) / 64), spans = (d->steps + 127) / 128;
  return check_grid(tiles * (spans > 0 ? spans : 1), d->steps <= 1 ? 64 : 512);
}

Sequence sequence_of(const dtst_recurrence_desc* d, const void* p, const int64_t (&st)[2], const char* name) {
  return Sequence{p, d->batch, d->steps, d->features, st, type_size(d->type), name};
}
Block of_features(const dtst_recurrence_desc* d, const void* p, int64_t rows, const char* name) {
  return Block{p, d->batch * d->features * rows * 4, name};
}

dtst_status recurrence(const dtst_recurrence_desc* d, const void* z, const void* v, const void* o, const float* h_zero,
                       const int32_t* lengths, void* y, float* h_out, float* states, void* workspace,
                       size_t workspace_bytes, void* stream) {
  DTST_TRY(check_sequence_sizes(d));
  if (d->batch == 0 || d->features == 0) return ok();
  const Sequence sz = sequence_of(d, z, d->z_stride, "z"), sv = sequence_of(d, v, d->v_stride, "v");
  const Sequence so = sequence_of(d, o, d->o_stride, "o"), sy = sequence_of(d, y, d->y_stride, "y");
  if (d->steps > 0) {
    DTST_TRY(check_sequence(sz));
    DTST_TRY(check_sequence(sv));
    if (o) DTST_TRY(check_sequence(so));
    DTST_TRY(check_sequence(sy));
    for (const Sequence* in : {&sz, &sv, &so}) DTST_TRY(check_no_share(sy, *in));
  }
  if (h_zero) DTST_TRY(check_align(h_zero, 4, "h_zero"));
  if (h_out) DTST_TRY(check_align(h_out, 4, "h_out"));
  if (states) DTST_TRY(check_align(states, 4, "states"));
  if (lengths) DTST_TRY(check_align(lengths, 4, "lengths"));
  const size_t need = recurrence_workspace(d->batch, d->steps, d->features, d->type);
  DTST_TRY(check_workspace(workspace, workspace_bytes, need));
  DTST_TRY(check_recurrence_grid(d));
  const Block bin = of_features(d, h_zero, 1, "h_zero"), bout = of_features(d, h_out, 1, "h_out");
  const Block bst = of_features(d, states, (d->steps + 127) / 128, "states"), bn{lengths, d->batch * 4, "lengths"};
  const Block bws{need ? workspace : nullptr, int64_t(need), "workspace"};
  for (const Block* b : {&bin, &bn, &bout, &bst, &bws}) DTST_TRY(check_no_share(sy, *b));
  for (const Block* out : {&bout, &bst, &bws}) {
    for (const Sequence* in : {&sz, &sv, &so}) DTST_TRY(check_no_share(*in, *out));
    if (out != &bout || h_out != h_zero) DTST_TRY(check_no_share(*out, bin));
    DTST_TRY(check_no_share(*out, bn));
  }
  DTST_TRY(check_no_share(bst, bout));
  DTST_TRY(check_no_share(bws, bout));
  DTST_TRY(check_no_share(bws, bst));
  const int e = timed(K_RECUR, stream, [&] {
    return launch_recurrence(*d, z, v, o, h_zero, lengths, y, h_out, states, workspace, stream);
  });
  return device_status(e, "recurrence launch");
}

dtst_status recurrence_adj(const dtst_recurrence_desc* d, const void* z, const void* v, const void* o,
                           const int32_t* lengths, const float* states, const void* g_y, const float* g_h, void* g_z,
                           void* g_v, void* g_o, float* g_hzero, void* workspace, size_t workspace_bytes,
                           void* stream) {
  DTST_TRY(check_sequence_sizes(d));
  if (d->batch == 0 || d->features == 0) return ok();
  if ((o != nullptr) != (g_o != nullptr) && d->steps > 0) return bad("g_o goes with o");
  const Sequence sz = sequence_of(d, z, d->z_stride, "z"), sv = sequence_of(d, v, d->v_stride, "v");
  const Sequence so = sequence_of(d, o, d->o_stride, "o"), sg = sequence_of(d, g_y, d->y_stride, "g_y");
  const Sequence gz = sequence_of(d, g_z, d->g_z_stride, "g_z"), gv = sequence_of(d, g_v, d->g_v_stride, "g_v");
  const Sequence go = sequence_of(d, g_o, d->g_o_stride, "g_o");
  if (d->steps > 0) {
    for (const Sequence* s : {&sz, &sv, &sg, &gz, &gv}) DTST_TRY(check_sequence(*s));
    if (o)
      for (const Sequence* s : {&so, &go}) DTST_TRY(check_sequence(*s));
    DTST_TRY(check_align(states, 4, "states"));
    for (const Sequence* in : {&sz, &sv, &so, &sg})
      for (const Sequence* out : {&gz, &gv, &go}) DTST_TRY(check_no_share(*out, *in));
    DTST_TRY(check_no_share(gz, gv));
    DTST_TRY(check_no_share(gz, go));
    DTST_TRY(check_no_share(gv, go));
  }
  if (g_h) DTST_TRY(check_align(g_h, 4, "g_h"));
  if (g_hzero) DTST_TRY(check_align(g_hzero, 4, "g_hzero"));
  if (lengths) DTST_TRY(check_align(lengths, 4, "lengths"));
  const size_t need = recurrence_workspace(d->batch, d->steps, d->features, d->type);
  DTST_TRY(check_workspace(workspace, workspace_bytes, need));
  DTST_TRY(check_recurrence_grid(d));
  const Block bst = of_features(d, d->steps > 0 ? states : nullptr, (d->steps + 127) / 128, "states");
  const Block bin = of_features(d, g_h, 1, "g_h"), bout = of_features(d, g_hzero, 1, "g_hzero");
  const Block bn{lengths, d->batch * 4, "lengths"}, bws{need ? workspace : nullptr, int64_t(need), "workspace"};
  for (const Sequence* out : {&gz, &gv, &go})
    for (const Block* b : {&bst, &bin, &bn, &bout, &bws}) DTST_TRY(check_no_share(*out, *b));
  for (const Block* out : {&bout, &bws}) {
    for (const Sequence* in : {&sz, &sv, &so, &sg}) DTST_TRY(check_no_share(*in, *out));
    DTST_TRY(check_no_share(*out, bst));
    if (out != &bout || g_hzero != g_h) DTST_TRY(check_no_share(*out, bin));
    DTST_TRY(check_no_share(*out, bn));
  }
  DTST_TRY(check_no_share(bws, bout));
  const int e = timed(K_RECUR_ADJ, stream, [&] {
    return launch_recurrence_adj(*d, z, v, o, lengths, states, g_y, g_h, g_z, g_v, g_o, g_hzero, workspace, stream);
  });
  return device_status(e, "recurrence backward launch");
}

}  // namespace

extern "C" {

dtst_status dtst_rms_norm(const dtst_norm_desc* d, const void* x, const void* res, const float* weight, void* sum_out,
                          void* y, void* scale, float* rstd, void* stream) {
  return guarded([&] { return norm(false, d, x, res, weight, nullptr, sum_out, y, scale, nullptr, rstd, stream); });
}

dtst_status dtst_rms_norm_adj_workspace(int64_t rows, int64_t cols, size_t* bytes) {
  return guarded([&] { return norm_adj_workspace(false, rows, cols, bytes); });
}

dtst_status dtst_rms_norm_adj(const dtst_norm_adj_desc* d, const void* g_y, const void* u, const float* weight,
                              const float* rstd, const void* g_sum, void* g_u, void* g_x, float* g_weight,
                              void* workspace, size_t workspace_bytes, void* stream) {
  return guarded([&] {
    return norm_adj(false, d, g_y, u, weight, nullptr, rstd, g_sum, g_u, g_x, g_weight, nullptr, workspace,
                    workspace_bytes, stream);
  });
}

dtst_status dtst_layer_norm(const dtst_norm_desc* d, const void* x, const void* res, const float* weight,
                            const float* bias, void* sum_out, void* y, void* scale, float* mean, float* rstd,
                            void* stream) {
  return guarded([&] { return norm(true, d, x, res, weight, bias, sum_out, y, scale, mean, rstd, stream); });
}

dtst_status dtst_layer_norm_adj_workspace(int64_t rows, int64_t cols, size_t* bytes) {
  return guarded([&] { return norm_adj_workspace(true, rows, cols, bytes); });
}

dtst_status dtst_layer_norm_adj(const dtst_norm_adj_desc* d, const void* g_y, const void* u, const float* weight,
                                const float* mean, const float* rstd, const void* g_sum, void* g_u, void* g_x,
                                float* g_weight, float* g_bias, void* workspace, size_t workspace_bytes, void* stream) {
  return guarded([&] {
    return norm_adj(true, d, g_y, u, weight, mean, rstd, g_sum, g_u, g_x, g_weight, g_bias, workspace, workspace_bytes,
                    stream);
  });
}

dtst_status dtst_quantise(const dtst_quantise_desc* d, const void* x, void* q, void* scale, void* qt, void* scale_t,
                          void* stream) {
  return guarded([&] { return quantise(d, x, q, scale, qt, scale_t, stream); });
}

dtst_status dtst_product(const dtst_product_desc* d, const void* a, const void* a_scale, const void* b,
                         const void* b_scale, const float* bias, void* c, void* stream) {
  return guarded([&] { return product(d, a, a_scale, b, b_scale, bias, c, stream); });
}

dtst_status dtst_recurrence_workspace(int64_t batch, int64_t steps, int64_t features, int type, size_t* bytes) {
  return guarded([&] {
    if (bytes == nullptr) return bad("bytes is null");
    dtst_recurrence_desc d{};
    d.batch = batch, d.steps = steps, d.features = features, d.type = type;
    DTST_TRY(check_sequence_sizes(&d));
    *bytes = recurrence_workspace(batch, steps, features, type);
    return ok();
  });
}

dtst_status dtst_recurrence(const dtst_recurrence_desc* d, const void* z, const void* v, const void* o,
                            const float* h_zero, const int32_t* lengths, void* y, float* h_out, float* states,
                            void* workspace, size_t workspace_bytes, void* stream) {
  return guarded([&] {
    return recurrence(d, z, v, o, h_zero, lengths, y, h_out, states, workspace, workspace_bytes, stream);
  });
}

dtst_status dtst_recurrence_adj(const dtst_recurrence_desc* d, const void* z, const void* v, const void* o,
                                const int32_t* lengths, const float* states, const void* g_y, const float* g_h,
                                void* g_z, void* g_v, void* g_o, float* g_hzero, void* workspace,
                                size_t workspace_bytes, void* stream) {
  return guarded([&] {
    return recurrence_adj(d, z, v, o, lengths, states, g_y, g_h, g_z, g_v, g_o, g_hzero, workspace, workspace_bytes,
                          stream);
  });
}

}  // extern "C"
