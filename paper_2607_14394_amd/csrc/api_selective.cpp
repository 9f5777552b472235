// C ABI of the operators of selective blocks (short convolution, state-space
// scan) and of gradient clipping: argument checks and dispatch, as in api_seq.cpp.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <initializer_list>
#include <string>
#include <vector>

#include "api_common.h"
#include "seq_checks.h"
#include "seq_internal.h"

namespace {

using namespace dtst;

// A range of memory; out: one that the call writes.
struct Range {
  uintptr_t at, end;
  bool out;
};

// Whether a written range shares a byte with any other.
bool any_shared(std::vector<Range>& r) {
  std::sort(r.begin(), r.end(), [](const Range& a, const Range& b) { return a.at < b.at; });
  uintptr_t read = 0, written = 0;  // the furthest ends so far
  for (const Range& x : r) {
    if (x.at < written || (x.out && x.at < read)) return true;
    uintptr_t& end = x.out ? written : read;
    end = std::max(end, x.end);
  }
  return false;
}

dtst_status check_tensors(const TensorList& l) {
  if (l.n < 0) return bad("need n >= 0");
  if (l.n > 0 && (l.p == nullptr || l.counts == nullptr || l.types == nullptr))
    return bad("tensors, counts or types is null");
  int64_t chunks = 0;
  for (int64_t i = 0; i < l.n; ++i) {
    const std::string name = "tensor " + std::to_string(i);
    if (l.counts[i] < 0 || l.counts[i] > kMost) return bad("count of " + name + " is out of range");
    if (!is_float_type(l.types[i])) return bad("type of " + name + " must be DTST_F32, DTST_BF16 or DTST_F16");
    if (l.counts[i] == 0) continue;
    DTST_TRY(check_align(l.p[i], type_size(l.types[i]), name.c_str()));
    if (l.out != nullptr) DTST_TRY(check_align(l.out[i], type_size(l.types[i]), ("out of " + name).c_str()));
    chunks += clip_chunks(l.counts[i]);
    if (chunks >= int64_t(1) << 31) return fail(DTST_ERR_UNSUPPORTED, "too many values");
  }
  return DTST_OK;
}

Range range_of(const void* p, int64_t bytes, bool out) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  return Range{at, at + uintptr_t(bytes), out};
}

dtst_status global_norm_workspace_of(int64_t n, const int64_t* counts, size_t* bytes) {
  if (bytes == nullptr) return bad("bytes is null");
  if (n < 0 || (n > 0 && counts == nullptr)) return bad("need n >= 0 and counts");
  for (int64_t i = 0; i < n; ++i)
    if (counts[i] < 0 || counts[i] > kMost) return bad("a count is out of range");
  *bytes = global_norm_workspace(TensorList{n, nullptr, nullptr, counts, nullptr});
  return ok();
}

dtst_status global_norm(const TensorList& l, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
  DTST_TRY(check_tensors(l));
  DTST_TRY(check_align(norm, 4, "norm"));
  const size_t need = global_norm_workspace(l);
  DTST_TRY(check_workspace(workspace, workspace_bytes, need));
  std::vector<Range> r{range_of(norm, 4, true), range_of(workspace, int64_t(need), true)};
  for (int64_t i = 0; i < l.n; ++i)
    if (l.counts[i] > 0) r.push_back(range_of(l.p[i], l.counts[i] * type_size(l.types[i]), false));
  if (need == 0) r.erase(r.begin() + 1);
  if (any_shared(r)) return bad("norm or workspace overlaps another array");
  const int e = timed(K_GLOBAL_NORM, stream, [&] { return launch_global_norm(l, norm, workspace, stream); });
  return device_status(e, "global norm launch");
}

dtst_status clip(const TensorList& l, const float* norm, float most, void* stream) {
  DTST_TRY(check_tensors(l));
  DTST_TRY(check_align(norm, 4, "norm"));
  if (!(most >= 0.f)) return bad("need most >= 0");
  std::vector<Range> r{range_of(norm, 4, false)};
  for (int64_t i = 0; i < l.n; ++i) {
    if (l.counts[i] == 0) continue;
    const int64_t bytes = l.counts[i] * type_size(l.types[i]);
    r.push_back(range_of(l.out != nullptr ? l.out[i] : l.p[i], bytes, true));
    if (l.out != nullptr && l.out[i] != l.p[i]) r.push_back(range_of(l.p[i], bytes, false));
  }
  if (any_shared(r)) return bad("a tensor that is written overlaps another array");
  const int e = timed(K_CLIP, stream, [&] { return launch_clip(l, norm, most, stream); });
  return device_status(e, "clip launch");
}

// The sizes of a scan (or, with states = taps - 1, of a convolution).
dtst_status check_sizes(int64_t batch, int64_t steps, int64_t features, int64_t states, int type) {
  if (batch < 0 || steps < 0 || features < 0) return bad("need batch, steps and features >= 0");
  if (!is_float_type(type)) return bad("type must be DTST_F32, DTST_BF16 or DTST_F16");
  if (features > (int64_t(1) << 28)) return fail(DTST_ERR_UNSUPPORTED, "features above 2^28");
  int64_t n = 0, m = 0;
  if (__builtin_mul_overflow(batch, steps, &n) || __builtin_mul_overflow(n, features, &m) || m > kMost ||
      __builtin_mul_overflow(n, states + 2, &m) || m > kMost || __builtin_mul_overflow(batch, features, &n) ||
      __builtin_mul_overflow(n, states + 2, &m) || m > kMost)
    return bad("problem size overflows the supported element counts");
  return DTST_OK;
}

dtst_status check_strides(std::initializer_list<const int64_t*> all) {
  for (const int64_t* s : all)
    for (int i = 0; i < 2; ++i)
      if (s[i] > kMost || s[i] < -kMost) return bad("a stride is too large");
  return DTST_OK;
}

dtst_status check_taps(int64_t taps) {
  if (taps < 1) return bad("need taps >= 1");
  if (taps > kConvMaxTaps) return fail(DTST_ERR_UNSUPPORTED, "taps above " + std::to_string(kConvMaxTaps));
  return DTST_OK;
}

dtst_status check_conv_desc(const dtst_conv_desc* d) {
  if (d == nullptr) return bad("descriptor is null");
  DTST_TRY(check_taps(d->taps));
  DTST_TRY(check_sizes(d->batch, d->steps, d->features, d->taps - 1, d->type));
  if (d->silu != 0 && d->silu != 1) return bad("silu must be 0 or 1");
  if (d->accumulate != 0 && d->accumulate != 1) return bad("accumulate must be 0 or 1");
  return check_strides({d->x_stride, d->y_stride, d->g_x_stride});
}

dtst_status check_states(int64_t states) {
  if (states < 1) return bad("need states >= 1");
  if (states > kScanMaxStates) return fail(DTST_ERR_UNSUPPORTED, "states above " + std::to_string(kScanMaxStates));
  return DTST_OK;
}

dtst_status check_scan_desc(const dtst_scan_desc* d) {
  if (d == nullptr) return bad("descriptor is null");
  DTST_TRY(check_states(d->states));
  DTST_TRY(check_sizes(d->batch, d->steps, d->features, d->states, d->type));
  if (d->accumulate != 0 && d->accumulate != 1) return bad("accumulate must be 0 or 1");
  return check_strides({d->x_stride, d->delta_stride, d->b_stride, d->c_stride, d->o_stride, d->y_stride, d->g_x_stride,
                        d->g_delta_stride, d->g_b_stride, d->g_c_stride, d->g_o_stride});
}

// (workgroups of 256 threads for 256 features of a segment; of up to 512 for 64 states
// that enter segments where there are several, of 256 to copy 256 where there are no steps)
dtst_status check_scan_grid(const dtst_scan_desc* d, bool adj) {
  const int64_t segments = scan_segments(d->batch, d->steps, d->features, d->states, adj);
  const int64_t states = d->batch * d->states * d->features;
  DTST_TRY(check_grid((d->features + 255) / 256 * segments * d->batch, 256));
  if (segments > 1) DTST_TRY(check_grid((states + 63) / 64, 512));
  return d->steps > 0 ? DTST_OK : check_grid((states + 255) / 256, 256);
}

dtst_status scan_workspace_of(int64_t batch, int64_t steps, int64_t features, int64_t states, bool adj, size_t* bytes) {
  if (bytes == nullptr) return bad("bytes is null");
  DTST_TRY(check_states(states));
  DTST_TRY(check_sizes(batch, steps, features, states, DTST_F32));
  dtst_scan_desc d{};
  d.batch = batch, d.steps = steps, d.features = features, d.states = states;
  *bytes = adj ? scan_adj_workspace(d) : scan_carry_bytes(d, false);
  return ok();
}

// Every written sequence and block apart from all others but those that it may be.
dtst_status check_outputs(std::initializer_list<const Sequence*> out, std::initializer_list<const Block*> out_blocks,
                          std::initializer_list<const Sequence*> in, std::initializer_list<const Block*> in_blocks,
                          const Block* inplace_out = nullptr, const Block* inplace_in = nullptr) {
  for (auto o = out.begin(); o != out.end(); ++o) {
    for (const Sequence* s : in) DTST_TRY(check_no_share(**o, *s));
    for (const Block* s : in_blocks) DTST_TRY(check_no_share(**o, *s));
    for (const Block* s : out_blocks) DTST_TRY(check_no_share(**o, *s));
    for (auto q = out.begin(); q != o; ++q) DTST_TRY(check_no_share(**o, **q));
  }
  for (auto o = out_blocks.begin(); o != out_blocks.end(); ++o) {
    for (const Sequence* s : in) DTST_TRY(check_no_share(*s, **o));
    for (const Block* s : in_blocks)
      if (!(*o == inplace_out && s == inplace_in && s->p == (*o)->p)) DTST_TRY(check_no_share(**o, *s));
    for (auto q = out_blocks.begin(); q != o; ++q) DTST_TRY(check_no_share(**o, **q));
  }
  return DTST_OK;
}

dtst_status conv(const dtst_conv_desc* d, const void* x, const float* weight, const float* bias, const void* state,
                 const int32_t* lengths, void* y, void* state_out, void* stream) {
  DTST_TRY(check_conv_desc(d));
  const int64_t B = d->batch, T = d->steps, F = d->features, rows = B * (d->taps - 1);
  if (B == 0 || F == 0) return ok();
  const int size = type_size(d->type);
  const Sequence sx{x, B, T, F, d->x_stride, size, "x"}, sy{y, B, T, F, d->y_stride, size, "y"};
  if (T > 0) {
    DTST_TRY(check_sequence(sx));
    DTST_TRY(check_sequence(sy));
    DTST_TRY(check_align(weight, 4, "weight"));
  }
  if (bias) DTST_TRY(check_align(bias, 4, "bias"));
  if (state) DTST_TRY(check_align(state, size, "state"));
  if (state_out) DTST_TRY(check_align(state_out, size, "state_out"));
  if (lengths) DTST_TRY(check_align(lengths, 4, "lengths"));
  DTST_TRY(check_grid(conv_groups(*d, false), 256));
  if (T == 0) DTST_TRY(check_grid((rows * F + 255) / 256, 256));  // (the state is copied)
  const Block bw{T > 0 ? weight : nullptr, d->taps * F * 4, "weight"}, bb{bias, F * 4, "bias"}, bn{lengths, B * 4, "lengths"};
  const Block bin{state, rows * F * size, "state"}, bout{state_out, rows * F * size, "state_out"};
  DTST_TRY(check_outputs({&sy}, {&bout}, {&sx}, {&bw, &bb, &bn, &bin}, &bout, &bin));
  const int e = timed(K_CONV, stream,
                      [&] { return launch_conv(*d, x, weight, bias, state, lengths, y, state_out, stream); });
  return device_status(e, "convolution launch");
}

dtst_status conv_adj(const dtst_conv_desc* d, const void* x, const float* weight, const float* bias, const void* state,
                     const int32_t* lengths, const void* g_y, const void* g_state_out, void* g_x, float* g_weight,
                     float* g_bias, void* g_state, void* workspace, size_t workspace_bytes, void* stream) {
  DTST_TRY(check_conv_desc(d));
  const int64_t B = d->batch, T = d->steps, F = d->features, rows = B * (d->taps - 1);
  if (F == 0) return ok();
  const bool steps = B > 0 && T > 0;
  const int size = type_size(d->type);
  const Sequence sx{x, B, T, F, d->x_stride, size, "x"}, sg{g_y, B, T, F, d->y_stride, size, "g_y"};
  const Sequence gx{g_x, B, T, F, d->g_x_stride, size, "g_x"};
  DTST_TRY(check_align(g_weight, 4, "g_weight"));
  if (steps) {
    for (const Sequence* s : {&sx, &sg, &gx}) DTST_TRY(check_sequence(*s));
    DTST_TRY(check_align(weight, 4, "weight"));
  }
  if (bias) DTST_TRY(check_align(bias, 4, "bias"));
  if (g_bias) DTST_TRY(check_align(g_bias, 4, "g_bias"));
  if (state) DTST_TRY(check_align(state, size, "state"));
  if (g_state_out) DTST_TRY(check_align(g_state_out, size, "g_state_out"));
  if (g_state) DTST_TRY(check_align(g_state, size, "g_state"));
  if (lengths) DTST_TRY(check_align(lengths, 4, "lengths"));
  const size_t need = conv_adj_workspace(*d);
  DTST_TRY(check_workspace(workspace, workspace_bytes, need));
  DTST_TRY(check_grid(conv_groups(*d, true), 256));
  if (!steps) DTST_TRY(check_grid((rows * F + 255) / 256, 256));  // (g_state_out is copied)
  DTST_TRY(check_grid(((d->taps + 1) * F + 31) / 32, 1024));
  const Block bw{steps ? weight : nullptr, d->taps * F * 4, "weight"}, bb{bias, F * 4, "bias"}, bn{lengths, B * 4, "lengths"};
  const Block bin{state, rows * F * size, "state"}, bgo{g_state_out, rows * F * size, "g_state_out"};
  const Block bgs{g_state, rows * F * size, "g_state"}, bgw{g_weight, d->taps * F * 4, "g_weight"};
  const Block bgb{g_bias, F * 4, "g_bias"}, bws{need ? workspace : nullptr, int64_t(need), "workspace"};
  DTST_TRY(check_outputs({&gx}, {&bgw, &bgb, &bgs, &bws}, {&sx, &sg}, {&bw, &bb, &bn, &bin, &bgo}));
  const int e = timed(K_CONV_ADJ, stream, [&] {
    return launch_conv_adj(*d, x, weight, bias, state, lengths, g_y, g_state_out, g_x, g_weight, g_bias, g_state,
                           workspace, stream);
  });
  return device_status(e, "convolution backward launch");
}

dtst_status scan(const dtst_scan_desc* d, const void* x, const void* delta, const float* a, const void* b,
                 const void* c, const float* skip, const void* o, const float* h_zero, const int32_t* lengths, void* y,
                 float* h_out, float* states, void* workspace, size_t workspace_bytes, void* stream) {
  DTST_TRY(check_scan_desc(d));
  if (d->batch == 0 || d->features == 0) return ok();
  const int64_t B = d->batch, T = d->steps, F = d->features, N = d->states;
  const int size = type_size(d->type);
  const Sequence sx{x, B, T, F, d->x_stride, size, "x"}, sd{delta, B, T, F, d->delta_stride, size, "delta"};
  const Sequence sb{b, B, T, N, d->b_stride, size, "b"}, sc{c, B, T, N, d->c_stride, size, "c"};
  const Sequence so{o, B, T, F, d->o_stride, size, "o"}, sy{y, B, T, F, d->y_stride, size, "y"};
  if (T > 0) {
    for (const Sequence* s : {&sx, &sd, &sb, &sc, &sy}) DTST_TRY(check_sequence(*s));
    if (o) DTST_TRY(check_sequence(so));
    DTST_TRY(check_align(a, 4, "a"));
  }
  if (skip) DTST_TRY(check_align(skip, 4, "d"));
  if (h_zero) DTST_TRY(check_align(h_zero, 4, "h_zero"));
  if (h_out) DTST_TRY(check_align(h_out, 4, "h_out"));
  if (states) DTST_TRY(check_align(states, 4, "states"));
  if (lengths) DTST_TRY(check_align(lengths, 4, "lengths"));
  const size_t need = scan_carry_bytes(*d, false);
  DTST_TRY(check_workspace(workspace, workspace_bytes, need));
  DTST_TRY(check_scan_grid(d, false));
  const int64_t one = B * N * F * 4, spans = (T + DTST_SCAN_SPAN - 1) / DTST_SCAN_SPAN;
  const Block ba{T > 0 ? a : nullptr, N * F * 4, "a"}, bd{skip, F * 4, "d"}, bn{lengths, B * 4, "lengths"};
  const Block bin{h_zero, one, "h_zero"}, bout{h_out, one, "h_out"}, bst{states, one * spans, "states"};
  const Block bws{need ? workspace : nullptr, int64_t(need), "workspace"};
  DTST_TRY(check_outputs({&sy}, {&bout, &bst, &bws}, {&sx, &sd, &sb, &sc, &so}, {&ba, &bd, &bn, &bin}, &bout, &bin));
  const int e = timed(K_SCAN, stream, [&] {
    return launch_scan(*d, x, delta, a, b, c, skip, o, h_zero, lengths, y, h_out, states, workspace, stream);
  });
  return device_status(e, "scan launch");
}

dtst_status scan_adj(const dtst_scan_desc* d, const void* x, const void* delta, const float* a, const void* b,
                     const void* c, const float* skip, const void* o, const int32_t* lengths, const float* states,
                     const void* g_y, const float* g_h, void* g_x, void* g_delta, float* g_a, void* g_b, void* g_c,
                     float* g_skip, void* g_o, float* g_hzero, void* workspace, size_t workspace_bytes, void* stream) {
  DTST_TRY(check_scan_desc(d));
  const int64_t B = d->batch, T = d->steps, F = d->features, N = d->states;
  if (F == 0) return ok();
  const bool steps = B > 0 && T > 0;
  if (steps && (o != nullptr) != (g_o != nullptr)) return bad("g_o goes with o");
  if (g_skip != nullptr && skip == nullptr) return bad("g_d goes with d");
  const int size = type_size(d->type);
  const Sequence sx{x, B, T, F, d->x_stride, size, "x"}, sd{delta, B, T, F, d->delta_stride, size, "delta"};
  const Sequence sb{b, B, T, N, d->b_stride, size, "b"}, sc{c, B, T, N, d->c_stride, size, "c"};
  const Sequence so{o, B, T, F, d->o_stride, size, "o"}, sg{g_y, B, T, F, d->y_stride, size, "g_y"};
  const Sequence gx{g_x, B, T, F, d->g_x_stride, size, "g_x"}, gd{g_delta, B, T, F, d->g_delta_stride, size, "g_delta"};
  const Sequence gb{g_b, B, T, N, d->g_b_stride, size, "g_b"}, gc{g_c, B, T, N, d->g_c_stride, size, "g_c"};
  const Sequence go{g_o, B, T, F, d->g_o_stride, size, "g_o"};
  DTST_TRY(check_align(g_a, 4, "g_a"));
  if (steps) {
    for (const Sequence* s : {&sx, &sd, &sb, &sc, &sg, &gx, &gd, &gb, &gc}) DTST_TRY(check_sequence(*s));
    if (o)
      for (const Sequence* s : {&so, &go}) DTST_TRY(check_sequence(*s));
    DTST_TRY(check_align(a, 4, "a"));
    DTST_TRY(check_align(states, 4, "states"));
  }
  if (skip) DTST_TRY(check_align(skip, 4, "d"));
  if (g_skip) DTST_TRY(check_align(g_skip, 4, "g_d"));
  if (g_h) DTST_TRY(check_align(g_h, 4, "g_h"));
  if (g_hzero) DTST_TRY(check_align(g_hzero, 4, "g_hzero"));
  if (lengths) DTST_TRY(check_align(lengths, 4, "lengths"));
  const size_t need = scan_adj_workspace(*d);
  DTST_TRY(check_workspace(workspace, workspace_bytes, need));
  DTST_TRY(check_scan_grid(d, true));
  // (a wave for 64 features of a segment; four waves for four times 64 of a span's g_b and g_c)
  DTST_TRY(check_grid((F + 63) / 64 * scan_segments(B, T, F, N, true) * B, 64));
  const int64_t one = B * N * F * 4, spans = (T + DTST_SCAN_SPAN - 1) / DTST_SCAN_SPAN;
  DTST_TRY(check_grid((B * spans * ((2 * N * DTST_SCAN_SPAN + 63) / 64) + 3) / 4, 256));
  DTST_TRY(check_grid(((N + 1) * F + 31) / 32, 1024));
  const Block ba{steps ? a : nullptr, N * F * 4, "a"}, bd{skip, F * 4, "d"}, bn{lengths, B * 4, "lengths"};
  const Block bst{steps ? states : nullptr, one * spans, "states"}, bin{g_h, one, "g_h"}, bout{g_hzero, one, "g_hzero"};
  const Block bga{g_a, N * F * 4, "g_a"}, bgd{g_skip, F * 4, "g_d"};
  const Block bws{need ? workspace : nullptr, int64_t(need), "workspace"};
  DTST_TRY(check_outputs({&gx, &gd, &gb, &gc, &go}, {&bga, &bgd, &bout, &bws}, {&sx, &sd, &sb, &sc, &so, &sg},
                         {&ba, &bd, &bn, &bst, &bin}, &bout, &bin));
  const int e = timed(K_SCAN_ADJ, stream, [&] {
    return launch_scan_adj(*d, x, delta, a, b, c, skip, o, lengths, states, g_y, g_h, g_x, g_delta, g_a, g_b, g_c, g_skip,
                           g_o, g_hzero, workspace, stream);
  });
  return device_status(e, "scan backward launch");
}

}  // namespace

extern "C" {

dtst_status dtst_conv(const dtst_conv_desc* d, const void* x, const float* weight, const float* bias, const void* state,
                      const int32_t* lengths, void* y, void* state_out, void* stream) {
  return guarded([&] { return conv(d, x, weight, bias, state, lengths, y, state_out, stream); });
}

dtst_status dtst_conv_adj_workspace(int64_t batch, int64_t steps, int64_t features, int64_t taps, size_t* bytes) {
  return guarded([&] {
    if (bytes == nullptr) return bad("bytes is null");
    DTST_TRY(check_taps(taps));
    DTST_TRY(check_sizes(batch, steps, features, taps - 1, DTST_F32));
    dtst_conv_desc d{};
    d.batch = batch, d.steps = steps, d.features = features, d.taps = taps;
    *bytes = conv_adj_workspace(d);
    return ok();
  });
}

dtst_status dtst_conv_adj(const dtst_conv_desc* d, const void* x, const float* weight, const float* bias,
                          const void* state, const int32_t* lengths, const void* g_y, const void* g_state_out, void* g_x,
                          float* g_weight, float* g_bias, void* g_state, void* workspace, size_t workspace_bytes,
                          void* stream) {
  return guarded([&] {
    return conv_adj(d, x, weight, bias, state, lengths, g_y, g_state_out, g_x, g_weight, g_bias, g_state, workspace,
                    workspace_bytes, stream);
  });
}

dtst_status dtst_scan_adj_workspace(int64_t batch, int64_t steps, int64_t features, int64_t states, size_t* bytes) {
  return guarded([&] { return scan_workspace_of(batch, steps, features, states, true, bytes); });
}

dtst_status dtst_scan_adj(const dtst_scan_desc* desc, const void* x, const void* delta, const float* a, const void* b,
                          const void* c, const float* d, const void* o, const int32_t* lengths, const float* states,
                          const void* g_y, const float* g_h, void* g_x, void* g_delta, float* g_a, void* g_b, void* g_c,
                          float* g_d, void* g_o, float* g_hzero, void* workspace, size_t workspace_bytes, void* stream) {
  return guarded([&] {
    return scan_adj(desc, x, delta, a, b, c, d, o, lengths, states, g_y, g_h, g_x, g_delta, g_a, g_b, g_c, g_d, g_o,
                    g_hzero, workspace, workspace_bytes, stream);
  });
}

dtst_status dtst_scan_workspace(int64_t batch, int64_t steps, int64_t features, int64_t states, size_t* bytes) {
  return guarded([&] { return scan_workspace_of(batch, steps, features, states, false, bytes); });
}

dtst_status dtst_scan(const dtst_scan_desc* desc, const void* x, const void* delta, const float* a, const void* b,
                      const void* c, const float* d, const void* o, const float* h_zero, const int32_t* lengths,
                      void* y, float* h_out, float* states, void* workspace, size_t workspace_bytes, void* stream) {
  return guarded([&] {
    return scan(desc, x, delta, a, b, c, d, o, h_zero, lengths, y, h_out, states, workspace, workspace_bytes, stream);
  });
}

dtst_status dtst_global_norm_workspace(int64_t n, const int64_t* counts, size_t* bytes) {
  return guarded([&] { return global_norm_workspace_of(n, counts, bytes); });
}

dtst_status dtst_global_norm(int64_t n, const void* const* tensors, const int64_t* counts, const int32_t* types,
                             float* norm, void* workspace, size_t workspace_bytes, void* stream) {
  return guarded([&] {
    return global_norm(TensorList{n, const_cast<void* const*>(tensors), nullptr, counts, types}, norm, workspace,
                       workspace_bytes, stream);
  });
}

dtst_status dtst_clip(int64_t n, void* const* tensors, const int64_t* counts, const int32_t* types, const float* norm,
                      float most, void* const* out, void* stream) {
  return guarded([&] { return clip(TensorList{n, tensors, out, counts, types}, norm, most, stream); });
}

}  // extern "C"
