// C ABI of the operators of selective blocks (short convolution, state-space
// scan) and of gradient clipping: argument checks and dispatch, as in api_seq.cpp.
#include <hip/hip_runtime.h>

#include <algorithm>
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

}  // namespace

extern "C" {

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
