// Argument checks that the operators on latent sequences share (api_seq.cpp,
// api_selective.cpp).  Host only.
#pragma once

#include <algorithm>
#include <cstdint>
#include <cstdlib>
#include <string>
#include <utility>

#include "api_common.h"

namespace dtst {

template <class F>
inline dtst_status guarded(F&& f) {
  try {
    return f();
  } catch (...) {
    return DTST_ERR_OUT_OF_MEMORY;  // (the host allocations of messages and event records are all that throws)
  }
}

inline dtst_status bad(const std::string& msg) { return fail(DTST_ERR_INVALID_ARG, msg); }

inline int type_size(int t) { return t == DTST_F32 ? 4 : t == DTST_E4M3 ? 1 : 2; }
inline bool is_float_type(int t) { return t == DTST_F32 || t == DTST_BF16 || t == DTST_F16; }

inline dtst_status check_align(const void* p, uintptr_t align, const char* name) {
  if (p == nullptr) return bad(std::string(name) + " is null");
  if (reinterpret_cast<uintptr_t>(p) % align != 0)
    return bad(std::string(name) + " is not aligned to " + std::to_string(align) + " bytes");
  return DTST_OK;
}

// Element counts and strides whose products stay far inside 64 bits.
constexpr int64_t kMost = int64_t(1) << 50;
inline dtst_status check_extent(int64_t rows, int64_t ld, const char* name) {
  int64_t n = 0;
  if (__builtin_mul_overflow(rows, ld, &n) || n > kMost) return bad(std::string(name) + " is too large");
  return DTST_OK;
}

// A strided (rows, cols) array.
struct Array {
  const void* p;
  int64_t rows, cols, ld;
  int size;
  const char* name;
};

inline dtst_status check_array(const Array& a, uintptr_t align) {
  DTST_TRY(check_align(a.p, align, a.name));
  if (a.ld < a.cols) return bad(std::string("stride of ") + a.name + " is below its row");
  return check_extent(a.rows, a.ld * a.size, a.name);
}

// The rows of a strided array in bytes: `outer` groups of `inner` rows of `row`
// bytes, each group's rows before the next group's first.
struct Rows {
  int64_t at, outer, outer_ld, inner, inner_ld, row;
};
inline bool is_dense(const Rows& r) {
  return (r.inner <= 1 || r.inner_ld == r.row) && (r.outer <= 1 || r.outer_ld == r.inner * r.row);
}
inline int64_t extent(const Rows& r) { return (r.outer - 1) * r.outer_ld + (r.inner - 1) * r.inner_ld + r.row; }

// Whether a row of r has a byte of [at, at + n).
inline bool share(const Rows& r, int64_t at, int64_t n) {
  const int64_t most = at + n - 1 - r.at;                           // a row that does starts here at the latest,
  const int64_t least = std::max<int64_t>(at - r.row + 1 - r.at, 0);  // here at the earliest
  if (n <= 0 || most < least) return false;
  const int64_t o = r.outer_ld > 0 ? std::min(least / r.outer_ld, r.outer - 1) : 0, rest = least - o * r.outer_ld;
  const int64_t i = r.inner_ld > 0 ? (rest + r.inner_ld - 1) / r.inner_ld : rest > 0 ? r.inner : 0;
  if (i < r.inner) return o * r.outer_ld + i * r.inner_ld <= most;
  return o + 1 < r.outer && (o + 1) * r.outer_ld <= most;
}

inline Rows rows_of(const Array& a) {
  return Rows{int64_t(reinterpret_cast<uintptr_t>(a.p)), a.rows, a.rows > 1 ? a.ld * a.size : 0, 1, 0, a.cols * a.size};
}

// Whether two arrays share an element.  Column ranges of one array (equal row
// strides, rows apart) do not; of unlike strides, where neither is without gaps,
// those that reach into each other's range are taken to.
inline bool share(const Array& a, const Array& b) {
  if (a.p == nullptr || b.p == nullptr || a.rows < 1 || b.rows < 1) return false;
  const uintptr_t pa = reinterpret_cast<uintptr_t>(a.p), pb = reinterpret_cast<uintptr_t>(b.p);
  const uintptr_t la = uintptr_t(a.ld) * a.size, lb = uintptr_t(b.ld) * b.size;
  const uintptr_t wa = uintptr_t(a.cols) * a.size, wb = uintptr_t(b.cols) * b.size;
  const uintptr_t ea = pa + (a.rows - 1) * la + wa, eb = pb + (b.rows - 1) * lb + wb;
  if (pa >= eb || pb >= ea) return false;
  const Rows ra = rows_of(a), rb = rows_of(b);
  if (is_dense(ra)) return share(rb, ra.at, extent(ra));
  if (is_dense(rb)) return share(ra, rb.at, extent(rb));
  if (la == lb && a.rows > 1 && b.rows > 1) {
    const uintptr_t off = pb >= pa ? (pb - pa) % la : (la - (pa - pb) % la) % la;  // b's column 0 in a's rows
    return off < wa || la - off < wb;
  }
  return true;
}

inline bool same(const Array& a, const Array& b) { return a.p == b.p && (a.ld == b.ld || a.rows <= 1) && a.size == b.size; }

inline dtst_status check_apart(const Array& out, const Array& other, bool may_be_same) {
  if (share(out, other) && !(may_be_same && same(out, other)))
    return bad(std::string(out.name) + " and " + other.name + " overlap");
  return DTST_OK;
}

// Codes and scales of an 8-bit (rows, k) array.
inline Array codes_of(const void* p, int64_t rows, int64_t k, int64_t ld, const char* name) {
  return Array{p, rows, (k + 127) / 128 * 128, ld, 1, name};
}
inline Array scales_of(const void* p, int64_t rows, int64_t k, int64_t ld, const char* name) {
  return Array{p, rows, ((k + 127) / 128 + 3) / 4 * 4, ld, 1, name};
}
inline dtst_status check_codes(const Array& q, const Array& s) {
  DTST_TRY(check_array(q, 16));
  DTST_TRY(check_array(s, 4));
  if (q.ld % 16 != 0) return bad(std::string("stride of ") + q.name + " is no multiple of 16");
  if (s.ld % 4 != 0) return bad(std::string("stride of ") + s.name + " is no multiple of 4");
  return DTST_OK;
}

// Workgroups of a launch: a dimension holds fewer than 2^32 threads.
inline dtst_status check_grid(int64_t groups, int64_t threads) {
  if (groups > (int64_t(1) << 32) / threads - 1) return fail(DTST_ERR_UNSUPPORTED, "too many rows for one launch");
  return DTST_OK;
}

inline dtst_status check_workspace(const void* ws, size_t have, size_t need) {
  if (need == 0) return DTST_OK;
  if (have < need)
    return bad("workspace too small: need " + std::to_string(need) + " bytes, got " + std::to_string(have));
  return check_ptr(ws, "workspace");
}

// A (batch, steps, features) array with strides of batch entries and steps.
struct Sequence {
  const void* p;
  int64_t batch, steps, features;
  const int64_t* st;
  int size;  // of an element
  const char* name;
};

inline dtst_status check_sequence(const Sequence& s) {
  DTST_TRY(check_align(s.p, s.size, s.name));
  const int64_t sb = s.st[0], t = s.st[1];
  if ((s.steps > 1 && t < s.features) || (s.batch > 1 && sb < s.features) || sb < 0 || t < 0)
    return bad(std::string("strides of ") + s.name + " are below its rows");
  // entries apart from each other: step rows inside an entry's stride, or entries inside a step's
  if (s.batch > 1 && s.steps > 1) {
    const bool by_entry = sb / t >= s.steps || (sb - (s.steps - 1) * t >= s.features && sb >= t);
    const bool by_step = t / sb >= s.batch || (t - (s.batch - 1) * sb >= s.features && t >= sb);
    if (!by_entry && !by_step) return bad(std::string("rows of ") + s.name + " overlap");
  }
  DTST_TRY(check_extent(s.batch, sb * s.size, s.name));
  return check_extent(s.steps, t * s.size, s.name);
}

inline bool is_empty(const Sequence& s) { return s.p == nullptr || s.batch < 1 || s.steps < 1 || s.features < 1; }

// (Of a sequence whose strides check_sequence takes.)
inline Rows rows_of(const Sequence& s) {
  Rows r{int64_t(reinterpret_cast<uintptr_t>(s.p)), s.batch, s.st[0] * s.size, s.steps, s.st[1] * s.size,
         s.features * s.size};
  if (r.outer <= 1) r.outer_ld = 0;
  if (r.inner <= 1) r.inner_ld = 0;
  if (r.outer_ld < r.inner_ld) std::swap(r.outer, r.inner), std::swap(r.outer_ld, r.inner_ld);
  return r;
}

// Whether two sequences share an element.  Of unlike strides, where neither is
// without gaps, only a common first element tells.
inline bool share(const Sequence& a, const Sequence& b) {
  if (is_empty(a) || is_empty(b)) return false;
  const Rows ra = rows_of(a), rb = rows_of(b);
  if (ra.at >= rb.at + extent(rb) || rb.at >= ra.at + extent(ra)) return false;
  if (is_dense(ra)) return share(rb, ra.at, extent(ra));
  if (is_dense(rb)) return share(ra, rb.at, extent(rb));
  if (ra.outer != rb.outer || ra.outer_ld != rb.outer_ld || ra.inner != rb.inner || ra.inner_ld != rb.inner_ld)
    return ra.at == rb.at;
  // Rows of the two lie j outer and i inner strides less delta apart: the nearest
  // of either sign.
  const auto below = [](int64_t x, int64_t ld) { return ld > 0 ? (x >= 0 ? x / ld : -((ld - 1 - x) / ld)) : 0; };
  const int64_t delta = rb.at - ra.at, j0 = below(delta, ra.outer_ld);
  for (int64_t j = j0; j <= j0 + 1; ++j) {
    if (j <= -ra.outer || j >= ra.outer) continue;
    const int64_t rest = delta - j * ra.outer_ld, i0 = below(rest, ra.inner_ld);
    for (int64_t i = i0; i <= i0 + 1; ++i)
      // (off: from a's row to b's)
      if (const int64_t off = rest - i * ra.inner_ld; i > -ra.inner && i < ra.inner && off < ra.row && -off < rb.row)
        return true;
  }
  return false;
}

inline dtst_status check_no_share(const Sequence& out, const Sequence& other) {
  if (share(out, other)) return bad(std::string(out.name) + " and " + other.name + " overlap");
  return DTST_OK;
}

// An array without gaps: states, lengths, the workspace.
struct Block {
  const void* p;
  int64_t bytes;
  const char* name;
};
inline dtst_status check_no_share(const Block& out, const Block& other) {
  if (out.p == nullptr || other.p == nullptr || out.bytes <= 0 || other.bytes <= 0) return DTST_OK;
  const uintptr_t a = reinterpret_cast<uintptr_t>(out.p), b = reinterpret_cast<uintptr_t>(other.p);
  if (a < b + uintptr_t(other.bytes) && b < a + uintptr_t(out.bytes)) return bad(std::string(out.name) + " and " + other.name + " overlap");
  return DTST_OK;
}
inline dtst_status check_no_share(const Sequence& s, const Block& b) {
  if (is_empty(s) || b.p == nullptr) return DTST_OK;
  if (share(rows_of(s), int64_t(reinterpret_cast<uintptr_t>(b.p)), b.bytes))
    return bad(std::string(s.name) + " and " + b.name + " overlap");
  return DTST_OK;
}

}  // namespace dtst
