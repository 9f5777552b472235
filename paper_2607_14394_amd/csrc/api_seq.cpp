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
#include "seq_internal.h"

namespace {

using namespace dtst;

template <class F>
dtst_status guarded(F&& f) {
  try {
    return f();
  } catch (...) {
    return DTST_ERR_OUT_OF_MEMORY;  // (the host allocations of messages and event records are all that throws)
  }
}

dtst_status bad(const std::string& msg) { return fail(DTST_ERR_INVALID_ARG, msg); }

int type_size(int t) { return t == DTST_F32 ? 4 : t == DTST_E4M3 ? 1 : 2; }
bool is_float_type(int t) { return t == DTST_F32 || t == DTST_BF16 || t == DTST_F16; }

dtst_status check_align(const void* p, uintptr_t align, const char* name) {
  if (p == nullptr) return bad(std::string(name) + " is null");
  if (reinterpret_cast<uintptr_t>(p) % align != 0)
    return bad(std::string(name) + " is not aligned to " + std::to_string(align) + " bytes");
  return DTST_OK;
}

// Element counts and strides whose products stay far inside 64 bits.
constexpr int64_t kMost = int64_t(1) << 50;
dtst_status check_extent(int64_t rows, int64_t ld, const char* name) {
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

dtst_status check_array(const Array& a, uintptr_t align) {
  DTST_TRY(check_align(a.p, align, a.name));
  if (a.ld < a.cols) return bad(std::string("stride of ") + a.name + " is below its row");
  return check_extent(a.rows, a.ld * a.size, a.name);
}

// The rows of a strided array in bytes: `outer` groups of `inner` rows of `row`
// bytes, each group's rows before the next group's first.
struct Rows {
  int64_t at, outer, outer_ld, inner, inner_ld, row;
};
bool is_dense(const Rows& r) {
  return (r.inner <= 1 || r.inner_ld == r.row) && (r.outer <= 1 || r.outer_ld == r.inner * r.row);
}
int64_t extent(const Rows& r) { return (r.outer - 1) * r.outer_ld + (r.inner - 1) * r.inner_ld + r.row; }

// Whether a row of r has a byte of [at, at + n).
bool share(const Rows& r, int64_t at, int64_t n) {
  const int64_t most = at + n - 1 - r.at;                           // a row that does starts here at the latest,
  const int64_t least = std::max<int64_t>(at - r.row + 1 - r.at, 0);  // here at the earliest
  if (n <= 0 || most < least) return false;
  const int64_t o = r.outer_ld > 0 ? std::min(least / r.outer_ld, r.outer - 1) : 0, rest = least - o * r.outer_ld;
  const int64_t i = r.inner_ld > 0 ? (rest + r.inner_ld - 1) / r.inner_ld : rest > 0 ? r.inner : 0;
  if (i < r.inner) return o * r.outer_ld + i * r.inner_ld <= most;
  return o + 1 < r.outer && (o + 1) * r.outer_ld <= most;
}

Rows rows_of(const Array& a) {
  return Rows{int64_t(reinterpret_cast<uintptr_t>(a.p)), a.rows, a.rows > 1 ? a.ld * a.size : 0, 1, 0, a.cols * a.size};
}

// Whether two arrays share an element.  Column ranges of one array (equal row
// strides, rows apart) do not; of unlike strides, where neither is without gaps,
// those that reach into each other's range are taken to.
bool share(const Array& a, const Array& b) {
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

bool same(const Array& a, const Array& b) { return a.p == b.p && (a.ld == b.ld || a.rows <= 1) && a.size == b.size; }

dtst_status check_apart(const Array& out, const Array& other, bool may_be_same) {
  if (share(out, other) && !(may_be_same && same(out, other)))
    return bad(std::string(out.name) + " and " + other.name + " overlap");
  return DTST_OK;
}

// Codes and scales of an 8-bit (rows, k) array.
Array codes_of(const void* p, int64_t rows, int64_t k, int64_t ld, const char* name) {
  return Array{p, rows, (k + 127) / 128 * 128, ld, 1, name};
}
Array scales_of(const void* p, int64_t rows, int64_t k, int64_t ld, const char* name) {
  return Array{p, rows, ((k + 127) / 128 + 3) / 4 * 4, ld, 1, name};
}
dtst_status check_codes(const Array& q, const Array& s) {
  DTST_TRY(check_array(q, 16));
  DTST_TRY(check_array(s, 4));
  if (q.ld % 16 != 0) return bad(std::string("stride of ") + q.name + " is no multiple of 16");
  if (s.ld % 4 != 0) return bad(std::string("stride of ") + s.name + " is no multiple of 4");
  return DTST_OK;
}

// Workgroups of a launch: a dimension holds fewer than 2^32 threads.
dtst_status check_grid(int64_t groups, int64_t threads) {
  if (groups > (int64_t(1) << 32) / threads - 1) return fail(DTST_ERR_UNSUPPORTED, "too many rows for one launch");
  return DTST_OK;
}

dtst_status check_workspace(const void* ws, size_t have, size_t need) {
  if (need == 0) return DTST_OK;
  if (have < need)
    return bad("workspace too small: need " + std::to_string(need) + " bytes, got " + std::to_string(have));
  return check_ptr(ws, "workspace");
}

dtst_status check_norm_types(int x_type, int res_type) {
  if (!is_float_type(x_type)) return bad("x_type must be DTST_F32, DTST_BF16 or DTST_F16");
  if (res_type != x_type && res_type != DTST_F32) return bad("res_type must be x_type or DTST_F32");
  return DTST_OK;
}

dtst_status check_rows_cols(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 1) return bad("need rows >= 0 and cols >= 1");
  return DTST_OK;
}

dtst_status rms_norm(const dtst_norm_desc* d, const void* x, const void* res, const float* weight, void* sum_out,
                     void* y, void* scale, float* rstd, void* stream) {
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
  DTST_TRY(check_array(ax, sx));
  DTST_TRY(check_align(weight, 4, "weight"));
  if (res) DTST_TRY(check_array(ar, sr));
  if (sum_out) DTST_TRY(check_array(as, sr));
  if (rstd) DTST_TRY(check_align(rstd, 4, "rstd"));
  DTST_TRY(q8 ? check_codes(ay, asc) : check_array(ay, sx));
  const NormGrid grid = rms_norm_grid(d->rows, d->cols);
  DTST_TRY(check_grid(grid.groups, grid.threads));
  DTST_TRY(check_apart(as, ar, true));
  DTST_TRY(check_apart(as, ax, res == nullptr));
  DTST_TRY(check_apart(ay, ax, !q8));
  for (const Array* out : {&as, &ay, &asc, &art}) DTST_TRY(check_apart(*out, aw, false));
  for (const Array* in : {&ax, &ar}) {
    DTST_TRY(check_apart(asc, *in, false));
    DTST_TRY(check_apart(art, *in, false));
  }
  DTST_TRY(check_apart(ay, ar, false));
  DTST_TRY(check_apart(ay, as, false));
  DTST_TRY(check_apart(asc, ay, false));
  DTST_TRY(check_apart(asc, as, false));
  for (const Array* out : {&as, &ay, &asc}) DTST_TRY(check_apart(art, *out, false));
  const int e = timed(K_NORM, stream,
                      [&] { return launch_rms_norm(*d, x, res, weight, sum_out, y, scale, rstd, stream); });
  return device_status(e, "norm launch");
}

dtst_status rms_norm_adj(const dtst_norm_adj_desc* d, const void* g_y, const void* u, const float* weight,
                         const float* rstd, const void* g_sum, void* g_u, void* g_x, float* g_weight, void* workspace,
                         size_t workspace_bytes, void* stream) {
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
  const Array agw{g_weight, 1, d->cols, d->cols, 4, "g_weight"};
  const size_t need = rms_norm_adj_workspace(d->rows, d->cols);
  const Array aws{workspace, 1, int64_t(need), int64_t(need), 1, "workspace"};
  DTST_TRY(check_align(g_weight, 4, "g_weight"));
  DTST_TRY(check_workspace(workspace, workspace_bytes, need));
  if (d->rows > 0) {
    DTST_TRY(check_array(ag, sx));
    DTST_TRY(check_array(au, sr));
    DTST_TRY(check_align(weight, 4, "weight"));
    DTST_TRY(check_align(rstd, 4, "rstd"));
    if (g_sum) DTST_TRY(check_array(as, sr));
    DTST_TRY(check_array(agu, sr));
    if (g_x) DTST_TRY(check_array(agx, sx));
    DTST_TRY(check_apart(agu, as, true));
    for (const Array* in : {&ag, &au, &aw, &art}) DTST_TRY(check_apart(agu, *in, false));
    for (const Array* in : {&ag, &au, &as, &aw, &art, &agu}) DTST_TRY(check_apart(agx, *in, false));
    for (const Array* in : {&ag, &au, &as, &aw, &art, &agu, &agx}) {
      DTST_TRY(check_apart(agw, *in, false));
      DTST_TRY(check_apart(aws, *in, false));
    }
  }
  DTST_TRY(check_apart(aws, agw, false));
  const int e = timed(K_NORM_ADJ, stream, [&] {
    return launch_rms_norm_adj(*d, g_y, u, weight, rstd, g_sum, g_u, g_x, g_weight, workspace, stream);
  });
  return device_status(e, "norm backward launch");
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

// A (batch, steps, features) array with strides of batch entries and steps.
struct Sequence {
  const void* p;
  const int64_t* st;
  const char* name;
};

dtst_status check_sequence(const dtst_recurrence_desc* d, const Sequence& s, int size) {
  DTST_TRY(check_align(s.p, size, s.name));
  const int64_t sb = s.st[0], t = s.st[1];
  if ((d->steps > 1 && t < d->features) || (d->batch > 1 && sb < d->features) || sb < 0 || t < 0)
    return bad(std::string("strides of ") + s.name + " are below its rows");
  // entries apart from each other: step rows inside an entry's stride, or entries inside a step's
  if (d->batch > 1 && d->steps > 1) {
    const bool by_entry = sb / t >= d->steps || (sb - (d->steps - 1) * t >= d->features && sb >= t);
    const bool by_step = t / sb >= d->batch || (t - (d->batch - 1) * sb >= d->features && t >= sb);
    if (!by_entry && !by_step) return bad(std::string("rows of ") + s.name + " overlap");
  }
  DTST_TRY(check_extent(d->batch, sb * size, s.name));
  return check_extent(d->steps, t * size, s.name);
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

// (Of a sequence whose strides check_sequence takes.)
Rows rows_of(const dtst_recurrence_desc* d, const Sequence& s, int size) {
  Rows r{int64_t(reinterpret_cast<uintptr_t>(s.p)), d->batch, s.st[0] * size, d->steps, s.st[1] * size, d->features * size};
  if (r.outer <= 1) r.outer_ld = 0;
  if (r.inner <= 1) r.inner_ld = 0;
  if (r.outer_ld < r.inner_ld) std::swap(r.outer, r.inner), std::swap(r.outer_ld, r.inner_ld);
  return r;
}

// Whether two sequences share an element.  Of unlike strides, where neither is
// without gaps, only a common first element tells.
bool share(const dtst_recurrence_desc* d, const Sequence& a, const Sequence& b, int size) {
  if (a.p == nullptr || b.p == nullptr || d->steps < 1) return false;
  const Rows ra = rows_of(d, a, size), rb = rows_of(d, b, size);
  if (ra.at >= rb.at + extent(rb) || rb.at >= ra.at + extent(ra)) return false;
  if (is_dense(ra)) return share(rb, ra.at, extent(ra));
  if (is_dense(rb)) return share(ra, rb.at, extent(rb));
  if (ra.outer != rb.outer || ra.outer_ld != rb.outer_ld || ra.inner_ld != rb.inner_ld) return ra.at == rb.at;
  // Rows of the two lie j outer and i inner strides less delta apart: the nearest
  // of either sign.
  const auto below = [](int64_t x, int64_t ld) { return ld > 0 ? (x >= 0 ? x / ld : -((ld - 1 - x) / ld)) : 0; };
  const int64_t delta = rb.at - ra.at, j0 = below(delta, ra.outer_ld);
  for (int64_t j = j0; j <= j0 + 1; ++j) {
    if (j <= -ra.outer || j >= ra.outer) continue;
    const int64_t rest = delta - j * ra.outer_ld, i0 = below(rest, ra.inner_ld);
    for (int64_t i = i0; i <= i0 + 1; ++i)
      if (i > -ra.inner && i < ra.inner && std::abs(rest - i * ra.inner_ld) < ra.row) return true;
  }
  return false;
}

// (one workgroup of 64 lanes a step's features, or of 512 for each 128 steps)
dtst_status check_recurrence_grid(const dtst_recurrence_desc* d) {
  const int64_t tiles = d->batch * ((d->features + 63) / 64), spans = (d->steps + 127) / 128;
  return check_grid(tiles * (spans > 0 ? spans : 1), d->steps <= 1 ? 64 : 512);
}

dtst_status check_no_share(const dtst_recurrence_desc* d, const Sequence& out, const Sequence& other, int size) {
  if (share(d, out, other, size)) return bad(std::string(out.name) + " and " + other.name + " overlap");
  return DTST_OK;
}

// An array without gaps: states, lengths, the workspace.
struct Block {
  const void* p;
  int64_t bytes;
  const char* name;
};
dtst_status check_no_share(const Block& out, const Block& other) {
  if (out.p == nullptr || other.p == nullptr || out.bytes <= 0 || other.bytes <= 0) return DTST_OK;
  const uintptr_t a = reinterpret_cast<uintptr_t>(out.p), b = reinterpret_cast<uintptr_t>(other.p);
  if (a < b + uintptr_t(other.bytes) && b < a + uintptr_t(out.bytes)) return bad(std::string(out.name) + " and " + other.name + " overlap");
  return DTST_OK;
}
dtst_status check_no_share(const dtst_recurrence_desc* d, const Sequence& s, const Block& b, int size) {
  if (s.p == nullptr || b.p == nullptr || d->steps < 1) return DTST_OK;
  if (share(rows_of(d, s, size), int64_t(reinterpret_cast<uintptr_t>(b.p)), b.bytes))
    return bad(std::string(s.name) + " and " + b.name + " overlap");
  return DTST_OK;
}
Block of_features(const dtst_recurrence_desc* d, const void* p, int64_t rows, const char* name) {
  return Block{p, d->batch * d->features * rows * 4, name};
}

dtst_status recurrence(const dtst_recurrence_desc* d, const void* z, const void* v, const void* o, const float* h_zero,
                       const int32_t* lengths, void* y, float* h_out, float* states, void* workspace,
                       size_t workspace_bytes, void* stream) {
  DTST_TRY(check_sequence_sizes(d));
  if (d->batch == 0 || d->features == 0) return ok();
  const int size = type_size(d->type);
  const Sequence sz{z, d->z_stride, "z"}, sv{v, d->v_stride, "v"}, so{o, d->o_stride, "o"}, sy{y, d->y_stride, "y"};
  if (d->steps > 0) {
    DTST_TRY(check_sequence(d, sz, size));
    DTST_TRY(check_sequence(d, sv, size));
    if (o) DTST_TRY(check_sequence(d, so, size));
    DTST_TRY(check_sequence(d, sy, size));
    for (const Sequence* in : {&sz, &sv, &so}) DTST_TRY(check_no_share(d, sy, *in, size));
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
  for (const Block* b : {&bin, &bn, &bout, &bst, &bws}) DTST_TRY(check_no_share(d, sy, *b, size));
  for (const Block* out : {&bout, &bst, &bws}) {
    for (const Sequence* in : {&sz, &sv, &so}) DTST_TRY(check_no_share(d, *in, *out, size));
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
  const int size = type_size(d->type);
  const Sequence sz{z, d->z_stride, "z"}, sv{v, d->v_stride, "v"}, so{o, d->o_stride, "o"}, sg{g_y, d->y_stride, "g_y"};
  const Sequence gz{g_z, d->g_z_stride, "g_z"}, gv{g_v, d->g_v_stride, "g_v"}, go{g_o, d->g_o_stride, "g_o"};
  if (d->steps > 0) {
    for (const Sequence* s : {&sz, &sv, &sg, &gz, &gv}) DTST_TRY(check_sequence(d, *s, size));
    if (o)
      for (const Sequence* s : {&so, &go}) DTST_TRY(check_sequence(d, *s, size));
    DTST_TRY(check_align(states, 4, "states"));
    for (const Sequence* in : {&sz, &sv, &so, &sg})
      for (const Sequence* out : {&gz, &gv, &go}) DTST_TRY(check_no_share(d, *out, *in, size));
    DTST_TRY(check_no_share(d, gz, gv, size));
    DTST_TRY(check_no_share(d, gz, go, size));
    DTST_TRY(check_no_share(d, gv, go, size));
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
    for (const Block* b : {&bst, &bin, &bn, &bout, &bws}) DTST_TRY(check_no_share(d, *out, *b, size));
  for (const Block* out : {&bout, &bws}) {
    for (const Sequence* in : {&sz, &sv, &so, &sg}) DTST_TRY(check_no_share(d, *in, *out, size));
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
  return guarded([&] { return rms_norm(d, x, res, weight, sum_out, y, scale, rstd, stream); });
}

dtst_status dtst_rms_norm_adj_workspace(int64_t rows, int64_t cols, size_t* bytes) {
  return guarded([&] {
    if (bytes == nullptr) return bad("bytes is null");
    DTST_TRY(check_rows_cols(rows, cols));
    if (cols > kNormMaxCols) return fail(DTST_ERR_UNSUPPORTED, "cols above " + std::to_string(kNormMaxCols));
    *bytes = rms_norm_adj_workspace(rows, cols);
    return ok();
  });
}

dtst_status dtst_rms_norm_adj(const dtst_norm_adj_desc* d, const void* g_y, const void* u, const float* weight,
                              const float* rstd, const void* g_sum, void* g_u, void* g_x, float* g_weight,
                              void* workspace, size_t workspace_bytes, void* stream) {
  return guarded([&] {
    return rms_norm_adj(d, g_y, u, weight, rstd, g_sum, g_u, g_x, g_weight, workspace, workspace_bytes, stream);
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
