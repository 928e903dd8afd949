// The C ABI of the operators that need no model (heads, orthogonalised updates) and of what hangs them into one: argument checks on
// the host, then the launches.
#include <algorithm>
#include <cmath>
#include <limits>
#include <new>

#include "model.h"

using spb::set_error;

namespace {

// Nothing thrown inside may leave a C entry.
template <class F>
int guarded(const char* who, F&& f) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    set_error("%s: out of host memory", who);
  } catch (...) {
    set_error("%s: unexpected failure on the host", who);
  }
  return SPB_ERR_HIP;
}

bool aligned(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

int check_rotary(const spb_rotary& r, int head_dim, const char* who) {
  SPB_REQUIRE(r.pairs >= 0 && 2 * (long long)r.pairs <= head_dim, SPB_ERR_INVALID_ARG, "%s: %d pairs in heads of %d", who, r.pairs, head_dim);
  if (r.pairs == 0) return SPB_OK;
  SPB_REQUIRE(r.axes >= 1 && r.axes <= SPB_MAX_AXES, SPB_ERR_INVALID_ARG, "%s: %d axes outside 1..%d", who, r.axes, SPB_MAX_AXES);
  for (int j = 0; j < r.pairs; ++j) {
    SPB_REQUIRE(r.axis[j] >= 0 && r.axis[j] < r.axes, SPB_ERR_INVALID_ARG, "%s: axis %d of pair %d outside 0..%d", who, r.axis[j], j, r.axes - 1);
    SPB_REQUIRE(std::isfinite(r.freq[j]), SPB_ERR_INVALID_ARG, "%s: frequency of pair %d is not finite", who, j);
  }
  return SPB_OK;
}

int check_heads(const spb_heads_desc* d, const char* who) {
  SPB_REQUIRE(d, SPB_ERR_INVALID_ARG, "%s: null description", who);
  SPB_REQUIRE(d->dtype == SPB_DTYPE_F32 || d->dtype == SPB_DTYPE_BF16, SPB_ERR_INVALID_ARG, "%s: dtype %d", who, d->dtype);
  SPB_REQUIRE(d->batch >= 0 && d->seq >= 0 && (long long)d->batch * d->seq <= 0x7FFFFFFFll, SPB_ERR_INVALID_ARG, "%s: %d sequences of %d tokens", who, d->batch, d->seq);
  SPB_REQUIRE(d->heads_q >= 1 && d->heads_k >= 0 && (long long)d->heads_q + d->heads_k <= 65535, SPB_ERR_INVALID_ARG, "%s: %d + %d heads", who, d->heads_q, d->heads_k);
  SPB_REQUIRE(d->head_dim >= 1 && d->head_dim <= SPB_MAX_HEAD_DIM, SPB_ERR_INVALID_ARG, "%s: head_dim %d outside 1..%d", who, d->head_dim, SPB_MAX_HEAD_DIM);
  SPB_REQUIRE(!d->norm || (d->eps > 0.f && std::isfinite(d->eps)), SPB_ERR_INVALID_ARG, "%s: eps must be positive", who);
  SPB_REQUIRE(d->norm || d->rotary.pairs != 0, SPB_ERR_INVALID_ARG, "%s: neither norm nor rotation", who);
  return check_rotary(d->rotary, d->head_dim, who);
}

// Strides of an input are any that are not negative; those of a result leave every row a place of its own.
int check_strides(const spb_heads_desc* d, const int64_t* s, bool result, const char* name, const char* who) {
  const long long extent[3] = {d->batch, d->seq, (long long)d->heads_q + d->heads_k};
  for (int i = 0; i < 3; ++i)
    SPB_REQUIRE(s[i] >= 0 && (__int128)s[i] * extent[i] <= ((__int128)1 << 60), SPB_ERR_INVALID_ARG, "%s: stride %lld of %s", who, (long long)s[i], name);
  if (!result) return SPB_OK;
  int order[3] = {0, 1, 2};
  std::sort(order, order + 3, [&](int a, int b) { return s[a] < s[b]; });
  __int128 span = d->head_dim;
  for (int i : order) {
    if (extent[i] <= 1) continue;
    SPB_REQUIRE((__int128)s[i] >= span, SPB_ERR_INVALID_ARG, "%s: rows of %s overlap", who, name);
    span = (__int128)s[i] * (extent[i] - 1) + span;
  }
  return SPB_OK;
}

// A result at an input's address takes that input's place row by row.
int check_in_place(const spb_heads_desc* d, const void* in, const int64_t* s, const void* out, const int64_t* o, const char* name, const char* who) {
  if (in != out) return SPB_OK;
  const long long extent[3] = {d->batch, d->seq, (long long)d->heads_q + d->heads_k};
  for (int i = 0; i < 3; ++i) SPB_REQUIRE(extent[i] <= 1 || s[i] == o[i], SPB_ERR_INVALID_ARG, "%s: in place of %s with other strides", who, name);
  return SPB_OK;
}

spb::HeadsProblem heads_problem(const spb_heads_desc* d, const int32_t* pos, int64_t pos_axis_stride, int64_t pos_batch_stride) {
  spb::HeadsProblem q;
  q.dtype = d->dtype == SPB_DTYPE_F32 ? spb::DType::F32 : spb::DType::BF16;
  q.batch = d->batch; q.seq = d->seq; q.heads_q = d->heads_q; q.heads_k = d->heads_k; q.head_dim = d->head_dim;
  q.norm = d->norm != 0; q.eps = d->eps;
  q.pairs = d->rotary.pairs; q.interleaved = d->rotary.interleaved != 0; q.axis = d->rotary.axis; q.freq = d->rotary.freq;
  q.pos = pos; q.pos_axis_stride = pos_axis_stride; q.pos_batch_stride = pos_batch_stride;
  return q;
}

int launched(hipError_t e, const char* who) {
  if (e == hipSuccess) return SPB_OK;
  (void)hipGetLastError();
  set_error("%s: %s", who, hipGetErrorString(e));
  return e == hipErrorInvalidValue ? SPB_ERR_INVALID_ARG : SPB_ERR_HIP;
}

// Whether a factor that kernels take in float32 stays finite there.
bool fits_f32(double v) { return std::isfinite((float)v); }

int check_config(const spb_muon_config* c, const char* who) {
  SPB_REQUIRE(c, SPB_ERR_INVALID_ARG, "%s: null configuration", who);
  SPB_REQUIRE(fits_f32(c->lr) && fits_f32(c->rms) && fits_f32(c->weight_decay) && fits_f32(c->momentum), SPB_ERR_INVALID_ARG,
              "%s: lr, rms, momentum and weight_decay must be finite in float32", who);
  SPB_REQUIRE(c->beta1 >= 0.0 && c->beta1 < 1.0 && c->beta2 >= 0.0 && c->beta2 < 1.0, SPB_ERR_INVALID_ARG, "%s: beta1 and beta2 must lie in [0, 1)", who);
  SPB_REQUIRE(c->ns_eps > 0.0 && c->adam_eps > 0.0 && std::isfinite(c->ns_eps) && std::isfinite(c->adam_eps), SPB_ERR_INVALID_ARG, "%s: ns_eps and adam_eps must be positive", who);
  // (ns_eps stays in float64; adam_eps as zero or with few bits would turn moments of zero into 0 / 0)
  SPB_REQUIRE((float)c->adam_eps >= std::numeric_limits<float>::min(), SPB_ERR_INVALID_ARG, "%s: adam_eps %g is below float32's normal numbers", who, c->adam_eps);
  SPB_REQUIRE(c->step >= 1, SPB_ERR_INVALID_ARG, "%s: step %lld", who, (long long)c->step);
  SPB_REQUIRE(c->ns_steps >= 1 && c->ns_steps <= 16, SPB_ERR_INVALID_ARG, "%s: ns_steps %d outside 1..16", who, c->ns_steps);
  return SPB_OK;
}

constexpr long long kMostEntries = 1ll << 33;   // of a tensor, and of all matrices of a call, padded: the grids behind them count their threads in 32 bits

int check_shape(long long rows, long long cols, int blocks, const char* name, const char* who) {
  SPB_REQUIRE(rows >= 1 && cols >= 1 && rows <= kMostEntries / cols, SPB_ERR_INVALID_ARG, "%s: %s is %lld x %lld", who, name, rows, cols);
  SPB_REQUIRE(blocks >= 0, SPB_ERR_INVALID_ARG, "%s: %d blocks of %s", who, blocks, name);
  if (blocks == 0) return SPB_OK;
  SPB_REQUIRE(rows % blocks == 0, SPB_ERR_INVALID_ARG, "%s: %lld rows of %s do not divide into %d blocks", who, rows, name, blocks);
  SPB_REQUIRE(rows / blocks <= SPB_MAX_MATRIX_SIDE && cols <= SPB_MAX_MATRIX_SIDE, SPB_ERR_INVALID_ARG, "%s: matrices of %s are %lld x %lld, sides reach %d", who, name,
              rows / blocks, cols, SPB_MAX_MATRIX_SIDE);
  return SPB_OK;
}

int check_workspace(const void* workspace, size_t bytes, size_t need, const char* who) {
  if (need == 0) return SPB_OK;
  SPB_REQUIRE(workspace && bytes >= need, SPB_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, bytes, need);
  SPB_REQUIRE(aligned(workspace, 256), SPB_ERR_WORKSPACE, "%s: workspace is not 256-byte aligned", who);
  return SPB_OK;
}

// Before anything is planned: the plan counts matrices in 32 bits.
int check_total(const std::vector<spb::MuonTensor>& t, const char* who) {
  __int128 padded = 0;
  for (const auto& x : t)
    if (x.blocks) padded += (__int128)x.blocks * ((x.rows / x.blocks + 255) / 256 * 256) * ((x.cols + 255) / 256 * 256);
  SPB_REQUIRE(padded <= kMostEntries, SPB_ERR_INVALID_ARG, "%s: too many matrices for one call", who);
  return SPB_OK;
}

// Nothing that a step writes may lie in anything else of it: workgroups take tensors, and parts of them, in any order.
int check_places(const std::vector<spb::MuonTensor>& t, const void* workspace, size_t workspace_bytes, const char* who) {
  struct Span { uintptr_t from, to; };
  auto span = [](const void* p, size_t bytes) { return Span{reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes}; };
  std::vector<Span> written;
  written.reserve(3 * t.size() + 1);
  for (const auto& x : t) {
    const size_t n = (size_t)(x.rows * x.cols);
    written.push_back(span(x.w, n * (x.dtype == spb::DType::F32 ? 4 : 2)));
    written.push_back(span(x.m, n * 4));
    if (x.v) written.push_back(span(x.v, n * 4));
  }
  if (workspace_bytes) written.push_back(span(workspace, workspace_bytes));
  std::sort(written.begin(), written.end(), [](const Span& a, const Span& b) { return a.from < b.from; });
  for (size_t i = 1; i < written.size(); ++i)
    SPB_REQUIRE(written[i].from >= written[i - 1].to, SPB_ERR_INVALID_ARG, "%s: a parameter, moment or the workspace lies in another", who);
  for (size_t i = 0; i < t.size(); ++i)
    for (int j = 0; j < t[i].count; ++j) {
      const Span g = span(t[i].g[j], (size_t)(t[i].rows * t[i].cols) * 4);
      const auto at = std::upper_bound(written.begin(), written.end(), g.from, [](uintptr_t from, const Span& s) { return from < s.to; });
      SPB_REQUIRE(at == written.end() || at->from >= g.to, SPB_ERR_INVALID_ARG, "%s: gradient %d of tensor %zu lies in what the step writes", who, j, i);
    }
  return SPB_OK;
}

// The factors of the parameter and of its update.
int check_rates(const std::vector<spb::MuonTensor>& t, const spb_muon_config& c, const char* who) {
  for (size_t i = 0; i < t.size(); ++i) {
    const double side = t[i].blocks ? std::sqrt((double)std::max(t[i].rows / t[i].blocks, t[i].cols)) : 1.0;
    SPB_REQUIRE(fits_f32(t[i].rate) && fits_f32(1.0 - t[i].rate * c.weight_decay) && fits_f32(t[i].rate * c.rms * side), SPB_ERR_INVALID_ARG,
                "%s: rate %g of tensor %zu leaves float32", who, t[i].rate, i);
  }
  return SPB_OK;
}

// shapes only: what the workspace goes by
int tensors_of(const spb_muon_tensor* in, int n, std::vector<spb::MuonTensor>* out, const char* who) {
  SPB_REQUIRE(n >= 0 && (in || n == 0), SPB_ERR_INVALID_ARG, "%s: null or negative list of tensors", who);
  for (int i = 0; i < n; ++i) {
    const spb_muon_tensor& s = in[i];
    const std::string name = "tensor " + std::to_string(i);
    SPB_REQUIRE(s.dtype == SPB_DTYPE_F32 || s.dtype == SPB_DTYPE_BF16, SPB_ERR_INVALID_ARG, "%s: dtype %d of %s", who, s.dtype, name.c_str());
    if (int rc = check_shape(s.rows, s.cols, s.blocks, name.c_str(), who)) return rc;
    spb::MuonTensor d;
    d.rows = s.rows; d.cols = s.cols; d.blocks = s.blocks;
    d.dtype = s.dtype == SPB_DTYPE_F32 ? spb::DType::F32 : spb::DType::BF16;
    out->push_back(d);
  }
  return SPB_OK;
}

}  // namespace

extern "C" {

int spb_rotary_sections(spb_rotary* out, int32_t axes, const int32_t* sections, double base, int32_t own_ladder, int32_t interleaved) {
  const char* who = "spb_rotary_sections";
  SPB_REQUIRE(out && sections, SPB_ERR_INVALID_ARG, "%s: null argument", who);
  SPB_REQUIRE(axes >= 1 && axes <= SPB_MAX_AXES, SPB_ERR_INVALID_ARG, "%s: %d axes outside 1..%d", who, axes, SPB_MAX_AXES);
  SPB_REQUIRE(base > 0.0 && std::isfinite(base), SPB_ERR_INVALID_ARG, "%s: base must be positive", who);
  long long total = 0;
  for (int a = 0; a < axes; ++a) {
    SPB_REQUIRE(sections[a] >= 0, SPB_ERR_INVALID_ARG, "%s: %d pairs for axis %d", who, sections[a], a);
    total += sections[a];
  }
  SPB_REQUIRE(total >= 1 && total <= SPB_MAX_PAIRS, SPB_ERR_INVALID_ARG, "%s: %lld pairs outside 1..%d", who, total, SPB_MAX_PAIRS);
  *out = spb_rotary{};
  out->pairs = (int32_t)total; out->axes = axes; out->interleaved = interleaved != 0;
  int j = 0;
  for (int a = 0; a < axes; ++a)
    for (int i = 0; i < sections[a]; ++i, ++j) {
      out->axis[j] = a;
      out->freq[j] = std::pow(base, own_ladder ? -(double)i / sections[a] : -(double)j / (double)total);
    }
  return SPB_OK;
}

int spb_heads_forward(const spb_heads_desc* d, const void* x, void* y, const int32_t* pos, int64_t pos_axis_stride, int64_t pos_batch_stride,
                      const void* gamma, const void* beta, void* stream) {
  const char* who = "spb_heads_forward";
  if (int rc = check_heads(d, who)) return rc;
  if (int rc = check_strides(d, d->x_stride, false, "x", who)) return rc;
  if (int rc = check_strides(d, d->y_stride, true, "y", who)) return rc;
  if (d->batch == 0 || d->seq == 0) return SPB_OK;
  const size_t size = d->dtype == SPB_DTYPE_F32 ? 4 : 2;
  SPB_REQUIRE(x && y && aligned(x, size) && aligned(y, size), SPB_ERR_INVALID_ARG, "%s: x or y null or misaligned", who);
  if (int rc = check_in_place(d, x, d->x_stride, y, d->y_stride, "x", who)) return rc;
  SPB_REQUIRE(!d->rotary.pairs || (pos && aligned(pos, 4)), SPB_ERR_INVALID_ARG, "%s: a rotation needs positions", who);
  SPB_REQUIRE(!d->norm || (gamma && aligned(gamma, size) && aligned(beta, size)), SPB_ERR_INVALID_ARG, "%s: gamma null, or gamma or beta misaligned", who);
  return guarded(who, [&] {
    spb::HeadsProblem q = heads_problem(d, pos, pos_axis_stride, pos_batch_stride);
    q.x = x; q.out = y;
    q.gamma = d->norm ? gamma : nullptr; q.beta = d->norm ? beta : nullptr;
    for (int i = 0; i < 3; ++i) { q.x_stride[i] = d->x_stride[i]; q.out_stride[i] = d->y_stride[i]; }
    return launched(spb::launch_heads_forward(q, static_cast<hipStream_t>(stream)), who);
  });
}

int spb_heads_workspace_size(const spb_heads_desc* d, size_t* bytes) {
  const char* who = "spb_heads_workspace_size";
  SPB_REQUIRE(bytes, SPB_ERR_INVALID_ARG, "%s: null argument", who);
  if (int rc = check_heads(d, who)) return rc;
  *bytes = d->norm ? spb::heads_partial_floats(d->batch, d->seq, d->heads_k, d->head_dim) * sizeof(float) : 0;
  return SPB_OK;
}

int spb_heads_backward(const spb_heads_desc* d, const void* x, const void* dy, void* dx, const int32_t* pos, int64_t pos_axis_stride,
                       int64_t pos_batch_stride, const void* gamma, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes, void* stream) {
  const char* who = "spb_heads_backward";
  if (int rc = check_heads(d, who)) return rc;
  if (d->norm)
    if (int rc = check_strides(d, d->x_stride, false, "x", who)) return rc;
  if (int rc = check_strides(d, d->y_stride, false, "dy", who)) return rc;
  if (int rc = check_strides(d, d->dx_stride, true, "dx", who)) return rc;
  const bool empty = d->batch == 0 || d->seq == 0;
  const size_t size = d->dtype == SPB_DTYPE_F32 ? 4 : 2;
  SPB_REQUIRE(empty || (dy && dx && aligned(dy, size) && aligned(dx, size)), SPB_ERR_INVALID_ARG, "%s: dy or dx null or misaligned", who);
  if (!empty) {
    if (int rc = check_in_place(d, dy, d->y_stride, dx, d->dx_stride, "dy", who)) return rc;
    if (d->norm)
      if (int rc = check_in_place(d, x, d->x_stride, dx, d->dx_stride, "x", who)) return rc;
  }
  SPB_REQUIRE(empty || !d->rotary.pairs || (pos && aligned(pos, 4)), SPB_ERR_INVALID_ARG, "%s: a rotation needs positions", who);
  if (d->norm) {
    SPB_REQUIRE(empty || (x && aligned(x, size)), SPB_ERR_INVALID_ARG, "%s: with norm x is needed", who);
    SPB_REQUIRE(gamma && dgamma && dbeta && aligned(gamma, size) && aligned(dgamma, 4) && aligned(dbeta, 4), SPB_ERR_INVALID_ARG, "%s: gamma, dgamma or dbeta null or misaligned", who);
    size_t need = 0;
    if (int rc = spb_heads_workspace_size(d, &need)) return rc;
    if (int rc = check_workspace(workspace, workspace_bytes, need, who)) return rc;
  }
  return guarded(who, [&] {
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (empty) {   // sums over nothing
      if (!d->norm) return SPB_OK;
      const size_t bytes = (size_t)(d->heads_k ? 2 : 1) * d->head_dim * 4;
      if (int rc = launched(spb::launch_fill_zero(dgamma, bytes, s), who)) return rc;
      return launched(spb::launch_fill_zero(dbeta, bytes, s), who);
    }
    spb::HeadsProblem q = heads_problem(d, pos, pos_axis_stride, pos_batch_stride);
    q.dy = dy; q.out = dx;
    for (int i = 0; i < 3; ++i) { q.x_stride[i] = d->x_stride[i]; q.dy_stride[i] = d->y_stride[i]; q.out_stride[i] = d->dx_stride[i]; }
    if (d->norm) { q.x = x; q.gamma = gamma; q.dgamma = dgamma; q.dbeta = dbeta; q.partial = static_cast<float*>(workspace); }
    return launched(spb::launch_heads_backward(q, s), who);
  });
}

int spb_muon_workspace_size(const spb_muon_tensor* tensors, int32_t n, size_t* bytes) {
  const char* who = "spb_muon_workspace_size";
  SPB_REQUIRE(bytes, SPB_ERR_INVALID_ARG, "%s: null argument", who);
  return guarded(who, [&] {
    std::vector<spb::MuonTensor> t;
    if (int rc = tensors_of(tensors, n, &t, who)) return rc;
    if (int rc = check_total(t, who)) return rc;
    *bytes = spb::muon_workspace_size(t.data(), n);
    return SPB_OK;
  });
}

int spb_muon_step(const spb_muon_tensor* tensors, int32_t n, const spb_muon_config* config, void* workspace, size_t workspace_bytes, void* stream) {
  const char* who = "spb_muon_step";
  if (int rc = check_config(config, who)) return rc;
  return guarded(who, [&] {
    std::vector<spb::MuonTensor> t;
    if (int rc = tensors_of(tensors, n, &t, who)) return rc;
    if (int rc = check_total(t, who)) return rc;
    for (int i = 0; i < n; ++i) {
      const spb_muon_tensor& s = tensors[i];
      const size_t size = s.dtype == SPB_DTYPE_F32 ? 4 : 2;
      SPB_REQUIRE(s.count >= 1 && s.count <= SPB_MAX_WORKERS && s.grads, SPB_ERR_INVALID_ARG, "%s: %d gradients of tensor %d", who, s.count, i);
      SPB_REQUIRE(s.w && s.m && (s.v || s.blocks) && aligned(s.w, size) && aligned(s.m, 4) && aligned(s.v, 4), SPB_ERR_INVALID_ARG,
                  "%s: w, m or v of tensor %d null or misaligned", who, i);
      SPB_REQUIRE(s.rate_scale >= 0.0 && std::isfinite(s.rate_scale), SPB_ERR_INVALID_ARG, "%s: rate_scale of tensor %d", who, i);
      t[i].w = s.w; t[i].m = s.m; t[i].v = s.blocks ? nullptr : s.v; t[i].count = s.count; t[i].rate = config->lr * s.rate_scale;
      for (int j = 0; j < s.count; ++j) {
        SPB_REQUIRE(s.grads[j] && aligned(s.grads[j], 4), SPB_ERR_INVALID_ARG, "%s: gradient %d of tensor %d null or misaligned", who, j, i);
        t[i].g[j] = s.grads[j];
      }
    }
    if (int rc = check_rates(t, *config, who)) return rc;
    const size_t need = spb::muon_workspace_size(t.data(), n);
    if (int rc = check_workspace(workspace, workspace_bytes, need, who)) return rc;
    if (int rc = check_places(t, workspace, need, who)) return rc;
    return launched(spb::launch_muon_step(t.data(), n, *config, workspace, static_cast<hipStream_t>(stream)), who);
  });
}

// rows and columns of parameter i
static void sides_of(const spb::ParamInfo& p, long long* rows, long long* cols) {
  *rows = p.shape[0];
  *cols = p.numel() / p.shape[0];
}

// shapes, types and blocks of the parameters of units from `unit` on, which is what the deepest worker of a step leaves to update
static int suffix_of(const spb::Model& im, const int32_t* blocks, int unit, std::vector<spb::MuonTensor>* t, const char* who) {
  for (size_t i = 0; i < im.params.size(); ++i) {
    if (im.params[i].unit < unit) continue;
    spb::MuonTensor d;
    sides_of(im.params[i], &d.rows, &d.cols);
    if (int rc = check_shape(d.rows, d.cols, blocks[i], im.params[i].name.c_str(), who)) return rc;
    d.blocks = blocks[i]; d.dtype = im.params[i].dtype;
    t->push_back(d);
  }
  return check_total(*t, who);
}

int spb_aggregate_muon_workspace_size(const spb_model* m, const int32_t* blocks, size_t* bytes) {
  const char* who = "spb_aggregate_muon_workspace_size";
  SPB_REQUIRE(m && blocks && bytes, SPB_ERR_INVALID_ARG, "%s: null argument", who);
  return guarded(who, [&] {
    size_t most = 0;
    // (fewer tensors may need more: how matrices are padded goes by what is launched with them)
    for (int unit = 0; unit < m->impl->num_units; ++unit) {
      std::vector<spb::MuonTensor> t;
      if (int rc = suffix_of(*m->impl, blocks, unit, &t, who)) return rc;
      most = std::max(most, spb::muon_workspace_size(t.data(), (int)t.size()));
    }
    *bytes = most;
    return SPB_OK;
  });
}

int spb_aggregate_muon(spb_model* m, int32_t n_workers, const int32_t* depths, void* const* worker_grads, const int32_t* blocks, void* const* first,
                       void* const* second, const spb_muon_config* config, int32_t scale_lr, void* workspace, size_t workspace_bytes, void* stream) {
  const char* who = "spb_aggregate_muon";
  SPB_REQUIRE(m && depths && worker_grads && blocks && first && second, SPB_ERR_INVALID_ARG, "%s: null argument", who);
  SPB_REQUIRE(n_workers >= 1 && n_workers <= SPB_MAX_WORKERS, SPB_ERR_INVALID_ARG, "%s: %d workers outside 1..%d", who, n_workers, SPB_MAX_WORKERS);
  if (int rc = check_config(config, who)) return rc;
  auto& im = *m->impl;
  for (int j = 0; j < n_workers; ++j)
    SPB_REQUIRE(depths[j] >= 0 && depths[j] <= im.num_units, SPB_ERR_DEPTH_RANGE, "%s: depth %d outside 0..%d", who, depths[j], im.num_units);
  SPB_REQUIRE(im.params_bound, SPB_ERR_STATE, "%s: parameters not bound", who);
  return guarded(who, [&] {
    const int n_params = (int)im.params.size();
    std::vector<spb::MuonTensor> t;
    for (int i = 0; i < n_params; ++i) {
      const char* name = im.params[i].name.c_str();
      spb::MuonTensor d;
      sides_of(im.params[i], &d.rows, &d.cols);
      if (int rc = check_shape(d.rows, d.cols, blocks[i], name, who)) return rc;
      for (int j = 0; j < n_workers; ++j) {
        if (im.params[i].unit < im.num_units - depths[j]) continue;   // worker j's suffix does not reach this unit
        const void* g = worker_grads[(size_t)j * n_params + i];
        SPB_REQUIRE(g && aligned(g, 16), SPB_ERR_INVALID_ARG, "%s: worker %d contributes to %s but its gradient pointer is null or not 16-byte aligned", who, j, name);
        d.g[d.count++] = static_cast<const float*>(g);
      }
      if (d.count == 0) continue;   // nobody reached it
      SPB_REQUIRE(first[i] && aligned(first[i], 16), SPB_ERR_INVALID_ARG, "%s: first moment of %s null or not 16-byte aligned", who, name);
      SPB_REQUIRE(blocks[i] || (second[i] && aligned(second[i], 16)), SPB_ERR_INVALID_ARG, "%s: second moment of %s null or not 16-byte aligned", who, name);
      d.w = im.param_ptrs[i]; d.m = static_cast<float*>(first[i]); d.v = blocks[i] ? nullptr : static_cast<float*>(second[i]);
      d.blocks = blocks[i]; d.dtype = im.params[i].dtype;
      d.rate = scale_lr ? config->lr * d.count / n_workers : config->lr;
      t.push_back(d);
    }
    if (int rc = check_total(t, who)) return rc;
    const size_t need = spb::muon_workspace_size(t.data(), (int)t.size());
    if (int rc = check_workspace(workspace, workspace_bytes, need, who)) return rc;
    if (int rc = check_places(t, workspace, need, who)) return rc;
    if (int rc = check_rates(t, *config, who)) return rc;
    return launched(spb::launch_muon_step(t.data(), (int)t.size(), *config, workspace, static_cast<hipStream_t>(stream)), who);
  });
}

int spb_encoder_heads(spb_model* m, const spb_rotary* rotary, const int32_t* pos, int64_t pos_axis_stride, int64_t pos_batch_stride, int32_t norm,
                      float eps) {
  const char* who = "spb_encoder_heads";
  SPB_REQUIRE(m, SPB_ERR_INVALID_ARG, "%s: null model", who);
  const int head_dim = m->impl->head_dim();
  SPB_REQUIRE(head_dim > 0, SPB_ERR_UNSUPPORTED, "%s: only encoders have heads", who);
  SPB_REQUIRE(!m->impl->params_bound && !m->impl->grads_bound, SPB_ERR_STATE, "%s: parameters or gradients are bound already", who);
  SPB_REQUIRE(head_dim <= SPB_MAX_HEAD_DIM, SPB_ERR_INVALID_ARG, "%s: heads of %d elements, at most %d", who, head_dim, SPB_MAX_HEAD_DIM);
  SPB_REQUIRE(!norm || (eps > 0.f && std::isfinite(eps)), SPB_ERR_INVALID_ARG, "%s: eps must be positive", who);
  if (rotary) {
    SPB_REQUIRE(rotary->pairs >= 1, SPB_ERR_INVALID_ARG, "%s: a rotation of no pairs", who);
    if (int rc = check_rotary(*rotary, head_dim, who)) return rc;
    SPB_REQUIRE(pos && aligned(pos, 4), SPB_ERR_INVALID_ARG, "%s: a rotation needs positions", who);
  }
  return guarded(who, [&] {
    m->impl->set_heads(rotary, pos, pos_axis_stride, pos_batch_stride, norm != 0, eps);
    return SPB_OK;
  });
}

}  // extern "C"
