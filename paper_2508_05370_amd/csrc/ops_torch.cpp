// ops_torch.cpp -- the layer operators of hetsim_ops.h on torch tensors: checks
// of types, shapes and devices, allocation of outputs and workspaces, and the
// call into libhetsim.so on torch's current stream.  A Python module of its own
// (ops.py is its face), so that the library itself knows no torch; as native
// code because a call on one token takes the card 3 us.
#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <c10/hip/HIPStream.h>
#include <dlfcn.h>
#include <torch/csrc/utils/pybind.h>

#include <string>
#include <vector>

#include "hetsim_ops.h"

namespace py = pybind11;
using at::Tensor;
typedef std::optional<Tensor> Maybe;

namespace {

struct Library {
  decltype(&sim_op_quantize) quantize;
  decltype(&sim_op_matmul_workspace) matmul_workspace;
  decltype(&sim_op_matmul) matmul;
  decltype(&sim_op_linear_workspace) linear_workspace;
  decltype(&sim_op_linear) linear;
  decltype(&sim_op_norm) norm;
  decltype(&sim_op_norm_backward_workspace) norm_backward_workspace;
  decltype(&sim_op_norm_backward) norm_backward;
  decltype(&sim_op_adamw) adamw;
} L;

void load(const std::string& path) {
  void* h = dlopen(path.c_str(), RTLD_NOW | RTLD_LOCAL);
  if (!h) throw std::runtime_error(dlerror());
  auto get = [&](auto& f, const char* name) {
    f = (std::remove_reference_t<decltype(f)>)dlsym(h, name);
    if (!f) throw std::runtime_error(path + " has no " + name);
  };
  get(L.quantize, "sim_op_quantize");
  get(L.matmul_workspace, "sim_op_matmul_workspace");
  get(L.matmul, "sim_op_matmul");
  get(L.linear_workspace, "sim_op_linear_workspace");
  get(L.linear, "sim_op_linear");
  get(L.norm, "sim_op_norm");
  get(L.norm_backward_workspace, "sim_op_norm_backward_workspace");
  get(L.norm_backward, "sim_op_norm_backward");
  get(L.adamw, "sim_op_adamw");
}

[[noreturn]] void refuse(const std::string& what) { throw py::value_error(what); }
void require(bool ok, const char* what) {
  if (!ok) refuse(what);
}
// The library's refusals and failures are binding.SimError.
void check(int code, const char* what) {
  if (code == SIM_OK) return;
  py::object type = py::module_::import("paper_2508_05370_amd.binding").attr("SimError");
  PyErr_SetObject(type.ptr(), type(code, what).ptr());
  throw py::error_already_set();
}

int type_of(at::ScalarType t) {
  return t == at::kBFloat16 ? SIM_BF16 : t == at::kHalf ? SIM_FP16 : t == at::kFloat ? SIM_FP32 : SIM_NONE;
}
int type_of(const Tensor& t, const char* what) {
  const int r = type_of(t.scalar_type());
  if (r == SIM_NONE) refuse(std::string(what) + ": type " + c10::toString(t.scalar_type()) + " is not bfloat16, float16 or float32");
  return r;
}
void* ptr(const Tensor& t) { return t.data_ptr(); }
void* ptr(const Maybe& t) { return t ? t->data_ptr() : nullptr; }

// Results have no history: a tensor whose gradient autograd is to record is
// refused, as an out argument of torch's own functions does.
void require_unrecorded(const Tensor& t) {
  if (t.requires_grad() && c10::GradMode::is_enabled())
    refuse("a tensor requires its gradient, which these calls do not record: pass it detached, or call under torch.no_grad()");
}

// The library writes through pointers: autograd is told, so that it notices a
// tensor that it saved.  (Tensors of inference mode have no counter.)
void written(const Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// Tensors are on the current GPU; its current stream.
struct Place {
  c10::Device device;
  void* stream;
  explicit Place(const Tensor& t, bool parameters = false) : device(t.device()), stream(nullptr) {
    if (!parameters) require_unrecorded(t);
    if (!t.is_cuda()) refuse("tensors must be on a GPU, not on " + device.str());
    const auto s = c10::hip::getCurrentHIPStream();
    if (s.device_index() != device.index()) refuse("tensors must be on the current GPU, not on " + device.str());
    stream = s.stream();
  }
  void on(const Tensor& t) const {
    require_unrecorded(t);
    if (t.device() != device) refuse("tensors on " + device.str() + " and " + t.device().str());
  }
  void on(const Maybe& t) const {
    if (t) on(*t);
  }
  Tensor empty(at::IntArrayRef size, at::ScalarType type) const {
    return at::empty(size, at::TensorOptions().dtype(type).device(device));
  }
  Tensor bytes(size_t n) const { return n ? empty({(int64_t)n}, at::kByte) : Tensor(); }
};
void* ptr_or_null(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

struct Matrix {
  void* p;
  int type;
  int64_t rows, cols, ld;
};
// A matrix with contiguous rows that do not overlap.
Matrix shape(const Tensor& t, const char* what) {
  if (t.dim() != 2) refuse(std::string(what) + ": a matrix");
  Matrix m = {t.data_ptr(), SIM_NONE, t.size(0), t.size(1), t.stride(0)};
  if ((t.stride(1) != 1 && m.cols > 1) || (m.ld < m.cols && m.rows > 1))
    refuse(std::string(what) + ": a matrix with contiguous rows that do not overlap");
  if (m.rows <= 1) m.ld = m.cols > 1 ? m.cols : 1;
  return m;
}
Matrix matrix(const Tensor& t, const char* what) {
  const int type = type_of(t, what);
  Matrix m = shape(t, what);
  m.type = type;
  return m;
}

constexpr at::ScalarType kE4m3 = at::kFloat8_e4m3fn;
int64_t blocks_of(int64_t n) { return n / SIM_BLOCK + (n % SIM_BLOCK != 0); }

sim_blocks block_form(const Tensor& codes, const Tensor& scales, int64_t k, const char* what, int64_t* rows) {
  if (codes.scalar_type() != kE4m3 || scales.scalar_type() != at::kFloat || codes.dim() != 2 || scales.dim() != 2)
    refuse(std::string(what) + ": matrices of e4m3 codes and of 32-bit scales");
  const Matrix c = shape(codes, what), s = shape(scales, what);
  const int64_t kb = blocks_of(k);
  if (c.cols < kb * SIM_BLOCK) refuse(std::string(what) + ": codes padded to whole blocks of 128 columns");
  if (s.rows != kb || (s.cols != c.rows && s.cols != blocks_of(c.rows)))
    refuse(std::string(what) + ": scales [blocks of columns, rows or blocks of rows]");
  *rows = c.rows;
  return {(uint8_t*)c.p, c.rows > 1 ? c.ld : c.cols, (float*)s.p, s.rows > 1 ? s.ld : s.cols,
          s.cols == c.rows ? 1u : (uint32_t)SIM_BLOCK};
}
sim_blocks new_blocks(const Place& at, int64_t rows, int64_t k, int64_t block_rows, Tensor* codes, Tensor* scales) {
  const int64_t kb = blocks_of(k), groups = block_rows == 1 ? rows : blocks_of(rows);
  *codes = at.empty({rows, kb * SIM_BLOCK}, kE4m3);
  *scales = at.empty({kb, groups}, at::kFloat);
  return {(uint8_t*)codes->data_ptr(), kb * SIM_BLOCK, (float*)scales->data_ptr(), groups, (uint32_t)block_rows};
}

py::tuple quantize(const Tensor& x, int64_t block_rows, bool rows, bool transposed) {
  const Matrix m = matrix(x, "x");
  require((block_rows == 1 || block_rows == SIM_BLOCK) && (rows || transposed), "block_rows is 1 or 128, and one form is wanted");
  const Place at(x);
  sim_blocks q = {}, qt = {};
  Tensor c, s, ct, st;
  if (rows) q = new_blocks(at, m.rows, m.cols, block_rows, &c, &s);
  if (transposed) qt = new_blocks(at, m.cols, m.rows, block_rows, &ct, &st);
  if (m.rows && m.cols)
    check(L.quantize(m.p, m.type, m.rows, m.cols, m.ld, rows ? &q : nullptr, transposed ? &qt : nullptr, at.stream), "sim_op_quantize");
  if (rows && transposed) return py::make_tuple(c, s, ct, st);
  return rows ? py::make_tuple(c, s) : py::make_tuple(ct, st);
}

Tensor matmul(const Tensor& a, const Tensor& a_scales, const Tensor& b, const Tensor& b_scales, int64_t k, at::ScalarType out_dtype,
              const Maybe& out, bool accumulate) {
  int64_t m, n;
  const sim_blocks ba = block_form(a, a_scales, k, "a", &m), bb = block_form(b, b_scales, k, "b", &n);
  const Place at(a);
  at.on(a_scales);
  at.on(b);
  at.on(b_scales);
  at.on(out);
  require(out || !accumulate, "accumulate needs out");
  const Tensor c = out ? *out : at.empty({m, n}, out_dtype);
  const Matrix o = matrix(c, "out");
  if (o.rows != m || o.cols != n) refuse("out: one row for each of a's, one column for each of b's rows");
  const size_t size = L.matmul_workspace(m, n, k);
  const Tensor ws = at.bytes(size);
  check(L.matmul(&ba, &bb, m, n, k, o.p, o.type, o.ld, accumulate, ptr_or_null(ws), size, at.stream), "sim_op_matmul");
  if (out) written(c);
  return c;
}

Tensor linear(const Tensor& x, const Tensor& codes, const Tensor& scales, const Maybe& out) {
  const Matrix m = matrix(x, "x");
  int64_t n;
  const sim_blocks w = block_form(codes, scales, m.cols, "weight", &n);
  const Place at(x);
  at.on(codes);
  at.on(scales);
  at.on(out);
  const Tensor y = out ? *out : at.empty({m.rows, n}, x.scalar_type());
  const Matrix o = matrix(y, "out");
  require(o.type == m.type && o.rows == m.rows && o.cols == n, "out: x's type, one column for each row of the weight");
  const size_t size = L.linear_workspace(m.rows, n, m.cols);
  const Tensor ws = at.bytes(size);
  check(L.linear(m.p, m.type, m.ld, &w, m.rows, n, m.cols, o.p, o.ld, ptr_or_null(ws), size, at.stream), "sim_op_linear");
  if (out) written(y);
  return y;
}

// ---------------------------------------------------------------- norms
float* vector_of(const Place& at, const Maybe& t, int64_t hidden, const char* what) {
  if (!t) return nullptr;
  at.on(t);
  if (t->scalar_type() != at::kFloat || t->numel() != hidden || !t->is_contiguous())
    refuse(std::string(what) + ": one 32-bit value for each channel");
  return (float*)t->data_ptr();
}
int64_t gate_of(const Place& at, const Maybe& gate, int64_t rows, int64_t hidden, const Tensor& y, const std::optional<int64_t>& per) {
  int64_t r = rows > 1 ? rows : 1;
  if (!gate) return r;
  at.on(gate);
  if (per) {
    require(*per >= 1, "rows_per_gate: at least 1");
    r = std::min(*per, r);
  }
  const int64_t groups = std::max<int64_t>(1, (rows + r - 1) / r);
  const Tensor& g = *gate;
  require(g.scalar_type() == y.scalar_type() && g.is_contiguous() && (g.dim() == 1 || g.dim() == 2) && g.size(-1) == hidden &&
              g.numel() == groups * hidden,
          "gate: y's type, a row of the hidden size for each rows_per_gate tokens");
  return r;
}
Matrix residual(const Tensor& h, int act) {
  const Matrix m = matrix(h, "h");
  require(act != SIM_NONE && (m.type == act || m.type == SIM_FP32), "h has y's type or 32 bits");
  require(m.cols >= 1, "h has columns");
  return m;
}
Matrix like(const Place& at, const Tensor& t, const char* what, int type, const Matrix& h) {
  at.on(t);
  const Matrix m = matrix(t, what);
  if (m.type != type || m.rows != h.rows || m.cols != h.cols) refuse(std::string(what) + ": the type and shape of what it belongs to");
  return m;
}

py::tuple norm(const Tensor& h, const Maybe& y, const Maybe& gate, const Maybe& post_weight, const Maybe& post_bias,
               const Maybe& pre_weight, const Maybe& pre_bias, int post, int pre, double alpha, double beta, double eps,
               const std::optional<int64_t>& rows_per_gate, bool quantized, const Maybe& out, const std::optional<at::ScalarType>& act_dtype) {
  const at::ScalarType act_type = y ? y->scalar_type() : act_dtype ? *act_dtype : h.scalar_type();
  const int act = type_of(act_type);
  const Matrix m = residual(h, act);
  const Place at(h);
  sim_norm_args a = {};
  a.rows = m.rows; a.hidden = m.cols; a.act = act; a.res = m.type; a.post = post; a.pre = pre;
  a.alpha = (float)alpha; a.beta = (float)beta; a.eps = (float)eps;
  a.h = m.p; a.ld_h = m.ld;
  a.post_weight = vector_of(at, post_weight, m.cols, "post_weight");
  a.post_bias = vector_of(at, post_bias, m.cols, "post_bias");
  a.pre_weight = vector_of(at, pre_weight, m.cols, "pre_weight");
  a.pre_bias = vector_of(at, pre_bias, m.cols, "pre_bias");
  Tensor sum = h, x, x_scale, post_stats, pre_stats;
  sim_blocks xq;
  a.rows_per_gate = 1;
  if (y) {
    const Matrix ym = like(at, *y, "y", act, m);
    a.y = ym.p; a.ld_y = ym.ld;
    a.rows_per_gate = gate_of(at, gate, m.rows, m.cols, *y, rows_per_gate);
    a.gate = ptr(gate);
    if (post) {
      post_stats = at.empty({2, m.rows}, at::kFloat);
      a.post_stats = (float*)post_stats.data_ptr();
    }
    sum = out ? *out : at.empty({m.rows, m.cols}, h.scalar_type());
    const Matrix o = like(at, sum, "out", m.type, m);
    a.h_out = o.p; a.ld_h_out = o.ld;
  } else {
    require(!gate && !out && !post, "gate, out and post need y");
  }
  if (pre) {
    pre_stats = at.empty({2, m.rows}, at::kFloat);
    a.pre_stats = (float*)pre_stats.data_ptr();
    if (quantized) {
      xq = new_blocks(at, m.rows, m.cols, 1, &x, &x_scale);
      a.xq = &xq;
    } else {
      x = at.empty({m.rows, m.cols}, act_type);
      a.x = x.data_ptr(); a.ld_x = m.cols;
    }
  } else {
    require(!quantized, "quantized needs pre");
  }
  if (m.rows) check(L.norm(&a, at.stream), "sim_op_norm");
  if (out) written(sum);
  auto give = [](const Tensor& t) { return t.defined() ? py::cast(t) : py::object(py::none()); };
  return py::make_tuple(sum, give(x), give(x_scale), give(post_stats), give(pre_stats));
}

py::tuple norm_backward(const Maybe& dh, const Maybe& dx, const Tensor& h, const Maybe& y, const Maybe& gate, const Maybe& post_weight,
                        const Maybe& post_bias, const Maybe& pre_weight, const Maybe& post_stats, const Maybe& pre_stats, int post,
                        int pre, double alpha, double beta, const std::optional<int64_t>& rows_per_gate, const Maybe& pre_bias) {
  require(y || dx, "y or dx is there");
  const at::ScalarType act_type = y ? y->scalar_type() : dx->scalar_type();
  const int act = type_of(act_type);
  const Matrix m = residual(h, act);
  const Place at(h);
  auto stats = [&](const Maybe& t, const char* what) {
    if (!t || t->scalar_type() != at::kFloat || !t->is_contiguous() || t->dim() != 2 || t->size(0) != 2 || t->size(1) != m.rows)
      refuse(std::string(what) + ": the forward pass's [2, rows]");
    at.on(t);
    return (const float*)t->data_ptr();
  };
  sim_norm_grad_args a = {};
  a.rows = m.rows; a.hidden = m.cols; a.act = act; a.res = m.type; a.post = post; a.pre = pre;
  a.alpha = (float)alpha; a.beta = (float)beta;
  a.h = m.p; a.ld_h = m.ld;
  if (dh) {
    const Matrix d = like(at, *dh, "dh", m.type, m);
    a.dh_out = d.p; a.ld_dh_out = d.ld;
  }
  if (pre) {
    require(dx.has_value(), "dx is needed with pre");
    const Matrix d = like(at, *dx, "dx", act, m);
    a.dx = d.p; a.ld_dx = d.ld;
    a.pre_stats = stats(pre_stats, "pre_stats");
  }
  Tensor dy, dgate, out = at.empty({m.rows, m.cols}, h.scalar_type()), sums[4];
  a.rows_per_gate = m.rows > 1 ? m.rows : 1;
  if (y) {
    const Matrix ym = like(at, *y, "y", act, m);
    a.y = ym.p; a.ld_y = ym.ld;
    a.rows_per_gate = gate_of(at, gate, m.rows, m.cols, *y, rows_per_gate);
    a.gate = ptr(gate);
    dy = at.empty({m.rows, m.cols}, act_type);
    a.dy = dy.data_ptr(); a.ld_dy = m.cols;
    if (gate) {
      dgate = at.empty(gate->sizes(), at::kFloat);
      a.dgate = (float*)dgate.data_ptr();
    }
    if (post) a.post_stats = stats(post_stats, "post_stats");
  } else {
    require(!gate && !post, "gate and post need y");
  }
  a.post_weight = vector_of(at, post_weight, m.cols, "post_weight");
  a.post_bias = vector_of(at, post_bias, m.cols, "post_bias");
  a.pre_weight = vector_of(at, pre_weight, m.cols, "pre_weight");
  a.dh = out.data_ptr(); a.ld_dh = m.cols;
  // a bias has a gradient after a layer norm, and wherever the forward pass took one (its values count in dgate alone)
  const bool post_sum = post == SIM_NORM_LAYER || (post != SIM_NORM_NONE && a.post_bias);
  const bool pre_sum = (vector_of(at, pre_bias, m.cols, "pre_bias") && pre != SIM_NORM_NONE) || pre == SIM_NORM_LAYER;
  const bool wanted[4] = {post != SIM_NORM_NONE, post_sum, pre != SIM_NORM_NONE, pre_sum};
  float** places[4] = {&a.dpost_weight, &a.dpost_bias, &a.dpre_weight, &a.dpre_bias};
  for (int i = 0; i < 4; ++i)
    if (wanted[i]) {
      sums[i] = at.empty({m.cols}, at::kFloat);
      *places[i] = (float*)sums[i].data_ptr();
    }
  if (m.rows) {
    const size_t size = L.norm_backward_workspace(m.rows, m.cols, a.rows_per_gate);
    const Tensor ws = at.bytes(size);
    check(L.norm_backward(&a, ptr_or_null(ws), size, at.stream), "sim_op_norm_backward");
  } else {
    for (Tensor& t : sums)
      if (t.defined()) t.zero_();
    if (dgate.defined()) dgate.zero_();
  }
  auto give = [](const Tensor& t) { return t.defined() ? py::cast(t) : py::object(py::none()); };
  return py::make_tuple(out, give(dy), give(dgate), give(sums[0]), give(sums[1]), give(sums[2]), give(sums[3]));
}

// ---------------------------------------------------------------- AdamW
typedef std::vector<Tensor> List;

void adamw(const List& p, const List& g, const List& m, const List& v, const std::optional<List>& copies, const std::optional<List>& m_scales,
           const std::optional<List>& v_scales, int64_t step, double lr, double beta1, double beta2, double eps,
           const std::vector<double>& decays, const Maybe& grad_scale, const Maybe& skip, uint64_t seed) {
  const size_t n = p.size();
  require(m_scales.has_value() == v_scales.has_value(), "both moments have scales, or none");
  const bool eight = m_scales.has_value();
  const List* lists[7] = {&p, &g, &m, &v, copies ? &*copies : nullptr, eight ? &*m_scales : nullptr, eight ? &*v_scales : nullptr};
  for (const List* l : lists) require(!l || l->size() == n, "lists of one length");
  require(decays.size() == 1 || decays.size() == n, "one weight decay, or one for each tensor");
  if (n == 0) return;
  const Place at(p[0], true);   // (parameters require gradients: a step on them is no part of what is recorded)
  for (const List* l : lists) {
    if (!l) continue;
    const at::ScalarType type = (*l)[0].scalar_type();
    for (const Tensor& t : *l)
      require(t.scalar_type() == type && t.device() == at.device && t.is_contiguous(), "contiguous tensors of one type on one device");
  }
  const at::ScalarType state = eight ? kE4m3 : at::kFloat;
  require(m[0].scalar_type() == state && v[0].scalar_type() == state, "moments in float32, or in e4m3 with scales");
  require(!eight || ((*m_scales)[0].scalar_type() == at::kFloat && (*v_scales)[0].scalar_type() == at::kFloat), "scales in float32");
  sim_adamw_args a = {};
  a.p_dtype = type_of(p[0], "parameters");
  a.grad_dtype = type_of(g[0], "gradients");
  a.copy_dtype = copies ? type_of((*copies)[0], "copies") : SIM_NONE;
  a.state_bits = eight ? 8 : 32;
  a.lr = lr; a.beta1 = beta1; a.beta2 = beta2; a.eps = eps; a.step = step; a.seed = seed;
  at.on(grad_scale);
  at.on(skip);
  require(!grad_scale || (grad_scale->scalar_type() == at::kFloat && grad_scale->numel() == 1), "grad_scale: one float32");
  require(!skip || (skip->scalar_type() == at::kInt && skip->numel() == 1), "skip: one int32");
  a.grad_scale = (const float*)ptr(grad_scale);
  a.skip = (const uint32_t*)ptr(skip);
  std::vector<sim_adamw_tensor> table(n);
  uint64_t first = 0;
  for (size_t i = 0; i < n; ++i) {
    const int64_t size = p[i].numel(), blocks = blocks_of(size);
    require(g[i].numel() == size && m[i].numel() == size && v[i].numel() == size && (!copies || (*copies)[i].numel() == size),
            "one size in every list for a tensor");
    require(!eight || ((*m_scales)[i].numel() == blocks && (*v_scales)[i].numel() == blocks), "a scale for each 128 elements of a tensor");
    table[i] = {ptr(p[i]), ptr(g[i]), ptr(m[i]), ptr(v[i]), eight ? (float*)ptr((*m_scales)[i]) : nullptr,
                eight ? (float*)ptr((*v_scales)[i]) : nullptr, copies ? ptr((*copies)[i]) : nullptr, size, first,
                (float)decays[decays.size() == 1 ? 0 : i]};
    first += (uint64_t)(blocks * SIM_BLOCK);
  }
  // (a failed call may have begun: all lists but the gradients' count as written)
  for (const List* l : lists)
    if (l && l != &g)
      for (const Tensor& t : *l) written(t);
  check(L.adamw(table.data(), (int64_t)n, &a, at.stream), "sim_op_adamw");
}

}  // namespace

PYBIND11_MODULE(_ops, m) {
  m.def("load", &load);
  m.def("quantize", &quantize);
  m.def("matmul", &matmul);
  m.def("linear", &linear);
  m.def("norm", &norm);
  m.def("norm_backward", &norm_backward);
  m.def("adamw", &adamw);
}
