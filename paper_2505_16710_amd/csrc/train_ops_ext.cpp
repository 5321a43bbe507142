// Binding of the operators around the training step (train_ops_api.cpp).  Third source of the extension module.
#include <algorithm>
#include <cstring>
#include <memory>

#include <ATen/hip/EmptyTensor.h>
#include <c10/core/DeviceGuard.h>

#include "binding_common.h"

namespace seco_ext {
namespace {

// A call's tensors are on one GPU, which is the current device while it runs; its stream, unless one is given, is that GPU's
// current one.
struct OnGpu {
  c10::DeviceGuard guard;
  void* s;
  OnGpu(const Tensor& t, PyObject* o) : guard(t.device()), s(o == Py_None ? c10::hip::getCurrentHIPStream(t.device().index()).stream() : stream(o)) {}
};
// Where a tensor's elements lie, of a buffer [B, H, N, D] those of rows [row, row + rows): all in [at, end)
struct Spread {
  uintptr_t at, end;
  const Tensor& t;
  int64_t rows;
  explicit Spread(const Tensor& t, int64_t row = 0, int64_t rows = -1) : t(t), rows(rows) {
    const int64_t e = t.element_size();
    at = reinterpret_cast<uintptr_t>(t.data_ptr()) + (uintptr_t)(rows < 0 ? 0 : row * t.stride(2) * e);
    end = at + (uintptr_t)e;
    for (int64_t i = 0; i < t.dim(); ++i) {
      if (size(i) == 0) {                        // nothing lies anywhere
        end = at;
        return;
      }
      end += (uintptr_t)((size(i) - 1) * t.stride(i) * e);
    }
  }
  int64_t size(int64_t i) const { return i == 2 && rows >= 0 ? rows : t.size(i); }
};
// The distances of two tensors' elements: sums of stride * i with first <= i <= last for every stride, and of pieces without
// gaps `width` bytes behind each.  Elements meet if such a sum comes to lie in a range.
struct Distances {
  struct Term {
    int64_t stride, first, last;
  };
  c10::SmallVector<Term, 8> terms;
  int budget = 1000;                             // sums looked at
  // the tensor's dimensions by their strides; those that leave no gap make a piece
  int64_t add(const Spread& x, int sign) {
    c10::SmallVector<std::pair<int64_t, int64_t>, 8> dims;
    for (int64_t i = 0; i < x.t.dim(); ++i)
      if (x.size(i) > 1) dims.emplace_back(x.t.stride(i) * (int64_t)x.t.element_size(), x.size(i) - 1);
    std::sort(dims.begin(), dims.end());
    int64_t width = x.t.element_size();
    size_t i = 0;
    for (; i < dims.size() && dims[i].first <= width; ++i) width += dims[i].first * dims[i].second;
    for (; i < dims.size(); ++i) {
      const int64_t stride = dims[i].first, last = dims[i].second;
      auto* at = std::find_if(terms.begin(), terms.end(), [&](const Term& t) { return t.stride == stride; });
      if (at == terms.end()) at = terms.insert(at, Term{stride, 0, 0});
      (sign > 0 ? at->last : at->first) += sign * last;
    }
    return width;
  }
  // whether a sum over the terms from the k-th on (largest strides first) lies in [low, high]; not, if the budget is used up
  bool reach(size_t k, int64_t low, int64_t high) {
    if (k == terms.size()) return low <= 0 && 0 <= high;
    int64_t least = 0, most = 0;                 // of what follows
    for (size_t i = k + 1; i < terms.size(); ++i) least += terms[i].stride * terms[i].first, most += terms[i].stride * terms[i].last;
    const Term& t = terms[k];
    auto down = [](int64_t a, int64_t b) { return a / b - (a % b < 0); };
    const int64_t first = std::max(t.first, -down(most - low, t.stride)), last = std::min(t.last, down(high - least, t.stride));
    for (int64_t i = first; i <= last && --budget >= 0; ++i)
      if (reach(k + 1, low - i * t.stride, high - i * t.stride)) return true;
    return false;
  }
};
// Whether two tensors share memory: their ranges first, then, where these meet (columns of one buffer), their elements.  Layouts that
// would take long to tell apart count as apart.
bool share(const Spread& a, const Spread& b) {
  if (a.end <= b.at || b.end <= a.at || a.at == a.end || b.at == b.end) return false;
  Distances x;
  const int64_t wide_a = x.add(a, 1), wide_b = x.add(b, -1), off = (int64_t)(a.at - b.at);
  std::sort(x.terms.begin(), x.terms.end(), [](const auto& p, const auto& q) { return p.stride > q.stride; });
  return x.reach(0, 1 - wide_a - off, wide_b - 1 - off);
}
void need_apart(const Spread& a, const Spread& b, const char* name, const char* other) {
  if (!share(a, b)) return;
  PyErr_Format(PyExc_ValueError, "%s overlaps %s", name, other);
  throw Raised{};
}
// a result in the place of an input lies there element for element; else it shares nothing with it, since other workgroups may
// have yet to read what one has written
void in_place_or_apart(const Tensor& out, const Tensor& in, const char* name, const char* other) {
  if (out.numel() == 0) return;
  if (out.data_ptr() != in.data_ptr()) return need_apart(Spread(out), Spread(in), name, other);
  for (int64_t i = 0; i < in.dim(); ++i)
    if (in.size(i) > 1 && out.stride(i) != in.stride(i)) {
      PyErr_Format(PyExc_ValueError, "%s: in the place of an input it needs that one's strides", name);
      throw Raised{};
    }
}
// A new tensor on a GPU tensor's device, without the way through the dispatcher: 0.3 us less of the host's time, which is what a
// short call takes (layer norm of 32 rows, four tensors: 7.2 -> 6.3 us)
Tensor fresh(at::IntArrayRef sizes, at::ScalarType type, const Tensor& there) {
  return Tensor(at::detail::empty_cuda(sizes, type, there.device(), std::nullopt));
}
// laid out like the other where that one is dense
Tensor fresh_like(const Tensor& t) { return t.is_contiguous() ? fresh(t.sizes(), t.scalar_type(), t) : at::empty_like(t, t.options().requires_grad(false)); }
void same_gpu(const Tensor& a, const Tensor& b) {
  if (!a.is_cuda() || a.device() != b.device()) raise(PyExc_ValueError, "the tensors must be on one GPU");
}

// [..., d] seen as rows of d elements at one distance from each other
struct Rows {
  int64_t n = 1, d = 0, stride = 0;
};
Rows rows_of(const Tensor& t, const char* name) {
  Rows r;
  const int64_t k = t.dim();
  if (k < 1 || t.size(k - 1) < 1 || (t.size(k - 1) > 1 && t.stride(k - 1) != 1)) {
    PyErr_Format(PyExc_ValueError, "%s: expected [..., d] with contiguous rows of at least one element", name);
    throw Raised{};
  }
  r.d = r.stride = t.size(k - 1);
  bool even = true;
  int64_t inner = 1;                             // rows in the dimensions behind this one
  for (int64_t i = k - 2; i >= 0; --i) {
    if (t.size(i) != 1) {
      if (inner == 1) r.stride = t.stride(i);
      else even = even && t.stride(i) == r.stride * inner;
      inner *= t.size(i);
    }
  }
  r.n = inner;
  if (!even && r.n > 0) {
    PyErr_Format(PyExc_ValueError, "%s: its rows must lie at one distance from each other", name);
    throw Raised{};
  }
  return r;
}
Rows rows_like(const Tensor& t, const Tensor& x, const char* name) {
  if (t.sizes() != x.sizes() || t.scalar_type() != x.scalar_type()) {
    PyErr_Format(PyExc_ValueError, "%s must have the shape and dtype of x", name);
    throw Raised{};
  }
  return rows_of(t, name);
}
void vector_of(const Tensor& t, int64_t d, at::ScalarType type, const char* name) {
  if (t.dim() != 1 || t.size(0) != d || !t.is_contiguous() || t.scalar_type() != type) {
    PyErr_Format(PyExc_ValueError, "%s: expected a contiguous [%lld] tensor of the gain's dtype", name, (long long)d);
    throw Raised{};
  }
}
// the type of gain and bias (none: given, or the rows')
at::ScalarType gain_type(const Tensor& x, const Tensor* gain, const Tensor* bias, PyObject* given = Py_None) {
  at::ScalarType t = gain ? gain->scalar_type() : bias ? bias->scalar_type() : x.scalar_type();
  if (given != Py_None) {
    if (!THPDtype_Check(given)) raise(PyExc_TypeError, "dtype must be a torch dtype");
    const at::ScalarType wanted = reinterpret_cast<THPDtype*>(given)->scalar_type;
    if (gain && wanted != t) raise(PyExc_TypeError, "dtype: with a gain, its dtype");
    t = wanted;
  }
  if (t != x.scalar_type() && t != at::kFloat) raise(PyExc_TypeError, "gain and bias must have x's dtype or float32");
  return t;
}
Tensor given_or(PyObject* o, const Tensor& like_t) {
  return o == Py_None ? fresh(like_t.sizes(), like_t.scalar_type(), like_t) : tensor(o);
}
PyObject* out_ref(PyObject* o, const Tensor& t) { return o == Py_None ? THPVariable_Wrap(t) : (Py_INCREF(o), o); }

layer_norm_desc norm_desc(const Tensor& x, const Rows& rows, at::ScalarType gain) {
  layer_norm_desc d{};
  d.rows = rows.n;
  d.d = rows.d;
  d.x_stride = d.residual_stride = d.out_stride = d.y_stride = rows.stride;
  d.dtype = dtype_code(x);
  d.gain_dtype = gain == at::kFloat ? SECO_F32 : SECO_BF16;
  return d;
}

// (x, gain, bias, eps, residual, y, x_out, stream) -> (y, mean, rstd) or, with a residual, (y, mean, rstd, x_out)
PyObject* norm_fwd(PyObject* const* a) {
  const Tensor& x = tensor(a[0]);
  const Tensor *gain = opt_tensor(a[1]), *bias = opt_tensor(a[2]), *res = opt_tensor(a[4]);
  const Rows rows = rows_of(x, "x");
  const at::ScalarType gt = gain_type(x, gain, bias);
  layer_norm_desc d = norm_desc(x, rows, gt);
  d.eps = (float)real(a[3]);
  if (gain) vector_of(*gain, rows.d, gt, "gain");
  if (bias) vector_of(*bias, rows.d, gt, "bias");
  if (res) d.residual_stride = rows_like(*res, x, "residual").stride;
  else if (a[6] != Py_None) raise(PyExc_ValueError, "x_out goes with a residual");
  const Tensor *y_given = opt_tensor(a[5]), *out_given = opt_tensor(a[6]);
  for (const Tensor* t : {y_given, out_given})
    if (t) {
      const char* name = t == y_given ? "y" : "x_out";
      rows_like(*t, x, name);
      in_place_or_apart(*t, x, name, "x");
      if (res) in_place_or_apart(*t, *res, name, "residual");
    }
  if (y_given && out_given) need_apart(Spread(*y_given), Spread(*out_given), "y", "x_out");
  for (const Tensor* t : {&x, gain, bias, res, y_given, out_given})
    if (t) same_gpu(x, *t);
  OnGpu on(x, a[7]);
  const Tensor y = given_or(a[5], x);
  Tensor out;
  if (res) out = given_or(a[6], x);
  const auto lead = x.sizes().slice(0, x.dim() - 1);
  const Tensor mean = fresh(lead, at::kFloat, x), rstd = fresh(lead, at::kFloat, x);
  d.y_stride = rows_of(y, "y").stride;
  if (res) d.out_stride = rows_of(out, "x_out").stride;
  if (rows.n > 0)
    check(lib.layer_norm_fwd(&d, ptr(x), ptr(res), ptr(gain), ptr(bias), res ? ptr(out) : nullptr, ptr(y), fptr(mean), fptr(rstd), on.s),
          "layer_norm_fwd");
  if (!res) return Py_BuildValue("NNN", out_ref(a[5], y), THPVariable_Wrap(mean), THPVariable_Wrap(rstd));
  return Py_BuildValue("NNNN", out_ref(a[5], y), THPVariable_Wrap(mean), THPVariable_Wrap(rstd), out_ref(a[6], out));
}

// (x, gain, mean, rstd, d_y, d_in, d_x, with_gain, with_bias, ws, stream, dtype or None) -> (d_x, d_gain or None, d_bias or None)
PyObject* norm_bwd(PyObject* const* a) {
  const Tensor &x = tensor(a[0]), &mean = tensor(a[2]), &rstd = tensor(a[3]), &dy = tensor(a[4]);
  const Tensor *gain = opt_tensor(a[1]), *in = opt_tensor(a[5]), *dx_given = opt_tensor(a[6]), *ws_given = opt_tensor(a[9]);
  const Rows rows = rows_of(x, "x");
  const at::ScalarType gt = gain_type(x, gain, nullptr, a[11]);
  layer_norm_desc d = norm_desc(x, rows, gt);
  if (gain) vector_of(*gain, rows.d, gt, "gain");
  for (const Tensor* t : {&mean, &rstd})
    if (t->scalar_type() != at::kFloat || !t->is_contiguous() || t->numel() != rows.n)
      raise(PyExc_ValueError, "mean, rstd: contiguous float32, one value per row");
  d.y_stride = rows_like(dy, x, "d_y").stride;
  if (in) d.residual_stride = rows_like(*in, x, "d_in").stride;
  if (dx_given) {
    rows_like(*dx_given, x, "d_x");
    for (const Tensor* t : {&x, &dy, in})
      if (t) in_place_or_apart(*dx_given, *t, "d_x", t == &x ? "x" : t == &dy ? "d_y" : "d_in");
  }
  for (const Tensor* t : {&mean, &rstd, &dy, gain, in, dx_given, ws_given})
    if (t) same_gpu(x, *t);
  const int with_gain = PyObject_IsTrue(a[7]), with_bias = PyObject_IsTrue(a[8]);
  if (with_gain < 0 || with_bias < 0) throw Raised{};
  OnGpu on(x, a[10]);
  const Tensor dx = given_or(a[6], x);
  d.out_stride = rows_of(dx, "d_x").stride;
  Tensor dg, db, ws;
  if (with_gain) dg = fresh({rows.d}, gt, x);
  if (with_bias) db = fresh({rows.d}, gt, x);
  if (with_gain || with_bias) {
    const size_t n = lib.layer_norm_workspace_bytes(&d);
    if (n == (size_t)-1) check(SECO_ERR_SHAPE, "layer_norm_workspace_bytes");
    if (n > 0) ws = ws_given ? *ws_given : scratch((int64_t)n, x, on.s);
  }
  // (an empty tensor has no address; nothing is read or written there)
  void* some = with_gain ? ptr(dg) : with_bias ? ptr(db) : nullptr;
  auto at_or = [&](void* p) { return p || rows.n > 0 ? p : some; };
  if (rows.n > 0 || some)
    check(lib.layer_norm_bwd(&d, at_or(ptr(x)), ptr(gain), static_cast<float*>(at_or(ptr(mean))), static_cast<float*>(at_or(ptr(rstd))),
                             at_or(ptr(dy)), rows.n > 0 ? ptr(in) : nullptr, at_or(ptr(dx)), with_gain ? ptr(dg) : nullptr,
                             with_bias ? ptr(db) : nullptr, ws.defined() ? ptr(ws) : nullptr, ws.defined() ? nbytes(ws) : 0, on.s),
          "layer_norm_bwd");
  auto wrap = [](const Tensor& t) { return t.defined() ? THPVariable_Wrap(t) : (Py_INCREF(Py_None), Py_None); };
  return Py_BuildValue("NNN", out_ref(a[6], dx), wrap(dg), wrap(db));
}

// ---- AdamW
struct Sequence {                                // of tensors, or none
  PyObject* s;
  Py_ssize_t n;
  explicit Sequence(PyObject* o) : s(nullptr), n(0) {
    if (o == Py_None) return;
    s = PySequence_Fast(o, "expected a sequence of tensors");
    if (!s) throw Raised{};
    n = PySequence_Fast_GET_SIZE(s);
  }
  ~Sequence() { Py_XDECREF(s); }
  Sequence(const Sequence&) = delete;
  PyObject* item(Py_ssize_t i) const { return PySequence_Fast_GET_ITEM(s, i); }
  const Tensor& operator[](Py_ssize_t i) const { return tensor(item(i)); }
};
[[noreturn]] void bad(PyObject* type, const char* what, Py_ssize_t i, const char* expected) {
  PyErr_Format(type, "%s[%zd]: %s", what, i, expected);
  throw Raised{};
}
// laid out like the parameter: the same elements at the same places
void same_places(const Tensor& t, const Tensor& p, const char* what, Py_ssize_t i) {
  bool same = t.sizes() == p.sizes();
  for (int64_t k = 0; same && k < p.dim(); ++k) same = p.size(k) < 2 || t.stride(k) == p.stride(k);
  if (!same) bad(PyExc_ValueError, what, i, "must have the shape and strides of its parameter");
  if (t.device() != p.device()) bad(PyExc_ValueError, what, i, "must be on its parameter's device");
}
const float* scalar_on(const Tensor& t, const Tensor& like_t, const char* what) {
  if (t.scalar_type() != at::kFloat || t.numel() != 1 || t.device() != like_t.device()) {
    PyErr_Format(PyExc_ValueError, "%s: a float, or a float32 tensor of one element on the parameters' device", what);
    throw Raised{};
  }
  return fptr(t);
}

// Sorts by merging the runs that are in order already: tensors that were made one behind the other mostly are.
void in_order(std::vector<std::pair<uintptr_t, uintptr_t>>& a) {
  std::vector<size_t> ends;                      // of the runs
  for (size_t i = 1; i <= a.size(); ++i)
    if (i == a.size() || a[i] < a[i - 1]) ends.push_back(i);
  std::vector<std::pair<uintptr_t, uintptr_t>> b(a.size());
  while (ends.size() > 1) {
    size_t begin = 0, kept = 0;
    for (size_t i = 0; i < ends.size(); i += 2) {
      const size_t end = ends[std::min(i + 1, ends.size() - 1)];
      std::merge(a.begin() + begin, a.begin() + ends[i], a.begin() + ends[i], a.begin() + end, b.begin() + begin);
      ends[kept++] = begin = end;
    }
    ends.resize(kept);
    a.swap(b);
  }
}

// (params, grads, m, v, step, lr, beta1, beta2, eps, weight_decay, masters, m_scales, v_scales, grad_scale, stream)
PyObject* adamw(PyObject* const* a) {
  const Sequence params(a[0]), grads(a[1]), ms(a[2]), vs(a[3]), masters(a[10]),
      m_scales(a[11]), v_scales(a[12]);
  const Tensor& step = tensor(a[4]);
  const Py_ssize_t n = params.n;
  if (grads.n != n || ms.n != n || vs.n != n || (masters.s && masters.n != n)) raise(PyExc_ValueError, "one gradient, m, v (and master) per parameter");
  if ((m_scales.s == nullptr) != (v_scales.s == nullptr) || (m_scales.s && (m_scales.n != n || v_scales.n != n)))
    raise(PyExc_ValueError, "states of 8 bits: one m_scale and one v_scale per parameter; states of 32: neither");
  if (step.scalar_type() != at::kLong || step.numel() != 2 || !step.is_contiguous())
    raise(PyExc_ValueError, "step: a contiguous int64 tensor of two elements, steps taken and 0");
  const bool eight = m_scales.s != nullptr, decays = !PyFloat_Check(a[9]) && !PyLong_Check(a[9]);
  std::vector<float> decay;
  if (decays) decay = floats(a[9]);
  if (decays && (Py_ssize_t)decay.size() != n) raise(PyExc_ValueError, "weight_decay: one value, or one per parameter");
  const float one_decay = decays ? 0.f : (float)real(a[9]);
  adamw_desc d{};
  if (THPVariable_Check(a[5])) d.lr_device = scalar_on(tensor(a[5]), step, "lr");
  else d.lr = real(a[5]);
  if (a[13] != Py_None) d.grad_scale_device = scalar_on(tensor(a[13]), step, "grad_scale");
  d.beta1 = real(a[6]);
  d.beta2 = real(a[7]);
  d.eps = real(a[8]);
  d.state_bits = eight ? 8 : 32;
  const auto list = std::make_unique<adamw_tensor[]>((size_t)n);
  for (Py_ssize_t i = 0; i < n; ++i) {
    const Tensor &p = params[i], &g = grads[i], &m = ms[i], &v = vs[i];
    adamw_tensor& t = list[i];
    if ((p.scalar_type() != at::kFloat && p.scalar_type() != at::kBFloat16) || (g.scalar_type() != at::kFloat && g.scalar_type() != at::kBFloat16))
      bad(PyExc_TypeError, "params", i, "parameter and gradient must be bfloat16 or float32");
    if (!p.is_non_overlapping_and_dense()) bad(PyExc_ValueError, "params", i, "must lie dense in memory, in any order of its dimensions");
    if (p.device() != step.device()) bad(PyExc_ValueError, "params", i, "must be on the device of step");
    const at::ScalarType state = eight ? at::kFloat8_e4m3fn : at::kFloat;
    if (m.scalar_type() != state || v.scalar_type() != state)
      bad(PyExc_TypeError, "m, v", i, eight ? "must be float8_e4m3fn beside scales" : "must be float32 without scales");
    same_places(g, p, "grads", i);
    same_places(m, p, "m", i);
    same_places(v, p, "v", i);
    t.n = p.numel();
    t.param = ptr(p);
    t.grad = ptr(g);
    t.m = ptr(m);
    t.v = ptr(v);
    t.param_dtype = dtype_code(p);
    t.grad_dtype = dtype_code(g);
    t.weight_decay = decays ? decay[(size_t)i] : one_decay;
    t.m_scale = t.v_scale = t.master = nullptr;
    if (eight) {
      for (const Tensor* x : {&m_scales[i], &v_scales[i]})
        if (x->scalar_type() != at::kFloat || !x->is_contiguous() || x->numel() != (t.n + 255) / 256 || x->device() != p.device())
          bad(PyExc_ValueError, "m_scales, v_scales", i, "one contiguous float32 per 256 elements of the parameter");
      t.m_scale = fptr(m_scales[i]);
      t.v_scale = fptr(v_scales[i]);
    }
    if (masters.s && masters.item(i) != Py_None) {
      const Tensor& w = masters[i];
      if (w.scalar_type() != at::kFloat || p.scalar_type() != at::kBFloat16) bad(PyExc_TypeError, "masters", i, "float32, of bfloat16 parameters only");
      same_places(w, p, "masters", i);
      t.master = fptr(w);
    }
  }
  std::vector<std::pair<uintptr_t, uintptr_t>> places;        // of what is written
  places.reserve((size_t)n * 6);
  auto written = [&](auto where) {
    for (Py_ssize_t i = 0; i < n; ++i) {
      const std::pair<void*, int64_t> w = where(list[i]);
      if (w.first && w.second > 0) places.emplace_back((uintptr_t)w.first, (uintptr_t)w.first + (uintptr_t)w.second);
    }
  };
  typedef std::pair<void*, int64_t> Place;
  written([](const adamw_tensor& t) { return Place(t.param, t.n * (t.param_dtype == SECO_BF16 ? 2 : 4)); });
  written([&](const adamw_tensor& t) { return Place(t.m, t.n * (eight ? 1 : 4)); });
  written([&](const adamw_tensor& t) { return Place(t.v, t.n * (eight ? 1 : 4)); });
  written([](const adamw_tensor& t) { return Place(t.m_scale, (t.n + 255) / 256 * 4); });
  written([](const adamw_tensor& t) { return Place(t.v_scale, (t.n + 255) / 256 * 4); });
  written([](const adamw_tensor& t) { return Place(t.master, t.n * 4); });
  in_order(places);
  for (size_t i = 1; i < places.size(); ++i)
    if (places[i].first < places[i - 1].second) raise(PyExc_ValueError, "params and their states: two of them overlap, or one is there twice");
  if (!step.is_cuda()) raise(PyExc_ValueError, "the tensors must be on one GPU");
  OnGpu on(step, a[14]);
  check(lib.adamw_step(&d, list.get(), (int32_t)n, static_cast<int64_t*>(ptr(step)), on.s), "adamw_step");
  // (what autograd has kept of a parameter's old values is out of date now)
  for (Py_ssize_t i = 0; i < n; ++i)
    if (!params[i].is_inference()) params[i].unsafeGetTensorImpl()->bump_version();
  Py_RETURN_NONE;
}

// ---- rotary positions with several axes
struct Axes {
  rope_axes x;
  int64_t head_dim = 0;
  explicit Axes(PyObject* o) {
    char* p;
    Py_ssize_t n;
    if (PyBytes_AsStringAndSize(o, &p, &n) < 0) throw Raised{};
    if (n != (Py_ssize_t)sizeof(x)) raise(PyExc_TypeError, "axes: expected a RopeAxes");
    memcpy(&x, p, sizeof(x));
    for (int i = 0; i < x.n_axes && i < SECO_ROPE_MAX_AXES; ++i) head_dim += 2 * (int64_t)x.sections[i];
  }
};
// int64 [axes, B or 1, rows]; strides in elements
void positions_of(const Tensor& t, const Axes& axes, int64_t B, int64_t rows, int64_t out[3]) {
  if (t.scalar_type() != at::kLong || t.dim() != 3 || t.size(0) != axes.x.n_axes || (t.size(1) != B && t.size(1) != 1) || t.size(2) != rows) {
    PyErr_Format(PyExc_ValueError, "positions: expected int64 [%d, %lld or 1, %lld]", (int)axes.x.n_axes, (long long)B, (long long)rows);
    throw Raised{};
  }
  for (int i = 0; i < 3; ++i) out[i] = t.size(i) == 1 ? 0 : t.stride(i);
}
void heads_tensor(const Tensor& t, const char* name, int64_t B, int64_t rows, int64_t D, at::ScalarType type) {
  if (t.dim() == 4 && t.size(0) == B && t.size(2) == rows && t.size(3) == D && t.stride(3) == 1 && t.scalar_type() == type) return;
  PyErr_Format(PyExc_ValueError, "%s: expected a [%lld, heads, %lld, %lld] tensor of the call's dtype with contiguous head_dim", name,
               (long long)B, (long long)rows, (long long)D);
  throw Raised{};
}
// k / v or their like: one shape and type
void like_each_other(const Tensor& a, const Tensor& b, const char* names) {
  if (a.sizes() == b.sizes() && a.scalar_type() == b.scalar_type()) return;
  PyErr_Format(PyExc_ValueError, "%s must share shape and dtype", names);
  throw Raised{};
}
// rows [begin, begin + n) of a cache or gradient buffer [B, H, N, D]
void rows_inside(const Tensor& t, const char* name, int64_t B, int64_t H, int64_t D, int64_t begin, int64_t n, at::ScalarType type) {
  if (t.dim() == 4 && t.size(0) == B && t.size(1) == H && t.size(3) == D && t.stride(3) == 1 && t.scalar_type() == type && begin >= 0 &&
      begin <= t.size(2) - n)
    return;
  PyErr_Format(PyExc_ValueError, "%s: expected [%lld, %lld, rows, %lld] with contiguous head_dim that holds rows %lld to %lld", name,
               (long long)B, (long long)H, (long long)D, (long long)begin, (long long)(begin + n));
  throw Raised{};
}
// what is written: every element at a place of its own
void writable(const Tensor& t, const char* name) {
  for (int64_t i = 0; i < t.dim(); ++i)
    if (t.size(i) > 1 && t.stride(i) == 0) {
      PyErr_Format(PyExc_ValueError, "%s: an expanded tensor cannot be written", name);
      throw Raised{};
    }
}
// whether a tensor lies element for element where those rows of a buffer do
bool in_place(const Spread& rows, const Tensor& t) {
  if (rows.at != reinterpret_cast<uintptr_t>(t.data_ptr()) || rows.t.scalar_type() != t.scalar_type()) return false;
  for (int i = 0; i < 4; ++i)
    if (t.size(i) > 1 && t.stride(i) != rows.t.stride(i)) return false;
  return true;
}
// a dimension of one element may have any stride; the library asks for one that keeps rows on their boundaries
void heads_strides(const Tensor& t, int64_t out[3]) {
  for (int i = 0; i < 3; ++i) out[i] = t.size(i) == 1 ? (i == 2 ? t.size(3) : 0) : t.stride(i);
}
// The library's calls take keys and values in one layout; where theirs differ, values take a call of their own.
bool one_layout(const Tensor& a, const Tensor& b) {
  for (int64_t i = 0; i < a.dim(); ++i)
    if (a.size(i) > 1 && a.stride(i) != b.stride(i)) return false;
  return true;
}
// ... of which nothing may be refused once the first is on its way: what the library asks of rows and their distances
void rows_aligned(const Tensor& t, const char* where) {
  int64_t st[3];
  heads_strides(t, st);
  const int64_t e = t.element_size();
  for (int i = 0; i < 3; ++i) {
    if (st[i] > (int64_t)1 << (i == 2 ? 30 : 40)) check(SECO_ERR_TOO_LARGE, where);
    if (st[i] * e % 16) check(SECO_ERR_ALIGN, where);
  }
  if (st[2] < t.size(3) || reinterpret_cast<uintptr_t>(t.data_ptr()) % 16) check(SECO_ERR_ALIGN, where);
}
seco_desc axes_desc(int64_t B, int64_t rows, int64_t D, at::ScalarType type, int64_t row_begin, const char* where) {
  if (B > 65535 || rows > 1 << 27 || D > 256 || row_begin > (int64_t)1 << 30) check(SECO_ERR_TOO_LARGE, where);
  seco_desc d{};
  d.q_start = (int32_t)row_begin;
  d.batch = (int32_t)B;
  d.n_q_heads = d.n_kv_heads = 1;
  d.chunk_len = (int32_t)rows;
  d.head_dim = (int32_t)D;
  d.dtype = type == at::kBFloat16 ? SECO_BF16 : SECO_F32;
  d.softmax_scale = 1.f;
  return d;
}
void fits_axes(const Axes& axes, int64_t D) {
  if (axes.head_dim == D) return;
  PyErr_Format(PyExc_ValueError, "axes: their sections make a head_dim of %lld, not %lld", (long long)axes.head_dim, (long long)D);
  throw Raised{};
}

// (x, positions, axes, inverse, out, stream) -> out
PyObject* rotate_axes(PyObject* const* a) {
  const Tensor &x = tensor(a[0]), &pos = tensor(a[1]);
  const Axes axes(a[2]);
  dtype_code(x);
  if (x.dim() != 4) raise(PyExc_ValueError, "x: expected a [batch, head, row, head_dim] tensor");
  const int64_t B = x.size(0), C = x.size(2), D = x.size(3);
  heads_tensor(x, "x", B, C, D, x.scalar_type());
  fits_axes(axes, D);
  seco_desc d = axes_desc(B, C, D, x.scalar_type(), 0, "rope_rotate_axes");
  int64_t ps[3];
  positions_of(pos, axes, B, C, ps);
  const int inv = PyObject_IsTrue(a[3]);
  if (inv < 0) throw Raised{};
  if (a[4] != Py_None) {
    const Tensor& o = tensor(a[4]);
    heads_tensor(o, "out", B, C, D, x.scalar_type());
    writable(o, "out");
    if (o.size(1) != x.size(1)) raise(PyExc_ValueError, "out must have the shape of x");
    in_place_or_apart(o, x, "out", "x");
    same_gpu(x, o);
  }
  same_gpu(x, pos);
  OnGpu on(x, a[5]);
  const Tensor out = a[4] == Py_None ? fresh_like(x) : tensor(a[4]);
  heads_strides(x, d.q_stride);
  heads_strides(out, d.o_stride);
  if (x.numel() > 0)
    check(lib.rope_rotate_axes(&d, &axes.x, (int32_t)x.size(1), ptr(x), ptr(out), static_cast<const int64_t*>(ptr(pos)), ps, inv, on.s),
          "rope_rotate_axes");
  return out_ref(a[4], out);
}

// (q or None, k_new, v_new, k_cache, v_cache, row_begin, positions, axes, q_out, stream) -> q_out or None
PyObject* append_axes(PyObject* const* a) {
  const Tensor* q = opt_tensor(a[0]);
  const Tensor &kn = tensor(a[1]), &vn = tensor(a[2]), &kc = tensor(a[3]), &vc = tensor(a[4]), &pos = tensor(a[6]);
  const Axes axes(a[7]);
  const int64_t row = integer(a[5]);
  dtype_code(kn);
  if (kn.dim() != 4) raise(PyExc_ValueError, "k_new: expected a [batch, head, row, head_dim] tensor");
  const int64_t B = kn.size(0), Hkv = kn.size(1), C = kn.size(2), D = kn.size(3);
  heads_tensor(kn, "k_new", B, C, D, kn.scalar_type());
  if (Hkv < 1) raise(PyExc_ValueError, "k_new: expected at least one head");
  fits_axes(axes, D);
  like_each_other(kn, vn, "k_new and v_new");
  like_each_other(kc, vc, "k_cache and v_cache");
  heads_tensor(vn, "v_new", B, C, D, kn.scalar_type());
  rows_inside(kc, "k_cache", B, Hkv, D, row, C, kn.scalar_type());
  rows_inside(vc, "v_cache", B, Hkv, D, row, C, kn.scalar_type());
  writable(kc, "k_cache");
  writable(vc, "v_cache");
  if (q) heads_tensor(*q, "q", B, C, D, kn.scalar_type());
  seco_desc d = axes_desc(B, C, D, kn.scalar_type(), row, "rope_append_axes");
  int64_t ps[3];
  positions_of(pos, axes, B, C, ps);
  if (a[8] != Py_None) {
    const Tensor& o = tensor(a[8]);
    heads_tensor(o, "q_out", B, C, D, kn.scalar_type());
    writable(o, "q_out");
    if (!q || o.size(1) != q->size(1)) raise(PyExc_ValueError, "q_out must have the shape of q");
    in_place_or_apart(o, *q, "q_out", "q");
    need_apart(Spread(o), Spread(kn), "q_out", "k_new");
    need_apart(Spread(o), Spread(vn), "q_out", "v_new");
    same_gpu(kn, o);
  }
  for (const Tensor* t : {&vn, &kc, &vc, &pos, q})
    if (t) same_gpu(kn, *t);
  const Spread k_rows(kc, row, C), v_rows(vc, row, C);          // what is written; keys and values may be there already
  need_apart(k_rows, v_rows, "k_cache", "v_cache");
  for (const Spread* rows : {&k_rows, &v_rows}) {
    const char* name = rows == &k_rows ? "k_cache" : "v_cache";
    if (q) need_apart(*rows, Spread(*q), name, "q");
    if (a[8] != Py_None) need_apart(*rows, Spread(tensor(a[8])), name, "q_out");
    for (const Tensor* t : {&kn, &vn})
      if ((rows == &k_rows) != (t == &kn) || !in_place(*rows, *t)) need_apart(*rows, Spread(*t), name, t == &kn ? "k_new" : "v_new");
  }
  OnGpu on(kn, a[9]);
  Tensor out;
  if (q) out = a[8] == Py_None ? fresh_like(*q) : tensor(a[8]);
  d.n_kv_heads = (int32_t)Hkv;
  heads_strides(kn, d.g_stride);
  heads_strides(kc, d.kv_stride);
  if (q) {
    d.n_q_heads = (int32_t)q->size(1);
    heads_strides(*q, d.q_stride);
    heads_strides(out, d.o_stride);
  }
  const int64_t* at = static_cast<const int64_t*>(ptr(pos));
  if (kn.numel() > 0) {
    const bool both = one_layout(kn, vn) && one_layout(kc, vc);
    for (const Tensor* t : {&vn, &vc})
      if (!both) rows_aligned(*t, "rope_append_axes");
    check(lib.rope_append_axes(&d, &axes.x, ptr(q), q ? ptr(out) : nullptr, ptr(kn), both ? ptr(vn) : nullptr, ptr(kc), both ? ptr(vc) : nullptr,
                               at, ps, on.s), "rope_append_axes");
    if (!both) {
      heads_strides(vn, d.g_stride);
      heads_strides(vc, d.kv_stride);
      check(lib.rope_append_axes(&d, &axes.x, nullptr, nullptr, nullptr, ptr(vn), nullptr, ptr(vc), at, ps, on.s), "rope_append_axes");
    }
  }
  if (!q) Py_RETURN_NONE;
  return out_ref(a[8], out);
}

// (d_q or None, gk, gv, row_begin, positions, axes, scaler, dq_out, d_k, d_v, dtype or None, stream) -> (dq_out or None, d_k, d_v)
PyObject* readout_axes(PyObject* const* a) {
  const Tensor *dq = opt_tensor(a[0]), *dk_given = opt_tensor(a[8]), *dv_given = opt_tensor(a[9]);
  const Tensor &gk = tensor(a[1]), &gv = tensor(a[2]), &pos = tensor(a[4]);
  const Axes axes(a[5]);
  const int64_t row = integer(a[3]);
  if (gk.dim() != 4 || pos.dim() != 3) raise(PyExc_ValueError, "expected [batch, head, row, head_dim] buffers and [axes, batch, row] positions");
  const int64_t B = gk.size(0), Hkv = gk.size(1), D = gk.size(3), C = pos.size(2);
  at::ScalarType type;
  if (a[10] != Py_None) {
    if (!THPDtype_Check(a[10])) raise(PyExc_TypeError, "dtype must be a torch dtype");
    type = reinterpret_cast<THPDtype*>(a[10])->scalar_type;
  } else if (dq || dk_given) {
    type = (dq ? *dq : *dk_given).scalar_type();
  } else {
    raise(PyExc_ValueError, "dtype: needed where neither d_q nor d_k is given");
  }
  if (type != at::kBFloat16 && type != at::kFloat) raise(PyExc_TypeError, "unsupported dtype: expected bfloat16 or float32");
  like_each_other(gk, gv, "gk and gv");
  if (Hkv < 1) raise(PyExc_ValueError, "gk: expected at least one head");
  rows_inside(gk, "gk", B, Hkv, D, row, C, at::kFloat);
  rows_inside(gv, "gv", B, Hkv, D, row, C, at::kFloat);
  fits_axes(axes, D);
  if (dq) heads_tensor(*dq, "d_q", B, C, D, type);
  if ((dk_given == nullptr) != (dv_given == nullptr)) raise(PyExc_ValueError, "d_k and d_v go together");
  if (dk_given) {
    like_each_other(*dk_given, *dv_given, "d_k and d_v");
    heads_tensor(*dk_given, "d_k", B, C, D, type);
    heads_tensor(*dv_given, "d_v", B, C, D, type);
    writable(*dk_given, "d_k");
    writable(*dv_given, "d_v");
    if (dk_given->size(1) != Hkv) raise(PyExc_ValueError, "d_k must have the heads of gk");
  }
  seco_desc d = axes_desc(B, C, D, type, row, "rope_readout_axes");
  int64_t ps[3];
  positions_of(pos, axes, B, C, ps);
  if (a[7] != Py_None) {
    const Tensor& o = tensor(a[7]);
    heads_tensor(o, "dq_out", B, C, D, type);
    writable(o, "dq_out");
    if (!dq || o.size(1) != dq->size(1)) raise(PyExc_ValueError, "dq_out must have the shape of d_q");
    in_place_or_apart(o, *dq, "dq_out", "d_q");
    same_gpu(gk, o);
  }
  for (const Tensor* t : {&gv, &pos, dq, dk_given, dv_given})
    if (t) same_gpu(gk, *t);
  const Spread gk_rows(gk, row, C), gv_rows(gv, row, C);
  auto results = [&](const Tensor* t, const char* name, const Spread* own) {      // own: what t may lie in the place of
    if (!t) return;
    if (own != &gk_rows || !in_place(gk_rows, *t)) need_apart(Spread(*t), gk_rows, name, "gk");
    if (own != &gv_rows || !in_place(gv_rows, *t)) need_apart(Spread(*t), gv_rows, name, "gv");
  };
  const Tensor* dq_given = opt_tensor(a[7]);
  results(dq_given, "dq_out", nullptr);
  results(dk_given, "d_k", &gk_rows);
  results(dv_given, "d_v", &gv_rows);
  if (dk_given) {
    need_apart(Spread(*dk_given), Spread(*dv_given), "d_k", "d_v");
    for (const Tensor* t : {dk_given, dv_given})
      for (const Tensor* other : {dq, dq_given})
        if (other) need_apart(Spread(*t), Spread(*other), t == dk_given ? "d_k" : "d_v", other == dq ? "d_q" : "dq_out");
  }
  OnGpu on(gk, a[11]);
  Tensor out, dk, dv;
  if (dq) out = a[7] == Py_None ? fresh_like(*dq) : tensor(a[7]);
  if (dk_given) {
    dk = *dk_given;
    dv = *dv_given;
  } else {
    dk = fresh({B, Hkv, C, D}, type, gk);
    dv = fresh({B, Hkv, C, D}, type, gk);
  }
  d.n_kv_heads = (int32_t)Hkv;
  heads_strides(gk, d.g_stride);
  heads_strides(dk, d.kv_stride);
  if (dq) {
    d.n_q_heads = (int32_t)dq->size(1);
    heads_strides(*dq, d.q_stride);
    heads_strides(out, d.o_stride);
  }
  const int64_t* at = static_cast<const int64_t*>(ptr(pos));
  const float scaler = (float)real(a[6]);
  if (dk.numel() > 0) {
    const bool both = one_layout(gk, gv) && one_layout(dk, dv);
    for (const Tensor* t : {&gv, (const Tensor*)&dv})
      if (!both) rows_aligned(*t, "rope_readout_axes");
    check(lib.rope_readout_axes(&d, &axes.x, ptr(dq), dq ? ptr(out) : nullptr, fptr(gk), both ? fptr(gv) : nullptr, ptr(dk), both ? ptr(dv) : nullptr,
                                scaler, at, ps, on.s), "rope_readout_axes");
    if (!both) {
      heads_strides(gv, d.g_stride);
      heads_strides(dv, d.kv_stride);
      check(lib.rope_readout_axes(&d, &axes.x, nullptr, nullptr, nullptr, fptr(gv), nullptr, ptr(dv), scaler, at, ps, on.s), "rope_readout_axes");
    }
  }
  PyObject* first = dq ? out_ref(a[7], out) : (Py_INCREF(Py_None), Py_None);
  return Py_BuildValue("NNN", first, out_ref(a[8], dk), out_ref(a[9], dv));
}

}  // namespace

PyMethodDef train_methods[] = {SECO_METHOD("rotate_axes", rotate_axes, 6), SECO_METHOD("append_axes", append_axes, 10),
                               SECO_METHOD("readout_axes", readout_axes, 12), SECO_METHOD("adamw", adamw, 15), SECO_METHOD("norm_fwd", norm_fwd, 8), SECO_METHOD("norm_bwd", norm_bwd, 12), {nullptr, nullptr, 0, nullptr}};

}  // namespace seco_ext
