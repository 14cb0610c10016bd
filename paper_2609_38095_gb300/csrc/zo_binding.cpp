// zo_binding.cpp -- Python's side of include/zo_forward.h: checks of arguments,
// tensors to pointers and strides, outputs, the current stream. (The same in
// Python took 15 to 22 us of a call on the GB300's host cores, most of them for
// reading attributes of tensors; the kernels of the smallest calls take 3 to 10.)
// No numeric step is done here, and the library is called through the pointers
// that forward.py hands to bind().
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/forward_grad.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <c10/core/AutogradState.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include <cmath>
#include <initializer_list>
#include <string>

#include "zo_forward.h"

namespace {

decltype(&zo_rotate_heads) g_rotate_heads = nullptr;
decltype(&zo_attention) g_attention = nullptr;
decltype(&zo_attention_decode) g_attention_decode = nullptr;
decltype(&zo_token_loss) g_token_loss = nullptr;

// Whether tensors may have tangents in this call: within a level of forward mode. (Asked once per call; asking each tensor
// took 0.5 us of a call of nine.)
thread_local bool g_tangents = false;
bool tangents() {
  return c10::AutogradState::get_tls_state().get_fw_grad_mode() && torch::autograd::ForwardADLevel::try_get_by_idx(0) != nullptr;
}

struct Refusal {  // an exception of Python's
  PyObject* type;
  std::string text;
};
[[noreturn]] void type_error(const std::string& s) { throw Refusal{PyExc_TypeError, s}; }
[[noreturn]] void value_error(const std::string& s) { throw Refusal{PyExc_ValueError, s}; }

int code(at::ScalarType t) {  // zo_dtype, -1 for others
  return t == at::kFloat ? ZO_F32 : t == at::kBFloat16 ? ZO_BF16 : t == at::kHalf ? ZO_F16 : -1;
}
int index_bytes(const at::Tensor& t) { return t.scalar_type() == at::kLong ? 8 : t.scalar_type() == at::kInt ? 4 : 0; }

const at::Tensor& cuda_tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) type_error(std::string(what) + " must be a CUDA tensor");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda()) type_error(std::string(what) + " must be a CUDA tensor");
  // reverse mode, or a tangent of forward mode (which no_grad leaves on)
  if ((t.requires_grad() && at::GradMode::is_enabled()) || (g_tangents && t._fw_grad(/*level=*/0).defined()))
    throw Refusal{PyExc_RuntimeError, std::string(what) + " asks for a gradient, which this operator does not have"};
  return t;
}

// A tensor of heads: of `like`'s type and on its device, contiguous within a head.
const at::Tensor& heads(PyObject* o, const char* what, int64_t dim, const at::Tensor* like = nullptr) {
  const at::Tensor& t = cuda_tensor(o, what);
  if (like == nullptr) {
    if (code(t.scalar_type()) < 0) type_error(std::string("unsupported dtype ") + c10::toString(t.scalar_type()));
  } else if (t.scalar_type() != like->scalar_type()) {
    type_error(std::string(what) + " must be " + c10::toString(like->scalar_type()) + ", got " + c10::toString(t.scalar_type()));
  } else if (t.device() != like->device()) {
    value_error(std::string(what) + " is on another device");
  }
  if (t.dim() != dim) value_error(std::string(what) + " must have " + std::to_string(dim) + " dimensions, got " + std::to_string(t.dim()));
  if (t.stride(-1) != 1 && t.size(-1) > 1) value_error(std::string(what) + ": the elements of a head must be contiguous");
  return t;
}

// A contiguous tensor of numbers beside the heads.
const at::Tensor& flat(PyObject* o, const char* what, std::initializer_list<at::ScalarType> types, const at::Tensor& like,
                       at::IntArrayRef shape) {
  const at::Tensor& t = cuda_tensor(o, what);
  bool known = false;
  for (const at::ScalarType s : types) known = known || t.scalar_type() == s;
  if (!known) type_error(std::string(what) + " has dtype " + c10::toString(t.scalar_type()));
  if (t.device() != like.device()) value_error(std::string(what) + " is on another device");
  if (t.sizes() != shape || !t.is_contiguous()) {
    std::string s = std::string(what) + " must be contiguous, of shape (";
    for (const int64_t n : shape) s += std::to_string(n) + ",";
    value_error(s + ")");
  }
  return t;
}

// A count as the library takes it.
int32_t count(int64_t n, const char* what) {
  if (n > INT32_MAX) value_error(std::string(what) + " is " + std::to_string(n) + ", more than the library counts");
  return static_cast<int32_t>(n);
}

bool given(PyObject* o) { return o != Py_None; }

double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw python_error();
  return v;
}

bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw python_error();
  return v != 0;
}

struct Output {  // a tensor and the object that is returned for it
  at::Tensor t;
  PyObject* o = nullptr;
  bool given = false;
  Output() = default;
  Output(const Output&) = delete;
  Output& operator=(const Output&) = delete;
  ~Output() { Py_XDECREF(o); }
  void is(PyObject* other) {
    t = THPVariable_Unpack(other);
    o = Py_NewRef(other);
    given = true;
  }
  void make(at::IntArrayRef shape, const at::Tensor& like, at::ScalarType type) {
    t = at::empty(shape, at::TensorOptions(like.device()).dtype(type));
    o = THPVariable_Wrap(t);
    if (o == nullptr) throw python_error();
  }
  // The object, once the call is on its stream. A tensor of the caller's has a new version then, so that a backward pass
  // that saved it before does not take it for the same (those of inference mode have none).
  PyObject* take() {
    if (given && !t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
    PyObject* r = o;
    o = nullptr;
    return r;
  }
};

// The launch, on the tensors' device and its current stream; a status that is not ZO_OK goes back as a number.
template <typename F>
int on_stream(const at::Tensor& t, F f) {
  const c10::cuda::OptionalCUDAGuard guard(t.device());
  return f(c10::cuda::getCurrentCUDAStream(t.device().index()).stream());
}

PyObject* first_or_both(Output& a, Output& b, bool both) {
  if (!both) return a.take();
  PyObject* r = PyTuple_New(2);
  if (r == nullptr) throw python_error();
  PyTuple_SET_ITEM(r, 0, a.take());
  PyTuple_SET_ITEM(r, 1, b.take());
  return r;
}

zo_rows rows_of(const at::Tensor& t) { return {t.data_ptr(), t.stride(0), t.stride(1)}; }
zo_pages pages_of(const at::Tensor& t) { return {t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)}; }

// What attention and decode_attention share: q, k, v, slopes, out.
struct Attention {
  const at::Tensor &q, &k, &v;
  int32_t n = 0, kv = 0, size = 0;  // query heads, key-value heads, head size
  const float* slopes = nullptr;
  float scale = 0.0f, softcap = 0.0f;
  Output out, lse;

  Attention(PyObject* const* a, int64_t dim, PyObject* scale_, PyObject* softcap_, PyObject* slopes_, PyObject* out_)
      : q(heads(a[0], "q", 3)), k(heads(a[1], "k", dim, &q)), v(heads(a[2], "v", dim, &q)) {
    if (k.sizes() != v.sizes() || k.size(-1) != q.size(2)) value_error("k and v must have the same shape and q's head size");
    if (k.size(-2) == 0 || q.size(1) % k.size(-2) != 0) value_error("the key-value heads must divide the query heads");
    n = count(q.size(1), "the number of heads"), kv = count(k.size(-2), "the number of heads"), size = count(q.size(2), "the head size");
    if (given(slopes_)) slopes = flat(slopes_, "slopes", {at::kFloat}, q, {q.size(1)}).const_data_ptr<float>();
    scale = given(scale_) ? static_cast<float>(number(scale_)) : static_cast<float>(1.0 / std::sqrt(static_cast<double>(q.size(2))));
    softcap = static_cast<float>(number(softcap_));
    if (given(out_)) {
      if (heads(out_, "out", 3, &q).sizes() != q.sizes()) value_error("out must have q's shape");
      out.is(out_);
    } else {
      out.make(q.sizes(), q, q.scalar_type());
    }
  }
};

PyObject* attention(PyObject* const* a) {  // q, k, v, spans, scale, softcap, slopes, out, with_lse
  Attention c(a, 3, a[4], a[5], a[6], a[7]);
  const int64_t tokens = c.q.size(0);
  const at::Tensor& spans = flat(a[3], "spans", {at::kInt}, c.q, {3, tokens});
  const bool with_lse = truth(a[8]);
  if (with_lse) c.lse.make({c.n, tokens}, c.q, at::kFloat);
  const zo_rows q = rows_of(c.q), k = rows_of(c.k), v = rows_of(c.v), out = rows_of(c.out.t);
  const int rc = on_stream(c.q, [&](void* stream) {
    return g_attention(&q, &k, &v, &out, tokens, c.k.size(0), c.n, c.kv, c.size, code(c.q.scalar_type()),
                       spans.const_data_ptr<int32_t>(), c.scale, c.softcap, c.slopes,
                       with_lse ? static_cast<float*>(c.lse.t.data_ptr()) : nullptr, stream);
  });
  return rc != ZO_OK ? PyLong_FromLong(rc) : first_or_both(c.out, c.lse, with_lse);
}

PyObject* decode_attention(PyObject* const* a) {  // q, k, v, pages, lengths, scale, softcap, slopes, out, with_lse
  Attention c(a, 4, a[5], a[6], a[7], a[8]);
  const int64_t batch = c.q.size(0);
  const at::Tensor& pages = cuda_tensor(a[3], "pages");
  if (pages.scalar_type() != at::kInt || pages.device() != c.q.device()) type_error("pages must be an int32 tensor on q's device");
  if (pages.dim() != 2 || pages.size(0) != batch || (pages.size(1) > 1 && pages.stride(1) != 1))
    value_error("pages must have one row per sequence, contiguous");
  const at::Tensor& lengths = flat(a[4], "lengths", {at::kInt}, c.q, {batch});
  if (c.k.size(1) < 1) value_error("a page must hold at least one row");
  const int32_t page_size = count(c.k.size(1), "the page size");
  const bool with_lse = truth(a[9]);
  if (with_lse) c.lse.make({batch, c.n}, c.q, at::kFloat);
  const zo_rows q = rows_of(c.q), out = rows_of(c.out.t);
  const zo_pages k = pages_of(c.k), v = pages_of(c.v);
  const int rc = on_stream(c.q, [&](void* stream) {
    return g_attention_decode(&q, &k, &v, &out, batch, c.n, c.kv, c.size, code(c.q.scalar_type()),
                              pages.const_data_ptr<int32_t>(), pages.stride(0), pages.size(1), c.k.size(0), page_size,
                              lengths.const_data_ptr<int32_t>(), c.scale, c.softcap, c.slopes,
                              with_lse ? static_cast<float*>(c.lse.t.data_ptr()) : nullptr, stream);
  });
  return rc != ZO_OK ? PyLong_FromLong(rc) : first_or_both(c.out, c.lse, with_lse);
}

// q, k, v, table, positions, q_weight, k_weight, eps, interleaved, q_out, k_out, v_out, slots
PyObject* rotate_heads(PyObject* const* a) {
  static const char* const names[3] = {"q", "k", "v"};
  static const char* const weights[2] = {"q_weight", "k_weight"};
  static const char* const outs[3] = {"q_out", "k_out", "v_out"};
  const at::Tensor& q = heads(a[0], "q", 3);
  const int64_t tokens = q.size(0), dim = count(q.size(2), "the head size");
  if (!given(a[1]) && (given(a[2]) || given(a[6]) || given(a[10]))) value_error("v, k_weight and k_out need k");
  if (!given(a[2]) && given(a[11])) value_error("v_out needs v");
  const at::Tensor& table = cuda_tensor(a[3], "table");
  flat(a[3], "table", {at::kFloat}, q, {table.size(0), table.dim() == 2 ? table.size(1) : 0});
  const at::Tensor& positions = flat(a[4], "positions", {at::kLong, at::kInt}, q, {tokens});
  const at::Tensor* slots = nullptr;
  if (given(a[12])) {
    if (!given(a[1]) || !given(a[10]) || given(a[2]) != given(a[11]))
      value_error("slots need k and the cache that it goes to, and v both or neither");
    slots = &flat(a[12], "slots", {positions.scalar_type()}, q, {tokens});
  }
  zo_head_part parts[3] = {};
  Output out[3];
  int n = 0;
  int64_t rows = 1, page_size = 1;
  for (int i = 0; i < 3; ++i) {
    if (!given(a[i])) continue;
    const at::Tensor& x = i == 0 ? q : heads(a[i], names[i], 3, &q);
    if (x.size(0) != tokens || x.size(2) != dim) value_error(std::string(names[i]) + " must have q's tokens and head size");
    parts[n].heads = count(x.size(1), "the number of heads");
    const bool slotted = i > 0 && slots != nullptr;
    if (given(a[9 + i])) {
      const bool paged = slotted && THPVariable_Check(a[9 + i]) && THPVariable_Unpack(a[9 + i]).dim() == 4;
      const at::Tensor& o = heads(a[9 + i], outs[i], paged ? 4 : 3, &q);
      if (o.size(-1) != dim || o.size(-2) != x.size(1) || (!slotted && o.size(0) != tokens))
        value_error(std::string(outs[i]) + " must have " + names[i] + "'s heads and, without slots, tokens");
      out[n].is(a[9 + i]);
    } else {
      out[n].make(x.sizes(), q, q.scalar_type());
    }
    const at::Tensor& o = out[n].t;
    zo_head_part& p = parts[n];
    p.in = rows_of(x);
    p.out = {o.data_ptr(), o.dim() == 4 ? o.stride(0) : 0, o.stride(-3), o.stride(-2)};
    if (i < 2 && given(a[5 + i])) {
      const at::Tensor& w = flat(a[5 + i], weights[i], {at::kFloat, at::kBFloat16, at::kHalf}, q, {dim});
      p.weight = w.const_data_ptr();
      p.weight_dtype = code(w.scalar_type());
    }
    p.flags = (i < 2 ? ZO_HEADS_ROTATE : 0) | (slotted ? ZO_HEADS_SLOTTED : 0);
    if (slotted) {
      const int64_t per_page = o.dim() == 4 ? o.size(1) : o.size(0), all = o.dim() == 4 ? o.size(0) * per_page : per_page;
      if (i == 2 && (all != rows || per_page != page_size)) value_error("k_out and v_out must have the same rows");
      rows = all;
      page_size = per_page;
    }
    ++n;
  }
  const double eps = number(a[7]);
  const int layout = truth(a[8]) ? ZO_ROTARY_INTERLEAVED : ZO_ROTARY_HALF;
  const int rc = on_stream(q, [&](void* stream) {
    return g_rotate_heads(parts, n, tokens, static_cast<int32_t>(dim), code(q.scalar_type()), table.const_data_ptr<float>(),
                          table.size(0), count(table.size(1), "the rotated part"), layout, positions.const_data_ptr(),
                          slots != nullptr ? slots->const_data_ptr() : nullptr, index_bytes(positions), rows,
                          page_size > 0 ? page_size : 1, static_cast<float>(eps), stream);
  });
  if (rc != ZO_OK) return PyLong_FromLong(rc);
  if (n == 1) return out[0].take();
  PyObject* r = PyTuple_New(n);
  if (r == nullptr) throw python_error();
  for (int i = 0; i < n; ++i) PyTuple_SET_ITEM(r, i, out[i].take());
  return r;
}

PyObject* token_loss(PyObject* const* a) {  // logits, targets, mean, add, out, float32, with_nll
  const at::Tensor& logits = heads(a[0], "logits", 2);
  const int64_t tokens = logits.size(0), vocab = logits.size(1);
  const at::Tensor& targets = flat(a[1], "targets", {at::kLong, at::kInt}, logits, {tokens});
  const bool add = truth(a[3]), with_nll = truth(a[6]);
  Output out, nll;
  if (given(a[4])) {
    flat(a[4], "out", {at::kDouble, at::kFloat}, logits, {1});
    out.is(a[4]);
  } else {
    if (add) value_error("add needs out");
    out.make({1}, logits, truth(a[5]) ? at::kFloat : at::kDouble);
  }
  if (with_nll) nll.make({tokens}, logits, at::kFloat);
  const at::Tensor work = at::empty({tokens > 0 ? tokens : 1}, at::TensorOptions(logits.device()).dtype(at::kDouble));
  const int flags = (truth(a[2]) ? ZO_LOSS_MEAN : 0) | (add ? ZO_LOSS_ADD : 0) | (out.t.scalar_type() == at::kFloat ? ZO_LOSS_F32 : 0);
  const int rc = on_stream(logits, [&](void* stream) {
    return g_token_loss(logits.const_data_ptr(), logits.stride(0), tokens, vocab, code(logits.scalar_type()),
                        targets.const_data_ptr(), index_bytes(targets), flags, out.t.data_ptr(),
                        with_nll ? static_cast<float*>(nll.t.data_ptr()) : nullptr, work.data_ptr(), work.numel() * 8, stream);
  });
  return rc != ZO_OK ? PyLong_FromLong(rc) : first_or_both(out, nll, with_nll);
}

// No exception leaves: a refusal becomes Python's, torch's own are translated by its macros.
template <PyObject* (*F)(PyObject* const*), Py_ssize_t N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "%zd arguments, %zd expected", n, N);
    return nullptr;
  }
  try {
    g_tangents = tangents();
    return F(args);
  } catch (const Refusal& r) {
    PyErr_SetString(r.type, r.text.c_str());
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {  // the addresses of the four entry points
  if (n != 4) {
    PyErr_SetString(PyExc_TypeError, "four addresses expected");
    return nullptr;
  }
  void* p[4];
  for (int i = 0; i < 4; ++i) {
    p[i] = PyLong_AsVoidPtr(args[i]);
    if (p[i] == nullptr) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "no address");
      return nullptr;
    }
  }
  g_rotate_heads = reinterpret_cast<decltype(g_rotate_heads)>(p[0]);
  g_attention = reinterpret_cast<decltype(g_attention)>(p[1]);
  g_attention_decode = reinterpret_cast<decltype(g_attention_decode)>(p[2]);
  g_token_loss = reinterpret_cast<decltype(g_token_loss)>(p[3]);
  Py_RETURN_NONE;
}

template <typename F>
PyCFunction fast(F f) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(f));
}

PyMethodDef g_methods[] = {{"bind", fast(&bind), METH_FASTCALL, nullptr},
                           {"rotate_heads", fast(&entry<rotate_heads, 13>), METH_FASTCALL, nullptr},
                           {"attention", fast(&entry<attention, 9>), METH_FASTCALL, nullptr},
                           {"decode_attention", fast(&entry<decode_attention, 10>), METH_FASTCALL, nullptr},
                           {"token_loss", fast(&entry<token_loss, 7>), METH_FASTCALL, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&g_module); }
