// Marshalling of the short calls (binding.py: rotary, attention_*, checkpoint_*) as an extension module: checks of the tensors, their
// pointers, strides and sizes, new outputs, the current stream, and the call of the C ABI.  A launch or two of these take some
// microseconds; the same steps in Python with ctypes took 10 to 20 (rotary positions of one token 13.3 us a call, of which the
// launch and two allocations are 5; a checkpoint stored 9.8; attention with its backward pass 38).  Nothing is computed
// here.  Errors are binding.HbpError, handed over by set_error.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "hbp.h"

namespace {

PyObject* g_error = nullptr;

struct Refused {};  // the Python error is set

// HbpError(code, "name: what")
[[noreturn]] void refuse(int code, const char* name, const char* what) {
  PyObject* where = PyUnicode_FromFormat("%s: %s", name, what);
  PyObject* e = where && g_error ? PyObject_CallFunction(g_error, "iO", code, where) : nullptr;
  Py_XDECREF(where);
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  } else if (!PyErr_Occurred()) {
    PyErr_SetString(PyExc_RuntimeError, what);
  }
  throw Refused();
}
void check(hbp_status st, const char* where) {
  if (st == HBP_OK) return;
  PyObject* e = g_error ? PyObject_CallFunction(g_error, "is", (int)st, where) : nullptr;
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  } else if (!PyErr_Occurred()) {
    PyErr_SetString(PyExc_RuntimeError, where);
  }
  throw Refused();
}

// A call of the library without Python's lock: a launch waits where the device's queue is full.  (The entries throw nothing; their arguments have been
// read from the tensors before, which the caller holds.)
template <typename... P, typename... A>
hbp_status unlocked(hbp_status (*call)(P...), A... args) {
  hbp_status st;
  Py_BEGIN_ALLOW_THREADS
  st = call(args...);
  Py_END_ALLOW_THREADS
  return st;
}

// One call: its name, and the device that all of its tensors are on.
struct Call {
  const char* name;
  int device = -1;
  bool any = false;
  explicit Call(const char* n) : name(n) {}

  const at::Tensor& tensor(PyObject* o, const char* what) {
    if (!THPVariable_Check(o)) refuse(HBP_ERR_INVALID_ARG, name, what);
    return on(THPVariable_Unpack(o));
  }
  const at::Tensor* maybe(PyObject* o, const char* what) { return o == Py_None ? nullptr : &tensor(o, what); }
  const at::Tensor& on(const at::Tensor& t) {
    // (what comes back has no gradient: without a word the step's parameters would be short of it)
    if (t.requires_grad() && at::GradMode::is_enabled())
      refuse(HBP_ERR_UNSUPPORTED, name, "a tensor asks for gradients, which are calls of their own here: torch.no_grad(), or an autograd.Function around them");
    const int at = t.is_cuda() ? (int)t.get_device() : -1;
    if (!any) {
      device = at;
      any = true;
      if (at < 0 || at != (int)c10::cuda::current_device()) refuse(HBP_ERR_INVALID_ARG, name, "a tensor is not on the current CUDA device");
    } else if (at != device) {
      refuse(HBP_ERR_INVALID_ARG, name, "the tensors are on different devices");
    }
    return t;
  }
  void* stream() const { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream(); }
  int32_t dtype(const at::Tensor& t) const {
    if (t.scalar_type() == at::kBFloat16) return HBP_BF16;
    if (t.scalar_type() == at::kFloat) return HBP_F32;
    refuse(HBP_ERR_DTYPE, name, "float or bfloat16 is wanted");
  }
  int64_t whole(PyObject* o) const {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused();
    return v;
  }
  int32_t whole32(PyObject* o) const {
    const int64_t v = whole(o);
    if (v != (int32_t)v) refuse(HBP_ERR_SHAPE, name, "a size does not fit 32 bits");
    return (int32_t)v;
  }
  double real(PyObject* o) const {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Refused();
    return v;
  }
  bool truth(PyObject* o) const {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Refused();
    return v != 0;
  }
  // [rows, heads, head_dim] with contiguous channels; a dimension of one element has any stride
  hbp_heads heads(const at::Tensor& t) const {
    if (t.dim() != 3) refuse(HBP_ERR_SHAPE, name, "wanted [rows, heads, head_dim]");
    if (t.stride(2) != 1 && t.size(2) != 1) refuse(HBP_ERR_SHAPE, name, "the channels are not contiguous");
    return {t.data_ptr(), t.size(0) > 1 ? t.stride(0) : 0, t.size(1) > 1 ? t.stride(1) : 0};
  }
  // rows of a matrix [rows, channels] with contiguous channels; a single row has no stride of its own
  int64_t apart(const at::Tensor& t) const {
    if (t.dim() != 2) refuse(HBP_ERR_SHAPE, name, "wanted [rows, channels]");
    if (t.stride(1) != 1 && t.size(1) != 1) refuse(HBP_ERR_SHAPE, name, "the channels are not contiguous");
    return t.size(0) > 1 ? t.stride(0) : t.size(1);
  }
  int32_t narrow(int64_t v) const {
    if (v != (int32_t)v) refuse(HBP_ERR_SHAPE, name, "a size does not fit 32 bits");
    return (int32_t)v;
  }
  // an output: given, and like `t`, or new
  at::Tensor output(PyObject* o, const at::Tensor& t, const char* what) {
    if (o == Py_None) return at::empty_like(t);
    const at::Tensor& g = tensor(o, what);
    if (g.sizes() != t.sizes() || g.scalar_type() != t.scalar_type()) refuse(HBP_ERR_SHAPE, name, what);
    return g;
  }
  void alike(const at::Tensor& g, const at::Tensor& t, const char* what) const {
    if (g.sizes() != t.sizes() || g.scalar_type() != t.scalar_type()) refuse(HBP_ERR_SHAPE, name, what);
  }
};

void wanted(Py_ssize_t got, Py_ssize_t want, const char* name) {
  if (got == want) return;
  PyErr_Format(PyExc_TypeError, "%s: %zd arguments, %zd are wanted", name, got, want);
  throw Refused();
}
PyObject* two(const at::Tensor& a, const at::Tensor& b) {
  PyObject *x = THPVariable_Wrap(a), *y = THPVariable_Wrap(b), *t = x && y ? PyTuple_Pack(2, x, y) : nullptr;
  Py_XDECREF(x);
  Py_XDECREF(y);
  return t;
}
PyObject* three(const at::Tensor& a, const at::Tensor& b, const at::Tensor& c) {
  PyObject *x = THPVariable_Wrap(a), *y = THPVariable_Wrap(b), *z = THPVariable_Wrap(c), *t = x && y && z ? PyTuple_Pack(3, x, y, z) : nullptr;
  Py_XDECREF(x);
  Py_XDECREF(y);
  Py_XDECREF(z);
  return t;
}

#define CALL_BEGIN HANDLE_TH_ERRORS try {
#define CALL_END \
  }              \
  catch (const Refused&) { return nullptr; } \
  END_HANDLE_TH_ERRORS

PyObject* set_error(PyObject*, PyObject* e) {
  Py_INCREF(e);
  Py_XSETREF(g_error, e);
  Py_RETURN_NONE;
}

// q, k, positions, first, period, rotary_dim, base, layout, scaling, factor, trained_length, fast, slow, amplitude, inverse, q_out, k_out
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
  CALL_BEGIN
  wanted(n, 17, "rotary");
  Call c("rotary");
  const at::Tensor& q = c.tensor(a[0], "q is no tensor");
  const at::Tensor* k = c.maybe(a[1], "k is no tensor");
  const at::Tensor* pos = c.maybe(a[2], "positions are no tensor");
  const hbp_heads qh = c.heads(q);
  const int64_t rows = q.size(0), head_dim = q.size(2);
  if (k && (k->dim() != 3 || k->size(0) != rows || k->size(2) != head_dim || k->scalar_type() != q.scalar_type()))
    refuse(HBP_ERR_SHAPE, c.name, "k is not like q");
  const hbp_heads kh = k ? c.heads(*k) : hbp_heads{};
  int32_t size = 0;
  if (pos) {
    size = pos->scalar_type() == at::kInt ? 4 : pos->scalar_type() == at::kLong ? 8 : 0;
    if (!size || pos->dim() != 1 || pos->size(0) != rows || !pos->is_contiguous()) refuse(HBP_ERR_SHAPE, c.name, "positions: wanted int32 or int64 [rows]");
  }
  hbp_rotary_spec s;
  s.rotary_dim = a[5] == Py_None ? c.narrow(head_dim) : c.whole32(a[5]);
  s.base = (float)c.real(a[6]);
  s.layout = c.whole32(a[7]);
  s.scaling = c.whole32(a[8]);
  s.factor = (float)c.real(a[9]);
  s.trained_length = (float)c.real(a[10]);
  s.fast = (float)c.real(a[11]);
  s.slow = (float)c.real(a[12]);
  s.amplitude = (float)c.real(a[13]);
  const int32_t type = c.dtype(q);
  const at::Tensor qo = c.output(a[15], q, "q_out is not like q"), ko = k ? c.output(a[16], *k, "k_out is not like k") : at::Tensor();
  const hbp_heads qoh = c.heads(qo), koh = k ? c.heads(ko) : hbp_heads{};
  check(unlocked(hbp_rotary, &s, c.truth(a[14]), type, rows, c.narrow(q.size(1)), k ? c.narrow(k->size(1)) : 0, c.narrow(head_dim), pos ? pos->data_ptr() : nullptr,
                   size, c.whole(a[3]), c.whole(a[4]), &qh, &qoh, &kh, &koh, c.stream()),
        "hbp_rotary");
  if (k) return two(qo, ko);
  PyObject* x = THPVariable_Wrap(qo);
  PyObject* t = x ? PyTuple_Pack(2, x, Py_None) : nullptr;
  Py_XDECREF(x);
  return t;
  CALL_END
}

// a[0..8]: sequences, q_len, kv_len, q_offsets, kv_offsets, causal, scale, status
hbp_attention attention_of(Call& c, const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, PyObject* const* a) {
  if (q.dim() != 3 || k.dim() != 3 || k.sizes() != v.sizes() || k.size(2) != q.size(2)) refuse(HBP_ERR_SHAPE, c.name, "q, k and v do not belong together");
  if (k.scalar_type() != q.scalar_type() || v.scalar_type() != q.scalar_type()) refuse(HBP_ERR_SHAPE, c.name, "q, k and v differ in type");
  hbp_attention s = {};
  s.dtype = c.dtype(q);
  s.causal = c.truth(a[5]);
  const at::Tensor* off[2] = {c.maybe(a[3], "q_offsets are no tensor"), c.maybe(a[4], "kv_offsets are no tensor")};
  int64_t sequences = a[0] == Py_None ? -1 : c.whole(a[0]);
  if (a[0] != Py_None && sequences < 0) refuse(HBP_ERR_SHAPE, c.name, "a negative number of sequences");
  for (const at::Tensor* t : off) {
    if (!t) continue;
    if (t->dim() != 1 || !t->is_contiguous() || t->scalar_type() != at::kInt || t->numel() < 1) refuse(HBP_ERR_SHAPE, c.name, "offsets: wanted int32 [sequences + 1]");
    if (sequences >= 0 && sequences != t->numel() - 1) refuse(HBP_ERR_SHAPE, c.name, "offsets of another number of sequences");
    sequences = t->numel() - 1;
  }
  if (sequences < 0) sequences = 1;
  s.sequences = c.narrow(sequences);
  s.q_rows = q.size(0);
  s.kv_rows = k.size(0);
  s.q_heads = c.narrow(q.size(1));
  s.kv_heads = c.narrow(k.size(1));
  s.head_dim = c.narrow(q.size(2));
  auto length = [&](PyObject* o, const at::Tensor* t, int64_t rows, const char* what) {
    if (o != Py_None) return c.whole32(o);
    if (t) refuse(HBP_ERR_SHAPE, c.name, what);
    if (sequences ? rows % sequences : rows) refuse(HBP_ERR_SHAPE, c.name, "the rows are no whole number of sequences of equal length");
    return c.narrow(sequences ? rows / sequences : 0);
  };
  s.q_len = length(a[1], off[0], s.q_rows, "q_len, the longest of the sequences, has to be given with q_offsets");
  s.kv_len = length(a[2], off[1], s.kv_rows, "kv_len, the longest of the sequences, has to be given with kv_offsets");
  s.q_offsets = off[0] ? off[0]->data_ptr<int32_t>() : nullptr;
  s.kv_offsets = off[1] ? off[1]->data_ptr<int32_t>() : nullptr;
  s.scale = a[6] == Py_None ? (float)(1.0 / std::sqrt((double)s.head_dim)) : (float)c.real(a[6]);
  const at::Tensor* status = c.maybe(a[7], "status is no tensor");
  if (status && (status->scalar_type() != at::kInt || status->numel() < 1)) refuse(HBP_ERR_SHAPE, c.name, "status: wanted an int32 tensor");
  s.status = status ? status->data_ptr<int32_t>() : nullptr;
  return s;
}
void lse_of(const Call& c, const at::Tensor& q, const at::Tensor& lse) {
  if (lse.dim() != 2 || lse.size(0) != q.size(1) || lse.size(1) != q.size(0) || !lse.is_contiguous() || lse.scalar_type() != at::kFloat)
    refuse(HBP_ERR_SHAPE, c.name, "lse: wanted float [q_heads, q_rows]");
}

// q, k, v, (as attention_of), o, lse
PyObject* attention_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  CALL_BEGIN
  wanted(n, 13, "attention_forward");
  Call c("attention_forward");
  const at::Tensor &q = c.tensor(a[0], "q is no tensor"), &k = c.tensor(a[1], "k is no tensor"), &v = c.tensor(a[2], "v is no tensor");
  hbp_attention s = attention_of(c, q, k, v, a + 3);
  const at::Tensor o = c.output(a[11], q, "o is not like q");
  const at::Tensor* given = c.maybe(a[12], "lse is no tensor");
  if (given) lse_of(c, q, *given);
  const at::Tensor lse = given ? *given : at::empty({q.size(1), q.size(0)}, q.options().dtype(at::kFloat));
  const hbp_heads qh = c.heads(q), kh = c.heads(k), vh = c.heads(v), oh = c.heads(o);
  s.fresh = (a[11] == Py_None ? HBP_FRESH_O : 0) | (given ? 0 : HBP_FRESH_LSE);
  check(unlocked(hbp_attention_forward, &s, &qh, &kh, &vh, &oh, lse.data_ptr<float>(), c.stream()), "hbp_attention_forward");
  return two(o, lse);
  CALL_END
}

// d_o, q, k, v, o, lse, (as attention_of), dq, dk, dv, scratch
PyObject* attention_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  CALL_BEGIN
  wanted(n, 18, "attention_backward");
  Call c("attention_backward");
  const at::Tensor &q = c.tensor(a[1], "q is no tensor"), &k = c.tensor(a[2], "k is no tensor"), &v = c.tensor(a[3], "v is no tensor");
  const at::Tensor &d_o = c.tensor(a[0], "d_o is no tensor"), &o = c.tensor(a[4], "o is no tensor"), &lse = c.tensor(a[5], "lse is no tensor");
  hbp_attention s = attention_of(c, q, k, v, a + 6);
  c.alike(d_o, q, "d_o is not like q");
  c.alike(o, q, "o is not like q");
  lse_of(c, q, lse);
  const at::Tensor dq = c.output(a[14], q, "dq is not like q"), dk = c.output(a[15], k, "dk is not like k"), dv = c.output(a[16], v, "dv is not like v");
  const at::Tensor* given = c.maybe(a[17], "scratch is no tensor");
  const at::Tensor scratch = given ? *given : at::empty_like(lse);
  const hbp_heads gh = c.heads(d_o), qh = c.heads(q), kh = c.heads(k), vh = c.heads(v), oh = c.heads(o), dqh = c.heads(dq), dkh = c.heads(dk), dvh = c.heads(dv);
  s.fresh = (a[14] == Py_None ? HBP_FRESH_DQ : 0) | (a[15] == Py_None ? HBP_FRESH_DK : 0) | (a[16] == Py_None ? HBP_FRESH_DV : 0);
  check(unlocked(hbp_attention_backward, &s, &gh, &qh, &kh, &vh, &oh, lse.data_ptr<float>(), &dqh, &dkh, &dvh, scratch.data_ptr(),
                               scratch.is_contiguous() ? scratch.nbytes() : 0, c.stream()),
        "hbp_attention_backward");
  return three(dq, dk, dv);
  CALL_END
}

// Codes and scales of an activation [rows, d], made where not given
struct Kept {
  at::Tensor codes, scales;
};
Kept kept(Call& c, const at::Tensor& like, PyObject* codes, PyObject* scales) {
  const int64_t rows = like.size(0), d = like.size(1), groups = (d + 31) / 32;
  Kept k;
  if (codes == Py_None) {
    k.codes = at::empty({rows, d}, like.options().dtype(at::kChar));
  } else {
    k.codes = c.tensor(codes, "codes are no tensor");
    if (k.codes.sizes() != like.sizes() || !k.codes.is_contiguous() || k.codes.scalar_type() != at::kChar) refuse(HBP_ERR_SHAPE, c.name, "codes: wanted int8 [rows, channels]");
  }
  if (scales == Py_None) {
    k.scales = at::empty({rows, groups}, like.options().dtype(at::kByte));
  } else {
    k.scales = c.tensor(scales, "scales are no tensor");
    if (k.scales.dim() != 2 || k.scales.size(0) != rows || k.scales.size(1) != groups || !k.scales.is_contiguous() || k.scales.scalar_type() != at::kByte)
      refuse(HBP_ERR_SHAPE, c.name, "scales: wanted uint8 [rows, channels / 32 rounded up]");
  }
  return k;
}
int8_t* codes_of(const Kept& k) { return k.codes.data_ptr<int8_t>(); }
uint8_t* scales_of(const Kept& k) { return k.scales.data_ptr<uint8_t>(); }
at::Tensor packed_like(const at::Tensor& t) { return at::empty(t.sizes(), t.options()); }

// x, codes, scales
PyObject* checkpoint_store(PyObject*, PyObject* const* a, Py_ssize_t n) {
  CALL_BEGIN
  wanted(n, 3, "checkpoint_store");
  Call c("checkpoint_store");
  const at::Tensor& x = c.tensor(a[0], "x is no tensor");
  const int64_t ld = c.apart(x);
  const int32_t type = c.dtype(x);
  const Kept k = kept(c, x, a[1], a[2]);
  check(unlocked(hbp_checkpoint_store, type, x.size(0), c.narrow(x.size(1)), x.data_ptr(), ld, codes_of(k), scales_of(k), c.stream()), "hbp_checkpoint_store");
  return two(k.codes, k.scales);
  CALL_END
}

// codes, scales, float or not, out
PyObject* checkpoint_load(PyObject*, PyObject* const* a, Py_ssize_t n) {
  CALL_BEGIN
  wanted(n, 4, "checkpoint_load");
  Call c("checkpoint_load");
  const at::Tensor& codes = c.tensor(a[0], "codes are no tensor");
  c.tensor(a[1], "scales are no tensor");
  if (codes.dim() != 2) refuse(HBP_ERR_SHAPE, c.name, "codes: wanted int8 [rows, channels]");
  const Kept k = kept(c, codes, a[0], a[1]);
  const at::Tensor* given = c.maybe(a[3], "out is no tensor");
  if (given && given->sizes() != codes.sizes()) refuse(HBP_ERR_SHAPE, c.name, "out is not like codes");
  const at::Tensor out = given ? *given : at::empty(codes.sizes(), codes.options().dtype(c.truth(a[2]) ? at::kFloat : at::kBFloat16));
  const int64_t ld = c.apart(out);
  check(unlocked(hbp_checkpoint_load, c.dtype(out), out.size(0), c.narrow(out.size(1)), codes_of(k), scales_of(k), out.data_ptr(), ld, c.stream()), "hbp_checkpoint_load");
  return THPVariable_Wrap(out);
  CALL_END
}

// z, act, codes, scales
PyObject* checkpoint_gelu(PyObject*, PyObject* const* a, Py_ssize_t n) {
  CALL_BEGIN
  wanted(n, 4, "checkpoint_gelu");
  Call c("checkpoint_gelu");
  const at::Tensor& z = c.tensor(a[0], "z is no tensor");
  const int64_t ldz = c.apart(z);
  const int32_t type = c.dtype(z);
  const at::Tensor act = a[1] == Py_None ? packed_like(z) : c.output(a[1], z, "act is not like z");
  const int64_t lda = c.apart(act);
  const Kept k = kept(c, z, a[2], a[3]);
  check(unlocked(hbp_checkpoint_gelu, type, z.size(0), c.narrow(z.size(1)), z.data_ptr(), ldz, act.data_ptr(), lda, codes_of(k), scales_of(k), c.stream()),
        "hbp_checkpoint_gelu");
  return three(act, k.codes, k.scales);
  CALL_END
}

// d_act, codes, scales, with_act, dz, act
PyObject* checkpoint_gelu_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  CALL_BEGIN
  wanted(n, 6, "checkpoint_gelu_backward");
  Call c("checkpoint_gelu_backward");
  const at::Tensor& g = c.tensor(a[0], "d_act is no tensor");
  c.tensor(a[1], "codes are no tensor");
  c.tensor(a[2], "scales are no tensor");
  const int64_t ldg = c.apart(g);
  const int32_t type = c.dtype(g);
  const Kept k = kept(c, g, a[1], a[2]);
  const at::Tensor dz = a[4] == Py_None ? packed_like(g) : c.output(a[4], g, "dz is not like d_act");
  const bool with_act = a[5] != Py_None || c.truth(a[3]);
  const at::Tensor act = !with_act ? at::Tensor() : a[5] == Py_None ? packed_like(g) : c.output(a[5], g, "act is not like d_act");
  check(unlocked(hbp_checkpoint_gelu_backward, type, g.size(0), c.narrow(g.size(1)), codes_of(k), scales_of(k), g.data_ptr(), ldg, dz.data_ptr(), c.apart(dz),
                                     with_act ? act.data_ptr() : nullptr, with_act ? c.apart(act) : 0, c.stream()),
        "hbp_checkpoint_gelu_backward");
  return with_act ? two(dz, act) : THPVariable_Wrap(dz);
  CALL_END
}

#define FAST(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {{"set_error", set_error, METH_O, nullptr}, FAST(rotary),          FAST(attention_forward),
                          FAST(attention_backward),                  FAST(checkpoint_store), FAST(checkpoint_load),
                          FAST(checkpoint_gelu),                     FAST(checkpoint_gelu_backward), {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&kModule); }
