// Calls on device tensors, from Python: checks, outputs and arguments without going through the interpreter (cos_verify_run, and the proposer's operators of
// cos_draft.h).
//
// What bounds small runs called from Python is the call itself: with its steps in Python one row of 5 x 2 x 32000 took 14.8 us a call, of
// which the device needs 12.4; now it takes 12.8.  Whatever does not fit here (other outputs, tensors that are not plain, anything to
// complain about) returns None, and the caller goes the long way, which has the messages.  Likewise drawing from one row 18.7 -> 9.2 us a call (the device's
// time), and distillation forward and backward of 16 rows 113 -> 60 us (of which the engine takes 52 for any graph), where the autograd function is a node of the engine's own kind.
#include <ATen/ops/as_strided.h>
#include <ATen/ops/empty.h>
#include <Python.h>
#include <c10/cuda/CUDAGraphsC10Utils.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/autograd/variable.h>

#include <new>
#include <optional>
#include <vector>

#include "cos_draft.h"
#include "cos_verify.h"

namespace {

using RunFn = cos_status (*)(cos_verify_ctx*, const cos_verify_args*, void*);

struct Callee {  // a context and what its calls have to look like
  RunFn run;
  cos_verify_ctx* ctx;
  int64_t n, positions, vocab;
  at::ScalarType dtype;
};
constexpr const char* kCapsule = "cos_verify.callee";

void drop(PyObject* capsule) { delete static_cast<Callee*>(PyCapsule_GetPointer(capsule, kCapsule)); }

// callee(address of cos_verify_run, address of the context, n, gamma + 1, vocab, dtype)
PyObject* callee(PyObject*, PyObject* args) {
  unsigned long long run = 0, ctx = 0;
  long long n = 0, positions = 0, vocab = 0;
  int dtype = 0;
  if (!PyArg_ParseTuple(args, "KKLLLi", &run, &ctx, &n, &positions, &vocab, &dtype)) return nullptr;
  Callee* c = new (std::nothrow) Callee{reinterpret_cast<RunFn>(run), reinterpret_cast<cos_verify_ctx*>(ctx), n, positions, vocab,
                                        dtype == COS_DTYPE_F32 ? at::kFloat : (dtype == COS_DTYPE_BF16 ? at::kBFloat16 : at::kHalf)};
  if (!c) return PyErr_NoMemory();
  PyObject* capsule = PyCapsule_New(c, kCapsule, drop);
  if (!capsule) delete c;
  return capsule;
}

// Without the interpreter's lock until the end of the scope, however that is left: what throws there (an allocation, a hook on saved tensors) becomes a Python error, which needs the lock.
struct Unlocked {
  PyThreadState* const state = PyEval_SaveThread();
  Unlocked() = default;
  Unlocked(const Unlocked&) = delete;
  Unlocked& operator=(const Unlocked&) = delete;
  ~Unlocked() { PyEval_RestoreThread(state); }
};

// A plain int32 device tensor that is contiguous, with anything in it.
bool plain_int32(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.scalar_type() == at::kInt && t.is_cuda() && t.is_contiguous();
}
bool as_word(PyObject* o, unsigned long long* v) {
  if (!PyLong_Check(o)) return false;
  *v = PyLong_AsUnsignedLongLongMask(o);
  return true;
}

// run(callee, logits, drafts, proposer, seed, offset, row_base, flags, bonus_model, offset_device): the outputs, or the status of a call
// that failed, or None.
PyObject* run(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  if (nargs != 10) {
    PyErr_SetString(PyExc_TypeError, "run takes 10 arguments");
    return nullptr;
  }
  const Callee* c = static_cast<Callee*>(PyCapsule_GetPointer(a[0], kCapsule));
  if (!c) return nullptr;
  HANDLE_TH_ERRORS  // (what the allocation of the outputs raises is what torch raises from Python)
  {
    if (!THPVariable_CheckExact(a[1]) || !plain_int32(a[3])) Py_RETURN_NONE;
    const at::Tensor &logits = THPVariable_Unpack(a[1]), &proposer = THPVariable_Unpack(a[3]);
    if (!logits.is_cuda() || logits.layout() != at::kStrided || logits.dim() != 4 || logits.scalar_type() != c->dtype) Py_RETURN_NONE;
    const int64_t B = logits.size(1), P = c->positions;
    if (logits.size(0) != c->n || logits.size(2) != P || logits.size(3) != c->vocab || logits.stride(3) != 1 || B < 1 || B > INT32_MAX) Py_RETURN_NONE;
    cos_verify_args v = {};
    unsigned long long row_base = 0, flags = 0, seed = 0, offset = 0;
    if (!as_word(a[4], &seed) || !as_word(a[5], &offset) || !as_word(a[6], &row_base) || !as_word(a[7], &flags)) Py_RETURN_NONE;
    if (proposer.dim() == 2) {
      if (proposer.size(0) != B || proposer.size(1) != P) Py_RETURN_NONE;
      flags |= COS_RUN_PROPOSER_PER_POSITION;
    } else if (proposer.numel() != B) {
      Py_RETURN_NONE;
    }
    if (a[8] != Py_None) {
      const long model = PyLong_Check(a[8]) ? PyLong_AsLong(a[8]) : -2;
      if (model < INT32_MIN || model > INT32_MAX || (model == -1 && PyErr_Occurred()) || !PyLong_Check(a[8])) {
        PyErr_Clear();
        Py_RETURN_NONE;
      }
      if (model >= 0) {
        flags |= COS_RUN_BONUS_FROM_MODEL;
        v.bonus_model = static_cast<int32_t>(model);
      }
    }
    if (a[2] != Py_None) {
      if (!THPVariable_CheckExact(a[2])) Py_RETURN_NONE;
      const at::Tensor& drafts = THPVariable_Unpack(a[2]);
      if (drafts.numel() > 0) {
        if (!plain_int32(a[2])) Py_RETURN_NONE;
        v.draft_tokens = static_cast<const int32_t*>(drafts.data_ptr());
      }
    }
    if (a[9] != Py_None) {
      if (!THPVariable_CheckExact(a[9])) Py_RETURN_NONE;
      const at::Tensor& t = THPVariable_Unpack(a[9]);
      if (t.scalar_type() != at::kLong || !t.is_cuda()) Py_RETURN_NONE;
      v.offset_device = static_cast<const uint64_t*>(t.data_ptr());
    }
    v.logits = logits.data_ptr();
    v.stride_model = logits.stride(0);
    v.stride_row = logits.stride(1);
    v.stride_pos = logits.stride(2);
    v.proposer = static_cast<const int32_t*>(proposer.data_ptr());
    v.batch = static_cast<int32_t>(B);
    v.flags = static_cast<int32_t>(flags);
    v.row_base = static_cast<int64_t>(row_base);
    v.seed = seed;
    v.offset = offset;
    // one allocation for the small outputs
    const at::Tensor buf = at::empty({B * (P + 3)}, logits.options().dtype(at::kInt).requires_grad(false));
    int32_t* at0 = static_cast<int32_t*>(buf.data_ptr());
    v.accept_count = at0;
    v.row_status = reinterpret_cast<uint32_t*>(at0 + B);
    v.bonus_prob = reinterpret_cast<float*>(at0 + 2 * B);
    v.out_tokens = at0 + 3 * B;
    void* stream = c10::cuda::getCurrentCUDAStream(logits.get_device()).stream();
    cos_status st;
    {
      const Unlocked unlocked;
      st = c->run(c->ctx, &v, stream);
    }
    if (st != COS_OK) return PyLong_FromLong(st);
    const at::Tensor outs[4] = {at::as_strided(buf, {B}, {1}, 0), at::as_strided(buf, {B, P}, {P, 1}, 3 * B), at::as_strided(buf, {B}, {1}, B),
                                at::as_strided(buf, {B}, {1}, 2 * B).view(at::kFloat)};
    static PyObject* const names[4] = {PyUnicode_InternFromString("accept_count"), PyUnicode_InternFromString("out_tokens"),
                                       PyUnicode_InternFromString("row_status"), PyUnicode_InternFromString("bonus_prob")};
    PyObject* d = PyDict_New();
    for (int k = 0; d && k < 4; ++k) {
      PyObject* t = THPVariable_Wrap(outs[k]);
      if (!t || PyDict_SetItem(d, names[k], t) != 0) Py_CLEAR(d);
      Py_XDECREF(t);
    }
    return d;
  }
  END_HANDLE_TH_ERRORS
}

// -- the proposer's operators ----------------------------------------------------------

template <class Args>
using CallFn = cos_status (*)(const Args*, void*);

template <class Args>
cos_status enqueue(unsigned long long fn, const Args& a, c10::DeviceIndex device) {
  void* stream = c10::cuda::getCurrentCUDAStream(device).stream();
  return reinterpret_cast<CallFn<Args>>(fn)(&a, stream);
}

// Rows of logits: a plain 2-D device tensor, contiguous along the vocabulary, of a type the library knows.
bool rows_of(PyObject* o, const at::Tensor** t, int64_t* stride, int32_t* dtype) {
  if (!THPVariable_CheckExact(o)) return false;
  const at::Tensor& x = THPVariable_Unpack(o);
  if (!x.is_cuda() || x.layout() != at::kStrided || x.dim() != 2) return false;
  const int64_t rows = x.size(0), vocab = x.size(1);
  if (rows < 1 || vocab < 1 || rows > INT32_MAX || vocab > INT32_MAX || (vocab > 1 && x.stride(1) != 1)) return false;
  switch (x.scalar_type()) {
    case at::kFloat: *dtype = COS_DTYPE_F32; break;
    case at::kBFloat16: *dtype = COS_DTYPE_BF16; break;
    case at::kHalf: *dtype = COS_DTYPE_F16; break;
    default: return false;
  }
  *t = &x;
  *stride = rows > 1 ? x.stride(0) : vocab;
  return true;
}
// The address of a contiguous tensor of that type and size on the device of `like`; nullptr where it is something else.
template <class T>
const T* plain(PyObject* o, const at::Tensor& like, int64_t numel, int64_t dims, at::ScalarType type) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.scalar_type() != type || t.layout() != at::kStrided || t.device() != like.device() || t.dim() != dims || t.numel() != numel || !t.is_contiguous()) return nullptr;
  return static_cast<const T*>(t.data_ptr());
}
// A number, or a tensor with one for each row.
template <class T>
bool of_rows(PyObject* o, const at::Tensor& like, int64_t rows, at::ScalarType type, T* one, const T** each) {
  if (THPVariable_CheckExact(o)) {
    *each = plain<T>(o, like, rows, 1, type);
    return *each != nullptr;
  }
  if (type == at::kInt) {
    if (!PyLong_Check(o)) return false;
    const long v = PyLong_AsLong(o);
    if (v < INT32_MIN || v > INT32_MAX || (v == -1 && PyErr_Occurred())) {
      PyErr_Clear();
      return false;
    }
    *one = static_cast<T>(v);
    return true;
  }
  if (!PyFloat_Check(o) && !PyLong_Check(o)) return false;
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  *one = static_cast<T>(v);
  return true;
}
bool number(PyObject* o, double* v) {
  const double* each = nullptr;
  return !THPVariable_Check(o) && of_rows(o, at::Tensor(), 0, at::kDouble, v, &each);
}
PyObject* dict_of(std::initializer_list<std::pair<const char*, at::Tensor>> items) {
  PyObject* d = PyDict_New();
  for (const auto& item : items) {
    if (!d || !item.second.defined()) continue;
    PyObject* t = THPVariable_Wrap(item.second);
    if (!t || PyDict_SetItemString(d, item.first, t) != 0) Py_CLEAR(d);
    Py_XDECREF(t);
  }
  return d;
}
bool address(PyObject* o, unsigned long long* fn) {
  *fn = PyLong_AsUnsignedLongLong(o);
  return !PyErr_Occurred();
}

// sample(cos_sample, logits, uniforms, temperature, top_k, top_p, min_p, filtered)
PyObject* sample(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  unsigned long long fn = 0;
  if (nargs != 8 || !address(a[0], &fn)) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "sample takes 8 arguments");
    return nullptr;
  }
  HANDLE_TH_ERRORS
  {
    const at::Tensor* logits = nullptr;
    cos_sample_args v = {};
    if (!rows_of(a[1], &logits, &v.stride_row, &v.dtype)) Py_RETURN_NONE;
    const int64_t rows = logits->size(0), vocab = logits->size(1);
    v.logits = logits->data_ptr();
    v.rows = static_cast<int32_t>(rows);
    v.vocab = static_cast<int32_t>(vocab);
    v.device = logits->get_device();
    v.uniforms = plain<float>(a[2], *logits, rows, 1, at::kFloat);
    if (!v.uniforms || !of_rows(a[3], *logits, rows, at::kFloat, &v.temperature, &v.row_temperature) || !of_rows(a[4], *logits, rows, at::kInt, &v.top_k, &v.row_top_k) ||
        !of_rows(a[5], *logits, rows, at::kFloat, &v.top_p, &v.row_top_p) || !of_rows(a[6], *logits, rows, at::kFloat, &v.min_p, &v.row_min_p))
      Py_RETURN_NONE;
    at::Tensor filtered;
    if (a[7] == Py_True) {
      filtered = at::empty({rows, vocab}, logits->options().requires_grad(false));
      v.filtered = filtered.data_ptr();
      v.stride_filtered = vocab;
    } else if (a[7] != Py_False) {
      Py_RETURN_NONE;
    }
    // one allocation for the small outputs
    const at::Tensor buf = at::empty({4, rows}, logits->options().dtype(at::kInt).requires_grad(false));
    int32_t* at0 = static_cast<int32_t*>(buf.data_ptr());
    v.tokens = at0;
    v.kept = at0 + rows;
    v.row_status = reinterpret_cast<uint32_t*>(at0 + 2 * rows);
    v.prob = reinterpret_cast<float*>(at0 + 3 * rows);
    cos_status st;
    {
      const Unlocked unlocked;
      st = enqueue(fn, v, logits->device().index());
    }
    if (st != COS_OK) return PyLong_FromLong(st);
    const auto part = [&](int64_t i) { return at::as_strided(buf, {rows}, {1}, i * rows); };
    return dict_of({{"tokens", part(0)}, {"prob", part(3).view(at::kFloat)}, {"kept", part(1)}, {"row_status", part(2)}, {"filtered", filtered}});
  }
  END_HANDLE_TH_ERRORS
}

// top_logits(cos_top_logits, logits, k, temperature)
PyObject* top_logits(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  unsigned long long fn = 0;
  if (nargs != 4 || !address(a[0], &fn)) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "top_logits takes 4 arguments");
    return nullptr;
  }
  HANDLE_TH_ERRORS
  {
    const at::Tensor* logits = nullptr;
    cos_top_args v = {};
    const int32_t* no_k = nullptr;
    if (!rows_of(a[1], &logits, &v.stride_row, &v.dtype) || THPVariable_Check(a[2])) Py_RETURN_NONE;
    if (!of_rows(a[2], *logits, 0, at::kInt, &v.k, &no_k) || !number(a[3], &v.temperature)) Py_RETURN_NONE;
    const int64_t rows = logits->size(0), vocab = logits->size(1), k = v.k;
    if (k < 1 || k > COS_TOP_MAX || k > vocab) Py_RETURN_NONE;
    const auto options = logits->options().requires_grad(false);
    const at::Tensor values = at::empty({rows, k}, options.dtype(at::kFloat)), ids = at::empty({rows, k}, options.dtype(at::kInt)), lse = at::empty({rows}, options.dtype(at::kFloat));
    v.logits = logits->data_ptr();
    v.rows = static_cast<int32_t>(rows);
    v.vocab = static_cast<int32_t>(vocab);
    v.device = logits->get_device();
    v.values = static_cast<float*>(values.data_ptr());
    v.ids = static_cast<int32_t*>(ids.data_ptr());
    v.lse = static_cast<float*>(lse.data_ptr());
    cos_status st;
    {
      const Unlocked unlocked;
      st = enqueue(fn, v, logits->device().index());
    }
    if (st != COS_OK) return PyLong_FromLong(st);
    return dict_of({{"values", values}, {"ids", ids}, {"lse", lse}});
  }
  END_HANDLE_TH_ERRORS
}

// The arguments that the calls of distillation share.
bool distill_of(PyObject* const* a, cos_distill_args* v, const at::Tensor** student) {
  if (!rows_of(a[0], student, &v->stride_student, &v->dtype) || !THPVariable_CheckExact(a[1])) return false;
  const at::Tensor &s = **student, &ids = THPVariable_Unpack(a[1]);
  const int64_t rows = s.size(0), dims = ids.dim();
  if ((dims != 2 && dims != 3) || ids.size(0) != rows) return false;
  const int64_t lists = dims == 2 ? 1 : ids.size(1), k = ids.size(dims - 1);
  if (lists < 1 || lists > COS_MAX_MODELS || k < 1 || k > COS_TOP_MAX || lists * k > COS_TOP_MAX) return false;
  v->ids = plain<int32_t>(a[1], s, rows * lists * k, dims, at::kInt);
  v->values = plain<float>(a[2], s, rows * lists * k, dims, at::kFloat);
  if (!v->ids || !v->values || THPVariable_Unpack(a[2]).sizes() != ids.sizes()) return false;
  if (a[3] != Py_None) {
    v->lse = plain<float>(a[3], s, rows * lists, dims - 1, at::kFloat);
    if (!v->lse || (dims == 3 && THPVariable_Unpack(a[3]).size(1) != lists)) return false;
  }
  if (a[4] == Py_None) {
    for (int64_t i = 0; i < lists; ++i) v->weights[i] = 1.0f;
  } else {
    if ((!PyList_Check(a[4]) && !PyTuple_Check(a[4])) || PySequence_Fast_GET_SIZE(a[4]) != lists) return false;
    for (int64_t i = 0; i < lists; ++i) {
      const float* none = nullptr;
      PyObject* w = PySequence_Fast_GET_ITEM(a[4], i);
      if (THPVariable_Check(w) || !of_rows(w, s, 0, at::kFloat, &v->weights[i], &none)) return false;
    }
  }
  if (!number(a[5], &v->temperature)) return false;
  v->student = s.data_ptr();
  v->rows = static_cast<int32_t>(rows);
  v->vocab = static_cast<int32_t>(s.size(1));
  v->device = s.get_device();
  v->lists = static_cast<int32_t>(lists);
  v->k = static_cast<int32_t>(k);
  return true;
}
at::Tensor floats(const at::Tensor& like, int64_t n) { return at::empty({n}, like.options().dtype(at::kFloat).requires_grad(false)); }
int64_t statistics_size(const cos_distill_args& v) { return static_cast<int64_t>(v.rows) * (COS_DISTILL_STATISTICS + v.lists * v.k); }

// A leaf whose gradient is taken up on the default stream (an eager graph of it is alive) has no backward pass in a capture: the engine would wait for that stream there, whose error nobody catches.
void refuse_capture(const at::Tensor& student) {
  if (!student.requires_grad() || !student.is_leaf() || c10::cuda::currentStreamCaptureStatusMayInitCtx() == c10::cuda::CaptureStatus::None) return;
  const auto takes = torch::autograd::impl::try_get_grad_accumulator(student);
  const auto on = takes ? takes->stream() : std::nullopt;
  TORCH_CHECK(!on || on->id() != 0, "distill_loss: a backward pass of this leaf cannot be captured while an eager graph of it is alive");
}

// refuse_capture(student): raises where that is so, for the autograd function of the long way.
PyObject* refuse_capture(PyObject*, PyObject* o) {
  HANDLE_TH_ERRORS
  if (THPVariable_Check(o)) refuse_capture(THPVariable_Unpack(o));
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

// The loss as a node of the autograd graph.  `grad_fn` is cos_distill_grad; `st` takes the status of the forward call.
struct DistillLoss : torch::autograd::Function<DistillLoss> {
  static at::Tensor forward(torch::autograd::AutogradContext* ctx, const at::Tensor& student, const at::Tensor& ids, const at::Tensor& values, const std::optional<at::Tensor>& lse, const cos_distill_args* args,
                            int64_t loss_fn, int64_t grad_fn, cos_status* st) {
    cos_distill_args v = *args;
    const at::Tensor loss = floats(student, v.rows), statistics = floats(student, statistics_size(v));
    v.loss = static_cast<float*>(loss.data_ptr());
    v.statistics = static_cast<float*>(statistics.data_ptr());
    *st = enqueue(static_cast<unsigned long long>(loss_fn), v, student.device().index());
    ctx->save_for_backward({student, ids, values, lse.value_or(at::Tensor()), statistics});
    std::vector<double> numbers = {v.temperature, static_cast<double>(v.lists), static_cast<double>(v.k)};
    for (int i = 0; i < v.lists; ++i) numbers.push_back(v.weights[i]);
    ctx->saved_data["numbers"] = numbers;
    ctx->saved_data["grad_fn"] = grad_fn;
    return loss;
  }
  static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list upstream) {
    torch::autograd::variable_list out(8);
    if (!upstream[0].defined()) return out;
    const auto saved = ctx->get_saved_variables();
    const auto numbers = ctx->saved_data["numbers"].toDoubleVector();
    const at::Tensor& student = saved[0];
    refuse_capture(student);
    at::Tensor grad;
    {
      const at::AutoGradMode off(false);
      const at::Tensor weights = upstream[0].contiguous();  // (an expanded scalar, of a mean or a sum)
      grad = at::empty({student.size(0), student.size(1)}, student.options().requires_grad(false));
      cos_distill_args v = {};
      v.student = student.data_ptr();
      v.rows = static_cast<int32_t>(student.size(0));
      v.vocab = static_cast<int32_t>(student.size(1));
      v.stride_student = v.rows > 1 ? student.stride(0) : v.vocab;
      v.dtype = student.scalar_type() == at::kFloat ? COS_DTYPE_F32 : (student.scalar_type() == at::kBFloat16 ? COS_DTYPE_BF16 : COS_DTYPE_F16);
      v.device = student.get_device();
      v.temperature = numbers[0];
      v.lists = static_cast<int32_t>(numbers[1]);
      v.k = static_cast<int32_t>(numbers[2]);
      for (int i = 0; i < v.lists; ++i) v.weights[i] = static_cast<float>(numbers[3 + i]);
      v.ids = static_cast<const int32_t*>(saved[1].data_ptr());
      v.values = static_cast<const float*>(saved[2].data_ptr());
      v.lse = saved[3].defined() ? static_cast<const float*>(saved[3].data_ptr()) : nullptr;
      v.statistics = static_cast<float*>(saved[4].data_ptr());
      v.row_weights = static_cast<const float*>(weights.data_ptr());
      v.grad = grad.data_ptr();
      v.stride_grad = v.vocab;
      const cos_status st = enqueue(static_cast<unsigned long long>(ctx->saved_data["grad_fn"].toInt()), v, student.device().index());
      TORCH_CHECK(st == COS_OK, "cos_distill_grad failed (", static_cast<int>(st), ")");
    }
    if (at::GradMode::is_enabled()) {  // (of create_graph: the gradient is there, its own is not)
      grad.requires_grad_(true);
      auto refuse = std::make_shared<torch::autograd::DelayedError>("distill_loss is differentiable once", 1);
      grad = (*refuse)({grad})[0];
    }
    out[0] = grad;
    return out;
  }
};

// distill_loss(cos_distill_loss, cos_distill_grad, student, ids, values, lse, weights, temperature)
PyObject* distill_loss(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  unsigned long long fn = 0, grad_fn = 0;
  if (nargs != 8 || !address(a[0], &fn) || !address(a[1], &grad_fn)) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "distill_loss takes 8 arguments");
    return nullptr;
  }
  HANDLE_TH_ERRORS
  {
    const at::Tensor* student = nullptr;
    cos_distill_args v = {};
    if (!distill_of(a + 2, &v, &student) || student->_fw_grad(0).defined()) Py_RETURN_NONE;  // (a tangent: refused)
    cos_status st = COS_OK;
    at::Tensor loss;
    if (at::GradMode::is_enabled() && student->requires_grad()) {
      const std::optional<at::Tensor> lse = a[5] == Py_None ? std::optional<at::Tensor>() : THPVariable_Unpack(a[5]);  // (an undefined tensor is no argument of a node)
      {
        const Unlocked unlocked;
        loss = DistillLoss::apply(*student, THPVariable_Unpack(a[3]), THPVariable_Unpack(a[4]), lse, &v, static_cast<int64_t>(fn), static_cast<int64_t>(grad_fn), &st);
      }
    } else {
      loss = floats(*student, v.rows);
      const at::Tensor statistics = floats(*student, statistics_size(v));
      v.loss = static_cast<float*>(loss.data_ptr());
      v.statistics = static_cast<float*>(statistics.data_ptr());
      {
        const Unlocked unlocked;
        st = enqueue(fn, v, student->device().index());
      }
    }
    if (st != COS_OK) return PyLong_FromLong(st);
    return THPVariable_Wrap(loss);
  }
  END_HANDLE_TH_ERRORS
}

// distill_step(cos_distill_step, student, ids, values, lse, weights, temperature, row_weights)
PyObject* distill_step(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  unsigned long long fn = 0;
  if (nargs != 8 || !address(a[0], &fn)) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "distill_step takes 8 arguments");
    return nullptr;
  }
  HANDLE_TH_ERRORS
  {
    const at::Tensor* student = nullptr;
    cos_distill_args v = {};
    if (!distill_of(a + 1, &v, &student)) Py_RETURN_NONE;
    v.row_weights = plain<float>(a[7], *student, v.rows, 1, at::kFloat);
    if (!v.row_weights) Py_RETURN_NONE;
    const at::Tensor loss = floats(*student, v.rows), statistics = floats(*student, statistics_size(v));
    const at::Tensor grad = at::empty({student->size(0), student->size(1)}, student->options().requires_grad(false));
    v.loss = static_cast<float*>(loss.data_ptr());
    v.statistics = static_cast<float*>(statistics.data_ptr());
    v.grad = grad.data_ptr();
    v.stride_grad = v.vocab;
    cos_status st;
    {
      const Unlocked unlocked;
      st = enqueue(fn, v, student->device().index());
    }
    if (st != COS_OK) return PyLong_FromLong(st);
    return dict_of({{"loss", loss}, {"grad", grad}});
  }
  END_HANDLE_TH_ERRORS
}

template <class F>
PyCFunction fast(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef methods[] = {{"callee", callee, METH_VARARGS, "a context, for run"},
                         {"run", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(run)), METH_FASTCALL, "one call of cos_verify_run"},
                         {"sample", fast(sample), METH_FASTCALL, "one call of cos_sample"},
                         {"top_logits", fast(top_logits), METH_FASTCALL, "one call of cos_top_logits"},
                         {"distill_loss", fast(distill_loss), METH_FASTCALL, "one call of cos_distill_loss, with its gradient"},
                         {"distill_step", fast(distill_step), METH_FASTCALL, "one call of cos_distill_step"},
                         {"refuse_capture", static_cast<PyCFunction>(refuse_capture), METH_O, "an error where a backward pass of this leaf must not be captured"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__call() { return PyModule_Create(&module); }
