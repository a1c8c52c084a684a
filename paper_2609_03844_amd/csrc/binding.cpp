// The Python entry points' call path in native code: argument checks, output tensors, the
// current stream and the libsbw call in one CPython function each.  Small calls are bound by
// the host; through ctypes a watermark call took 6.3 us of host time and a decoding call
// 13 us, most of it attribute reads and argument marshalling.
//
// These functions take the calls whose arguments are what the documentation asks for: plain
// strided tensors on the current device, Python numbers, the current stream.  For anything
// else they return None and do nothing, and the Python code of the entry point handles the
// call or names what is wrong with it.  Otherwise they return the sbw status, or for the
// functions with outputs the tuple of them (the status where it is not SBW_OK).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <c10/core/TensorImpl.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <exception>

#include "sbw.h"
#include "sbw_step.h"

namespace {

using at::Tensor;

// Keys of a plain tensor on the GPU; a fake, batched, functional or wrapped one has others.
const c10::DispatchKeySet kPlainKeys({c10::DispatchKey::CUDA, c10::DispatchKey::AutogradCUDA,
                                      c10::DispatchKey::ADInplaceOrView,
                                      c10::DispatchKey::AutocastCUDA});

bool plain(const Tensor& t) {
  return t.defined() && t.has_storage() && t.layout() == at::kStrided &&
         (t.key_set().raw_repr() & ~kPlainKeys.raw_repr()) == 0;
}

// The tensor behind a Python object, or null where it is not a plain one of this device,
// type and (for contiguous operands) layout.
const Tensor* tensor_of(PyObject* o, c10::DeviceIndex device) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const Tensor& t = THPVariable_Unpack(o);
  return plain(t) && t.get_device() == device ? &t : nullptr;
}
const Tensor* packed_of(PyObject* o, at::ScalarType type, c10::DeviceIndex device) {
  const Tensor* t = tensor_of(o, device);
  return t != nullptr && t->scalar_type() == type && t->is_contiguous() ? t : nullptr;
}

struct Call {
  const Tensor* matrix = nullptr;    // logits or texts
  int64_t rows, columns, row_stride;
  sbw_dtype_t dtype = SBW_F32;
  const Tensor* context = nullptr;
  int64_t width = 1;
  uint64_t key;
  double gamma, delta = 0.0;
  sbw_seeding_t seeding;
  c10::DeviceIndex device;
};

bool number(PyObject* o, double* out) {
  if (PyFloat_Check(o)) {
    *out = PyFloat_AS_DOUBLE(o);
    return true;
  }
  if (!PyLong_CheckExact(o)) return false;
  *out = PyLong_AsDouble(o);
  if (*out == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  return true;
}

bool integer(PyObject* o, int64_t* out) {
  if (!PyLong_CheckExact(o)) return false;
  int overflow = 0;
  *out = PyLong_AsLongLongAndOverflow(o, &overflow);
  return overflow == 0;
}

bool key_of(PyObject* o, uint64_t* out) {   // the low 64 bits of any integer
  if (!PyLong_CheckExact(o)) return false;
  *out = PyLong_AsUnsignedLongLongMask(o);
  return true;
}

bool seeding_of(PyObject* o, sbw_seeding_t* out) {
  if (!PyUnicode_CheckExact(o)) return false;
  if (PyUnicode_CompareWithASCIIString(o, "context") == 0) *out = SBW_SEED_CONTEXT;
  else if (PyUnicode_CompareWithASCIIString(o, "self_salt") == 0) *out = SBW_SEED_SELF_SALT;
  else return false;
  return true;
}

// A non-empty matrix with unit stride along its rows, on the current device.
bool matrix_of(PyObject* o, Call* c) {
  if (!THPVariable_CheckExact(o)) return false;
  const Tensor& t = THPVariable_Unpack(o);
  if (!plain(t) || t.dim() != 2 || t.numel() == 0 || t.stride(1) != 1) return false;
  c->device = c10::hip::current_device();
  if (t.get_device() != c->device) return false;
  c->matrix = &t;
  c->rows = t.size(0);
  c->columns = t.size(1);
  c->row_stride = c->rows > 1 ? t.stride(0) : std::max(c->columns, t.stride(0));
  return true;
}

// logits, context, key, gamma, delta, seeding
bool logits_call(PyObject* logits, PyObject* context, PyObject* key, PyObject* gamma, PyObject* delta,
                 PyObject* seeding, Call* c) {
  if (!matrix_of(logits, c)) return false;
  if (c->matrix->scalar_type() == at::kBFloat16) c->dtype = SBW_BF16;
  else if (c->matrix->scalar_type() != at::kFloat) return false;
  c->context = packed_of(context, at::kInt, c->device);
  if (c->context == nullptr || c->context->dim() < 1 || c->context->dim() > 2 ||
      c->context->size(0) != c->rows)
    return false;
  c->width = c->context->dim() == 2 ? c->context->size(1) : 1;
  return key_of(key, &c->key) && number(gamma, &c->gamma) && number(delta, &c->delta) &&
         seeding_of(seeding, &c->seeding);
}

void* stream_of(const Call& c) { return c10::hip::getCurrentHIPStream(c.device).stream(); }

// The caller's output vector, or a new one for None.
bool output_of(PyObject* o, int64_t n, at::ScalarType type, const Call& c, Tensor* out) {
  if (o == Py_None) {
    *out = at::empty({n}, c.matrix->options().dtype(type));
    return plain(*out);
  }
  const Tensor* t = packed_of(o, type, c.device);
  if (t == nullptr || t->dim() != 1 || t->size(0) != n) return false;
  *out = *t;
  return true;
}

PyObject* object_of(PyObject* given, const Tensor& t) {
  if (given != Py_None) {
    Py_INCREF(given);
    return given;
  }
  return THPVariable_Wrap(t);
}

template <typename F>
PyObject* guarded(F&& f) {
  try {
    return f();
  } catch (const std::exception&) {   // the Python path meets the same error and reports it
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

template <typename F>
sbw_status_t unlocked(F&& f) {
  sbw_status_t s;
  Py_BEGIN_ALLOW_THREADS
  s = f();
  Py_END_ALLOW_THREADS
  return s;
}

// Two or three objects in a tuple, built before the launch so that nothing fails after it.
PyObject* tuple_of(PyObject* a, PyObject* b, PyObject* c) {
  PyObject* t = a != nullptr && b != nullptr ? PyTuple_New(c != nullptr ? 3 : 2) : nullptr;
  if (t == nullptr) {
    Py_XDECREF(a);
    Py_XDECREF(b);
    Py_XDECREF(c);
    return nullptr;
  }
  PyTuple_SET_ITEM(t, 0, a);
  PyTuple_SET_ITEM(t, 1, b);
  if (c != nullptr) PyTuple_SET_ITEM(t, 2, c);
  return t;
}

PyObject* outputs_or_status(PyObject* outputs, sbw_status_t s) {
  if (s == SBW_OK) return outputs;
  Py_DECREF(outputs);
  return PyLong_FromLong(s);
}

// watermark(logits, context, key, gamma, delta, seeding, v_offset)
PyObject* watermark(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Call c;
    int64_t v_offset;
    if (n != 7 || !logits_call(a[0], a[1], a[2], a[3], a[4], a[5], &c) || !integer(a[6], &v_offset))
      Py_RETURN_NONE;
    void* logits = c.matrix->data_ptr();
    const auto* context = static_cast<const int32_t*>(c.context->data_ptr());
    void* stream = stream_of(c);
    return PyLong_FromLong(unlocked([&] {
      return sbw_watermark_shard(logits, c.dtype, c.rows, c.columns, c.row_stride, context, c.width,
                                 v_offset, c.key, c.gamma, static_cast<float>(c.delta), c.seeding, stream);
    }));
  });
}

// watermark_candidates(logits, context, candidates, key, gamma, delta, seeding)
PyObject* watermark_candidates(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Call c;
    if (n != 7 || !logits_call(a[0], a[1], a[3], a[4], a[5], a[6], &c)) Py_RETURN_NONE;
    const Tensor* cand = packed_of(a[2], at::kInt, c.device);
    if (cand == nullptr || cand->dim() != 2 || cand->size(0) != c.rows) Py_RETURN_NONE;
    void* logits = c.matrix->data_ptr();
    const auto* context = static_cast<const int32_t*>(c.context->data_ptr());
    const auto* ids = static_cast<const int32_t*>(cand->data_ptr());
    const int64_t k = cand->size(1);
    void* stream = stream_of(c);
    return PyLong_FromLong(unlocked([&] {
      return sbw_watermark_candidates(logits, c.dtype, c.rows, c.columns, c.row_stride, ids, k, context,
                                      c.width, c.key, c.gamma, static_cast<float>(c.delta), c.seeding,
                                      stream);
    }));
  });
}

// decode(logits, context, key, gamma, delta, seeding, seeds or None, inv_temperature,
//        tokens, values, workspace, with_values, v_offset): greedy without seeds
PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Call c;
    int64_t v_offset;
    double inv_t = 1.0;
    if (n != 13 || !logits_call(a[0], a[1], a[2], a[3], a[4], a[5], &c) || !number(a[7], &inv_t) ||
        !PyBool_Check(a[11]) || !integer(a[12], &v_offset))
      Py_RETURN_NONE;
    const bool sample = a[6] != Py_None;
    const Tensor* seeds = nullptr;
    if (sample) {
      seeds = packed_of(a[6], at::kLong, c.device);
      if (seeds == nullptr || seeds->dim() != 1 || seeds->size(0) != c.rows) Py_RETURN_NONE;
    }
    const bool with_values = a[9] != Py_None || a[11] == Py_True;
    const int64_t need = sbw_watermark_argmax_workspace(c.rows, c.columns);
    Tensor tokens, values, workspace;
    if (!output_of(a[8], c.rows, at::kInt, c, &tokens)) Py_RETURN_NONE;
    if (with_values && !output_of(a[9], c.rows, at::kFloat, c, &values)) Py_RETURN_NONE;
    if (a[10] == Py_None) {
      if (!output_of(Py_None, need, at::kLong, c, &workspace)) Py_RETURN_NONE;
    } else {
      const Tensor* w = packed_of(a[10], at::kLong, c.device);
      if (w == nullptr || w->numel() < need) Py_RETURN_NONE;
      workspace = *w;
    }
    const void* logits = c.matrix->data_ptr();
    const auto* context = static_cast<const int32_t*>(c.context->data_ptr());
    auto* token = static_cast<int32_t*>(tokens.data_ptr());
    auto* value = with_values ? static_cast<float*>(values.data_ptr()) : nullptr;
    auto* partials = static_cast<uint64_t*>(workspace.data_ptr());
    const auto* seed = sample ? static_cast<const uint64_t*>(seeds->data_ptr()) : nullptr;
    void* stream = stream_of(c);
    PyObject* second;
    if (with_values) {
      second = object_of(a[9], values);
    } else {
      Py_INCREF(Py_None);
      second = Py_None;
    }
    PyObject* outputs = tuple_of(object_of(a[8], tokens), second, nullptr);
    if (outputs == nullptr) return nullptr;
    return outputs_or_status(outputs, unlocked([&] {
      const float delta = static_cast<float>(c.delta);
      if (sample)
        return sbw_watermark_sample_shard(logits, c.dtype, c.rows, c.columns, c.row_stride, context, c.width,
                                          v_offset, c.key, c.gamma, delta, c.seeding, seed,
                                          static_cast<float>(inv_t), token, value, partials, stream);
      return sbw_watermark_argmax_shard(logits, c.dtype, c.rows, c.columns, c.row_stride, context, c.width,
                                        v_offset, c.key, c.gamma, delta, c.seeding, token, value, partials,
                                        stream);
    }));
  });
}

// detect(tokens, key, gamma, seeding, width, lengths, ignore_repeated, counts, z[, scored]):
// without `scored` the scored positions are left out (two outputs)
PyObject* detect(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Call c;
    if (n < 9 || n > 10 || !matrix_of(a[0], &c) || c.matrix->scalar_type() != at::kInt || !key_of(a[1], &c.key) ||
        !number(a[2], &c.gamma) || !seeding_of(a[3], &c.seeding) || !integer(a[4], &c.width) ||
        !PyBool_Check(a[6]))
      Py_RETURN_NONE;
    const Tensor* lengths = nullptr;
    if (a[5] != Py_None) {
      lengths = packed_of(a[5], at::kInt, c.device);
      if (lengths == nullptr || lengths->dim() != 1 || lengths->size(0) != c.rows) Py_RETURN_NONE;
    }
    const bool with_scored = n == 10;
    Tensor counts, scored, z;
    if (!output_of(a[7], c.rows, at::kInt, c, &counts) ||
        (with_scored && !output_of(a[9], c.rows, at::kInt, c, &scored)) ||
        !output_of(a[8], c.rows, at::kDouble, c, &z))
      Py_RETURN_NONE;
    const auto* tokens = static_cast<const int32_t*>(c.matrix->data_ptr());
    const auto* length = lengths != nullptr ? static_cast<const int32_t*>(lengths->data_ptr()) : nullptr;
    auto* count = static_cast<int32_t*>(counts.data_ptr());
    auto* positions = with_scored ? static_cast<int32_t*>(scored.data_ptr()) : nullptr;
    auto* score = static_cast<double*>(z.data_ptr());
    const uint32_t flags = a[6] == Py_True ? SBW_DETECT_IGNORE_REPEATED : 0u;
    void* stream = stream_of(c);
    PyObject* first = object_of(a[7], counts);
    PyObject* last = object_of(a[8], z);
    PyObject* outputs = with_scored ? tuple_of(first, object_of(a[9], scored), last)
                                    : tuple_of(first, last, nullptr);
    if (outputs == nullptr) return nullptr;
    return outputs_or_status(outputs, unlocked([&] {
      return sbw_detect_ex(tokens, c.rows, c.columns, c.row_stride, length, c.width, c.key, c.gamma,
                           c.seeding, flags, count, positions, score, stream);
    }));
  });
}

// ---- the operators of sbw_step.h ---------------------------------------------------------

// A tuple of `count` new objects (an array whose unset places are None); all or nothing.
template <size_t count>
PyObject* tuple_of(PyObject* (&objects)[count]) {
  PyObject* t = PyTuple_New(count);
  for (size_t i = 0; i < count; ++i) {
    if (objects[i] == nullptr) {
      Py_INCREF(Py_None);
      objects[i] = Py_None;
    }
    if (t != nullptr) PyTuple_SET_ITEM(t, i, objects[i]);
    else Py_DECREF(objects[i]);
  }
  return t;
}

// Outputs of four-byte elements side by side in one allocation (an allocation costs the host about a
// microsecond, a tensor on a part of one a tenth), behind a workspace that is small; a larger one has an
// allocation of its own, so that no output keeps it alive.
constexpr int64_t kSmallWorkspace = 8192;   // 64 KiB
struct Block {
  Tensor whole, own_workspace;
  int64_t used = 0;
  Block(int64_t workspace, int64_t elements, const Call& c) {
    const auto options = c.matrix->options().requires_grad(false);
    if (workspace <= kSmallWorkspace) used = 2 * workspace;
    else own_workspace = at::empty({workspace}, options.dtype(at::kLong));
    whole = at::empty({used + elements}, options.dtype(at::kFloat));
  }
  uint64_t* workspace() const {
    return static_cast<uint64_t*>((own_workspace.defined() ? own_workspace : whole).data_ptr());
  }
  Tensor take(at::ScalarType type, at::IntArrayRef sizes) {
    auto impl = c10::make_intrusive<c10::TensorImpl>(c10::Storage(whole.storage()), whole.key_set(),
                                                     at::scalarTypeToTypeMeta(type));
    impl->set_sizes_contiguous(sizes);
    impl->set_storage_offset(used);
    used += impl->numel();
    return Tensor(std::move(impl));
  }
};

// Whether a gradient is asked for, or a tangent: the Python path refuses them for outputs that carry none.
bool followed(const Tensor& t) { return t.requires_grad() && c10::GradMode::is_enabled(); }
bool dual(const Tensor& t) { return t._fw_grad(0).defined(); }

// logits and, unless None, tokens [rows] or [rows, n]
bool tokens_call(PyObject* logits, PyObject* tokens, Call* c, const Tensor** ids, int64_t* n) {
  if (!matrix_of(logits, c) || (c->rows > 1 && c->row_stride < c->columns)) return false;
  if (c->matrix->scalar_type() == at::kBFloat16) c->dtype = SBW_BF16;
  else if (c->matrix->scalar_type() != at::kFloat) return false;
  if (dual(*c->matrix)) return false;
  *ids = nullptr;
  *n = 0;
  if (tokens == Py_None) return true;
  const Tensor* t = packed_of(tokens, at::kInt, c->device);
  if (t == nullptr || t->dim() < 1 || t->dim() > 2 || t->size(0) != c->rows) return false;
  *ids = t;
  *n = t->dim() == 2 ? t->size(1) : 1;
  return true;
}

// None (a null pointer), or a packed float tensor of this shape.
bool floats_of(PyObject* o, at::IntArrayRef shape, const Call& c, const float** out) {
  *out = nullptr;
  if (o == Py_None) return true;
  const Tensor* t = packed_of(o, at::kFloat, c.device);
  if (t == nullptr || t->sizes() != shape || dual(*t)) return false;
  *out = static_cast<const float*>(t->data_ptr());
  return true;
}

// token_logprobs(logits, tokens or None, inv_temperature, top): the six outputs
PyObject* token_logprobs(PyObject*, PyObject* const* a, Py_ssize_t count) {
  return guarded([&]() -> PyObject* {
    Call c;
    const Tensor* ids;
    int64_t n, top;
    double inv_t;
    if (count != 4 || !tokens_call(a[0], a[1], &c, &ids, &n) || !number(a[2], &inv_t) || !integer(a[3], &top) ||
        top < 0 || top > SBW_STEP_MAX_TOKENS || n > SBW_STEP_MAX_TOKENS)
      Py_RETURN_NONE;
    Block block(sbw_token_logprobs_workspace(c.rows, c.columns, top), c.rows * (4 + n + 2 * top), c);
    Tensor stats = block.take(at::kFloat, {c.rows, 2});
    Tensor lse = block.take(at::kFloat, {c.rows}), entropy = block.take(at::kFloat, {c.rows});
    Tensor logprobs, top_ids, top_logprobs;
    if (ids != nullptr) logprobs = block.take(at::kFloat, ids->sizes());
    if (top > 0) {
      top_ids = block.take(at::kInt, {c.rows, top});
      top_logprobs = block.take(at::kFloat, {c.rows, top});
    }
    const void* logits = c.matrix->data_ptr();
    const auto* token = ids != nullptr ? static_cast<const int32_t*>(ids->data_ptr()) : nullptr;
    const auto address = [](const Tensor& t) { return t.defined() ? static_cast<float*>(t.data_ptr()) : nullptr; };
    float *lp = address(logprobs), *l = address(lse), *h = address(entropy), *st = address(stats);
    float* tl = address(top_logprobs);
    auto* ti = top > 0 ? static_cast<int32_t*>(top_ids.data_ptr()) : nullptr;
    uint64_t* scratch = block.workspace();
    void* stream = stream_of(c);
    PyObject* objects[6] = {};
    const Tensor* outputs[6] = {&logprobs, &lse, &entropy, &stats, &top_ids, &top_logprobs};
    for (int i = 0; i < 6; ++i)
      if (outputs[i]->defined()) objects[i] = THPVariable_Wrap(*outputs[i]);
    PyObject* result = tuple_of(objects);
    if (result == nullptr) return nullptr;
    return outputs_or_status(result, unlocked([&] {
      return sbw_token_logprobs(logits, c.dtype, c.rows, c.columns, c.row_stride, token, n,
                                static_cast<float>(inv_t), top, lp, l, h, st, ti, tl, scratch, stream);
    }));
  });
}

// token_logprobs_grad(logits, tokens or None, stats, entropy, grad_logprobs, grad_lse, grad_entropy (each or
//                     None), inv_temperature): the gradient
PyObject* token_logprobs_grad(PyObject*, PyObject* const* a, Py_ssize_t count) {
  return guarded([&]() -> PyObject* {
    Call c;
    const Tensor* ids;
    int64_t n;
    double inv_t;
    const float *stats, *entropy, *g, *g_lse, *g_entropy;
    if (count != 8 || !tokens_call(a[0], a[1], &c, &ids, &n) || a[2] == Py_None ||
        (a[4] != Py_None && ids == nullptr) || !floats_of(a[2], {c.rows, 2}, c, &stats) ||
        !floats_of(a[3], {c.rows}, c, &entropy) ||
        !floats_of(a[4], ids != nullptr ? ids->sizes() : at::IntArrayRef(), c, &g) ||
        !floats_of(a[5], {c.rows}, c, &g_lse) || !floats_of(a[6], {c.rows}, c, &g_entropy) || !number(a[7], &inv_t) ||
        (g_entropy != nullptr && entropy == nullptr))
      Py_RETURN_NONE;
    Tensor grad = at::empty({c.rows, c.columns}, c.matrix->options().requires_grad(false));
    const void* logits = c.matrix->data_ptr();
    const auto* token = ids != nullptr ? static_cast<const int32_t*>(ids->data_ptr()) : nullptr;
    void* out = grad.data_ptr();
    void* stream = stream_of(c);
    PyObject* result = THPVariable_Wrap(grad);
    if (result == nullptr) return nullptr;
    return outputs_or_status(result, unlocked([&] {
      return sbw_token_logprobs_grad(logits, c.dtype, c.rows, c.columns, c.row_stride, token, n, stats, entropy, g,
                                     g_lse, g_entropy, static_cast<float>(inv_t), out, c.columns, stream);
    }));
  });
}

// top_candidates(logits, k, v_offset): ids and values
PyObject* top_candidates(PyObject*, PyObject* const* a, Py_ssize_t count) {
  return guarded([&]() -> PyObject* {
    Call c;
    const Tensor* none;
    int64_t n, k, v_offset;
    if (count != 3 || !tokens_call(a[0], Py_None, &c, &none, &n) || !integer(a[1], &k) || k < 1 ||
        !integer(a[2], &v_offset) || k > SBW_STEP_MAX_TOKENS || followed(*c.matrix))
      Py_RETURN_NONE;
    Block block(sbw_top_candidates_workspace(c.rows, c.columns, k), 2 * c.rows * k, c);
    Tensor ids = block.take(at::kInt, {c.rows, k}), values = block.take(at::kFloat, {c.rows, k});
    const void* logits = c.matrix->data_ptr();
    auto* id = static_cast<int32_t*>(ids.data_ptr());
    auto* value = static_cast<float*>(values.data_ptr());
    uint64_t* scratch = block.workspace();
    void* stream = stream_of(c);
    PyObject* result = tuple_of(THPVariable_Wrap(ids), THPVariable_Wrap(values), nullptr);
    if (result == nullptr) return nullptr;
    return outputs_or_status(result, unlocked([&] {
      return sbw_top_candidates(logits, c.dtype, c.rows, c.columns, c.row_stride, v_offset, k, id, value, scratch,
                                stream);
    }));
  });
}

// head_logits(hidden, codes, scales, whether the logits are bfloat16): the logits
PyObject* head_logits(PyObject*, PyObject* const* a, Py_ssize_t count) {
  return guarded([&]() -> PyObject* {
    Call c;
    if (count != 4 || !matrix_of(a[0], &c) || c.matrix->scalar_type() != at::kBFloat16 || !PyBool_Check(a[3]) ||
        (c.rows > 1 && c.row_stride < c.columns) || followed(*c.matrix) || dual(*c.matrix))
      Py_RETURN_NONE;
    const Tensor* codes = packed_of(a[1], at::kByte, c.device);
    if (codes == nullptr || codes->dim() != 2 || 2 * codes->size(1) != c.columns || codes->size(0) == 0)
      Py_RETURN_NONE;
    const int64_t V = codes->size(0);
    const Tensor* scales = packed_of(a[2], at::kFloat, c.device);
    sbw_dtype_t scale_dtype = SBW_F32;
    if (scales == nullptr) {
      scales = packed_of(a[2], at::kBFloat16, c.device);
      scale_dtype = SBW_BF16;
    }
    if (scales == nullptr || scales->dim() != 2 || scales->size(0) != V || scales->size(1) == 0 ||
        c.columns % scales->size(1) != 0 || followed(*scales) || dual(*scales))
      Py_RETURN_NONE;
    const bool bf16 = a[3] == Py_True;
    Tensor logits = at::empty({c.rows, V}, c.matrix->options().dtype(bf16 ? at::kBFloat16 : at::kFloat)
                                               .requires_grad(false));
    const void* hidden = c.matrix->data_ptr();
    const auto* code = static_cast<const uint8_t*>(codes->data_ptr());
    const void* scale = scales->data_ptr();
    const int64_t group = c.columns / scales->size(1);
    void* out = logits.data_ptr();
    void* stream = stream_of(c);
    PyObject* result = THPVariable_Wrap(logits);
    if (result == nullptr) return nullptr;
    return outputs_or_status(result, unlocked([&] {
      return sbw_head_logits(hidden, c.rows, c.columns, c.row_stride, code, scale, scale_dtype, group, V, out,
                             bf16 ? SBW_BF16 : SBW_F32, V, stream);
    }));
  });
}

PyCFunction fast(PyObject* (*f)(PyObject*, PyObject* const*, Py_ssize_t)) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}

PyMethodDef methods[] = {
    {"watermark", fast(watermark), METH_FASTCALL, nullptr},
    {"watermark_candidates", fast(watermark_candidates), METH_FASTCALL, nullptr},
    {"decode", fast(decode), METH_FASTCALL, nullptr},
    {"detect", fast(detect), METH_FASTCALL, nullptr},
    {"token_logprobs", fast(token_logprobs), METH_FASTCALL, nullptr},
    {"token_logprobs_grad", fast(token_logprobs_grad), METH_FASTCALL, nullptr},
    {"top_candidates", fast(top_candidates), METH_FASTCALL, nullptr},
    {"head_logits", fast(head_logits), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
