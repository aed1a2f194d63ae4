// fastcall.cpp -- the argument checks of the calls that programs make once per ply, in native code.
//
// With small batches a ply takes the GPU 4 to 6 us, and the Python checks of the up to seven tensors of a call (dtype, device,
// contiguity, shape, pointer: 0.4 us each) took longer than that.  Each function here checks the tensors of one call exactly as
// binding.py does and calls the library's C entry point, whose address it is given; it returns the entry point's code, or None when
// anything is not as it has to be, and then the Python path runs and raises its error.  Nothing is kept between calls.
#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/GradMode.h>
#include <c10/core/StreamGuard.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdint>

#include "pgxcache.h"
#include "pgxpolicy.h"
#include "pgxrotary.h"

namespace {

// pointer of a contiguous cuda tensor of the given type and shape; false: not such a tensor (or one of a subclass)
bool take(PyObject* o, at::ScalarType type, int64_t d0, int64_t d1, void** out) {
  if (!THPVariable_CheckExact(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  const int64_t dim = d1 < 0 ? 1 : 2;
  if (t.scalar_type() != type || !t.is_cuda() || t.dim() != dim || t.size(0) != d0 || (dim == 2 && t.size(1) != d1) || !t.is_contiguous()) return false;
  *out = t.data_ptr();
  return true;
}
// the same, None gives a null pointer
bool take_or_null(PyObject* o, at::ScalarType type, int64_t d0, int64_t d1, void** out) {
  if (o == Py_None) { *out = nullptr; return true; }
  return take(o, type, d0, d1, out);
}

template <class F>
PyObject* guarded(F&& f) {   // f: prepares and calls; returns -1000 when the Python path has to look at the call
  int rc = -1000;
  try {
    rc = f();
  } catch (...) {
    rc = -1000;
  }
  if (PyErr_Occurred()) PyErr_Clear();
  if (rc == -1000) Py_RETURN_NONE;
  return PyLong_FromLong(rc);
}
template <class F>
int without_gil(F&& f) {   // launching can wait for room in the queue
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f();
  Py_END_ALLOW_THREADS
  return rc;
}
void* pointer(PyObject* o) { return PyLong_AsVoidPtr(o); }
uint32_t u32(PyObject* o) { return (uint32_t)PyLong_AsUnsignedLongLong(o); }

constexpr auto kInt = at::kInt;
constexpr auto kByte = at::kByte;
constexpr auto kFloat = at::kFloat;

// (address, handle, batch, actions)
PyObject* step(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&] {
    void* actions;
    if (n != 4) return -1000;
    void *fn = pointer(a[0]), *h = pointer(a[1]);
    const int64_t B = PyLong_AsLongLong(a[2]);
    if (PyErr_Occurred() || !take(a[3], kInt, B, -1, &actions)) return -1000;
    return without_gil([&] { return ((int (*)(void*, const int32_t*))fn)(h, (const int32_t*)actions); });
  });
}

// (address, handle, batch, actions, seed, t, start_t, out)
PyObject* step_sample(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&] {
    void *actions, *start, *out;
    if (n != 8) return -1000;
    void *fn = pointer(a[0]), *h = pointer(a[1]);
    const int64_t B = PyLong_AsLongLong(a[2]);
    const uint32_t seed = u32(a[4]), t = u32(a[5]);
    if (PyErr_Occurred() || !take(a[3], kInt, B, -1, &actions) || !take_or_null(a[6], kInt, B, -1, &start) || !take(a[7], kInt, B, -1, &out)) return -1000;
    return without_gil([&] {
      return ((int (*)(void*, const int32_t*, uint32_t, uint32_t, const int32_t*, int32_t*))fn)(h, (const int32_t*)actions, seed, t, (const int32_t*)start,
                                                                                               (int32_t*)out);
    });
  });
}

// (address, handle, batch, seed, t, start_t, out)
PyObject* random_actions(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&] {
    void *start, *out;
    if (n != 7) return -1000;
    void *fn = pointer(a[0]), *h = pointer(a[1]);
    const int64_t B = PyLong_AsLongLong(a[2]);
    const uint32_t seed = u32(a[3]), t = u32(a[4]);
    if (PyErr_Occurred() || !take_or_null(a[5], kInt, B, -1, &start) || !take(a[6], kInt, B, -1, &out)) return -1000;
    return without_gil([&] { return ((int (*)(void*, uint32_t, uint32_t, const int32_t*, int32_t*))fn)(h, seed, t, (const int32_t*)start, (int32_t*)out); });
  });
}

// (address, handle, mask_pitch, obs_pitch, src, actions, dst, mask, obs, rewards, terminated)
PyObject* step_slots(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&] {
    void *src, *actions, *dst, *mask, *obs, *rew, *term;
    if (n != 11 || !THPVariable_CheckExact(a[4])) return -1000;
    void *fn = pointer(a[0]), *h = pointer(a[1]);
    const int64_t mask_pitch = PyLong_AsLongLong(a[2]), obs_pitch = PyLong_AsLongLong(a[3]);
    const at::Tensor& s = THPVariable_Unpack(a[4]);
    if (PyErr_Occurred() || s.dim() != 1 || s.size(0) > INT32_MAX) return -1000;
    const int64_t N = s.size(0);
    if (!take(a[4], kInt, N, -1, &src) || !take_or_null(a[5], kInt, N, -1, &actions) || !take(a[6], kInt, N, -1, &dst) ||
        !take_or_null(a[7], kByte, N, mask_pitch, &mask) || !take_or_null(a[8], kByte, N, obs_pitch, &obs) || !take_or_null(a[9], kFloat, N, 2, &rew) ||
        !take_or_null(a[10], kByte, N, -1, &term))
      return -1000;
    return without_gil([&] {
      return ((int (*)(void*, int32_t, const int32_t*, const int32_t*, const int32_t*, uint8_t*, uint8_t*, float*, uint8_t*))fn)(
          h, (int32_t)N, (const int32_t*)src, (const int32_t*)actions, (const int32_t*)dst, (uint8_t*)mask, (uint8_t*)obs, (float*)rew, (uint8_t*)term);
    });
  });
}

// ---- the policy's calls: from logits to actions, and the loss --------------------------------------------------------------------------
const at::Tensor* tensor(PyObject* o) { return THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr; }
bool dense_rows(const at::Tensor& t) { return t.numel() == 0 || t.size(-1) == 1 || t.stride(-1) == 1; }

struct Row {   // what the calls know of the logits
  int64_t rows, actions, pitch;
  int32_t type;
  c10::Device device;
  const void* data;
};
bool take_logits(PyObject* o, Row* r) {
  const at::Tensor* t = tensor(o);
  if (!t || !t->is_cuda() || t->dim() != 2 || !dense_rows(*t)) return false;
  const auto s = t->scalar_type();
  if (s != at::kFloat && s != at::kHalf && s != at::kBFloat16) return false;
  *r = Row{t->size(0), t->size(1), t->stride(0), s == at::kFloat ? PGXPOLICY_F32 : s == at::kHalf ? PGXPOLICY_F16 : PGXPOLICY_BF16, t->device(), t->data_ptr()};
  return r->actions >= 1 && r->actions <= PGXPOLICY_MAX_ACTIONS && r->rows <= INT32_MAX;
}
// one value per row, or None
bool take_per_row(PyObject* o, const Row& r, at::ScalarType type, void** out) {
  *out = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = tensor(o);
  if (!t || t->scalar_type() != type || t->device() != r.device || t->dim() != 1 || t->size(0) != r.rows || !dense_rows(*t)) return false;
  *out = t->data_ptr();
  return true;
}
// float32 [rows][actions], or None
bool take_matrix(PyObject* o, const Row& r, at::ScalarType type, void** out, int64_t* pitch) {
  *out = nullptr;
  *pitch = 0;
  if (o == Py_None) return true;
  const at::Tensor* t = tensor(o);
  if (!t || t->scalar_type() != type || t->device() != r.device || t->dim() != 2 || t->size(0) != r.rows || t->size(1) != r.actions || !dense_rows(*t)) return false;
  *out = t->data_ptr();
  *pitch = t->stride(0);
  return true;
}
bool number(PyObject* o, float* out) {
  if (!PyFloat_Check(o) && !PyLong_Check(o)) return false;
  *out = (float)PyFloat_AsDouble(o);
  return !PyErr_Occurred();
}
// (mask, bias, record, begin, end, repetition, frequency, presence, temperature)
constexpr int kAdjustArgs = 9;
bool take_adjust(PyObject* const* a, const Row& r, pgxpolicy_adjust* d) {
  *d = pgxpolicy_adjust{};
  if (a[0] != Py_None) {
    const at::Tensor* t = tensor(a[0]);
    if (!t || (t->scalar_type() != kByte && t->scalar_type() != at::kBool) || t->device() != r.device || t->dim() != 2 || t->size(0) != r.rows ||
        t->size(1) < r.actions || !dense_rows(*t))
      return false;
    d->mask_dev = (const uint8_t*)t->data_ptr();
    d->mask_pitch = t->stride(0);
  }
  if (a[1] != Py_None) {
    const at::Tensor* t = tensor(a[1]);
    if (!t || t->scalar_type() != kFloat || t->device() != r.device || (t->dim() != 1 && t->dim() != 2) || t->size(-1) != r.actions ||
        (t->dim() == 2 && t->size(0) != r.rows) || !dense_rows(*t))
      return false;
    d->bias_dev = (const float*)t->data_ptr();
    d->bias_pitch = t->dim() == 1 ? 0 : t->stride(0);
  }
  if (!number(a[5], &d->repetition) || !number(a[6], &d->frequency) || !number(a[7], &d->presence)) return false;
  if (!(d->repetition > 0.0f) || !std::isfinite(d->repetition)) return false;
  if (a[2] != Py_None) {
    const at::Tensor* t = tensor(a[2]);
    void *begin, *end;
    if (!t || t->scalar_type() != kInt || t->device() != r.device || t->dim() != 2 || t->size(0) != r.rows || t->size(1) > PGXPOLICY_MAX_RECORD) return false;
    if (!take_per_row(a[3], r, kInt, &begin) || !take_per_row(a[4], r, kInt, &end)) return false;
    d->record_dev = (const int32_t*)t->data_ptr();
    d->record_row_stride = t->stride(0);
    d->record_ply_stride = t->stride(1);
    d->record_len = (int32_t)t->size(1);
    d->begin_dev = (const int32_t*)begin;
    d->end_dev = (const int32_t*)end;
  } else if (a[3] != Py_None || a[4] != Py_None || d->repetition != 1.0f || d->frequency != 0.0f || d->presence != 0.0f) {
    return false;
  }
  if (a[8] == Py_None) return true;
  if (number(a[8], &d->temperature)) return d->temperature > 0.0f && std::isfinite(d->temperature);
  void* t;
  if (!take_per_row(a[8], r, kFloat, &t)) return false;
  d->temperature_dev = (const float*)t;
  return true;
}
PyObject* g_raw_stream;   // callable: device index -> the current stream's address
bool current_stream(c10::Device d, void** out) {
  PyObject* index = PyLong_FromLong(d.index());
  PyObject* s = index && g_raw_stream ? PyObject_CallOneArg(g_raw_stream, index) : nullptr;
  Py_XDECREF(index);
  if (!s) return false;
  *out = PyLong_AsVoidPtr(s);
  Py_DECREF(s);
  return !PyErr_Occurred();
}
at::Tensor fresh(at::IntArrayRef shape, at::ScalarType type, c10::Device d) { return at::empty(shape, at::TensorOptions().dtype(type).device(d)); }
void* data_or_null(const at::Tensor& t) { return t.numel() ? t.data_ptr() : nullptr; }
// the given output or a new one
bool output(PyObject* o, at::IntArrayRef shape, at::ScalarType type, c10::Device d, at::Tensor* out) {
  if (o == Py_None) {
    *out = fresh(shape, type, d);
    return true;
  }
  const at::Tensor* t = tensor(o);
  if (!t || t->scalar_type() != type || t->device() != d || t->sizes() != shape || !dense_rows(*t)) return false;
  *out = *t;
  return true;
}
// the code, or the outputs once the call has succeeded
PyObject* outputs(int rc, std::initializer_list<std::pair<PyObject*, at::Tensor>> list) {
  if (rc != 0) return PyLong_FromLong(rc);
  PyObject* tuple = PyTuple_New((Py_ssize_t)list.size());
  if (!tuple) return nullptr;
  Py_ssize_t i = 0;
  for (const auto& [given, t] : list) {
    PyObject* o = given == Py_None ? THPVariable_Wrap(t) : Py_NewRef(given);
    if (!o) { Py_DECREF(tuple); return nullptr; }
    PyTuple_SET_ITEM(tuple, i++, o);
  }
  return tuple;
}
template <class F>
PyObject* guarded_outputs(F&& f) {   // f: prepares, calls and returns the outputs; nullptr when the Python path has to look at the call
  PyObject* o = nullptr;
  try {
    o = f();
  } catch (...) {
    o = nullptr;
  }
  if (PyErr_Occurred()) { PyErr_Clear(); Py_CLEAR(o); }
  if (!o) Py_RETURN_NONE;
  return o;
}

PyObject* set_raw_stream(PyObject*, PyObject* f) {
  Py_XDECREF(g_raw_stream);
  g_raw_stream = Py_NewRef(f);
  Py_RETURN_NONE;
}

// (address, logits, adjust..., normalize, out)
PyObject* policy_logits(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded_outputs([&]() -> PyObject* {
    Row r{0, 0, 0, 0, c10::Device(c10::kCPU), nullptr};
    pgxpolicy_adjust d;
    at::Tensor out;
    void* stream;
    if (n != 4 + kAdjustArgs || !take_logits(a[1], &r) || !take_adjust(a + 2, r, &d)) return nullptr;
    PyObject* given = a[3 + kAdjustArgs];
    const int normalize = PyObject_IsTrue(a[2 + kAdjustArgs]);
    const c10::DeviceGuard guard(r.device);
    if (!output(given, {r.rows, r.actions}, kFloat, r.device, &out) || !current_stream(r.device, &stream)) return nullptr;
    auto* fn = (decltype(&pgxpolicy_logits))pointer(a[0]);
    const int rc = without_gil([&] { return fn((int32_t)r.rows, (int32_t)r.actions, r.data, r.type, r.pitch, &d, normalize, (float*)data_or_null(out), out.stride(0), stream); });
    return outputs(rc, {{given, out}});
  });
}

// (address, logits, noise, adjust..., out, logp)
PyObject* policy_sample(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded_outputs([&]() -> PyObject* {
    Row r{0, 0, 0, 0, c10::Device(c10::kCPU), nullptr};
    pgxpolicy_adjust d;
    at::Tensor out, logp;
    void *noise, *stream;
    int64_t pitch;
    if (n != 5 + kAdjustArgs || !take_logits(a[1], &r) || !take_matrix(a[2], r, kFloat, &noise, &pitch) || !take_adjust(a + 3, r, &d)) return nullptr;
    PyObject *given = a[3 + kAdjustArgs], *given_logp = a[4 + kAdjustArgs];
    const c10::DeviceGuard guard(r.device);
    if (!output(given, {r.rows}, kInt, r.device, &out) || !output(given_logp, {r.rows}, kFloat, r.device, &logp) || !current_stream(r.device, &stream)) return nullptr;
    auto* fn = (decltype(&pgxpolicy_sample))pointer(a[0]);
    const int rc = without_gil([&] {
      return fn((int32_t)r.rows, (int32_t)r.actions, r.data, r.type, r.pitch, &d, (const float*)noise, pitch, (int32_t*)data_or_null(out), (float*)data_or_null(logp), stream);
    });
    return outputs(rc, {{given, out}, {given_logp, logp}});
  });
}

// (address, logits, target, weight, entropy, grad_scale, adjust..., grad)
PyObject* policy_loss(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded_outputs([&]() -> PyObject* {
    Row r{0, 0, 0, 0, c10::Device(c10::kCPU), nullptr};
    pgxpolicy_adjust d;
    at::Tensor loss, entropies, grad;
    void *shares = nullptr, *taken = nullptr, *weight, *stream;
    int64_t pitch = 0;
    float bonus, scale;
    if (n != 7 + kAdjustArgs || !take_logits(a[1], &r) || !take_adjust(a + 6, r, &d) || !take_per_row(a[3], r, kFloat, &weight)) return nullptr;
    const at::Tensor* target = tensor(a[2]);
    if (!target || (target->dim() == 1 ? !take_per_row(a[2], r, kInt, &taken) : !take_matrix(a[2], r, kFloat, &shares, &pitch))) return nullptr;
    if (!number(a[4], &bonus) || !number(a[5], &scale)) return nullptr;
    PyObject* given = a[6 + kAdjustArgs];
    const c10::DeviceGuard guard(r.device);
    const auto type = tensor(a[1])->scalar_type();
    if (!output(given, {r.rows, r.actions}, type, r.device, &grad) || !current_stream(r.device, &stream)) return nullptr;
    loss = fresh({r.rows}, kFloat, r.device);
    entropies = fresh({r.rows}, kFloat, r.device);
    auto* fn = (decltype(&pgxpolicy_loss))pointer(a[0]);
    const int rc = without_gil([&] {
      return fn((int32_t)r.rows, (int32_t)r.actions, r.data, r.type, r.pitch, &d, (const float*)shares, pitch, (const int32_t*)taken, (const float*)weight, bonus, scale,
                (float*)data_or_null(loss), (float*)data_or_null(entropies), data_or_null(grad), grad.stride(0), stream);
    });
    return outputs(rc, {{Py_None, loss}, {Py_None, entropies}, {given, grad}});
  });
}

// ---- the paged cache -------------------------------------------------------------------------------------------------------------------
// (address, handle, shape, ...) where shape = (slots, kv_heads, head_dim, type, device index, the handle's stream as torch numbers it)
struct CacheShape {
  int64_t slots, kv_heads, head_dim;
  at::ScalarType type;
  c10::Device device;
  c10::StreamId stream;
};
bool take_shape(PyObject* o, CacheShape* s) {
  if (!PyTuple_CheckExact(o) || PyTuple_GET_SIZE(o) != 6) return false;
  int64_t v[6];
  for (int i = 0; i < 6; ++i) v[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(o, i));
  if (PyErr_Occurred()) return false;
  *s = CacheShape{v[0], v[1], v[2], v[3] == PGXCACHE_F16 ? at::kHalf : at::kBFloat16, c10::Device(c10::kCUDA, (c10::DeviceIndex)v[4]), v[5]};
  return true;
}
// a contiguous tensor of one value per entry, on the cache's device
bool take_entries(PyObject* o, const CacheShape& s, at::ScalarType type, int64_t n, void** out) {
  return take(o, type, n, -1, out) && tensor(o)->device() == s.device;
}
bool take_status(PyObject* o, const CacheShape& s, int64_t n, void** out) {
  *out = nullptr;
  return o == Py_None || take_entries(o, s, kByte, n, out);
}
bool take_list(PyObject* o, const CacheShape& s, int64_t* n, void** out) {
  *n = s.slots;
  *out = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = tensor(o);
  if (!t || t->dim() != 1 || t->size(0) > s.slots) return false;
  *n = t->size(0);
  return take_entries(o, s, kInt, *n, out);
}
// [n][heads][head_dim] of the cache's type, strides in elements
bool take_heads(PyObject* o, const CacheShape& s, int64_t n, int64_t heads, void** out, int64_t* entry, int64_t* head) {
  const at::Tensor* t = tensor(o);
  if (!t || t->scalar_type() != s.type || t->device() != s.device || t->dim() != 3 || t->size(0) != n || t->size(1) != heads || t->size(2) != s.head_dim || t->stride(2) != 1)
    return false;
  *out = t->data_ptr();
  *entry = t->stride(0);
  *head = t->stride(1);
  return true;
}

// (address, handle, shape, slots, counts, status)
PyObject* cache_advance(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded([&] {
    CacheShape s{0, 0, 0, kFloat, c10::Device(c10::kCPU), 0};
    int64_t n, count = 0;
    void *slots, *counts = nullptr, *status;
    if (n_args != 6 || !take_shape(a[2], &s) || !take_list(a[3], s, &n, &slots) || !take_status(a[5], s, n, &status)) return -1000;
    if (PyLong_CheckExact(a[4])) {
      count = PyLong_AsLongLong(a[4]);
      if (PyErr_Occurred() || count < 0 || count > INT32_MAX) return -1000;
    } else if (!take_entries(a[4], s, kInt, n, &counts)) {
      return -1000;
    }
    auto* fn = (decltype(&pgxcache_advance))pointer(a[0]);
    void* h = pointer(a[1]);
    return without_gil([&] { return fn((pgxcache_t)h, (int32_t)n, (const int32_t*)slots, (const int32_t*)counts, (int32_t)count, (uint8_t*)status); });
  });
}

// (address, handle, shape, src, dst, status)
PyObject* cache_fork(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded([&] {
    CacheShape s{0, 0, 0, kFloat, c10::Device(c10::kCPU), 0};
    int64_t n;
    void *src, *dst, *status;
    if (n_args != 6 || a[3] == Py_None || !take_shape(a[2], &s) || !take_list(a[3], s, &n, &src) || !take_entries(a[4], s, kInt, n, &dst) ||
        !take_status(a[5], s, n, &status))
      return -1000;
    auto* fn = (decltype(&pgxcache_fork))pointer(a[0]);
    void* h = pointer(a[1]);
    return without_gil([&] { return fn((pgxcache_t)h, (int32_t)n, (const int32_t*)src, (const int32_t*)dst, (uint8_t*)status); });
  });
}

// (address, handle, shape, slots)
PyObject* cache_free(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded([&] {
    CacheShape s{0, 0, 0, kFloat, c10::Device(c10::kCPU), 0};
    int64_t n;
    void* slots;
    if (n_args != 4 || !take_shape(a[2], &s) || !take_list(a[3], s, &n, &slots)) return -1000;
    auto* fn = (decltype(&pgxcache_free))pointer(a[0]);
    void* h = pointer(a[1]);
    return without_gil([&] { return fn((pgxcache_t)h, (int32_t)n, (const int32_t*)slots); });
  });
}

// keys or values of new tokens: [n][kv_heads][head_dim] or [n][tokens][kv_heads][head_dim]
bool take_tokens(PyObject* o, const CacheShape& s, int64_t n, int64_t* tokens, void** out, int64_t* entry, int64_t* token, int64_t* head) {
  const at::Tensor* t = tensor(o);
  if (!t || (t->dim() != 3 && t->dim() != 4)) return false;
  const bool many = t->dim() == 4;
  if (t->scalar_type() != s.type || t->device() != s.device || t->size(0) != n || t->size(-2) != s.kv_heads || t->size(-1) != s.head_dim || t->stride(-1) != 1) return false;
  *tokens = many ? t->size(1) : 1;
  *out = t->data_ptr();
  *entry = t->stride(0);
  *token = many ? t->stride(1) : 0;
  *head = t->stride(-2);
  return *tokens <= INT32_MAX;
}

// (address, handle, shape, layer, k, v, slots)
PyObject* cache_write(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded([&] {
    CacheShape s{0, 0, 0, kFloat, c10::Device(c10::kCPU), 0};
    int64_t n, tokens, tokens_v, ke, kt, kh, ve, vt, vh;
    void *slots, *k, *v;
    if (n_args != 7 || !take_shape(a[2], &s) || !take_list(a[6], s, &n, &slots) || !take_tokens(a[4], s, n, &tokens, &k, &ke, &kt, &kh) ||
        !take_tokens(a[5], s, n, &tokens_v, &v, &ve, &vt, &vh) || tokens != tokens_v || tensor(a[4])->dim() != tensor(a[5])->dim())
      return -1000;
    const long layer = PyLong_AsLong(a[3]);
    if (PyErr_Occurred() || layer < 0 || layer > INT32_MAX) return -1000;
    auto* fn = (decltype(&pgxcache_write))pointer(a[0]);
    void* h = pointer(a[1]);
    return without_gil([&] { return fn((pgxcache_t)h, (int32_t)layer, (int32_t)n, (const int32_t*)slots, (int32_t)tokens, k, ke, kt, kh, v, ve, vt, vh); });
  });
}

// (address, handle, shape, layer, tokens, slots, first, k, v)
PyObject* cache_read(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded_outputs([&]() -> PyObject* {
    CacheShape s{0, 0, 0, kFloat, c10::Device(c10::kCPU), 0};
    int64_t n, first = 0, got;
    void *slots, *firsts = nullptr, *at[2];
    int64_t entry[2], token[2], head[2];
    at::Tensor out[2];
    if (n_args != 9 || !take_shape(a[2], &s) || !take_list(a[5], s, &n, &slots) || !PyLong_CheckExact(a[4])) return nullptr;
    const int64_t tokens = PyLong_AsLongLong(a[4]);
    const long layer = PyLong_AsLong(a[3]);
    if (PyErr_Occurred() || layer < 0 || layer > INT32_MAX || tokens < 0 || tokens > INT32_MAX) return nullptr;
    if (PyLong_CheckExact(a[6])) {
      first = PyLong_AsLongLong(a[6]);
      if (PyErr_Occurred() || first < 0 || first > INT32_MAX) return nullptr;
    } else if (!take_entries(a[6], s, kInt, n, &firsts)) {
      return nullptr;
    }
    const c10::StreamGuard guard(c10::Stream(c10::Stream::UNSAFE, s.device, s.stream));   // new outputs belong to the stream that writes them
    for (int i = 0; i < 2; ++i) {
      if (a[7 + i] == Py_None) {
        out[i] = fresh({n, tokens, s.kv_heads, s.head_dim}, s.type, s.device);
        at[i] = data_or_null(out[i]);
        entry[i] = out[i].stride(0); token[i] = out[i].stride(1); head[i] = out[i].stride(2);
      } else {
        if (!tensor(a[7 + i]) || tensor(a[7 + i])->dim() != 4 || !take_tokens(a[7 + i], s, n, &got, &at[i], &entry[i], &token[i], &head[i]) || got != tokens) return nullptr;
        out[i] = *tensor(a[7 + i]);
      }
    }
    auto* fn = (decltype(&pgxcache_read))pointer(a[0]);
    void* h = pointer(a[1]);
    const int rc = without_gil([&] {
      return fn((pgxcache_t)h, (int32_t)layer, (int32_t)n, (const int32_t*)slots, (const int32_t*)firsts, (int32_t)first, (int32_t)tokens, at[0], entry[0], token[0], head[0], at[1],
                entry[1], token[1], head[1]);
    });
    return outputs(rc, {{a[7], out[0]}, {a[8], out[1]}});
  });
}

// (address, handle, shape, layer, q, slots, k, v, scale, out, lse)
PyObject* cache_attend(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded_outputs([&]() -> PyObject* {
    CacheShape s{0, 0, 0, kFloat, c10::Device(c10::kCPU), 0};
    int64_t n, qe, qh, ke = 0, kh = 0, ve = 0, vh = 0;
    void *slots, *q, *k = nullptr, *v = nullptr, *lse_data = nullptr;
    float scale;
    at::Tensor out, lse;
    if (n_args != 11 || !take_shape(a[2], &s) || !take_list(a[5], s, &n, &slots) || n == 0) return nullptr;
    const at::Tensor* qt = tensor(a[4]);
    if (!qt || qt->dim() != 3 || qt->size(1) < 1 || qt->size(1) % s.kv_heads != 0 || !take_heads(a[4], s, n, qt->size(1), &q, &qe, &qh)) return nullptr;
    const int64_t heads = qt->size(1);
    if ((a[6] == Py_None) != (a[7] == Py_None)) return nullptr;
    if (a[6] != Py_None && (!take_heads(a[6], s, n, s.kv_heads, &k, &ke, &kh) || !take_heads(a[7], s, n, s.kv_heads, &v, &ve, &vh))) return nullptr;
    if (!number(a[8], &scale)) return nullptr;
    const long layer = PyLong_AsLong(a[3]);
    if (PyErr_Occurred() || layer < 0 || layer > INT32_MAX) return nullptr;
    const c10::StreamGuard guard(c10::Stream(c10::Stream::UNSAFE, s.device, s.stream));   // new outputs belong to the stream that writes them
    if (!output(a[9], {n, heads, s.head_dim}, s.type, s.device, &out)) return nullptr;
    PyObject* given_lse = a[10] == Py_True ? Py_None : a[10];
    if (a[10] != Py_False) {
      if (!output(given_lse, {n, heads}, kFloat, s.device, &lse) || !lse.is_contiguous()) return nullptr;
      lse_data = lse.data_ptr();
    }
    auto* fn = (decltype(&pgxcache_attend))pointer(a[0]);
    void* h = pointer(a[1]);
    const int rc = without_gil([&] {
      return fn((pgxcache_t)h, (int32_t)layer, (int32_t)n, (const int32_t*)slots, (int32_t)heads, q, qe, qh, k, ke, kh, v, ve, vh, scale, out.data_ptr(), out.stride(0), out.stride(1),
                (float*)lse_data);
    });
    if (lse_data) return outputs(rc, {{a[9], out}, {given_lse, lse}});
    return outputs(rc, {{a[9], out}});
  });
}

// ---- rotary positions ------------------------------------------------------------------------------------------------------------------
// a tensor, or a tuple or list of one or two; the number of them, 0: neither
int take_tensors(PyObject* o, PyObject** items) {
  if (PyTuple_CheckExact(o) || PyList_CheckExact(o)) {
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(o);
    if (n < 1 || n > PGXROTARY_MAX_PARTS) return 0;
    for (Py_ssize_t k = 0; k < n; ++k)
      if (!tensor(items[k] = PySequence_Fast_GET_ITEM(o, k))) return 0;
    return (int)n;
  }
  items[0] = o;
  return tensor(o) ? 1 : 0;
}
// (address, x, positions, frequencies, interleaved, magnitude, inverse, out); returns the outputs as a tuple
PyObject* rotate(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded_outputs([&]() -> PyObject* {
    PyObject *xs[PGXROTARY_MAX_PARTS], *given[PGXROTARY_MAX_PARTS] = {Py_None, Py_None};
    at::Tensor outs[PGXROTARY_MAX_PARTS];
    pgxrotary_part parts[PGXROTARY_MAX_PARTS];
    void* stream;
    float magnitude;
    const int n = n_args == 8 ? take_tensors(a[1], xs) : 0;
    if (n == 0) return nullptr;
    const at::Tensor &first = *tensor(xs[0]), *p = tensor(a[2]), *f = tensor(a[3]);
    const auto type = first.scalar_type();
    const int64_t dim = first.dim();
    if (!first.is_cuda() || (dim != 3 && dim != 4) || (type != at::kFloat && type != at::kHalf && type != at::kBFloat16) || first.numel() == 0) return nullptr;
    const int64_t D = first.size(-1), entries = first.size(0), tokens = dim == 4 ? first.size(1) : 1;
    if (entries * tokens > INT32_MAX || D > PGXROTARY_MAX_HEAD_DIM) return nullptr;
    if (!p || p->scalar_type() != kInt || p->device() != first.device() || p->dim() != dim - 2 || p->size(0) != entries || (dim == 4 && p->size(1) != tokens)) return nullptr;
    if (!f || f->scalar_type() != at::kDouble || f->device() != first.device() || f->dim() != 1 || !f->is_contiguous() || f->size(0) < 1 || 2 * f->size(0) > D) return nullptr;
    if (!number(a[5], &magnitude) || !std::isfinite(magnitude)) return nullptr;
    const int interleaved = PyObject_IsTrue(a[4]), inverse = PyObject_IsTrue(a[6]);
    if (interleaved < 0 || inverse < 0) return nullptr;
    if (a[7] != Py_None && take_tensors(a[7], given) != n) return nullptr;
    const c10::DeviceGuard guard(first.device());
    for (int k = 0; k < n; ++k) {
      const at::Tensor& x = *tensor(xs[k]);
      if (x.scalar_type() != type || x.device() != first.device() || x.dim() != dim || x.size(0) != entries || (dim == 4 && x.size(1) != tokens) || x.size(-1) != D ||
          x.size(-2) > 65536 || !dense_rows(x) || !output(given[k], x.sizes(), type, first.device(), &outs[k]))
        return nullptr;
      const at::Tensor& o = outs[k];
      if (c10::GradMode::is_enabled() && (x.requires_grad() || o.requires_grad())) return nullptr;
      parts[k] = pgxrotary_part{data_or_null(x), x.stride(0), dim == 4 ? x.stride(1) : 0, x.stride(-2), data_or_null(o), o.stride(0), dim == 4 ? o.stride(1) : 0, o.stride(-2),
                                (int32_t)x.size(-2)};
    }
    if (!current_stream(first.device(), &stream)) return nullptr;
    auto* fn = (decltype(&pgxrotary_turn))pointer(a[0]);
    const int rc = without_gil([&] {
      return fn((int32_t)entries, (int32_t)tokens, (int32_t)D, (int32_t)(2 * f->size(0)), type == at::kFloat ? PGXROTARY_F32 : type == at::kHalf ? PGXROTARY_F16 : PGXROTARY_BF16,
                (const int32_t*)p->data_ptr(), p->stride(0), dim == 4 ? p->stride(1) : 0, (const double*)f->data_ptr(), magnitude, interleaved, inverse, n, parts, stream);
    });
    for (int k = 0; k < n && rc == 0; ++k)   // what autograd has kept of a given output is no longer what it was
      if (given[k] != Py_None && !outs[k].is_inference()) outs[k].unsafeGetTensorImpl()->bump_version();
    if (n == 1) return outputs(rc, {{given[0], outs[0]}});
    return outputs(rc, {{given[0], outs[0]}, {given[1], outs[1]}});
  });
}

PyMethodDef kMethods[] = {
    {"step", (PyCFunction)(void*)step, METH_FASTCALL, nullptr},
    {"step_sample", (PyCFunction)(void*)step_sample, METH_FASTCALL, nullptr},
    {"random_actions", (PyCFunction)(void*)random_actions, METH_FASTCALL, nullptr},
    {"step_slots", (PyCFunction)(void*)step_slots, METH_FASTCALL, nullptr},
    {"set_raw_stream", set_raw_stream, METH_O, nullptr},
    {"policy_logits", (PyCFunction)(void*)policy_logits, METH_FASTCALL, nullptr},
    {"policy_sample", (PyCFunction)(void*)policy_sample, METH_FASTCALL, nullptr},
    {"policy_loss", (PyCFunction)(void*)policy_loss, METH_FASTCALL, nullptr},
    {"cache_advance", (PyCFunction)(void*)cache_advance, METH_FASTCALL, nullptr},
    {"cache_fork", (PyCFunction)(void*)cache_fork, METH_FASTCALL, nullptr},
    {"cache_free", (PyCFunction)(void*)cache_free, METH_FASTCALL, nullptr},
    {"cache_write", (PyCFunction)(void*)cache_write, METH_FASTCALL, nullptr},
    {"cache_read", (PyCFunction)(void*)cache_read, METH_FASTCALL, nullptr},
    {"cache_attend", (PyCFunction)(void*)cache_attend, METH_FASTCALL, nullptr},
    {"rotate", (PyCFunction)(void*)rotate, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject* PyInit__fastcall() { return PyModule_Create(&kModule); }
