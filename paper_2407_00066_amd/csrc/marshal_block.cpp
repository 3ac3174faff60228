// The binding of cts_block.h's calls (host code, torch's C++ API): a decode
// step's calls take the GPU a few microseconds each, less than checking their
// tensors attribute by attribute in Python.  A function here takes the C entry point's
// address, torch's current stream and the Python call's arguments, checks the
// tensors, allocates what the caller did not give, and makes the call.  It returns
// the outputs with the call's status, or None if an argument is not as it has to
// be: the Python side then finds out what is wrong and says so.  An allocation that
// fails raises torch's own error for it.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/Device.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <exception>
#include <optional>

#include "cts_block.h"

namespace {

// What an argument that is not as it has to be ends a call with.
struct Refused {};
void need(bool ok) {
  if (!ok) throw Refused{};
}

// What an allocation that failed ends a call with.
struct Failed { std::exception_ptr why; };
at::Tensor allocate(at::IntArrayRef shape, c10::ScalarType dt, c10::Device dev) {
  try {
    return at::empty(shape, at::TensorOptions().dtype(dt).device(dev));
  } catch (...) {
    throw Failed{std::current_exception()};
  }
}
PyObject* raise(const Failed& f) {
  HANDLE_TH_ERRORS
  std::rethrow_exception(f.why);
  END_HANDLE_TH_ERRORS
}

const at::Tensor& tensor(PyObject* o) {
  need(THPVariable_Check(o));
  const at::Tensor& t = THPVariable_Unpack(o);
  need(t.layout() == c10::kStrided);
  return t;
}

long long integer(PyObject* o) {
  PyObject* i = PyNumber_Index(o);
  need(i != nullptr);
  const long long v = PyLong_AsLongLong(i);
  Py_DECREF(i);
  need(!(v == -1 && PyErr_Occurred()));
  return v;
}
int32_t int32(PyObject* o) {
  const long long v = integer(o);
  need(v >= INT32_MIN && v <= INT32_MAX);
  return static_cast<int32_t>(v);
}
int32_t int32(int64_t v) {
  need(v >= INT32_MIN && v <= INT32_MAX);
  return static_cast<int32_t>(v);
}
double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  need(!(v == -1.0 && PyErr_Occurred()));
  return v;
}
template <typename F> F entry(PyObject* o) { return reinterpret_cast<F>(static_cast<uintptr_t>(integer(o))); }
void* stream(PyObject* o) { return reinterpret_cast<void*>(static_cast<uintptr_t>(integer(o))); }

int dtype_code(c10::ScalarType t) {
  need(t == at::kFloat || t == at::kBFloat16);
  return t == at::kFloat ? CTS_F32 : CTS_BF16;
}

void* data(const at::Tensor& t) { return t.numel() ? t.data_ptr() : nullptr; }

// A contiguous array of this shape.
void* dense(const at::Tensor& t, c10::Device dev, c10::ScalarType dt, at::IntArrayRef shape) {
  need(t.device() == dev && t.scalar_type() == dt && t.sizes() == shape && t.is_contiguous());
  return data(t);
}

// An array of this shape whose rows (the first dimension) are contiguous each.
struct Rows { void* p; int64_t ld; };
Rows rows(const at::Tensor& t, c10::Device dev, c10::ScalarType dt, at::IntArrayRef shape) {
  need(t.device() == dev && t.scalar_type() == dt && t.sizes() == shape);
  int64_t width = 1;
  for (int64_t i = t.dim() - 1; i > 0; --i) {
    need(t.size(i) == 1 || t.stride(i) == width);
    width *= t.size(i);
  }
  return {data(t), t.size(0) > 1 ? t.stride(0) : width};       // (a single row's stride is arbitrary)
}

at::Tensor fresh(PyObject* given, at::IntArrayRef shape, c10::ScalarType dt, c10::Device dev) {
  return given != Py_None ? tensor(given) : allocate(shape, dt, dev);
}

c10::Device device_of(PyObject* o) {
  need(THPDevice_Check(o));
  const c10::Device d = reinterpret_cast<THPDevice*>(o)->device;
  need(d.type() == c10::DeviceType::CUDA);
  return d;
}

const cts_kv_cache& cache_of(PyObject* o) {
  return *reinterpret_cast<const cts_kv_cache*>(static_cast<uintptr_t>(integer(o)));
}

// The sections of a rotary call (host numbers, one for each axis), into sec; null for None.
const int32_t* sections_of(PyObject* given, int64_t axes, int32_t* sec) {
  if (given == Py_None) return nullptr;
  PyObject* list = PySequence_Fast(given, "sections");
  need(list != nullptr);
  const bool fits = PySequence_Fast_GET_SIZE(list) == axes && axes <= 16;
  bool ok = fits;
  for (int64_t i = 0; ok && i < axes; ++i) {
    const long long v = PyLong_AsLongLong(PySequence_Fast_GET_ITEM(list, i));
    ok = !(v == -1 && PyErr_Occurred()) && v >= INT32_MIN && v <= INT32_MAX;
    sec[i] = static_cast<int32_t>(v);
  }
  Py_DECREF(list);
  need(ok);
  return sec;
}

PyObject* wrap(const at::Tensor& t) { return THPVariable_Wrap(t); }

// Runs f; None for a refusal, and for tensors whose sizes or storage cannot be had (they
// only stand for others, or raise errors of their own, which come again with Python's checks).
template <typename F> PyObject* call(Py_ssize_t n, Py_ssize_t want, F f) {
  if (n != want) {
    PyErr_Format(PyExc_TypeError, "%zd arguments, expected %zd", n, want);
    return nullptr;
  }
  try {
    return f();
  } catch (const Refused&) {
  } catch (const Failed& f) {
    return raise(f);
  } catch (const std::exception&) {
  }
  PyErr_Clear();
  Py_RETURN_NONE;
}

}  // namespace

// kv_write(entry, stream, device, cache, k, v, slots) -> status
PyObject* cts_marshal_kv_write(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 7, [&]() -> PyObject* {
    const c10::Device dev = device_of(a[2]);
    const cts_kv_cache& c = cache_of(a[3]);
    const at::Tensor &k = tensor(a[4]), &v = tensor(a[5]), &slots = tensor(a[6]);
    const c10::ScalarType dt = k.scalar_type();
    const int code = dtype_code(dt);
    need(k.dim() == 3);
    const int64_t T = k.size(0);
    const int64_t shape[3] = {T, c.n_heads, c.head_dim};
    const Rows kr = rows(k, dev, dt, shape), vr = rows(v, dev, dt, shape);
    const void* s = dense(slots, dev, at::kLong, {T});
    return PyLong_FromLong(entry<decltype(&cts_kv_write)>(a[0])(&c, int32(T), kr.p, kr.ld, vr.p, vr.ld,
                                                                static_cast<const int64_t*>(s), code, stream(a[1])));
  });
}

// kv_read(entry, stream, device, cache, slots, dtype, k_out, v_out) -> (k, v, status)
PyObject* cts_marshal_kv_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 8, [&]() -> PyObject* {
    const c10::Device dev = device_of(a[2]);
    const cts_kv_cache& c = cache_of(a[3]);
    const at::Tensor& slots = tensor(a[4]);
    need(THPDtype_Check(a[5]));
    c10::ScalarType dt = reinterpret_cast<THPDtype*>(a[5])->scalar_type;
    if (a[6] != Py_None) dt = tensor(a[6]).scalar_type();
    const int code = dtype_code(dt);
    const int64_t T = slots.numel();
    const int64_t shape[3] = {T, c.n_heads, c.head_dim};
    const void* s = dense(slots, dev, at::kLong, {T});
    const at::Tensor k = fresh(a[6], shape, dt, dev), v = fresh(a[7], shape, dt, dev);
    const Rows kr = rows(k, dev, dt, shape), vr = rows(v, dev, dt, shape);
    const int st = entry<decltype(&cts_kv_read)>(a[0])(&c, int32(T), static_cast<const int64_t*>(s), kr.p, kr.ld, vr.p,
                                                       vr.ld, code, stream(a[1]));
    return Py_BuildValue("(NNi)", wrap(k), wrap(v), st);
  });
}

// kv_attention(entry, size entry, stream, device, cache, q, block_table, kv_len, q_start, max_q, max_kv, scale, window,
//              out, workspace) -> (out, status)
PyObject* cts_marshal_kv_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 15, [&]() -> PyObject* {
    const c10::Device dev = device_of(a[3]);
    const cts_kv_cache& c = cache_of(a[4]);
    const at::Tensor &q = tensor(a[5]), &table = tensor(a[6]), &len = tensor(a[7]);
    const c10::ScalarType dt = q.scalar_type();
    need(q.dim() == 3 && table.dim() == 2);
    const int64_t T = q.size(0), heads = q.size(1), B = table.size(0), cols = table.size(1);
    const int64_t shape[3] = {T, heads, c.head_dim};
    const Rows qr = rows(q, dev, dt, shape);
    cts_attn_problem p{};
    p.T = int32(T); p.B = int32(B); p.n_q_heads = int32(heads); p.max_pages = int32(cols);
    p.dtype = dtype_code(dt);
    // (all rows may be one sequence's)
    p.max_q = a[9] != Py_None ? int32(a[9]) : a[8] == Py_None ? 1 : int32(std::max<int64_t>(T, 1));
    p.max_kv = a[10] == Py_None ? int32(cols * c.page_size) : int32(a[10]);
    p.scale = static_cast<float>(number(a[11]));
    p.window = int32(a[12]);
    const void* tp = dense(table, dev, at::kInt, {B, cols});
    const void* lp = dense(len, dev, at::kInt, {B});
    const void* sp = a[8] == Py_None ? nullptr : dense(tensor(a[8]), dev, at::kInt, {B + 1});
    const at::Tensor out = fresh(a[13], shape, dt, dev);
    const Rows orr = rows(out, dev, dt, shape);
    at::Tensor ws;
    if (a[14] != Py_None) {
      ws = tensor(a[14]);
      need(ws.device() == dev && ws.scalar_type() == at::kByte && ws.is_contiguous());
    } else {
      const int64_t bytes = entry<decltype(&cts_kv_attention_workspace_size)>(a[1])(&p, &c);
      ws = allocate({bytes > 0 ? bytes : 1}, at::kByte, dev);
    }
    const int st = entry<decltype(&cts_kv_attention)>(a[0])(
        &p, &c, qr.p, qr.ld, static_cast<const int32_t*>(tp), static_cast<const int32_t*>(lp),
        static_cast<const int32_t*>(sp), orr.p, orr.ld, data(ws), static_cast<size_t>(ws.numel()), stream(a[2]));
    return Py_BuildValue("(Ni)", wrap(out), st);
  });
}

// block_norm(entry, stream, device, x, weight, y, post_weight, gate, scale, eps, h_out, n_out) -> (h, n, status)
PyObject* cts_marshal_block_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 12, [&]() -> PyObject* {
    const c10::Device dev = device_of(a[2]);
    const at::Tensor& x = tensor(a[3]);
    const c10::ScalarType dt = x.scalar_type();
    const int code = dtype_code(dt);
    need(x.dim() == 2);
    const int64_t T = x.size(0), d = x.size(1);
    const int64_t shape[2] = {T, d};
    const Rows xr = rows(x, dev, dt, shape);
    const void* wp = dense(tensor(a[4]), dev, dt, {d});
    Rows yr{}, gr{}, hr{};
    const void* pp = nullptr;
    std::optional<at::Tensor> h;
    if (a[5] != Py_None) {
      yr = rows(tensor(a[5]), dev, dt, shape);
      if (a[6] != Py_None) pp = dense(tensor(a[6]), dev, dt, {d});
      if (a[7] != Py_None) {
        const at::Tensor& g = tensor(a[7]);
        if (g.dim() == 1) gr = {dense(g, dev, dt, {d}), 0};
        else gr = rows(g, dev, dt, shape);
      }
      h = fresh(a[10], shape, dt, dev);
      hr = rows(*h, dev, dt, shape);
    } else {
      need(a[6] == Py_None && a[7] == Py_None && a[10] == Py_None);
    }
    const at::Tensor out = fresh(a[11], shape, dt, dev);
    const Rows nr = rows(out, dev, dt, shape);
    const int st = entry<decltype(&cts_block_norm)>(a[0])(
        int32(T), int32(d), code, xr.p, xr.ld, yr.p, yr.ld, pp, gr.p, gr.ld, static_cast<float>(number(a[8])),
        static_cast<float>(number(a[9])), wp, hr.p, hr.ld, nr.p, nr.ld, stream(a[1]));
    return Py_BuildValue("(NNi)", wrap(h ? *h : x), wrap(out), st);
  });
}

// rotary(entry, stream, device, q, k, cos, sin, positions, sections, interleaved, q_out, k_out) -> (q', k', status)
PyObject* cts_marshal_rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 12, [&]() -> PyObject* {
    const c10::Device dev = device_of(a[2]);
    const at::Tensor &some = tensor(a[3] != Py_None ? a[3] : a[4]), &cos = tensor(a[5]), &pos = tensor(a[7]);
    const c10::ScalarType dt = some.scalar_type();
    const int code = dtype_code(dt);
    need(some.dim() == 3 && cos.dim() == 2 && (pos.dim() == 1 || pos.dim() == 2));
    const int64_t T = some.size(0), d = some.size(2), n_pos = cos.size(0), half = cos.size(1);
    const int64_t axes = pos.dim() == 1 ? 1 : pos.size(0);
    Rows in[2] = {}, out[2] = {};
    int64_t heads[2] = {0, 0};
    std::optional<at::Tensor> o[2];
    for (int i = 0; i < 2; ++i) {
      if (a[3 + i] == Py_None) {
        need(a[10 + i] == Py_None);
        continue;
      }
      const at::Tensor& t = tensor(a[3 + i]);
      need(t.dim() == 3);
      heads[i] = t.size(1);
      const int64_t shape[3] = {T, heads[i], d};
      in[i] = rows(t, dev, dt, shape);
      o[i] = fresh(a[10 + i], shape, dt, dev);
      out[i] = rows(*o[i], dev, dt, shape);
    }
    int32_t sec[16];
    const int32_t* const sections = sections_of(a[8], axes, sec);
    const void* cp = dense(cos, dev, at::kFloat, {n_pos, half});
    const void* sp = dense(tensor(a[6]), dev, at::kFloat, {n_pos, half});
    const void* pp = pos.dim() == 1 ? dense(pos, dev, at::kInt, {T}) : dense(pos, dev, at::kInt, {axes, T});
    const int inter = PyObject_IsTrue(a[9]);
    need(inter >= 0);
    const int st = entry<decltype(&cts_rotary)>(a[0])(
        int32(T), int32(heads[0]), int32(heads[1]), int32(d), int32(2 * half), code, in[0].p, in[0].ld, in[1].p, in[1].ld,
        static_cast<const float*>(cp), static_cast<const float*>(sp), int32(n_pos), static_cast<const int32_t*>(pp),
        int32(axes), sections, inter, out[0].p, out[0].ld, out[1].p, out[1].ld, stream(a[1]));
    PyObject* r[2];
    for (int i = 0; i < 2; ++i) {
      if (o[i]) r[i] = wrap(*o[i]);
      else { Py_INCREF(Py_None); r[i] = Py_None; }
    }
    return Py_BuildValue("(NNi)", r[0], r[1], st);
  });
}

// kv_append(entry, stream, device, cache, q, k, v, slots, cos, sin, positions, sections, interleaved, q_out, k_out)
//   -> (q', status)
PyObject* cts_marshal_kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 15, [&]() -> PyObject* {
    const c10::Device dev = device_of(a[2]);
    const cts_kv_cache& c = cache_of(a[3]);
    const at::Tensor &k = tensor(a[5]), &v = tensor(a[6]), &slots = tensor(a[7]), &cos = tensor(a[8]), &pos = tensor(a[10]);
    const c10::ScalarType dt = k.scalar_type();
    const int code = dtype_code(dt);
    need(k.dim() == 3 && cos.dim() == 2 && (pos.dim() == 1 || pos.dim() == 2));
    const int64_t T = k.size(0), n_pos = cos.size(0), half = cos.size(1), axes = pos.dim() == 1 ? 1 : pos.size(0);
    const int64_t shape[3] = {T, c.n_heads, c.head_dim};
    const Rows kr = rows(k, dev, dt, shape), vr = rows(v, dev, dt, shape);
    const void* s = dense(slots, dev, at::kLong, {T});
    Rows qr{}, qo{}, ko{};
    int64_t heads = 0;
    std::optional<at::Tensor> out;
    if (a[4] != Py_None) {
      const at::Tensor& q = tensor(a[4]);
      need(q.dim() == 3);
      heads = q.size(1);
      const int64_t q_shape[3] = {T, heads, c.head_dim};
      qr = rows(q, dev, dt, q_shape);
      out = fresh(a[13], q_shape, dt, dev);
      qo = rows(*out, dev, dt, q_shape);
    } else {
      need(a[13] == Py_None);
    }
    if (a[14] != Py_None) ko = rows(tensor(a[14]), dev, dt, shape);
    const void* cp = dense(cos, dev, at::kFloat, {n_pos, half});
    const void* sp = dense(tensor(a[9]), dev, at::kFloat, {n_pos, half});
    const void* pp = pos.dim() == 1 ? dense(pos, dev, at::kInt, {T}) : dense(pos, dev, at::kInt, {axes, T});
    int32_t sec[16];
    const int32_t* const sections = sections_of(a[11], axes, sec);
    const int inter = PyObject_IsTrue(a[12]);
    need(inter >= 0);
    const int st = entry<decltype(&cts_kv_append)>(a[0])(
        &c, int32(T), int32(heads), int32(2 * half), code, qr.p, qr.ld, kr.p, kr.ld, vr.p, vr.ld,
        static_cast<const int64_t*>(s), static_cast<const float*>(cp), static_cast<const float*>(sp), int32(n_pos),
        static_cast<const int32_t*>(pp), int32(axes), sections, inter, qo.p, qo.ld, ko.p, ko.ld, stream(a[1]));
    if (out) return Py_BuildValue("(Ni)", wrap(*out), st);
    return Py_BuildValue("(Oi)", Py_None, st);
  });
}

// kv_tree_attention(entry, size entry, stream, device, cache, q, block_table, kv_len, mask, q_start, max_q, max_kv, scale,
//                   window, positions, out, workspace) -> (out, status)
PyObject* cts_marshal_kv_tree_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 17, [&]() -> PyObject* {
    const c10::Device dev = device_of(a[3]);
    const cts_kv_cache& c = cache_of(a[4]);
    const at::Tensor &q = tensor(a[5]), &table = tensor(a[6]), &len = tensor(a[7]), &mask = tensor(a[8]);
    const c10::ScalarType dt = q.scalar_type();
    need(q.dim() == 3 && table.dim() == 2 && mask.dim() == 2);
    const int64_t T = q.size(0), heads = q.size(1), B = table.size(0), cols = table.size(1), words = mask.size(1);
    const int64_t shape[3] = {T, heads, c.head_dim};
    const Rows qr = rows(q, dev, dt, shape);
    cts_attn_problem p{};
    p.T = int32(T); p.B = int32(B); p.n_q_heads = int32(heads); p.max_pages = int32(cols);
    p.dtype = dtype_code(dt);
    // (all rows may be one sequence's: drafts past the mask's bits would be left out)
    need(a[10] != Py_None || a[9] == Py_None || T <= std::min<int64_t>(32 * words, 512));
    p.max_q = a[10] != Py_None ? int32(a[10]) : a[9] == Py_None ? 1 : int32(std::max<int64_t>(T, 1));
    p.max_kv = a[11] == Py_None ? int32(cols * c.page_size) : int32(a[11]);
    p.scale = static_cast<float>(number(a[12]));
    p.window = int32(a[13]);
    const void* tp = dense(table, dev, at::kInt, {B, cols});
    const void* lp = dense(len, dev, at::kInt, {B});
    const void* mp = dense(mask, dev, at::kInt, {T, words});
    const void* sp = a[9] == Py_None ? nullptr : dense(tensor(a[9]), dev, at::kInt, {B + 1});
    const void* pp = a[14] == Py_None ? nullptr : dense(tensor(a[14]), dev, at::kInt, {T});
    const at::Tensor out = fresh(a[15], shape, dt, dev);
    const Rows orr = rows(out, dev, dt, shape);
    at::Tensor ws;
    if (a[16] != Py_None) {
      ws = tensor(a[16]);
      need(ws.device() == dev && ws.scalar_type() == at::kByte && ws.is_contiguous());
    } else {
      const int64_t bytes = entry<decltype(&cts_kv_tree_attention_workspace_size)>(a[1])(&p, &c);
      ws = allocate({bytes > 0 ? bytes : 1}, at::kByte, dev);
    }
    const int st = entry<decltype(&cts_kv_tree_attention)>(a[0])(
        &p, &c, qr.p, qr.ld, static_cast<const int32_t*>(tp), static_cast<const int32_t*>(lp),
        static_cast<const int32_t*>(sp), static_cast<const uint32_t*>(mp), words, static_cast<const int32_t*>(pp), orr.p,
        orr.ld, data(ws), static_cast<size_t>(ws.numel()), stream(a[2]));
    return Py_BuildValue("(Ni)", wrap(out), st);
  });
}

// kv_keep(entry, stream, device, cache, block_table, kv_len, q_start, path, n_path) -> status
PyObject* cts_marshal_kv_keep(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 9, [&]() -> PyObject* {
    const c10::Device dev = device_of(a[2]);
    const cts_kv_cache& c = cache_of(a[3]);
    const at::Tensor &table = tensor(a[4]), &path = tensor(a[7]);
    need(table.dim() == 2 && path.dim() == 2);
    const int64_t B = table.size(0), cols = table.size(1), most = path.size(1);
    const void* tp = dense(table, dev, at::kInt, {B, cols});
    const void* lp = dense(tensor(a[5]), dev, at::kInt, {B});
    const void* sp = dense(tensor(a[6]), dev, at::kInt, {B + 1});
    const void* pp = dense(path, dev, at::kInt, {B, most});
    const void* np = dense(tensor(a[8]), dev, at::kInt, {B});
    return PyLong_FromLong(entry<decltype(&cts_kv_keep)>(a[0])(
        &c, int32(B), int32(cols), static_cast<const int32_t*>(tp), static_cast<const int32_t*>(lp),
        static_cast<const int32_t*>(sp), int32(most), static_cast<const int32_t*>(pp), static_cast<const int32_t*>(np),
        stream(a[1])));
  });
}
