// The decoder operators' calls from Python, for decoder.py: argument checks, result tensors and the C call in one step.  A step of a small batch is bound by what its calls cost on the
// host: through ctypes and tensor methods 5 to 8 us each beyond the launch, here 1 (0.1 to 0.3 of it for the device's guard and the question whether a graph is being captured).  Marshalling only, as binding.py; PyTorch supplies memory and streams.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <hip/hip_runtime_api.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <string>

#include "rnswino.h"

namespace {

struct Refused {};  // a Python error is set

PyObject *g_check = nullptr;  // binding._check(code, name)

[[noreturn]] void refuse(const std::string &what) {
  PyErr_SetString(PyExc_ValueError, what.c_str());
  throw Refused();
}

std::string shape_of(at::IntArrayRef s) {
  std::string out = "(";
  for (int64_t v : s) out += std::to_string(v) + ", ";
  return out + ")";
}

const at::Tensor &tensor(PyObject *o, const char *name) {
  if (!THPVariable_Check(o)) refuse(std::string(name) + " must be a tensor");
  return THPVariable_Unpack(o);
}

// A contiguous tensor of this type and shape on the GPU `device`.
void expect(const at::Tensor &t, const char *name, at::ScalarType type, std::initializer_list<int64_t> shape, c10::Device device) {
  const at::IntArrayRef want(shape.begin(), shape.size());
  if (t.scalar_type() == type && t.sizes() == want && t.is_contiguous() && t.device() == device && t.is_cuda()) return;
  refuse(std::string(name) + " must be a contiguous " + c10::toString(type) + " tensor of shape " + shape_of(want) + " on " + device.str() + ", not " + c10::toString(t.scalar_type()) + " " +
         shape_of(t.sizes()) + " with strides " + shape_of(t.strides()) + " on " + t.device().str());
}

const at::Tensor &indices(PyObject *o, const char *name, at::ScalarType type, std::initializer_list<int64_t> shape, c10::Device device) {
  const at::Tensor &t = tensor(o, name);
  expect(t, name, type, shape, device);
  return t;
}

int64_t integer(PyObject *o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused();
  return v;
}
template <typename T>
T *address(PyObject *o) { return reinterpret_cast<T *>(static_cast<intptr_t>(integer(o))); }

// A cache by one of its tensors, which says where it lies.
void expect_cache(PyObject *held, c10::Device device) {
  const at::Tensor &t = tensor(held, "cache");
  if (t.device() != device) refuse("the cache must be on " + device.str() + ", not " + t.device().str());
}

int type_of(const at::Tensor &t, const char *name) {
  if (t.scalar_type() == at::kBFloat16) return RNSWINO_TYPE_BF16;
  if (t.scalar_type() == at::kHalf) return RNSWINO_TYPE_F16;
  refuse(std::string(name) + " must be bfloat16 or float16, not " + c10::toString(t.scalar_type()));
}

// Rows [n][width], contiguous within a row, on a GPU; the stride to the next (a single row has none that matters).
int64_t rows(const at::Tensor &t, const char *name, int64_t width, int64_t &stride) {
  if (t.dim() != 2 || t.size(1) != width || (width > 1 && t.stride(1) != 1) || !t.is_cuda())
    refuse(std::string(name) + " must be rows of " + std::to_string(width) + " contiguous elements on the GPU, not " + shape_of(t.sizes()) + " with strides " + shape_of(t.strides()) + " on " +
           t.device().str());
  stride = t.size(0) > 1 ? t.stride(0) : (width + 7) / 8 * 8;
  return t.size(0);
}
// The same for [n][heads][dim] with contiguous heads and dimensions.
int64_t head_rows(const at::Tensor &t, const char *name, int64_t heads, int64_t dim, int64_t &stride) {
  if (t.dim() != 3 || t.size(1) != heads || t.size(2) != dim || t.stride(2) != 1 || (heads > 1 && t.stride(1) != dim) || !t.is_cuda())
    refuse(std::string(name) + " must be [n][" + std::to_string(heads) + "][" + std::to_string(dim) + "] with contiguous heads on the GPU, not " + shape_of(t.sizes()) + " with strides " +
           shape_of(t.strides()) + " on " + t.device().str());
  stride = t.size(0) > 1 ? t.stride(0) : heads * dim;
  return t.size(0);
}

// (The library launches on the current device, and the handle of a device's default stream names no device: calls are made under a DeviceGuard of their tensors'.)
void *stream_of(const at::Tensor &t) { return c10::hip::getCurrentHIPStream(t.device().index()).stream(); }

// (at::empty finds its way here through the dispatcher, 0.3 us each time: rows into the cache and back, three results, 8.8 -> 8.0 us)
at::Tensor make(at::IntArrayRef shape, at::ScalarType type, c10::Device device) { return at::detail::empty_cuda(shape, type, device, std::nullopt); }

void succeeded(int code, const char *name) {
  if (!code) return;
  PyObject *r = PyObject_CallFunction(g_check, "is", code, name);  // raises
  Py_XDECREF(r);
  throw Refused();
}

PyObject *pair(at::Tensor a, PyObject *b) {  // takes b's reference
  PyObject *first = THPVariable_Wrap(std::move(a));
  PyObject *both = first && b ? PyTuple_Pack(2, first, b) : nullptr;
  Py_XDECREF(first);
  Py_XDECREF(b);
  return both;
}

// Whether what is enqueued on `stream` goes into a graph (yes, where that cannot be said).
bool captured(void *stream) {
  hipStreamCaptureStatus status;
  if (hipStreamIsCapturing(static_cast<hipStream_t>(stream), &status) == hipSuccess) return status != hipStreamCaptureStatusNone;
  (void)hipGetLastError();  // not the launch's
  return true;
}

// A workspace of at least `bytes`: the given one (None: none yet) or a new one, as a new reference.  A graph that is captured keeps its address, so it goes into the list `kept` too: the object
// that owns the list may then take a larger one for other calls, and replays still write into this one and into nothing else.
PyObject *workspace(PyObject *given, PyObject *kept, size_t bytes, c10::Device device, void *stream, void *&data) {
  data = nullptr;
  PyObject *held = nullptr;
  if (given != Py_None) {
    const at::Tensor &t = tensor(given, "workspace");
    if ((size_t)t.numel() >= bytes && t.device() == device) {
      data = bytes ? t.data_ptr() : nullptr;
      Py_INCREF(held = given);
    }
  }
  if (!held && !bytes) Py_INCREF(held = given);
  if (!held) {
    at::Tensor made = make({(int64_t)bytes}, at::kByte, device);
    data = made.data_ptr();
    held = THPVariable_Wrap(std::move(made));
  }
  if (held && bytes && kept && captured(stream)) {
    const Py_ssize_t n = PyList_Size(kept);
    if (n < 0 || ((n == 0 || PyList_GetItem(kept, n - 1) != held) && PyList_Append(kept, held))) Py_CLEAR(held);
  }
  if (!held) throw Refused();
  return held;
}

// What throws ends as a Python error, PyTorch's errors as its own.  From `wanted` to `most` arguments (0: as many).
template <typename F>
PyObject *guarded(Py_ssize_t n, Py_ssize_t wanted, F f, Py_ssize_t most = 0) {
  if (n < wanted || n > (most ? most : wanted)) {
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", wanted, n);
    return nullptr;
  }
  try {
    return f();
  } catch (const Refused &) {
  } catch (...) {
    torch::translate_exception_to_python(std::current_exception());
  }
  return nullptr;
}

// (cached, fresh, free_pages, table, row_start, lens, slots, positions, needed, page_size); the last five tensors are the caller's own results
PyObject *tables(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 10, [&]() -> PyObject * {
    const at::Tensor &table = tensor(a[3], "table"), &row_start = tensor(a[4], "row_start"), &lens = tensor(a[5], "lens"), &slots = tensor(a[6], "slots"), &positions = tensor(a[7], "positions"),
                     &needed = tensor(a[8], "needed");
    const int64_t requests = lens.numel(), tokens = slots.numel();
    const c10::Device device = lens.device();
    if (table.dim() != 2) refuse("table must be int32 [requests][width], not " + shape_of(table.sizes()));
    expect(table, "table", at::kInt, {requests, table.size(1)}, device);
    const at::Tensor &cached = indices(a[0], "cached", at::kInt, {requests}, device), &fresh = indices(a[1], "fresh", at::kInt, {requests}, device), &free_pages = tensor(a[2], "free_pages");
    expect(free_pages, "free_pages", at::kInt, {free_pages.numel()}, device);
    const c10::DeviceGuard guard(device);
    succeeded(rnswino_block_tables(cached.const_data_ptr<int32_t>(), fresh.const_data_ptr<int32_t>(), (int32_t)requests, free_pages.const_data_ptr<int32_t>(), (int32_t)free_pages.numel(),
                                   (int32_t)integer(a[9]), table.data_ptr<int32_t>(), (int32_t)table.size(1), row_start.data_ptr<int32_t>(), lens.data_ptr<int32_t>(), slots.data_ptr<int64_t>(),
                                   positions.data_ptr<int32_t>(), (int32_t)tokens, needed.data_ptr<int32_t>(), stream_of(lens)),
              "rnswino_block_tables");
    Py_RETURN_NONE;
  });
}

struct Rope {
  rnswino_rope_t d;
  at::Tensor qkv;
  const char *q, *k, *v;
  const void *wq = nullptr, *wk = nullptr;
  const float *angles = nullptr;
  const int32_t *positions;
};
// (descriptor, angles, wq, wk, qkv, positions); with_v: the rows hold values too
Rope rope_of(PyObject *const *a, bool with_v) {
  Rope r = {*address<rnswino_rope_t>(a[0]), tensor(a[4], "qkv")};
  rnswino_rope_t &d = r.d;
  const int64_t q_width = (int64_t)d.q_heads * d.head_dim, k_width = (int64_t)d.kv_heads * d.head_dim;
  int64_t stride;
  const int64_t n = rows(r.qkv, "qkv", q_width + k_width * (with_v ? 2 : 1), stride);
  const c10::Device device = r.qkv.device();
  d.type = type_of(r.qkv, "qkv");
  d.n_tokens = (int32_t)n;
  d.q_stride = d.k_stride = d.v_stride = stride;
  d.q_out_stride = q_width, d.k_out_stride = k_width;
  r.q = (const char *)r.qkv.const_data_ptr();
  r.k = r.q + 2 * q_width, r.v = r.k + 2 * k_width;
  r.positions = indices(a[5], "positions", at::kInt, {n}, device).const_data_ptr<int32_t>();
  if (d.rotary) r.angles = indices(a[1], "angles", at::kFloat, {d.max_position, d.rotary}, device).const_data_ptr<float>();
  if (a[2] != Py_None) r.wq = indices(a[2], "wq", r.qkv.scalar_type(), {d.head_dim}, device).const_data_ptr();
  if (a[3] != Py_None) r.wk = indices(a[3], "wk", r.qkv.scalar_type(), {d.head_dim}, device).const_data_ptr();
  return r;
}

PyObject *rope(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 6, [&]() -> PyObject * {
    const Rope r = rope_of(a, false);
    const c10::DeviceGuard guard(r.qkv.device());
    at::Tensor q = make({r.d.n_tokens, r.d.q_heads, r.d.head_dim}, r.qkv.scalar_type(), r.qkv.device()), k = make({r.d.n_tokens, r.d.kv_heads, r.d.head_dim}, r.qkv.scalar_type(), r.qkv.device());
    succeeded(rnswino_qk_norm_rope(&r.d, r.q, r.k, r.wq, r.wk, r.angles, r.positions, q.data_ptr(), k.data_ptr(), stream_of(r.qkv)), "rnswino_qk_norm_rope");
    return pair(std::move(q), THPVariable_Wrap(std::move(k)));
  });
}

// (descriptor, angles, wq, wk, qkv, positions, slots, cache, one of its tensors)
PyObject *append(PyObject *, PyObject *const *a, Py_ssize_t n) {
  const auto call = [&]() -> PyObject * {
    const Rope r = rope_of(a, true);
    const at::Tensor &slots = indices(a[6], "slots", at::kLong, {r.d.n_tokens}, r.qkv.device());
    const c10::DeviceGuard guard(r.qkv.device());
    if (n > 8) expect_cache(a[8], r.qkv.device());
    at::Tensor q = make({r.d.n_tokens, r.d.q_heads, r.d.head_dim}, r.qkv.scalar_type(), r.qkv.device());
    succeeded(rnswino_qk_norm_rope_cache4(&r.d, r.q, r.k, r.v, r.wq, r.wk, r.angles, r.positions, slots.const_data_ptr<int64_t>(), q.data_ptr(), address<rnswino_cache4_t>(a[7]), stream_of(r.qkv)),
              "rnswino_qk_norm_rope_cache4");
    return THPVariable_Wrap(std::move(q));
  };
  return guarded(n, 8, call, 9);
}

// (cache, slots, half precision, one of the cache's tensors)
PyObject *read(PyObject *, PyObject *const *a, Py_ssize_t n) {
  const auto call = [&]() -> PyObject * {
    const rnswino_cache4_t *cache = address<rnswino_cache4_t>(a[0]);
    const at::Tensor &slots = tensor(a[1], "slots");
    expect(slots, "slots", at::kLong, {slots.numel()}, slots.device());
    if (n > 3) expect_cache(a[3], slots.device());
    const c10::DeviceGuard guard(slots.device());
    const bool half = integer(a[2]) != 0;
    at::Tensor k = make({slots.numel(), cache->kv_heads, cache->head_dim}, half ? at::kHalf : at::kBFloat16, slots.device()), v = make(k.sizes(), k.scalar_type(), k.device());
    succeeded(rnswino_cache4_read(cache, slots.const_data_ptr<int64_t>(), slots.numel(), half ? RNSWINO_TYPE_F16 : RNSWINO_TYPE_BF16, k.data_ptr(), v.data_ptr(), stream_of(slots)),
              "rnswino_cache4_read");
    return pair(std::move(k), THPVariable_Wrap(std::move(v)));
  };
  return guarded(n, 3, call, 4);
}

// (cache, descriptor, q, table, lens, row_start, max_fresh, max_len, out or None, workspace or None, list of workspaces that graphs have, one of the cache's tensors) -> (out, workspace)
PyObject *attend(PyObject *, PyObject *const *a, Py_ssize_t n) {
  const auto call = [&]() -> PyObject * {
    const rnswino_cache4_t *cache = address<rnswino_cache4_t>(a[0]);
    rnswino_attention_t d = *address<rnswino_attention_t>(a[1]);
    const at::Tensor &q = tensor(a[2], "q"), &table = tensor(a[3], "table");
    const c10::Device device = q.device();
    d.n_tokens = (int32_t)head_rows(q, "q", d.q_heads, cache->head_dim, d.q_stride);
    d.type = type_of(q, "q");
    if (n > 11) expect_cache(a[11], device);
    if (table.dim() != 2) refuse("table must be int32 [requests][width], not " + shape_of(table.sizes()));
    d.n_requests = (int32_t)table.size(0), d.table_width = (int32_t)table.size(1);
    expect(table, "table", at::kInt, {d.n_requests, d.table_width}, device);
    const at::Tensor &lens = indices(a[4], "lens", at::kInt, {d.n_requests}, device), &row_start = indices(a[5], "row_start", at::kInt, {d.n_requests + 1}, device);
    d.max_fresh = (int32_t)integer(a[6]), d.max_len = (int32_t)integer(a[7]);
    const c10::DeviceGuard guard(device);
    at::Tensor out;
    if (a[8] == Py_None) {
      out = make(q.sizes(), q.scalar_type(), device);
      d.out_stride = (int64_t)d.q_heads * cache->head_dim;
    } else {
      out = tensor(a[8], "out");
      if (head_rows(out, "out", d.q_heads, cache->head_dim, d.out_stride) != d.n_tokens || out.scalar_type() != q.scalar_type() || out.device() != device)
        refuse("out must have the shape, type and device of q, not " + shape_of(out.sizes()) + " " + c10::toString(out.scalar_type()) + " on " + out.device().str());
    }
    void *const stream = stream_of(q), *scratch;
    PyObject *held = workspace(a[9], n > 10 ? a[10] : nullptr, rnswino_cache4_attention_workspace_bytes(cache, &d), device, stream, scratch);
    const int code = rnswino_cache4_attention(cache, &d, q.const_data_ptr(), table.const_data_ptr<int32_t>(), lens.const_data_ptr<int32_t>(), row_start.const_data_ptr<int32_t>(), out.data_ptr(), scratch,
                                              stream);
    if (code) Py_DECREF(held);
    succeeded(code, "rnswino_cache4_attention");
    return pair(std::move(out), held);
  };
  return guarded(n, 10, call, 12);
}

// (codes, scales, inputs, x, y or None, workspace or None, list of workspaces that graphs have) -> (y, workspace)
PyObject *linear(PyObject *, PyObject *const *a, Py_ssize_t n) {
  const auto call = [&]() -> PyObject * {
    const at::Tensor &codes = tensor(a[0], "codes"), &scales = tensor(a[1], "scales"), &x = tensor(a[3], "x");
    const int64_t inputs = integer(a[2]), outputs = codes.size(0);
    const c10::Device device = codes.device();
    int64_t x_stride, y_stride;
    const int64_t count = rows(x, "x", inputs, x_stride);
    const int type = type_of(x, "x");
    if (x.device() != device) refuse("x must be on the weights' " + device.str() + ", not " + x.device().str());
    const c10::DeviceGuard guard(device);
    at::Tensor y = a[4] == Py_None ? make({count, outputs}, x.scalar_type(), device) : tensor(a[4], "y");
    if (rows(y, "y", outputs, y_stride) != count || y.scalar_type() != x.scalar_type() || y.device() != device)
      refuse("y must be " + std::to_string(count) + " rows of the type of x on its device, not " + shape_of(y.sizes()) + " " + c10::toString(y.scalar_type()) + " on " + y.device().str());
    void *const stream = stream_of(x), *scratch;
    PyObject *held = workspace(a[5], n > 6 ? a[6] : nullptr, rnswino_fp8_linear_workspace_bytes((int32_t)count, (int32_t)outputs, (int32_t)inputs), device, stream, scratch);
    const int code = rnswino_fp8_linear(x.const_data_ptr(), x_stride, (const uint8_t *)codes.const_data_ptr(), scales.const_data_ptr<float>(), (int32_t)count, (int32_t)outputs, (int32_t)inputs, type,
                                        y.data_ptr(), y_stride, scratch, stream);
    if (code) Py_DECREF(held);
    succeeded(code, "rnswino_fp8_linear");
    return pair(std::move(y), held);
  };
  return guarded(n, 6, call, 7);
}

PyMethodDef kMethods[] = {
    {"tables", (PyCFunction)(void (*)(void))tables, METH_FASTCALL, nullptr}, {"rope", (PyCFunction)(void (*)(void))rope, METH_FASTCALL, nullptr},
    {"append", (PyCFunction)(void (*)(void))append, METH_FASTCALL, nullptr}, {"read", (PyCFunction)(void (*)(void))read, METH_FASTCALL, nullptr},
    {"attend", (PyCFunction)(void (*)(void))attend, METH_FASTCALL, nullptr}, {"linear", (PyCFunction)(void (*)(void))linear, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_decoder", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__decoder(void) {
  PyObject *binding = PyImport_ImportModule("paper_2007_12216_amd.binding");
  if (!binding) return nullptr;
  g_check = PyObject_GetAttrString(binding, "_check");
  Py_DECREF(binding);
  return g_check ? PyModule_Create(&kModule) : nullptr;
}
