// The extension module's calls on tensors that lie on devices that are not there: the library's entry points write down which device is current when they are called.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/core/impl/FakeGuardImpl.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdlib>
#include <string>
#include <vector>

namespace stand_in {
using Devices = c10::impl::FakeGuardImpl<c10::DeviceType::CUDA>;
const c10::impl::DeviceGuardImplRegistrar registrar(c10::DeviceType::CUDA, new Devices());

at::Tensor tensor(at::IntArrayRef shape, at::ScalarType type, int device) {
  int64_t n = 1;
  for (int64_t v : shape) n *= v;
  const size_t bytes = (size_t)n * c10::elementSize(type);
  const size_t room = (bytes / 256 + 1) * 256;
  void *memory = aligned_alloc(256, room);  // never given back: the process ends with the test
  c10::Storage storage(c10::Storage::use_byte_size_t(), bytes, c10::DataPtr(memory, c10::Device(c10::kCUDA, (c10::DeviceIndex)device)), nullptr, false);
  at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(std::move(storage), c10::DispatchKeySet(c10::DispatchKey::CUDA), caffe2::TypeMeta::fromScalarType(type));
  t.unsafeGetTensorImpl()->set_sizes_contiguous(shape);
  return t;
}

struct Stream {
  void *handle;
  void *stream() const { return handle; }
};
std::vector<std::string> launches;
int launched(const char *name, void *stream) {
  launches.push_back(std::string(name) + " on " + std::to_string(Devices::getDeviceIndex()) + ", stream of " + std::to_string((intptr_t)stream));
  return 0;
}
}  // namespace stand_in

namespace c10::hip {
inline stand_in::Stream stand_in_stream(int device) { return {(void *)(intptr_t)device}; }
}  // namespace c10::hip
namespace at::detail {
inline at::Tensor stand_in_empty(at::IntArrayRef shape, at::ScalarType type, std::optional<c10::Device> device, std::optional<c10::MemoryFormat>) {
  return stand_in::tensor(shape, type, device->index());
}
}  // namespace at::detail
#define getCurrentHIPStream stand_in_stream
#define empty_cuda stand_in_empty
#include "decoder_binding.cpp"

extern "C" {
int rnswino_block_tables(const int32_t *, const int32_t *, int32_t, const int32_t *, int32_t, int32_t, int32_t *, int32_t, int32_t *, int32_t *, int64_t *, int32_t *, int32_t, int32_t *,
                         void *stream) {
  return stand_in::launched("tables", stream);
}
int rnswino_qk_norm_rope(const rnswino_rope_t *, const void *, const void *, const void *, const void *, const float *, const int32_t *, void *, void *, void *stream) {
  return stand_in::launched("rope", stream);
}
int rnswino_qk_norm_rope_cache4(const rnswino_rope_t *, const void *, const void *, const void *, const void *, const void *, const float *, const int32_t *, const int64_t *, void *,
                                const rnswino_cache4_t *, void *stream) {
  return stand_in::launched("append", stream);
}
int rnswino_cache4_read(const rnswino_cache4_t *, const int64_t *, int64_t, int32_t, void *, void *, void *stream) { return stand_in::launched("read", stream); }
size_t rnswino_cache4_attention_workspace_bytes(const rnswino_cache4_t *, const rnswino_attention_t *) { return 0; }
int rnswino_cache4_attention(const rnswino_cache4_t *, const rnswino_attention_t *, const void *, const int32_t *, const int32_t *, const int32_t *, void *, void *, void *stream) {
  return stand_in::launched("attend", stream);
}
size_t rnswino_fp8_linear_workspace_bytes(int32_t, int32_t, int32_t) { return 0; }
int rnswino_fp8_linear(const void *, int64_t, const uint8_t *, const float *, int32_t, int32_t, int32_t, int32_t, void *, int64_t, void *, void *stream) {
  return stand_in::launched("linear", stream);
}
}

namespace {
// (device, type, sizes ...): a tensor of "int", "long", "float", "byte" or "bf16"
PyObject *make_on(PyObject *, PyObject *const *a, Py_ssize_t n) {
  std::vector<int64_t> shape;
  for (Py_ssize_t i = 2; i < n; ++i) shape.push_back(PyLong_AsLongLong(a[i]));
  const std::string type = PyUnicode_AsUTF8(a[1]);
  const at::ScalarType of = type == "int" ? at::kInt : type == "long" ? at::kLong : type == "float" ? at::kFloat : type == "byte" ? at::kByte : at::kBFloat16;
  return THPVariable_Wrap(stand_in::tensor(shape, of, (int)PyLong_AsLong(a[0])));
}
PyObject *launches(PyObject *, PyObject *const *, Py_ssize_t) {
  PyObject *all = PyList_New(0);
  for (const std::string &s : stand_in::launches) {
    PyObject *one = PyUnicode_FromString(s.c_str());
    PyList_Append(all, one);
    Py_DECREF(one);
  }
  stand_in::launches.clear();
  return all;
}
PyObject *current(PyObject *, PyObject *const *, Py_ssize_t) { return PyLong_FromLong(stand_in::Devices::getDeviceIndex()); }
PyMethodDef kStandIns[] = {{"make", (PyCFunction)(void (*)(void))make_on, METH_FASTCALL, nullptr},
                           {"launches", (PyCFunction)(void (*)(void))launches, METH_FASTCALL, nullptr},
                           {"current", (PyCFunction)(void (*)(void))current, METH_FASTCALL, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef kStandInModule = {PyModuleDef_HEAD_INIT, "decoder_devices", nullptr, -1, kStandIns, nullptr, nullptr, nullptr, nullptr};
}  // namespace
PyMODINIT_FUNC PyInit_decoder_devices(void) { return PyModule_Create(&kStandInModule); }
