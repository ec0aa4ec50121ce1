// What the Python side of the gradient sets and of group norm does per call, in C++: reading tensors (pointers, types,
// strides), refusing what does not fit, allocating outputs and calling the entry points of include/sae.h.  A model has
// hundreds of gradient tensors, and looking at four properties of each in Python took 0.25 us a tensor, more than the kernels.
// No arithmetic happens here.
#include "../../include/sae.h"

#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <cuda_runtime_api.h>
#include <torch/extension.h>

#include <cstring>
#include <vector>

namespace py = pybind11;
using at::Tensor;

namespace {

int type_of(at::ScalarType t) {
  return t == at::kFloat ? SAE_TYPE_FLOAT : t == at::kBFloat16 ? SAE_TYPE_BFLOAT : t == at::kHalf ? SAE_TYPE_HALF : -1;
}

[[noreturn]] void refuse(const std::string& why) { throw py::value_error(why); }

// A new tensor, straight from the CUDA allocator (the dispatcher's way costs three times the time).
Tensor fresh(at::IntArrayRef sizes, at::ScalarType type, at::Device device) {
  return at::detail::empty_cuda(sizes, type, device, std::nullopt);
}

const Tensor& tensor_of(PyObject* o) {
  if (!THPVariable_Check(o)) refuse("tensors are wanted");
  return THPVariable_Unpack(o);
}

// ---- gradient sets ----------------------------------------------------------------------------------------------------
struct Shape { std::vector<int64_t> sizes, strides; };

class GradPlan {
 public:
  GradPlan(int64_t handle, int K, std::vector<int64_t> sizes, std::vector<int> types, int device, int64_t stream,
           std::vector<std::pair<std::vector<int64_t>, std::vector<int64_t>>> like)
      : h_(reinterpret_cast<sae_grads*>(handle)), K_(K), T_((int)sizes.size()), d_(0), device_(device),
        stream_(reinterpret_cast<cudaStream_t>(stream)), sizes_(std::move(sizes)), types_(std::move(types)) {
    for (int64_t n : sizes_) d_ += n;
    for (auto& p : like) like_.push_back({p.first, p.second});
  }

  std::tuple<int, Tensor> norm(py::handle tensors, int kind) {
    const Rows r = pointers(tensors, false);
    Tensor norms = rows();
    return {on_stream([&] { return sae_grads_norm(h_, r.ptrs.data(), kind, norms.data_ptr<float>()); }), norms};
  }
  std::tuple<int, Tensor> clip(py::handle tensors, int kind, float max_norm) {
    const Rows r = pointers(tensors, true);
    Tensor norms = rows();
    const int rc = on_stream([&] { return sae_grads_clip(h_, const_cast<void* const*>(r.ptrs.data()), kind, max_norm, norms.data_ptr<float>()); });
    if (rc == SAE_OK) written(r);
    return {rc, norms};
  }
  std::tuple<int, Tensor, std::optional<Tensor>> pack(py::handle tensors, std::optional<Tensor> out, int kind, float max_norm) {
    if (!out) out = fresh({K_, d_}, at::kFloat, device());
    const int64_t stride = vector(*out, "out", false);
    const Rows r = pointers(tensors, false);
    std::optional<Tensor> norms;
    if (kind != SAE_NORM_NONE) norms = rows();
    const int rc = on_stream([&] {
      return sae_grads_pack(h_, r.ptrs.data(), kind, max_norm, (float*)out->data_ptr(), stride, norms ? norms->data_ptr<float>() : nullptr);
    });
    if (rc == SAE_OK) written(*out);
    return {rc, *out, norms};
  }
  int unpack(const Tensor& v, py::handle tensors) {
    const int64_t stride = vector(v, "vector", true);
    const Rows r = pointers(tensors, true);
    const int rc = on_stream([&] { return sae_grads_unpack(h_, (const float*)v.data_ptr(), stride, const_cast<void* const*>(r.ptrs.data())); });
    if (rc == SAE_OK) written(r);
    return rc;
  }

 private:
  at::Device device() const { return at::Device(at::kCUDA, (c10::DeviceIndex)device_); }
  Tensor rows() const { return fresh({K_}, at::kFloat, device()); }

  // The row stride of a [d] (one row, or the same for all) or [K, d] float32 tensor.
  int64_t vector(const Tensor& v, const char* what, bool same) const {
    if (v.scalar_type() != at::kFloat || !v.is_cuda() || v.get_device() != device_)
      refuse(std::string(what) + " must be a float32 tensor on the set's device");
    if (v.dim() == 1 && v.size(0) == d_ && (K_ == 1 || same) && (d_ < 2 || v.stride(0) == 1)) return 0;
    if (v.dim() == 2 && v.size(0) == K_ && v.size(1) == d_ && (d_ < 2 || v.stride(1) == 1) && (K_ == 1 || v.stride(0) >= d_))
      return K_ > 1 ? v.stride(0) : 0;
    refuse(std::string(what) + " must have " + std::to_string(K_) + " rows of " + std::to_string(d_) + " elements without gaps");
  }

  void check_type(const Tensor& t, int j) const {
    if (type_of(t.scalar_type()) != types_[j] || !t.is_cuda() || t.get_device() != device_) refuse("a tensor's dtype or device is not the set's");
  }

  // A call's tensors: their addresses, the sequences that hold them, and themselves where the call writes them.  A generator's
  // tensors may have no other owner; without one their memory would be the next allocation's (the norms') before the kernels have read it.
  struct Rows {
    std::vector<const void*> ptrs;
    std::vector<py::object> held;
    std::vector<const Tensor*> tensors;
  };

  // What a call has written counts as changed in place: autograd refuses a backward pass that would need the old values.
  static void written(const Tensor& t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
  }
  static void written(const Rows& r) {
    for (const Tensor* t : r.tensors) written(*t);
  }

  void row(py::handle tensors, Rows& out, bool writes) const {
    py::object seq = py::reinterpret_steal<py::object>(PySequence_Fast(tensors.ptr(), "a row is a sequence of tensors"));
    if (!seq) throw py::error_already_set();
    out.held.push_back(seq);
    if (PySequence_Fast_GET_SIZE(seq.ptr()) != T_)
      refuse("a row has " + std::to_string(T_) + " tensors, got " + std::to_string(PySequence_Fast_GET_SIZE(seq.ptr())));
    PyObject** items = PySequence_Fast_ITEMS(seq.ptr());
    const size_t at = out.ptrs.size();
    out.ptrs.resize(at + (size_t)T_);
    const void** const ptrs = out.ptrs.data() + at;
    for (int j = 0; j < T_; ++j) {
      const Tensor& t = tensor_of(items[j]);
      check_type(t, j);
      if (like_.empty()) {
        if (t.numel() != sizes_[j] || !t.is_contiguous()) refuse("tensors must be contiguous and of the set's sizes");
      } else {
        const Shape& s = like_[j];
        bool same = t.sizes() == at::IntArrayRef(s.sizes);
        for (size_t i = 0; same && sizes_[j] && i < s.sizes.size(); ++i) same = s.sizes[i] == 1 || t.stride((int64_t)i) == s.strides[i];
        if (!same) refuse("tensors must have the shapes and strides that the set was made like");
      }
      ptrs[j] = t.data_ptr();
      if (writes) out.tensors.push_back(&t);
    }
  }

  Rows pointers(py::handle tensors, bool writes) const {
    Rows out;
    out.ptrs.reserve((size_t)K_ * T_);
    out.held.reserve((size_t)K_ + 1);
    if (writes) out.tensors.reserve((size_t)K_ * T_);
    if (THPVariable_Check(tensors.ptr())) {
      const Tensor& t = THPVariable_Unpack(tensors.ptr());
      if (T_ != 1 || t.dim() != 2 || t.size(0) != K_ || t.size(1) != sizes_[0] || (t.size(1) > 1 && t.stride(1) != 1) ||
          (K_ > 1 && t.stride(0) < t.size(1)))
        refuse("one tensor stands for [num_rows, n] of a set of one tensor, rows without gaps");
      check_type(t, 0);
      out.tensors.push_back(&t);
      for (int k = 0; k < K_; ++k) out.ptrs.push_back((const char*)t.data_ptr() + (int64_t)k * t.stride(0) * t.element_size());
      return out;
    }
    py::object seq = py::reinterpret_steal<py::object>(PySequence_Fast(tensors.ptr(), "tensors: a sequence of tensors, or of rows of tensors"));
    if (!seq) throw py::error_already_set();
    out.held.push_back(seq);
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq.ptr());
    PyObject** items = PySequence_Fast_ITEMS(seq.ptr());
    if (K_ == 1 && n > 0 && THPVariable_Check(items[0])) {
      row(seq, out, writes);
    } else {
      if (n != K_) refuse("tensors of " + std::to_string(K_) + " rows are wanted, got " + std::to_string(n));
      for (Py_ssize_t k = 0; k < n; ++k) {
        if (THPVariable_Check(items[k])) refuse("a row is a sequence of tensors");
        row(items[k], out, writes);
      }
    }
    return out;
  }

  // The set's work is on its own stream.  Where another is current, the two are ordered both ways, so that the call may
  // read what the current stream has made and the current stream may use what it gives.
  template <typename F>
  int on_stream(F call) const {
    cudaStream_t current = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device_).stream();
    if (current == stream_) return call();
    c10::cuda::CUDAGuard guard((c10::DeviceIndex)device_);
    cudaEvent_t e = nullptr;
    if (cudaEventCreateWithFlags(&e, cudaEventDisableTiming) != cudaSuccess) return SAE_ERR_CUDA;
    int rc = cudaEventRecord(e, current) == cudaSuccess && cudaStreamWaitEvent(stream_, e, 0) == cudaSuccess ? SAE_OK : SAE_ERR_CUDA;
    if (rc == SAE_OK) rc = call();
    const bool back = cudaEventRecord(e, stream_) == cudaSuccess && cudaStreamWaitEvent(current, e, 0) == cudaSuccess;
    cudaEventDestroy(e);
    return rc == SAE_OK && !back ? SAE_ERR_CUDA : rc;
  }

  sae_grads* h_;
  int K_, T_;
  int64_t d_;
  int device_;
  cudaStream_t stream_;
  std::vector<int64_t> sizes_;
  std::vector<int> types_;
  std::vector<Shape> like_;
};

// ---- group norm -----------------------------------------------------------------------------------------------------------

// (sample, pixel) strides of an [n, c, *space] tensor whose channels are neighbours in memory and whose pixels follow one
// another at one stride.
void strides_of(const Tensor& t, const char* what, int64_t& sample, int64_t& pixel) {
  sample = pixel = 0;
  if (t.numel() == 0) return;
  if (t.size(1) > 1 && t.stride(1) != 1) refuse(std::string(what) + " must be channels last: neighbouring channels next to each other in memory");
  int64_t run = 1;
  for (int64_t i = t.dim() - 1; i >= 2; --i) {
    if (t.size(i) == 1) continue;
    if (run == 1) pixel = t.stride(i);
    else if (t.stride(i) != run * pixel) refuse(std::string(what) + ": the pixels of a sample must follow one another at one stride");
    run *= t.size(i);
  }
  sample = t.size(0) > 1 ? t.stride(0) : 0;
}

void input(const Tensor& t, const Tensor& x, const char* what, int64_t& sample, int64_t& pixel) {
  if (t.sizes() != x.sizes() || t.scalar_type() != x.scalar_type() || t.device() != x.device())
    refuse(std::string(what) + " must have the shape, dtype and device of x");
  strides_of(t, what, sample, pixel);
}

typedef std::optional<Tensor> Maybe;

sae_group_norm_desc describe(const Tensor& x, int64_t groups, const Maybe& weight, const Maybe& bias, double eps, int act, const Maybe& residual) {
  if (!x.is_cuda() || type_of(x.scalar_type()) < 0 || x.dim() < 2) refuse("x must be a float32, bfloat16 or float16 CUDA tensor [n, c, *space]");
  const int64_t c = x.size(1);
  if (groups < 1 || c < 1 || c % groups || groups > INT32_MAX) refuse("the number of groups must divide the number of channels");
  sae_group_norm_desc d;
  std::memset(&d, 0, sizeof(d));                 // padding too: descriptions are compared
  d.type = type_of(x.scalar_type());
  d.param_type = SAE_TYPE_FLOAT;
  for (int i = 0; i < 2; ++i) {
    const Maybe& t = i ? bias : weight;
    if (!t) continue;
    if (t->dim() != 1 || t->size(0) != c || type_of(t->scalar_type()) < 0 || t->device() != x.device() || !t->is_contiguous())
      refuse(std::string(i ? "bias" : "weight") + " must be a contiguous [c] tensor on x's device");
    d.param_type = type_of(t->scalar_type());
  }
  if (weight && bias && weight->scalar_type() != bias->scalar_type()) refuse("weight and bias must have the same dtype");
  d.activation = act;
  d.groups = (int32_t)groups;
  d.samples = x.size(0);
  d.channels = c;
  d.pixels = 1;
  for (int64_t i = 2; i < x.dim(); ++i) d.pixels *= x.size(i);
  d.eps = (float)eps;
  strides_of(x, "x", d.x_sample, d.x_pixel);
  if (residual) input(*residual, x, "residual", d.residual_sample, d.residual_pixel);
  return d;
}

// A new tensor of x's shape, channels last without gaps.
Tensor dense(const Tensor& x) {
  c10::SmallVector<int64_t, 6> st(x.dim());
  int64_t run = x.size(1);
  st[1] = 1;
  for (int64_t i = x.dim() - 1; i >= 2; --i) { st[i] = run; run *= std::max<int64_t>(1, x.size(i)); }
  st[0] = run;
  return at::detail::empty_strided_cuda(x.sizes(), st, x.scalar_type(), x.device());
}

void* ptr(const Maybe& t) { return t ? t->data_ptr() : nullptr; }

Tensor workspace(const sae_group_norm_desc& d, const Tensor& x, int backward, size_t& bytes) {
  // asked for once for a description: a layer's calls have the same one over and over
  static thread_local sae_group_norm_desc last[2];
  static thread_local int64_t last_bytes[2] = {-1, -1};
  static thread_local int last_device[2] = {-1, -1};
  const int device = x.get_device();
  if (last_device[backward] != device || std::memcmp(&last[backward], &d, sizeof(d)) != 0) {
    last_bytes[backward] = sae_group_norm_workspace(&d, backward);
    last[backward] = d;
    last_device[backward] = device;
  }
  bytes = last_bytes[backward] > 0 ? (size_t)last_bytes[backward] : 0;
  return bytes ? fresh({(int64_t)bytes}, at::kByte, x.device()) : Tensor();
}

std::tuple<int, Tensor, Tensor, Tensor> group_norm_forward(const Tensor& x, int64_t groups, const Maybe& weight, const Maybe& bias,
                                                           double eps, int act, const Maybe& residual) {
  const sae_group_norm_desc d = describe(x, groups, weight, bias, eps, act, residual);
  c10::cuda::CUDAGuard guard(x.device());
  Tensor y = dense(x);
  Tensor mean = fresh({x.size(0), groups}, at::kFloat, x.device()), rstd = fresh({x.size(0), groups}, at::kFloat, x.device());
  size_t bytes;
  Tensor ws = workspace(d, x, 0, bytes);
  const int rc = sae_group_norm_forward(&d, x.data_ptr(), ptr(residual), ptr(weight), ptr(bias), y.data_ptr(), (float*)mean.data_ptr(),
                                        (float*)rstd.data_ptr(), bytes ? ws.data_ptr() : nullptr, bytes,
                                        c10::cuda::getCurrentCUDAStream(x.get_device()).stream());
  return {rc, y, mean, rstd};
}

std::tuple<int, Tensor, Maybe, Maybe, Maybe> group_norm_backward(const Tensor& dy, const Tensor& x, const Tensor& mean, const Tensor& rstd,
                                                                 int64_t groups, const Maybe& weight, const Maybe& bias, int act,
                                                                 const Maybe& residual, bool need_residual, bool need_params) {
  sae_group_norm_desc d = describe(x, groups, weight, bias, 0.0, act, residual);
  input(dy, x, "dy", d.dy_sample, d.dy_pixel);
  for (const Tensor* t : {&mean, &rstd})
    if (t->dim() != 2 || t->size(0) != x.size(0) || t->size(1) != groups || t->scalar_type() != at::kFloat || t->device() != x.device() || !t->is_contiguous())
      refuse("mean and rstd must be the float32 [n, groups] tensors of the forward call");
  c10::cuda::CUDAGuard guard(x.device());
  Tensor dx = dense(x);
  Maybe dres, dweight, dbias;
  if (residual && need_residual) dres = dense(x);
  if (weight && need_params) dweight = fresh(weight->sizes(), weight->scalar_type(), x.device());
  if (bias && need_params) dbias = fresh(bias->sizes(), bias->scalar_type(), x.device());
  size_t bytes;
  Tensor ws = workspace(d, x, 1, bytes);
  const int rc = sae_group_norm_backward(&d, dy.data_ptr(), x.data_ptr(), ptr(residual), (const float*)mean.data_ptr(), (const float*)rstd.data_ptr(),
                                         ptr(weight), ptr(bias), dx.data_ptr(), ptr(dres), ptr(dweight), ptr(dbias),
                                         bytes ? ws.data_ptr() : nullptr, bytes, c10::cuda::getCurrentCUDAStream(x.get_device()).stream());
  return {rc, dx, dres, dweight, dbias};
}

}  // namespace

PYBIND11_MODULE(TORCH_EXTENSION_NAME, m) {
  py::class_<GradPlan>(m, "GradPlan")
      .def(py::init<int64_t, int, std::vector<int64_t>, std::vector<int>, int, int64_t,
                    std::vector<std::pair<std::vector<int64_t>, std::vector<int64_t>>>>())
      .def("norm", &GradPlan::norm)
      .def("clip", &GradPlan::clip)
      .def("pack", &GradPlan::pack)
      .def("unpack", &GradPlan::unpack);
  m.def("group_norm_forward", &group_norm_forward);
  m.def("group_norm_backward", &group_norm_backward);
}
