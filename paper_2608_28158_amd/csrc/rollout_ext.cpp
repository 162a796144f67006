// Python binding of the generation calls (harts_rollout.h) for torch tensors:
// checks of the arguments, allocation of the results and the call, in one step.
// A generated token is many small calls, and each of these took 5 to 7 us of
// Python around a 3 us launch (one linear-attention step of one sequence: 11.3 us,
// of which the kernel takes 3; so 5.1).  The library's functions are handed over by
// address (bind), so that it is the one library that the package has loaded.
#include <ATen/Functions.h>
#include <ATen/core/Tensor.h>
#include <c10/core/AutogradState.h>
#include <c10/core/DeviceGuard.h>
#include <pybind11/pybind11.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/pybind.h>

#include <cmath>
#include <cstdint>
#include <optional>
#include <sstream>
#include <string>
#include <vector>

#include "harts_rollout.h"

namespace py = pybind11;
using at::Tensor;
using OptTensor = std::optional<Tensor>;

namespace {

struct Calls {
  decltype(&harts_cache_write) cache_write = nullptr;
  decltype(&harts_cache_read) cache_read = nullptr;
  decltype(&harts_gen_attn) gen_attn = nullptr;
  decltype(&harts_la_step) la_step = nullptr;
  decltype(&harts_kda_step) kda_step = nullptr;
  py::object* fail = nullptr;      // (code, where): raises the package's error
} L;

void bind(uintptr_t cache_write, uintptr_t cache_read, uintptr_t gen_attn, uintptr_t la_step, uintptr_t kda_step,
          const py::object& fail) {
  L.cache_write = reinterpret_cast<decltype(L.cache_write)>(cache_write);
  L.cache_read = reinterpret_cast<decltype(L.cache_read)>(cache_read);
  L.gen_attn = reinterpret_cast<decltype(L.gen_attn)>(gen_attn);
  L.la_step = reinterpret_cast<decltype(L.la_step)>(la_step);
  L.kda_step = reinterpret_cast<decltype(L.kda_step)>(kda_step);
  L.fail = new py::object(fail);   // (kept for the process: no destructor after the interpreter's end)
}

void ok(int code, const char* where) {
  if (code != HARTS_OK) (*L.fail)(code, where);
}

// Tensors on one GPU, contiguous, of a given type and shape, none recording a
// gradient or carrying a tangent while those are on.
struct Checker {
  c10::Device device;
  bool grad = c10::AutogradState::get_tls_state().get_grad_mode();
  bool tangents = c10::AutogradState::get_tls_state().get_fw_grad_mode();
  explicit Checker(const Tensor& first) : device(first.device()) {
    if (!device.is_cuda()) throw std::runtime_error("generation runs on the GPU only");
  }
  explicit Checker(int64_t index) : device(at::kCUDA, static_cast<c10::DeviceIndex>(index)) {}
  void operator()(const char* name, const Tensor& t, at::ScalarType type, at::IntArrayRef shape) const {
    if (t.scalar_type() != type || t.sizes() != shape || !t.is_contiguous()) {
      std::ostringstream s;
      s << name << " must be contiguous " << type << " " << shape << ", got " << t.scalar_type() << " " << t.sizes();
      if (!t.is_contiguous()) s << " with strides " << t.strides();
      throw py::value_error(s.str());
    }
    if (t.device() != device) {
      std::ostringstream s;
      s << name << " is on " << t.device() << ", expected " << device;
      throw py::value_error(s.str());
    }
    if (grad && t.requires_grad())
      throw std::runtime_error(std::string(name) + " requires a gradient; generation is not differentiable");
    if (tangents && t._fw_grad(0).defined())
      throw std::runtime_error(std::string(name) + " carries a tangent; generation is not differentiable");
  }
};

// A tensor that a call has written counts as modified, for a backward pass that saved it.
void written(const Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

void* ptr(const OptTensor& t) { return t ? t->data_ptr() : nullptr; }
const int32_t* ints(const OptTensor& t) { return static_cast<const int32_t*>(ptr(t)); }

const harts_cache* cache_at(uintptr_t p) { return reinterpret_cast<const harts_cache*>(p); }

// cells: the tensors that hold the cache (the package's own tuple)
void cache_write(uintptr_t desc, int64_t device, uintptr_t stream, const py::tuple& cells, const Tensor& rows,
                 const Tensor& k, const Tensor& v) {
  const harts_cache* c = cache_at(desc);
  const Checker check(device);
  const int64_t n = rows.dim() > 0 ? rows.size(0) : 0;
  check("rows", rows, at::kInt, {n, 2});
  check("k", k, at::kBFloat16, {n, c->H, c->d});
  check("v", v, at::kBFloat16, {n, c->H, c->d});
  const c10::DeviceGuard on(check.device);
  ok(L.cache_write(c, rows.const_data_ptr<int32_t>(), n, k.const_data_ptr(), v.const_data_ptr(),
                   reinterpret_cast<void*>(stream)), "harts_cache_write");
  for (const py::handle t : cells) written(THPVariable_Unpack(t.ptr()));
}

py::tuple cache_read(uintptr_t desc, int64_t device, uintptr_t stream, const Tensor& rows) {
  const harts_cache* c = cache_at(desc);
  const Checker check(device);
  const int64_t n = rows.dim() > 0 ? rows.size(0) : 0;
  check("rows", rows, at::kInt, {n, 2});
  const auto options = rows.options().dtype(at::kBFloat16);
  const Tensor k = at::empty({n, c->H, c->d}, options), v = at::empty({n, c->H, c->d}, options);
  const c10::DeviceGuard on(check.device);
  ok(L.cache_read(c, rows.const_data_ptr<int32_t>(), n, k.data_ptr(), v.data_ptr(), reinterpret_cast<void*>(stream)),
     "harts_cache_read");
  return py::make_tuple(k, v);
}

py::tuple attend(uintptr_t desc, uintptr_t sizes_at, uintptr_t items, uintptr_t order, uintptr_t part_off,
                 int64_t q_heads, int64_t ws_bytes, int64_t device, uintptr_t stream, const Tensor& q,
                 std::optional<double> scale, const OptTensor& out) {
  const harts_cache* c = cache_at(desc);
  const auto* sizes = reinterpret_cast<const harts_gen_sizes*>(sizes_at);
  const Checker check(device);
  check("q", q, at::kBFloat16, {sizes->n_rows, q_heads, c->d});
  if (out) check("out", *out, at::kBFloat16, {sizes->n_rows, q_heads, c->d});
  const Tensor o = out ? *out : at::empty_like(q);
  // (workspace from the allocator at every call: calls on other streams, or captured into other graphs, share none)
  const Tensor lse = at::empty({sizes->n_rows, q_heads}, q.options().dtype(at::kFloat));
  const Tensor ws = ws_bytes > 0 ? at::empty({ws_bytes}, q.options().dtype(at::kByte)) : Tensor();
  const c10::DeviceGuard on(check.device);
  ok(L.gen_attn(c, sizes, reinterpret_cast<const int32_t*>(items), reinterpret_cast<const int32_t*>(order),
                reinterpret_cast<const int32_t*>(part_off), static_cast<int32_t>(q_heads),
                static_cast<float>(scale ? *scale : 1.0 / std::sqrt(static_cast<double>(c->d))), q.const_data_ptr(),
                o.data_ptr(), lse.data_ptr<float>(), ws_bytes > 0 ? ws.data_ptr() : nullptr,
                static_cast<size_t>(ws_bytes), reinterpret_cast<void*>(stream)), "harts_gen_attn");
  if (out) written(o);
  return py::make_tuple(o, lse);
}

// beta only for KDA.
Tensor step(bool kda, const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& g, const OptTensor& beta,
            const Tensor& S, const OptTensor& S_out_, const OptTensor& idx_in, const OptTensor& idx_out_,
            const OptTensor& row_off, std::optional<double> scale, const OptTensor& out, const py::object& stream_of) {
  const at::ScalarType type = q.scalar_type();
  if (q.dim() != 3 || (type != at::kBFloat16 && type != at::kFloat))
    throw py::value_error("q must be float32 or bfloat16 [rows, H, d]");
  const Checker check(q);
  const int64_t n_rows = q.size(0), H = q.size(1), d = q.size(2);
  check("q", q, type, {n_rows, H, d});
  check("k", k, type, {n_rows, H, d});
  check("v", v, type, {n_rows, H, d});
  if (out) check("out", *out, type, {n_rows, H, d});
  if (kda) check("g", g, at::kFloat, {n_rows, H, d});
  else check("g", g, at::kFloat, {n_rows, H});
  if (kda) {
    if (!beta) throw py::value_error("beta must be float32 [rows, H], got None");
    check("beta", *beta, at::kFloat, {n_rows, H});
  }
  int64_t n_seq = n_rows;
  if (row_off) {
    n_seq = row_off->numel() - 1;
    if (n_seq < 0) throw py::value_error("row_off has one entry more than there are sequences");
    check("row_off", *row_off, at::kInt, {n_seq + 1});
  }
  const bool inside = !S_out_ || S_out_->is_same(S);      // an update in place
  if (inside && idx_out_ && !(S_out_ && idx_in && idx_out_->is_same(*idx_in)))
    throw py::value_error("an update in place leaves every state where it was: S_out and idx_out have to be None");
  const Tensor& S_out = inside ? S : *S_out_;
  const OptTensor& idx_out = inside ? idx_in : idx_out_;
  const auto pool = [&](const char* name, const Tensor& t, const char* index_name, const OptTensor& idx) {
    const int64_t n = t.dim() > 0 ? t.size(0) : 0;
    check(name, t, at::kFloat, {n, H, d, d});
    if (idx) check(index_name, *idx, at::kInt, {n_seq});
    else if (n < n_seq)
      throw py::value_error(std::string(name) + " has " + std::to_string(n) + " states for " + std::to_string(n_seq) +
                            " sequences and no index");
    return n;
  };
  const int64_t n_in = pool("S", S, "idx_in", idx_in);
  const int64_t n_out = inside ? n_in : pool("S_out", S_out, "idx_out", idx_out);
  const Tensor o = out ? *out : at::empty_like(q);
  const c10::DeviceGuard on(check.device);
  void* stream = reinterpret_cast<void*>(stream_of(static_cast<int64_t>(check.device.index())).cast<uintptr_t>());
  const int32_t code = type == at::kBFloat16 ? HARTS_BF16 : HARTS_F32;
  const float f = static_cast<float>(scale ? *scale : 1.0 / std::sqrt(static_cast<double>(d)));
  if (kda)
    ok(L.kda_step(code, n_seq, n_rows, static_cast<int32_t>(H), static_cast<int32_t>(d), f, q.const_data_ptr(),
                  k.const_data_ptr(), v.const_data_ptr(), g.const_data_ptr<float>(), beta->const_data_ptr<float>(),
                  ints(row_off), S.const_data_ptr<float>(), ints(idx_in), n_in, S_out.data_ptr<float>(), ints(idx_out),
                  n_out, o.data_ptr(), stream), "harts_kda_step");
  else
    ok(L.la_step(code, n_seq, n_rows, static_cast<int32_t>(H), static_cast<int32_t>(d), f, q.const_data_ptr(),
                 k.const_data_ptr(), v.const_data_ptr(), g.const_data_ptr<float>(), ints(row_off),
                 S.const_data_ptr<float>(), ints(idx_in), n_in, S_out.data_ptr<float>(), ints(idx_out), n_out,
                 o.data_ptr(), stream), "harts_la_step");
  written(S_out);
  if (out) written(o);
  return o;
}

}  // namespace

PYBIND11_MODULE(_rollout, m) {
  m.def("bind", &bind);
  m.def("cache_write", &cache_write);
  m.def("cache_read", &cache_read);
  m.def("attend", &attend);
  m.def("step", &step);
}
