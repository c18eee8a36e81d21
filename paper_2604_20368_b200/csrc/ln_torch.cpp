// Argument marshalling of the query / key preparation and of softmax attention for torch tensors: checks, outputs and
// workspaces, the current stream of the tensors' device, and the C ABI.  A serving step's kernels take a few microseconds; the same
// marshalling through ctypes took 34 us a call, most of the step.
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/extension.h>

#include <optional>
#include <sstream>
#include <string>

#include "laplace_nystrom.h"

namespace {

namespace py = pybind11;
using at::Tensor;
using Maybe = std::optional<Tensor>;

// Entry points of the CUDA library, and the package's error class (see bind).
struct Api {
  decltype(&rope_fwd) rope_fwd_ = nullptr;
  decltype(&rope_bwd) rope_bwd_ = nullptr;
  decltype(&qk_norm_rope_fwd) qkn_fwd = nullptr;
  decltype(&qk_norm_rope_bwd_workspace_bytes) qkn_bytes = nullptr;
  decltype(&qk_norm_rope_bwd) qkn_bwd = nullptr;
  decltype(&softmax_attention_workspace_bytes) sm_bytes = nullptr;
  decltype(&softmax_attention_fwd) sm_fwd = nullptr;
  decltype(&softmax_attention_bwd) sm_bwd = nullptr;
  PyObject* error = nullptr;
} api;

[[noreturn]] void refuse(const std::string& what) { throw py::value_error(what); }

void check(int status, const char* where) {
  if (status == LN_OK) return;
  py::object e = py::reinterpret_borrow<py::object>(api.error)(status, where);
  PyErr_SetObject(api.error, e.ptr());
  throw py::error_already_set();
}

template <typename S> std::string text(const S& sizes) {
  std::ostringstream o;
  o << sizes;
  return o.str();
}

// What every tensor of a call shares.
struct Like {
  at::ScalarType type;
  c10::Device device;
  int dtype;
  explicit Like(const Tensor& q) : type(q.scalar_type()), device(q.device()) {
    if (!device.is_cuda()) refuse("tensor must live on a CUDA device (there is no CPU path)");
    if (q.dim() != 4) refuse("Q must be [B, H, n, d]");
    if (type == at::kFloat) dtype = LN_F32;
    else if (type == at::kBFloat16) dtype = LN_BF16;
    else refuse(std::string("unsupported storage dtype ") + c10::toString(type));
  }
};

// One [B, H, n, d] tensor.
ln_view view(const char* name, const Tensor& t, at::IntArrayRef shape, const Like& like) {
  if (t.sizes() != shape) refuse(std::string(name) + ": shape " + text(t.sizes()) + ", expected " + text(shape));
  if (t.scalar_type() != like.type || t.device() != like.device)
    refuse(std::string(name) + ": " + c10::toString(t.scalar_type()) + " on " + t.device().str() + ", expected " + c10::toString(like.type) + " on " + like.device.str());
  if (t.stride(3) != 1) refuse(std::string(name) + ": the channels of a row must be adjacent");
  return ln_view{t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)};
}

// An optional contiguous tensor; its pointer.
template <typename T> T* vector(const char* name, const Maybe& t, at::ScalarType type, at::IntArrayRef shape, c10::Device device) {
  if (!t) return nullptr;
  if (t->scalar_type() != type || t->sizes() != shape || t->device() != device || !t->is_contiguous())
    refuse(std::string(name) + ": " + c10::toString(t->scalar_type()) + " " + text(t->sizes()) + " on " + t->device().str() + ", expected a contiguous " +
           c10::toString(type) + " " + text(shape) + " on " + device.str());
  return static_cast<T*>(t->data_ptr());
}

int32_t narrow(int64_t v, const char* what) {
  if (v < INT32_MIN || v > INT32_MAX) refuse(std::string(what) + " does not fit 32 bits");
  return (int32_t)v;
}

void* stream_of(c10::Device d) { return c10::cuda::getCurrentCUDAStream(d.index()).stream(); }

Tensor bytes(size_t n, c10::Device d) { return at::empty({(int64_t)(n < 16 ? 16 : n)}, at::TensorOptions().dtype(at::kByte).device(d)); }

// ------------------------------------------------------------------------------------------ rotary positions, head norms
struct RopePlan {
  int32_t d, r;
  bool interleaved;
  float factor;
  Maybe turns;
};

struct QkCall {
  Like like;
  int64_t B, Hq, n, d, Hk;
  int64_t qs[4], ks[4];
  ln_rope p;
  QkCall(const RopePlan& rope, const Tensor& Q, const Maybe& K, const Maybe& pos, int64_t start) : like(Q), B(Q.size(0)), Hq(Q.size(1)), n(Q.size(2)), d(Q.size(3)), Hk(0) {
    if (K) {
      if (K->dim() != 4) refuse("K must be [B, H, n, d]");
      Hk = K->size(1);
    }
    if (d != rope.d) refuse("Rope of " + std::to_string(rope.d) + " channels for heads of " + std::to_string(d));
    const int64_t q[4] = {B, Hq, n, d}, k[4] = {B, Hk, n, d};
    std::copy(q, q + 4, qs);
    std::copy(k, k + 4, ks);
    if (rope.turns && rope.turns->device() != like.device) refuse("Rope on " + rope.turns->device().str() + " for tensors on " + like.device.str());
    p = ln_rope{rope.d, rope.r, rope.interleaved ? 1 : 0, like.dtype, rope.turns ? reinterpret_cast<const uint64_t*>(rope.turns->data_ptr()) : nullptr,
                rope.factor, nullptr, 0, 0, narrow(start, "start")};
    if (pos) {
      const int64_t dim = pos->dim();
      if (pos->scalar_type() != at::kInt || pos->device() != like.device || dim < 1 || dim > 2 || pos->size(dim - 1) != n ||
          (dim == 2 && pos->size(0) != 1 && pos->size(0) != B))
        refuse(std::string("pos: ") + c10::toString(pos->scalar_type()) + " " + text(pos->sizes()) + " on " + pos->device().str() + ", expected int32 [" +
               std::to_string(B) + ", " + std::to_string(n) + "] or [" + std::to_string(n) + "] on " + like.device.str());
      p.pos = static_cast<const int32_t*>(pos->data_ptr());
      p.pos_batch = dim == 2 && pos->size(0) > 1 ? pos->stride(0) : 0;
      p.pos_token = pos->stride(dim - 1);
    }
    narrow(B, "B"); narrow(Hq, "Hq"); narrow(Hk, "Hk"); narrow(n, "n");
  }
  at::IntArrayRef q() const { return {qs, 4}; }
  at::IntArrayRef k() const { return {ks, 4}; }
  Tensor out(const Maybe& given, bool keys, const Tensor& model) const { return given ? *given : at::empty(keys ? k() : q(), model.options()); }
};

py::object or_none(bool have, const Tensor& t) { return have ? py::cast(t) : py::none(); }

py::tuple rope(bool backward, const RopePlan& plan, const Tensor& Q, const Maybe& K, const Maybe& pos, int64_t start, const Maybe& Qo, const Maybe& Ko) {
  const QkCall c(plan, Q, K, pos, start);
  const c10::cuda::CUDAGuard on(c.like.device);
  const Tensor yq = c.out(Qo, false, Q), yk = K ? c.out(Ko, true, Q) : Tensor();
  const ln_view x0 = view("Q", Q, c.q(), c.like), y0 = view("output of Q", yq, c.q(), c.like);
  ln_view x1{}, y1{};
  if (K) { x1 = view("K", *K, c.k(), c.like); y1 = view("output of K", yk, c.k(), c.like); }
  check((backward ? api.rope_bwd_ : api.rope_fwd_)(&c.p, (int32_t)c.B, (int32_t)c.n, (int32_t)c.Hq, (int32_t)c.Hk, &x0, K ? &x1 : nullptr, &y0,
                                                 K ? &y1 : nullptr, stream_of(c.like.device)),
        backward ? "rope_bwd" : "rope_fwd");
  return py::make_tuple(yq, or_none(K.has_value(), yk));
}

py::tuple norm_rope_fwd(const RopePlan& plan, const Tensor& Q, const Maybe& K, const Maybe& gq, const Maybe& gk, double eps, const Maybe& pos, int64_t start,
                        const Maybe& Qo, const Maybe& Ko) {
  const QkCall c(plan, Q, K, pos, start);
  const c10::cuda::CUDAGuard on(c.like.device);
  const float *g0 = vector<float>("gq", gq, at::kFloat, {c.d}, c.like.device), *g1 = vector<float>("gk", gk, at::kFloat, {c.d}, c.like.device);
  const Tensor yq = c.out(Qo, false, Q), yk = K ? c.out(Ko, true, Q) : Tensor();
  const ln_view x0 = view("Q", Q, c.q(), c.like), y0 = view("Qr", yq, c.q(), c.like);
  ln_view x1{}, y1{};
  if (K) { x1 = view("K", *K, c.k(), c.like); y1 = view("Kr", yk, c.k(), c.like); }
  check(api.qkn_fwd(&c.p, (int32_t)c.B, (int32_t)c.n, (int32_t)c.Hq, (int32_t)c.Hk, (float)eps, g0, g1, &x0, K ? &x1 : nullptr, &y0, K ? &y1 : nullptr,
                    stream_of(c.like.device)),
        "qk_norm_rope_fwd");
  return py::make_tuple(yq, or_none(K.has_value(), yk));
}

py::tuple norm_rope_bwd(const RopePlan& plan, const Tensor& Q, const Maybe& K, const Tensor& dQr, const Maybe& dKr, const Maybe& gq, const Maybe& gk, double eps,
                        const Maybe& pos, int64_t start, const Maybe& dQ, const Maybe& dK) {
  const QkCall c(plan, Q, K, pos, start);
  if (K.has_value() != dKr.has_value()) refuse("K and dKr go together");
  const c10::cuda::CUDAGuard on(c.like.device);
  const float *g0 = vector<float>("gq", gq, at::kFloat, {c.d}, c.like.device), *g1 = vector<float>("gk", gk, at::kFloat, {c.d}, c.like.device);
  const Tensor yq = c.out(dQ, false, Q), yk = K ? c.out(dK, true, Q) : Tensor();
  const bool sq = gq.has_value(), sk = gk.has_value() && K.has_value();
  const Tensor dgq = sq ? at::empty_like(*gq) : Tensor(), dgk = sk ? at::empty_like(*gk) : Tensor();
  const ln_view x0 = view("Q", Q, c.q(), c.like), d0 = view("dQr", dQr, c.q(), c.like), y0 = view("dQ", yq, c.q(), c.like);
  ln_view x1{}, d1{}, y1{};
  if (K) { x1 = view("K", *K, c.k(), c.like); d1 = view("dKr", *dKr, c.k(), c.like); y1 = view("dK", yk, c.k(), c.like); }
  const Tensor ws = bytes(sq || sk ? api.qkn_bytes(&c.p, (int32_t)c.B, (int32_t)c.n, (int32_t)c.Hq, (int32_t)c.Hk) : 0, c.like.device);
  check(api.qkn_bwd(&c.p, (int32_t)c.B, (int32_t)c.n, (int32_t)c.Hq, (int32_t)c.Hk, (float)eps, g0, g1, &x0, K ? &x1 : nullptr, &d0, K ? &d1 : nullptr, &y0,
                    K ? &y1 : nullptr, sq ? dgq.data_ptr<float>() : nullptr, sk ? dgk.data_ptr<float>() : nullptr, ws.data_ptr(), (size_t)ws.numel(),
                    stream_of(c.like.device)),
        "qk_norm_rope_bwd");
  return py::make_tuple(yq, or_none(K.has_value(), yk), or_none(sq, dgq), or_none(sk, dgk));
}

// ------------------------------------------------------------------------------------------ softmax attention
struct SmPlan {                                        // the fields of SoftmaxAttention
  std::optional<double> scale;
  double cap;
  bool causal;
  Maybe prefix, slopes, doc_q, doc_k, kv_len;
};

struct SmCall {
  Like like;
  int64_t qs[4], ks[4];
  ln_softmax p;
  SmCall(const SmPlan& s, const Tensor& Q, const Tensor& K) : like(Q) {
    if (K.dim() != 4) refuse("K must be [B, H, n, d]");
    const int64_t B = Q.size(0), Hq = Q.size(1), nq = Q.size(2), d = Q.size(3), Hk = K.size(1), nk = K.size(2);
    const int64_t q[4] = {B, Hq, nq, d}, k[4] = {B, Hk, nk, d};
    std::copy(q, q + 4, qs);
    std::copy(k, k + 4, ks);
    const auto ints = [&](const char* name, const Maybe& t, at::IntArrayRef shape) { return vector<int32_t>(name, t, at::kInt, shape, like.device); };
    p = ln_softmax{narrow(B, "B"), narrow(Hq, "Hq"), narrow(Hk, "Hk"), narrow(nq, "nq"), narrow(nk, "nk"), narrow(d, "d"), like.dtype,
                   (float)(s.scale ? *s.scale : 1.0 / std::sqrt((double)(d > 0 ? d : 1))), (float)s.cap, s.causal ? 1 : 0, ints("prefix", s.prefix, {B}),
                   ints("kv_len", s.kv_len, {B}), vector<float>("slopes", s.slopes, at::kFloat, {Hq}, like.device), ints("doc_q", s.doc_q, {B, nq}),
                   ints("doc_k", s.doc_k, {B, nk})};
  }
  at::IntArrayRef q() const { return {qs, 4}; }
  at::IntArrayRef k() const { return {ks, 4}; }
  Tensor workspace(const Maybe& given, int backward) const {
    if (!given) return bytes(api.sm_bytes(&p, backward), like.device);
    if (given->device() != like.device || given->scalar_type() != at::kByte || !given->is_contiguous()) refuse("ws: expected a contiguous uint8 tensor on " + like.device.str());
    return *given;
  }
  int32_t* status(const Maybe& t) const { return vector<int32_t>("dev_status", t, at::kInt, {qs[0] * qs[1]}, like.device); }
};

int64_t softmax_bytes(const SmPlan& s, const Tensor& Q, const Tensor& K, bool backward) {
  const SmCall c(s, Q, K);
  return (int64_t)api.sm_bytes(&c.p, backward ? 1 : 0);
}

py::tuple softmax_fwd(const SmPlan& s, const Tensor& Q, const Tensor& K, const Tensor& V, const Maybe& O, const Maybe& lse, const Maybe& ws, const Maybe& dev_status) {
  const SmCall c(s, Q, K);
  const c10::cuda::CUDAGuard on(c.like.device);
  const at::IntArrayRef rows(c.qs, 3);
  const Tensor o = O ? *O : at::empty(c.q(), Q.options()), l = lse ? *lse : at::empty(rows, Q.options().dtype(at::kFloat)), w = c.workspace(ws, 0);
  const ln_view q = view("Q", Q, c.q(), c.like), k = view("K", K, c.k(), c.like), v = view("V", V, c.k(), c.like), y = view("O", o, c.q(), c.like);
  check(api.sm_fwd(&c.p, &q, &k, &v, &y, vector<float>("lse", l, at::kFloat, rows, c.like.device), w.data_ptr(), (size_t)w.numel(), c.status(dev_status),
                   stream_of(c.like.device)),
        "softmax_attention_fwd");
  return py::make_tuple(o, l);
}

py::tuple softmax_bwd(const SmPlan& s, const Tensor& Q, const Tensor& K, const Tensor& V, const Tensor& O, const Tensor& lse, const Tensor& dO, const Maybe& dQ,
                      const Maybe& dK, const Maybe& dV, const Maybe& ws, const Maybe& dev_status) {
  const SmCall c(s, Q, K);
  const c10::cuda::CUDAGuard on(c.like.device);
  const Tensor gq = dQ ? *dQ : at::empty(c.q(), Q.options()), gk = dK ? *dK : at::empty(c.k(), Q.options()), gv = dV ? *dV : at::empty(c.k(), Q.options());
  const Tensor w = c.workspace(ws, 1);
  const ln_view q = view("Q", Q, c.q(), c.like), k = view("K", K, c.k(), c.like), v = view("V", V, c.k(), c.like), o = view("O", O, c.q(), c.like),
                g = view("dO", dO, c.q(), c.like), a = view("dQ", gq, c.q(), c.like), b = view("dK", gk, c.k(), c.like), e = view("dV", gv, c.k(), c.like);
  check(api.sm_bwd(&c.p, &q, &k, &v, &o, vector<float>("lse", lse, at::kFloat, {c.qs, 3}, c.like.device), &g, &a, &b, &e, w.data_ptr(), (size_t)w.numel(),
                   c.status(dev_status), stream_of(c.like.device)),
        "softmax_attention_bwd");
  return py::make_tuple(gq, gk, gv);
}

// Addresses of the C ABI by name, from the library that the package has loaded, and its error class.
void bind(const py::dict& at, const py::object& error) {
  const auto put = [&](const char* name, auto& fn) { fn = reinterpret_cast<std::remove_reference_t<decltype(fn)>>(at[name].cast<uintptr_t>()); };
  put("rope_fwd", api.rope_fwd_);
  put("rope_bwd", api.rope_bwd_);
  put("qk_norm_rope_fwd", api.qkn_fwd);
  put("qk_norm_rope_bwd_workspace_bytes", api.qkn_bytes);
  put("qk_norm_rope_bwd", api.qkn_bwd);
  put("softmax_attention_workspace_bytes", api.sm_bytes);
  put("softmax_attention_fwd", api.sm_fwd);
  put("softmax_attention_bwd", api.sm_bwd);
  api.error = error.inc_ref().ptr();
}

}  // namespace

PYBIND11_MODULE(TORCH_EXTENSION_NAME, m) {
  m.def("bind", &bind);
  py::class_<RopePlan>(m, "RopePlan").def(py::init([](int32_t d, int32_t r, bool interleaved, double factor, const Maybe& turns) {
    return RopePlan{d, r, interleaved, (float)factor, turns};
  }));
  py::class_<SmPlan>(m, "SmPlan").def(py::init([](std::optional<double> scale, double cap, bool causal, const Maybe& prefix, const Maybe& slopes, const Maybe& doc_q,
                                                 const Maybe& doc_k, const Maybe& kv_len) {
    return SmPlan{scale, cap, causal, prefix, slopes, doc_q, doc_k, kv_len};
  }));
  m.def("rope", &rope);
  m.def("qk_norm_rope_fwd", &norm_rope_fwd);
  m.def("qk_norm_rope_bwd", &norm_rope_bwd);
  m.def("softmax_bytes", &softmax_bytes);
  m.def("softmax_fwd", &softmax_fwd);
  m.def("softmax_bwd", &softmax_bwd);
}
