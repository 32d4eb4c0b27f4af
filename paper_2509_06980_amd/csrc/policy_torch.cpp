// The policy update's operators on torch tensors: checks of the arguments, results and workspaces from torch's allocator, then the
// calls of include/rl_rollout.h.  Host code only; small calls take as long as their launch, so it is compiled.
#include <ATen/ATen.h>
#include <ATen/MemoryOverlap.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/utils/pybind.h>

#include <optional>
#include <string>
#include <tuple>

#include "../../include/rl_rollout.h"

namespace py = pybind11;
using at::Tensor;
using Maybe = std::optional<Tensor>;

namespace {

struct Refused {
  int code;
  std::string message;
};
void check(bool ok, const char* message) {
  if (!ok) throw Refused{RL_E_ARG, message};
}
void done(int rc) {
  if (rc != RL_OK) throw Refused{rc, rl_last_error()};
}

// the element type of a call's tensors, all of one type on one GPU
int type_of(const Tensor& x) {
  check(x.scalar_type() == at::kFloat || x.scalar_type() == at::kBFloat16, "tensors have to be float32 or bfloat16");
  check(x.is_cuda(), "tensors have to be on the GPU");
  return x.scalar_type() == at::kFloat ? RL_DTYPE_F32 : RL_DTYPE_BF16;
}
void like(const Tensor& x, const Tensor& first) {
  check(x.scalar_type() == first.scalar_type() && x.device() == first.device(), "tensors of one call have one type and one device");
}
void plain(const Tensor& x, at::ScalarType type, const Tensor& first, const char* message) {
  check(x.scalar_type() == type && x.device() == first.device() && x.is_contiguous(), message);
}
Tensor fresh(at::IntArrayRef shape, const Tensor& first) { return at::empty(shape, first.options()); }
Tensor floats(at::IntArrayRef shape, const Tensor& first) { return at::empty(shape, first.options().dtype(at::kFloat)); }
Tensor bytes(int64_t n, const Tensor& first) { return at::empty({std::max<int64_t>(n, 1)}, first.options().dtype(at::kByte)); }
void* at_stream(int64_t stream) { return reinterpret_cast<void*>(stream); }
bool rows_contiguous(const Tensor& x) { return x.dim() > 0 && (x.stride(-1) == 1 || x.size(-1) <= 1); }
int32_t small(int64_t n, const char* message) {
  check(n >= 0 && n <= 0x7fffffff, message);
  return (int32_t)n;
}

// Rows of x in two steps of strides; a copy only where two cannot say where they are.
struct Rows {
  Tensor x;
  int64_t outer, outer_stride, inner_stride;
  int32_t inner, width;
};
Rows rows_of(const Tensor& x) {
  const int64_t w = x.size(-1);
  if (x.is_contiguous() || !rows_contiguous(x) || x.dim() > 3) {
    const Tensor c = x.contiguous();
    return {c, w ? c.numel() / w : 0, w, 0, 1, small(w, "rows are too long")};
  }
  if (x.dim() < 3) return {x, x.dim() == 2 ? x.size(0) : 1, x.dim() == 2 ? x.stride(0) : w, 0, 1, small(w, "rows are too long")};
  return {x, x.size(0), x.stride(0), x.stride(1), small(x.size(1), "too many rows in one group"), small(w, "rows are too long")};
}

std::tuple<Tensor, Maybe, Tensor> norm_forward(const Tensor& x, const Tensor& weight, const Maybe& bias, double eps, bool centered,
                                               int64_t stream) {
  const int dt = type_of(x);
  like(weight, x);
  check(x.dim() >= 1 && weight.dim() == 1 && weight.size(0) == x.size(-1) && weight.is_contiguous(), "weight has to be contiguous, of the length of a row");
  if (bias) {
    like(*bias, x);
    check(bias->sizes() == weight.sizes() && bias->is_contiguous(), "bias has to be contiguous, of the length of a row");
  }
  const c10::DeviceGuard guard(x.device());
  const Rows r = rows_of(x);
  Tensor y = fresh(x.sizes(), x), rstd = floats(x.sizes().slice(0, x.dim() - 1), x);
  Maybe mean;
  if (centered) mean = at::empty_like(rstd);
  if (r.inner > 0 && r.width > 0)
    done(rl_norm_forward(r.x.data_ptr(), r.outer, r.inner, r.width, r.outer_stride, r.inner_stride, weight.data_ptr(),
                         bias ? bias->data_ptr() : nullptr, (float)eps, centered, dt, y.data_ptr(), mean ? mean->data_ptr<float>() : nullptr,
                         rstd.data_ptr<float>(), at_stream(stream)));
  return {y, mean, rstd};
}

std::tuple<Tensor, Tensor, Maybe> norm_backward(const Tensor& dy, const Tensor& x, const Tensor& weight, const Maybe& mean, const Tensor& rstd,
                                                bool centered, bool biased, int64_t stream) {
  const int dt = type_of(x);
  like(dy, x);
  like(weight, x);
  check(x.dim() >= 1 && dy.sizes() == x.sizes(), "dy has to have x's shape");
  check(weight.dim() == 1 && weight.size(0) == x.size(-1) && weight.is_contiguous(), "weight has to be contiguous, of the length of a row");
  plain(rstd, at::kFloat, x, "rstd has to be contiguous float32 on the same GPU");
  check(rstd.sizes() == x.sizes().slice(0, x.dim() - 1), "rstd is one number a row");
  if (centered) {
    check(mean.has_value() && mean->sizes() == rstd.sizes(), "mean is one number a row");
    plain(*mean, at::kFloat, x, "mean has to be contiguous float32 on the same GPU");
  }
  const c10::DeviceGuard guard(x.device());
  Rows r = rows_of(x), d = rows_of(dy);
  if (r.inner != d.inner) {      // one of the two lies in two steps: the other, contiguous, in the same two
    const int64_t n = std::max(r.inner, d.inner), w = r.width;
    const int64_t outer = n ? r.x.numel() / std::max<int64_t>(w, 1) / n : 0;
    Rows& flat = r.inner < d.inner ? r : d;
    flat = {flat.x, outer, n * w, w, (int32_t)n, flat.width};
  }
  Tensor dx = fresh(x.sizes(), x), dweight = at::empty_like(weight);
  Maybe dbias;
  if (biased) dbias = at::empty_like(weight);
  const int64_t n = rl_norm_workspace(r.outer * r.inner, r.width, biased);
  const Tensor ws = bytes(n, x);
  if (r.width > 0)
    done(rl_norm_backward(d.x.data_ptr(), d.outer_stride, d.inner_stride, r.x.data_ptr(), r.inner ? r.outer : 0, std::max(r.inner, 1), r.width,
                          r.outer_stride, r.inner_stride, weight.data_ptr(), centered ? mean->data_ptr<float>() : nullptr, rstd.data_ptr<float>(),
                          centered, dt, dx.data_ptr(), dweight.data_ptr(), biased ? dbias->data_ptr() : nullptr, ws.data_ptr(), n,
                          at_stream(stream)));
  return {dx, dweight, dbias};
}

std::tuple<Tensor, Maybe> rotary(const Tensor& q, const Maybe& k, const Tensor& positions, const Tensor& table, bool interleaved, bool inverse,
                                 const Maybe& q_out, const Maybe& k_out, int64_t stream) {
  const int dt = type_of(q);
  check(q.dim() == 3, "q is [tokens, heads, head_dim]");
  if (k) {
    like(*k, q);
    check(k->dim() == 3 && k->size(0) == q.size(0) && k->size(2) == q.size(2), "k is [tokens, heads, head_dim]");
  }
  plain(positions, at::kInt, q, "positions have to be contiguous int32 on the same GPU");
  plain(table, at::kFloat, q, "table has to be contiguous float32 on the same GPU");
  check(positions.dim() == 1 && positions.size(0) == q.size(0), "one position a token");
  check(table.dim() == 3 && table.size(2) == 2 && 2 * table.size(1) <= q.size(2), "table is [positions, rot_dim / 2, 2], rot_dim at most head_dim");
  const c10::DeviceGuard guard(q.device());
  auto in = [](const Tensor& x) { return rows_contiguous(x) ? x : x.contiguous(); };
  auto out = [&](const Tensor& x, const Maybe& given) {
    if (!given) return fresh(x.sizes(), x);
    like(*given, q);
    check(given->sizes() == x.sizes() && rows_contiguous(*given), "an output has its input's shape and contiguous heads");
    // written behind autograd's back: no gradient may be wanted of it, none of its elements may share memory
    check(!(c10::GradMode::is_enabled() && given->requires_grad()), "an output that requires a gradient (use rotate)");
    check(at::has_internal_overlap(*given) != at::MemOverlap::Yes, "elements of an output share memory");
    return *given;
  };
  const Tensor a = in(q), y = out(q, q_out);
  Tensor b, z;
  if (k) b = in(*k), z = out(*k, k_out);
  // whoever kept the old contents for a backward pass is told
  for (const Maybe& given : {q_out, k ? k_out : Maybe()})
    if (given) given->unsafeGetTensorImpl()->bump_version();
  auto stride = [](const Tensor& x, int i) { return x.defined() ? x.stride(i) : 0; };
  if (a.size(1) > 0)
    done(rl_rotary(a.data_ptr(), y.data_ptr(), small(a.size(1), "too many heads"), a.stride(0), a.stride(1), y.stride(0), y.stride(1),
                   k ? b.data_ptr() : nullptr, k ? z.data_ptr() : nullptr, k ? small(b.size(1), "too many heads") : 0, stride(b, 0), stride(b, 1),
                   stride(z, 0), stride(z, 1), a.size(0), small(a.size(2), "heads are too long"), small(2 * table.size(1), "heads are too long"),
                   interleaved, inverse, positions.data_ptr<int32_t>(), table.data_ptr<float>(), small(table.size(0), "too many positions"), dt,
                   at_stream(stream)));
  return {y, k ? Maybe(z) : Maybe()};
}

// What both directions of attention check and pass on.
struct Packed {
  Tensor q, k, v;
  int dt;
  int32_t n_seq, total_q, total_k, nq, nkv, d;
  float scale;
};
Packed packed(const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& cu_q, const Tensor& cu_k, const std::optional<double>& scale) {
  const int dt = type_of(q);
  like(k, q);
  like(v, q);
  check(q.dim() == 3 && k.dim() == 3 && v.sizes() == k.sizes() && k.size(2) == q.size(2), "q is [tokens, heads, head_dim], k and v [tokens, KV heads, head_dim]");
  plain(cu_q, at::kInt, q, "cu_q has to be contiguous int32 on the same GPU");
  plain(cu_k, at::kInt, q, "cu_k has to be contiguous int32 on the same GPU");
  check(cu_q.dim() == 1 && cu_q.sizes() == cu_k.sizes() && cu_q.size(0) >= 1, "cu_q and cu_k are offsets of the same sequences");
  auto in = [](const Tensor& x) { return rows_contiguous(x) ? x : x.contiguous(); };
  const double d = q.size(2) > 0 ? 1.0 / std::sqrt((double)q.size(2)) : 1.0;
  return {in(q), in(k), in(v), dt, small(cu_q.size(0) - 1, "too many sequences"), small(q.size(0), "too many tokens"), small(k.size(0), "too many tokens"),
          small(q.size(1), "too many heads"), small(k.size(1), "too many heads"), small(q.size(2), "heads are too long"), (float)scale.value_or(d)};
}

std::tuple<Tensor, Tensor> attention_forward(const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& cu_q, const Tensor& cu_k, bool causal,
                                             const std::optional<double>& scale, int64_t stream) {
  const Packed p = packed(q, k, v, cu_q, cu_k, scale);
  const c10::DeviceGuard guard(q.device());
  Tensor o = fresh(q.sizes(), q), lse = floats({q.size(1), q.size(0)}, q);
  done(rl_attention_forward(p.q.data_ptr(), p.q.stride(0), p.q.stride(1), p.k.data_ptr(), p.k.stride(0), p.k.stride(1), p.v.data_ptr(),
                            p.v.stride(0), p.v.stride(1), cu_q.data_ptr<int32_t>(), cu_k.data_ptr<int32_t>(), p.n_seq, p.total_q, p.total_k, p.nq,
                            p.nkv, p.d, p.scale, causal, p.dt, o.data_ptr(), lse.data_ptr<float>(), at_stream(stream)));
  return {o, lse};
}

std::tuple<Tensor, Tensor, Tensor> attention_backward(const Tensor& dout, const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& o,
                                                      const Tensor& lse, const Tensor& cu_q, const Tensor& cu_k, bool causal,
                                                      const std::optional<double>& scale, int64_t stream) {
  const Packed p = packed(q, k, v, cu_q, cu_k, scale);
  like(dout, q);
  like(o, q);
  check(dout.sizes() == q.sizes() && o.sizes() == q.sizes(), "do and o have to have q's shape");
  plain(lse, at::kFloat, q, "lse has to be contiguous float32 on the same GPU");
  check(lse.dim() == 2 && lse.size(0) == q.size(1) && lse.size(1) == q.size(0), "lse is [heads, tokens]");
  const c10::DeviceGuard guard(q.device());
  const Tensor g = dout.contiguous(), oc = o.contiguous();
  Tensor dq = fresh(q.sizes(), q), dk = fresh(k.sizes(), q), dv = fresh(v.sizes(), q);
  const int64_t n = rl_attention_fast_workspace(p.n_seq, p.total_q, p.total_k, p.nq, p.nkv, p.d, p.dt);
  const Tensor ws = bytes(n, q);
  done(rl_attention_backward(g.data_ptr(), p.q.data_ptr(), p.q.stride(0), p.q.stride(1), p.k.data_ptr(), p.k.stride(0), p.k.stride(1),
                             p.v.data_ptr(), p.v.stride(0), p.v.stride(1), oc.data_ptr(), lse.data_ptr<float>(), cu_q.data_ptr<int32_t>(),
                             cu_k.data_ptr<int32_t>(), p.n_seq, p.total_q, p.total_k, p.nq, p.nkv, p.d, p.scale, causal, p.dt, dq.data_ptr(),
                             dk.data_ptr(), dv.data_ptr(), ws.data_ptr(), n, at_stream(stream)));
  return {dq, dk, dv};
}

int head(const Tensor& hidden, const Tensor& weight, const Tensor& targets) {
  const int dt = type_of(hidden);
  like(weight, hidden);
  check(hidden.dim() == 2 && weight.dim() == 2 && weight.size(1) == hidden.size(1) && targets.dim() == 1 && targets.size(0) == hidden.size(0),
        "hidden is [rows, hidden], weight [vocab, hidden], targets [rows]");
  check(weight.is_contiguous(), "weight has to be contiguous");
  plain(targets, at::kInt, hidden, "targets have to be contiguous int32 on the same GPU");
  return dt;
}

std::tuple<Tensor, Tensor> token_logprobs_forward(const Tensor& hidden, const Tensor& weight, const Tensor& targets, double temperature,
                                                  int64_t stream) {
  const int dt = head(hidden, weight, targets);
  const c10::DeviceGuard guard(hidden.device());
  const Tensor h = rows_contiguous(hidden) ? hidden : hidden.contiguous();
  Tensor logp = floats({hidden.size(0)}, hidden), lse = floats({hidden.size(0)}, hidden);
  const int32_t rows = small(h.size(0), "too many rows"), width = small(h.size(1), "rows are too long"), vocab = small(weight.size(0), "vocabulary too large");
  const int64_t n = rl_token_logprobs_workspace(rows, width, vocab, dt, 0);
  const Tensor ws = bytes(n, hidden);
  done(rl_token_logprobs_forward(h.data_ptr(), h.stride(0), rows, width, weight.data_ptr(), vocab, targets.data_ptr<int32_t>(), (float)temperature, dt,
                                 logp.data_ptr<float>(), lse.data_ptr<float>(), ws.data_ptr(), n, at_stream(stream)));
  return {logp, lse};
}

std::tuple<Tensor, Tensor> token_logprobs_backward(const Tensor& dlogp, const Tensor& hidden, const Tensor& weight, const Tensor& targets,
                                                   const Tensor& lse, double temperature, int64_t stream) {
  const int dt = head(hidden, weight, targets);
  plain(dlogp, at::kFloat, hidden, "dlogp has to be contiguous float32 on the same GPU");
  plain(lse, at::kFloat, hidden, "lse has to be contiguous float32 on the same GPU");
  check(dlogp.sizes() == targets.sizes() && lse.sizes() == targets.sizes(), "dlogp and lse are one number a row");
  const c10::DeviceGuard guard(hidden.device());
  const Tensor h = rows_contiguous(hidden) ? hidden : hidden.contiguous();
  Tensor dhidden = fresh(hidden.sizes(), hidden), dweight = fresh(weight.sizes(), hidden);
  const int32_t rows = small(h.size(0), "too many rows"), width = small(h.size(1), "rows are too long"), vocab = small(weight.size(0), "vocabulary too large");
  const int64_t n = rl_token_logprobs_workspace(rows, width, vocab, dt, 1);
  const Tensor ws = bytes(n, hidden);
  done(rl_token_logprobs_backward(dlogp.data_ptr<float>(), h.data_ptr(), h.stride(0), rows, width, weight.data_ptr(), vocab,
                                  targets.data_ptr<int32_t>(), lse.data_ptr<float>(), (float)temperature, dt, dhidden.data_ptr(), dweight.data_ptr(),
                                  ws.data_ptr(), n, at_stream(stream)));
  return {dhidden, dweight};
}

}  // namespace

PYBIND11_MODULE(_policy_torch, m) {
  static py::object error = py::module_::import("paper_2509_06980_amd.binding").attr("RolloutError");
  py::register_exception_translator([](std::exception_ptr p) {
    try {
      if (p) std::rethrow_exception(p);
    } catch (const Refused& r) {
      PyErr_SetObject(error.ptr(), error(r.code, r.message).ptr());
    }
  });
  m.def("norm_forward", &norm_forward);
  m.def("norm_backward", &norm_backward);
  m.def("rotary", &rotary);
  m.def("attention_forward", &attention_forward);
  m.def("attention_backward", &attention_backward);
  m.def("token_logprobs_forward", &token_logprobs_forward);
  m.def("token_logprobs_backward", &token_logprobs_backward);
}
