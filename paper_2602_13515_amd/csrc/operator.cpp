// The differentiable operators in native code, as autograd functions over the C ABI: block-sparse attention (pattern from q
// and k, forward, backward) and the velocity distillation loss, with the results, checks and errors of the Python functions in
// autograd.py and distill.py, which stay for the calls that this module does not take (a pattern asked for, overlapping
// backward kernels, tracing, function transforms, tensors that are not plain CUDA tensors); and the operators around the
// attention (block.py), which have no other route.
//
// Why: the Python route cost more host time than the kernels take on small layers.  Two heads of 2,048 tokens, forward and
// backward: 82 us of kernels and the gaps between them, 226 us a pass, in which the backward pass waited for the
// interpreter lock twice.  Here a pass allocates one buffer for the pattern (six tensors before) and one scratch buffer for
// mask and forward, and the backward pass runs in the engine's thread without the interpreter: 90 us (82 with the
// kernels as they are now).  24 heads of 1,281 tokens 223 -> 133 us (116); sampling on 1,000 tokens, two heads 46 -> 28 us (17).
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPGraphsC10Utils.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/extension.h>

#include <unordered_set>

#include "spa2.h"

namespace {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::Variable;
using torch::autograd::variable_list;

// A negative return code of the C ABI as the exception the Python binding raises for it.
void check(int code, const char* where) {
  if (code == SPA2_OK) return;
  py::gil_scoped_acquire gil;
  const py::object e = py::module_::import("paper_2602_13515_amd.binding").attr("Spa2Error")(code, where);
  PyErr_SetObject((PyObject*)Py_TYPE(e.ptr()), e.ptr());
  throw py::error_already_set();
}

void* stream_of(const Tensor& x) { return (void*)c10::hip::getCurrentHIPStream(x.device().index()).stream(); }

Tensor like(const Tensor& x) { return at::empty_strided(x.sizes(), x.strides(), x.options()); }

Tensor bytes(int64_t n, const Tensor& x) { return at::empty({n}, x.options().dtype(at::kByte)); }

// x with ref's strides (the kernels take one stride triple for all token tensors of a call).
Tensor match(const Tensor& x, const Tensor& ref) {
  if (x.strides() == ref.strides()) return x;
  Tensor y = like(ref);
  y.copy_(x);
  return y;
}

// Whether x starts where the kernels read 16 bytes at a time.  (Upstream gradients need not: the backward of a concatenation
// hands out views of its buffer at any element.)
bool aligned(const Tensor& x) { return (reinterpret_cast<uintptr_t>(x.data_ptr()) & 15) == 0; }

constexpr const char* ONE_LAYOUT = "all token tensors of one call share shape, strides, dtype and device";

void same_layout(const Tensor& ref, std::initializer_list<const Tensor*> others) {
  for (const Tensor* t : others)
    TORCH_CHECK_VALUE(t->sizes() == ref.sizes() && t->strides() == ref.strides() &&
                      t->scalar_type() == ref.scalar_type() && t->device() == ref.device(), ONE_LAYOUT);
}

void check_inputs(const Tensor& q, const Tensor& k, const Tensor& v) {
  const std::pair<const char*, const Tensor*> named[] = {{"q", &q}, {"k", &k}, {"v", &v}};
  for (const auto& [name, t] : named) {
    TORCH_CHECK_VALUE(t->is_cuda(), name, " must live on the GPU: the operator has no CPU path");
    TORCH_CHECK_VALUE(t->scalar_type() == at::kBFloat16 && t->dim() == 4, name, " must be a bf16 [B, H, N, d] view");
  }
  TORCH_CHECK_VALUE(k.sizes() == q.sizes() && v.sizes() == q.sizes(), "self-attention: q, k, v share one shape");
  TORCH_CHECK_VALUE(q.stride(3) == 1, "the head dimension must be contiguous");
  TORCH_CHECK_VALUE(k.device() == q.device() && v.device() == q.device(), ONE_LAYOUT);
}

// What saved-tensor hooks bring back is checked before a kernel gets its address.  (The sizes are those of the upstream
// gradient, which the engine has compared with the output's.)
void check_saved(const Tensor& q, const Tensor& lse, int64_t gpu) {
  TORCH_CHECK_VALUE(q.is_cuda() && q.device().index() == gpu && q.scalar_type() == at::kBFloat16 && q.dim() == 4 &&
                    q.stride(3) == 1, "saved token tensors come back as bf16 [B, H, N, d] views on their GPU, d contiguous");
  TORCH_CHECK_VALUE(lse.device() == q.device() && lse.scalar_type() == at::kFloat && lse.is_contiguous() &&
                    lse.numel() == q.size(0) * q.size(1) * q.size(2), "the log-sum-exp comes back as B * H * N contiguous fp32 numbers");
}

spa2_shape shape_of(const Tensor& q) {
  spa2_shape s;
  s.B = (int32_t)q.size(0); s.H = (int32_t)q.size(1); s.N = (int32_t)q.size(2); s.d = (int32_t)q.size(3);
  s.bq = SPA2_BQ; s.bkv = SPA2_BKV;
  s.sb = q.stride(0); s.sh = q.stride(1); s.sn = q.stride(2);
  return s;
}

// The arrays of a pattern of our own in one buffer.  The backward pass makes the column lists (spa2_bwd_rows).
struct PatternLayout {
  int64_t off[3] = {0, 0, 0}, total = 0;
  explicit PatternLayout(const spa2_shape& s) {
    const int64_t bh = (int64_t)s.B * s.H;
    const int64_t tm = ((int64_t)s.N + SPA2_BQ - 1) / SPA2_BQ, tn = ((int64_t)s.N + SPA2_BKV - 1) / SPA2_BKV;
    const int64_t size[3] = {bh * tm * tn, 4 * bh * tm, 4 * bh * tm * tn};
    for (int x = 0; x < 3; ++x) { off[x] = total; total += (size[x] + 255) & ~(int64_t)255; }
  }
  spa2_pattern in(const Tensor& buf) const {
    char* p = (char*)buf.data_ptr();
    spa2_pattern r = {};
    r.mask = (uint8_t*)(p + off[0]);
    r.row_cnt = (int32_t*)(p + off[1]); r.row_idx = (int32_t*)(p + off[2]);
    return r;
  }
};

// A caller's pattern: mask, row_cnt, row_idx, col_cnt, col_idx, row_order, col_order (undefined: not there).
spa2_pattern given_pattern(const std::vector<Tensor>& t) {
  auto at = [&](int x) -> void* { return t[x].defined() ? t[x].data_ptr() : nullptr; };
  spa2_pattern r;
  r.mask = (uint8_t*)at(0);
  r.row_cnt = (int32_t*)at(1); r.row_idx = (int32_t*)at(2);
  r.col_cnt = (int32_t*)at(3); r.col_idx = (int32_t*)at(4);
  r.row_order = (int32_t*)at(5); r.col_order = (int32_t*)at(6);
  return r;
}

struct Attention : torch::autograd::Function<Attention> {
  static Tensor forward(AutogradContext* ctx, const Tensor& q, const Tensor& k_in, const Tensor& v_in, double k_frac,
                        double top_p, double scale, bool training, const std::vector<Tensor>& given) {
    const c10::DeviceGuard device(q.device());
    const Tensor k = match(k_in, q), v = match(v_in, q);
    const spa2_shape s = shape_of(q);
    const bool build = given.empty();
    const PatternLayout layout(s);
    const Tensor buf = build ? bytes(layout.total, q) : Tensor();
    spa2_pattern pattern = build ? layout.in(buf) : given_pattern(given);
    // one scratch buffer for mask and forward; a log-sum-exp that nobody reads lies behind it
    const int64_t need = (int64_t)(build ? spa2_mask_fwd_workspace_bytes(&s) : spa2_fwd_workspace_bytes(&s));
    const int64_t lse_at = (need + 255) & ~(int64_t)255;
    const Tensor ws = bytes(training ? lse_at : lse_at + 4 * q.size(0) * q.size(1) * q.size(2), q);
    void* stream = stream_of(q);
    const int32_t tn = (int32_t)((q.size(2) + SPA2_BKV - 1) / SPA2_BKV);
    const Tensor o = like(q);
    Tensor o_res, lse;
    if (training) {
      o_res = like(q);
      lse = at::empty({q.size(0), q.size(1), q.size(2)}, q.options().dtype(at::kFloat));
    }
    float* lse_p = training ? (float*)lse.data_ptr() : (float*)((char*)ws.data_ptr() + lse_at);
    void* o_res_p = training ? o_res.data_ptr() : nullptr;
    if (build)
      check(spa2_mask_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), &s, spa2_topk_blocks(k_frac, tn), (float)top_p,
                          (float)scale, &pattern, o.data_ptr(), o_res_p, lse_p, ws.data_ptr(), (size_t)need, stream),
            "spa2_mask_fwd");
    else
      check(spa2_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), &s, &pattern, (float)scale, o.data_ptr(), o_res_p, lse_p,
                     ws.data_ptr(), (size_t)need, stream), "spa2_fwd");
    if (training) {
      ctx->save_for_backward({q, k, v, o, o_res, lse});
      ctx->saved_data["pattern"] = build ? std::vector<Tensor>{buf} : given;
      ctx->saved_data["scale"] = scale;
      ctx->saved_data["gpu"] = (int64_t)q.device().index();
    }
    return o;
  }

  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    const variable_list saved = ctx->get_saved_variables();
    const Tensor &q = saved[0], &k = saved[1], &v = saved[2], &o = saved[3], &o_res = saved[4], &lse = saved[5];
    check_saved(q, lse, ctx->saved_data["gpu"].toInt());
    const c10::DeviceGuard device(q.device());
    const Tensor up = grads[0].to(at::kBFloat16), d_o = match(aligned(up) ? up : up.clone(), q);
    // (all of them, not d_o alone: saved-tensor hooks may bring a tensor back in another layout)
    same_layout(q, {&k, &v, &o, &o_res, &d_o});
    const spa2_shape s = shape_of(q);
    const std::vector<Tensor> kept = ctx->saved_data["pattern"].toTensorVector();
    const bool built = kept.size() == 1;
    const spa2_pattern pattern = built ? PatternLayout(s).in(kept[0]) : given_pattern(kept);
    const Tensor dq = like(q), dk = like(q), dv = like(q);
    const int64_t need = (int64_t)(built ? spa2_bwd_rows_workspace_bytes(&s) : spa2_bwd_workspace_bytes(&s));
    const Tensor ws = bytes(need, q);
    check((built ? spa2_bwd_rows : spa2_bwd)(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), o_res.data_ptr(),
                                             d_o.data_ptr(), (const float*)lse.data_ptr(), &s, &pattern,
                                             (float)ctx->saved_data["scale"].toDouble(), dq.data_ptr(), dk.data_ptr(),
                                             dv.data_ptr(), ws.data_ptr(), (size_t)need, stream_of(q)),
          built ? "spa2_bwd_rows" : "spa2_bwd");
    return {dq, dk, dv, Variable(), Variable(), Variable(), Variable(), Variable()};
  }
};

// given: a caller's pattern (see given_pattern), or none: it is built from q and k
Tensor attention(const Tensor& q, const Tensor& k, const Tensor& v, double k_frac, double top_p, double scale,
                 const std::vector<std::optional<Tensor>>& given) {
  check_inputs(q, k, v);
  // Without a backward pass to come (sampling) nobody reads the column lists or the output's residual.
  const bool training = at::GradMode::is_enabled() && (q.requires_grad() || k.requires_grad() || v.requires_grad());
  std::vector<Tensor> pattern;
  for (const auto& t : given) pattern.push_back(t.value_or(Tensor()));
  return Attention::apply(q, k, v, k_frac, top_p, scale, training, pattern);
}

// ------------------------------------------------------------------ velocity distillation loss
int32_t vd_type(const Tensor& x) { return x.scalar_type() == at::kBFloat16 ? 0 : 1; }

void vd_check(const Tensor& us, const Tensor& uf) {
  TORCH_CHECK_VALUE(us.is_cuda() && uf.is_cuda(), "spa2 runs on the GPU only: predictions must be CUDA tensors");
  TORCH_CHECK_VALUE((us.scalar_type() == at::kBFloat16 || us.scalar_type() == at::kFloat) &&
                    uf.scalar_type() == us.scalar_type(), "predictions are bfloat16 or float32, both of the same type");
  TORCH_CHECK_VALUE(us.sizes() == uf.sizes() && us.is_contiguous() && uf.is_contiguous() && us.device() == uf.device(),
                    "predictions are contiguous tensors of one shape");
}

// One pass for the loss, one for the gradient.  (Not spa2_vd_loss_and_grad: what the upstream derivative is, and whether a
// backward pass comes at all, is known only after the loss.  With it, 2 x 201 MB of fp32, us: upstream 1 172 -> 115, but upstream
// 0.5 171 -> 191 and the loss alone 74 -> 111, and a gradient that is multiplied afterwards is rounded once more.)
struct VelocityLoss : torch::autograd::Function<VelocityLoss> {
  static Tensor forward(AutogradContext* ctx, const Tensor& us, const Tensor& uf, double weight) {
    vd_check(us, uf);
    const c10::DeviceGuard device(us.device());
    const Tensor loss = at::empty({}, us.options().dtype(at::kDouble));
    const int64_t n = (int64_t)spa2_vd_loss_workspace_bytes();
    const Tensor ws = bytes(n, us);
    check(spa2_vd_loss(us.data_ptr(), uf.data_ptr(), us.numel(), vd_type(us), weight, (double*)loss.data_ptr(),
                       ws.data_ptr(), (size_t)n, stream_of(us)), "spa2_vd_loss");
    ctx->save_for_backward({us, uf});
    ctx->saved_data["weight"] = weight;
    return loss;
  }

  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    const variable_list saved = ctx->get_saved_variables();
    const Tensor &us = saved[0], &uf = saved[1];
    vd_check(us, uf);
    const c10::DeviceGuard device(us.device());
    const Tensor upstream = grads[0].contiguous();
    TORCH_CHECK_VALUE(upstream.scalar_type() == at::kDouble && upstream.numel() == 1 && upstream.is_cuda(),
                      "upstream is a float64 CUDA tensor of one element");
    const Tensor grad = at::empty_like(us);
    check(spa2_vd_loss_grad(us.data_ptr(), uf.data_ptr(), us.numel(), vd_type(us), ctx->saved_data["weight"].toDouble(),
                            (const double*)upstream.data_ptr(), grad.data_ptr(), stream_of(us)), "spa2_vd_loss_grad");
    return {grad, Variable(), Variable()};
  }
};

Tensor velocity_loss(const Tensor& u_sparse, const Tensor& u_full, double weight) {
  return VelocityLoss::apply(u_sparse.contiguous(), u_full.detach().contiguous(), weight);
}

// ------------------------------------------------------------------ around the attention
using OptTensor = std::optional<Tensor>;

Tensor or_none(const OptTensor& t) { return t.value_or(Tensor()); }
const void* ptr(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
int32_t dtype_of(const Tensor& t) { return t.scalar_type() == at::kBFloat16 ? SPA2_DTYPE_BF16 : SPA2_DTYPE_F32; }
bool float_kind(const Tensor& t) { return t.scalar_type() == at::kBFloat16 || t.scalar_type() == at::kFloat; }

// A [B, H, N, d] tensor without gaps, tokens outside the heads where x has them so (what a projection leaves and takes).
Tensor dense_like(const Tensor& x, at::ScalarType dtype) {
  const int64_t h = x.size(1), n = x.size(2), d = x.size(3);
  const bool tokens_outside = x.stride(2) > x.stride(1);
  return at::empty_strided(x.sizes(), {h * n * d, tokens_outside ? d : n * d, tokens_outside ? h * d : d, 1}, x.options().dtype(dtype));
}
// Whether a call is one that autograd has to see: with a gradient to come, or a tangent (which it refuses).
bool differentiated(std::initializer_list<const Tensor*> inputs) {
  const bool grad = at::GradMode::is_enabled();
  for (const Tensor* t : inputs)
    if (t->defined() && ((grad && t->requires_grad()) || t->_fw_grad(0).defined())) return true;
  return false;
}
// Strides as the kernels read them: a dimension of one element has none.
std::array<int64_t, 3> strides_of(const Tensor& x) {
  std::array<int64_t, 3> s;
  for (int i = 0; i < 3; ++i) s[i] = x.size(i) > 1 ? x.stride(i) : 0;
  return s;
}

// x in the memory order of ref (of another type maybe), from a 16-byte boundary.
Tensor in_order(const Tensor& x, const Tensor& ref) {
  if (x.stride(3) == 1 && strides_of(x) == strides_of(ref) && aligned(x)) return x;
  const Tensor y = at::empty_strided(ref.sizes(), ref.strides(), x.options());
  y.copy_(x);
  return y;
}

// The results of a backward pass, which is no differentiable function itself: differentiating them is an error, not zero.
variable_list once(variable_list grads, bool graph, const char* name) {
  if (!graph) return grads;
  variable_list there;
  for (const auto& g : grads) if (g.defined()) there.push_back(g.detach().requires_grad_());
  const int64_t n = (int64_t)there.size();
  const auto error = std::make_shared<torch::autograd::DelayedError>(std::string(name) + " has no second derivative", n);
  const at::AutoGradMode with_graph(true);
  const variable_list out = (*error)(std::move(there));
  size_t at = 0;
  for (auto& g : grads) if (g.defined()) g = out[at++];
  return grads;
}

// A backward pass that is captured while an eager graph of the same leaf lives would hand that leaf's gradient to the stream
// the eager graph was made on.  If that is the default stream, which cannot take part in a capture, this breaks the capture and
// with it the process: refused here, before anything is captured, for the inputs and all that they were computed from.
// (Other streams are joined to the capture, as that of a warm-up whose loss is still held.)
void capture_check(const Tensor& on, std::initializer_list<Tensor> inputs) {
  if (!at::GradMode::is_enabled()) return;
  const c10::DeviceGuard device(on.device());
  if (c10::hip::currentStreamCaptureStatusMayInitCtx() == c10::hip::CaptureStatus::None) return;
  const auto eager = c10::hip::getDefaultHIPStream();
  std::vector<std::shared_ptr<torch::autograd::Node>> open;
  std::unordered_set<const torch::autograd::Node*> seen;
  auto visit = [&](const std::shared_ptr<torch::autograd::Node>& node) {
    if (node && seen.insert(node.get()).second) open.push_back(node);
  };
  for (const Tensor& t : inputs)
    if (t.defined() && t.requires_grad()) visit(t.is_leaf() ? torch::autograd::impl::try_get_grad_accumulator(t) : t.grad_fn());
  while (!open.empty()) {
    const std::shared_ptr<torch::autograd::Node> node = std::move(open.back());
    open.pop_back();
    const auto made_on = node->stream();
    TORCH_CHECK(!made_on || made_on->id() != eager.id() || made_on->device_index() != eager.device_index(),
                "an eager graph of one of the inputs, or of what they were computed from, is still alive: let go of its outputs "
                "before capturing a backward pass (or capture without gradients)");
    for (const auto& edge : node->next_edges()) visit(edge.function);
  }
}

struct NormShape {
  spa2_norm_shape s = {};
  NormShape(const Tensor& q, const Tensor& k, const Tensor& cos, const Tensor& positions, bool interleaved, const Tensor& qo,
            const Tensor& ko) {
    s.B = (int32_t)q.size(0); s.Hq = (int32_t)q.size(1); s.Hk = (int32_t)k.size(1); s.N = (int32_t)q.size(2); s.d = (int32_t)q.size(3);
    s.dtype = dtype_of(q);
    if (cos.defined()) { s.rot = (int32_t)(2 * cos.size(1)); s.table_rows = (int32_t)cos.size(0); }
    s.interleaved = interleaved;
    if (positions.defined()) {
      s.pos_bits = positions.scalar_type() == at::kInt ? 32 : 64;
      s.pos_sb = positions.dim() == 2 && positions.size(0) > 1 ? q.size(2) : 0;
    }
    const auto a = strides_of(q), b = strides_of(k), c = strides_of(qo), d = strides_of(ko);
    s.q_sb = a[0]; s.q_sh = a[1]; s.q_sn = a[2]; s.k_sb = b[0]; s.k_sh = b[1]; s.k_sn = b[2];
    s.qo_sb = c[0]; s.qo_sh = c[1]; s.qo_sn = c[2]; s.ko_sb = d[0]; s.ko_sh = d[1]; s.ko_sn = d[2];
  }
};

void norm_check(const Tensor& q, const Tensor& k, const Tensor& wq, const Tensor& wk, const Tensor& cos, const Tensor& sin,
                const Tensor& positions) {
  for (const Tensor* t : {&q, &k}) {
    TORCH_CHECK_VALUE(t->is_cuda(), "q and k must live on the GPU: the operator has no CPU path");
    TORCH_CHECK_VALUE(t->dim() == 4 && float_kind(*t), "q and k are bf16 or fp32 [B, H, N, d] views");
    TORCH_CHECK_VALUE(t->stride(3) == 1, "the head dimension must be contiguous");
  }
  TORCH_CHECK_VALUE(k.scalar_type() == q.scalar_type() && k.device() == q.device() && k.size(0) == q.size(0) &&
                    k.size(2) == q.size(2) && k.size(3) == q.size(3),
                    "q and k share type, device, batch, tokens and head dimension");
  for (const Tensor* t : {&wq, &wk})
    TORCH_CHECK_VALUE(!t->defined() || (t->scalar_type() == at::kFloat && t->dim() == 1 && t->size(0) == q.size(3) &&
                                        t->is_contiguous() && t->device() == q.device()),
                      "weights are vectors of d elements, bf16 or fp32, on the device of q");
  TORCH_CHECK_VALUE(cos.defined() == sin.defined(), "cos and sin come together");
  for (const Tensor* t : {&cos, &sin})
    TORCH_CHECK_VALUE(!t->defined() || (t->scalar_type() == at::kFloat && t->dim() == 2 && t->sizes() == cos.sizes() &&
                                        t->is_contiguous() && t->device() == q.device()),
                      "cos and sin are contiguous fp32 tables [rows, rotated channels / 2] on the device of q");
  for (const Tensor* t : {&cos, &sin})
    TORCH_CHECK_VALUE(!t->defined() || !differentiated({t}), "cos and sin get no gradient: detach them");
  if (positions.defined()) {
    TORCH_CHECK_VALUE(cos.defined(), "positions without tables");
    TORCH_CHECK_VALUE((positions.scalar_type() == at::kInt || positions.scalar_type() == at::kLong) &&
                      positions.device() == q.device() && positions.is_contiguous() &&
                      ((positions.dim() == 1 && positions.size(0) == q.size(2)) ||
                       (positions.dim() == 2 && positions.size(1) == q.size(2) &&
                        (positions.size(0) == 1 || positions.size(0) == q.size(0)))),
                      "positions are int32 or int64 numbers [N] or [B, N] on the device of q");
  } else {
    TORCH_CHECK_VALUE(!cos.defined() || cos.size(0) >= q.size(2), "the tables have fewer rows than there are tokens");
  }
}

std::pair<Tensor, Tensor> norm_rotate_call(const Tensor& q, const Tensor& k, const Tensor& wq, const Tensor& wk, const Tensor& cos,
                                           const Tensor& sin, const Tensor& positions, double eps, bool interleaved) {
  const c10::DeviceGuard device(q.device());
  const Tensor qo = dense_like(q, at::kBFloat16), ko = dense_like(k, at::kBFloat16);
  const NormShape n(q, k, cos, positions, interleaved, qo, ko);
  check(spa2_norm_rotate(q.data_ptr(), k.data_ptr(), (const float*)ptr(wq), (const float*)ptr(wk), (const float*)ptr(cos),
                         (const float*)ptr(sin), ptr(positions), &n.s, (float)eps, qo.data_ptr(), ko.data_ptr(),
                         stream_of(q)), "spa2_norm_rotate");
  return {qo, ko};
}

struct NormRotate : torch::autograd::Function<NormRotate> {
  static variable_list forward(AutogradContext* ctx, const Tensor& q, const Tensor& k, const OptTensor& q_weight,
                               const OptTensor& k_weight, const OptTensor& cos_, const OptTensor& sin_,
                               const OptTensor& positions_, double eps, bool interleaved, bool weight_grads) {
    const Tensor wq = or_none(q_weight), wk = or_none(k_weight), cos = or_none(cos_), sin = or_none(sin_), positions = or_none(positions_);
    const auto [qo, ko] = norm_rotate_call(q, k, wq, wk, cos, sin, positions, eps, interleaved);
    ctx->save_for_backward({q, k, wq, wk, cos, sin, positions});
    ctx->saved_data["eps"] = eps;
    ctx->saved_data["interleaved"] = interleaved;
    ctx->saved_data["weight_grads"] = weight_grads;
    return {qo, ko};
  }

  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    const bool graph = at::GradMode::is_enabled();
    const at::NoGradGuard no_graph;
    const variable_list s = ctx->get_saved_variables();
    const Tensor &q = s[0], &k = s[1], &wq = s[2], &wk = s[3], &cos = s[4], &sin = s[5], &positions = s[6];
    // (saved-tensor hooks may bring something else back)
    norm_check(q, k, wq, wk, cos, sin, positions);
    TORCH_CHECK_VALUE(grads[0].sizes() == q.sizes() && grads[1].sizes() == k.sizes() && grads[0].device() == q.device() &&
                      grads[1].device() == q.device(), "saved q and k come back in their shapes on their GPU");
    const c10::DeviceGuard device(q.device());
    const Tensor dq = dense_like(q, q.scalar_type()), dk = dense_like(k, k.scalar_type());
    const Tensor dqo = in_order(grads[0].to(at::kBFloat16), dq), dko = in_order(grads[1].to(at::kBFloat16), dk);
    const bool weights = ctx->saved_data["weight_grads"].toBool();
    const NormShape n(q, k, cos, positions, ctx->saved_data["interleaved"].toBool(), dq, dk);
    Tensor dwq, dwk, ws;
    if (weights) {
      if (wq.defined()) dwq = at::empty_like(wq);
      if (wk.defined()) dwk = at::empty_like(wk);
      ws = bytes((int64_t)spa2_norm_rotate_bwd_workspace_bytes(&n.s), q);
    }
    check(spa2_norm_rotate_bwd(q.data_ptr(), k.data_ptr(), (const float*)ptr(wq), (const float*)ptr(wk), (const float*)ptr(cos),
                               (const float*)ptr(sin), ptr(positions), dqo.data_ptr(), dko.data_ptr(), &n.s,
                               (float)ctx->saved_data["eps"].toDouble(), dq.data_ptr(), dk.data_ptr(), (float*)ptr(dwq),
                               (float*)ptr(dwk), (void*)ptr(ws), weights ? (size_t)ws.numel() : 0, stream_of(q)),
          "spa2_norm_rotate_bwd");
    return once({dq, dk, dwq, dwk, Variable(), Variable(), Variable(), Variable(), Variable(), Variable()}, graph,
                "qk_norm_rotate");
  }
};

// weights of any float type, anywhere in memory: the kernels read fp32 from a 16-byte boundary (PyTorch differentiates this)
OptTensor as_weight(const OptTensor& w) {
  if (!w || !w->defined()) return std::nullopt;
  const Tensor x = w->to(at::kFloat).contiguous();
  return aligned(x) ? x : x.clone();
}

std::tuple<Tensor, Tensor> norm_rotate(const Tensor& q, const Tensor& k, const OptTensor& q_weight, const OptTensor& k_weight,
                                       const OptTensor& cos, const OptTensor& sin, const OptTensor& positions, double eps,
                                       bool interleaved) {
  const OptTensor wq = as_weight(q_weight), wk = as_weight(k_weight);
  norm_check(q, k, or_none(wq), or_none(wk), or_none(cos), or_none(sin), or_none(positions));
  const Tensor w0 = or_none(wq), w1 = or_none(wk);
  if (!differentiated({&q, &k, &w0, &w1}))
    return norm_rotate_call(q, k, w0, w1, or_none(cos), or_none(sin), or_none(positions), eps, interleaved);
  capture_check(q, {q, k, or_none(q_weight), or_none(k_weight)});
  const bool weight_grads = at::GradMode::is_enabled() && ((wq && wq->requires_grad()) || (wk && wk->requires_grad()));
  const variable_list out = NormRotate::apply(q, k, wq, wk, cos, sin, positions, eps, interleaved, weight_grads);
  return {out[0], out[1]};
}

// ---- attention to another sequence
struct CrossShape {
  spa2_cross_shape s = {};
  // strides of a dimension of one element are never used: any that pass the checks
  static void set(const Tensor& x, int64_t& sb, int64_t& sh, int64_t& sn) {
    const int64_t any = (x.size(3) + 7) & ~(int64_t)7;
    sb = x.size(0) > 1 ? x.stride(0) : any; sh = x.size(1) > 1 ? x.stride(1) : any; sn = x.size(2) > 1 ? x.stride(2) : any;
  }
  CrossShape(const Tensor& q, const Tensor& k, const Tensor& dk) {
    s.B = (int32_t)q.size(0); s.Hq = (int32_t)q.size(1); s.Hk = (int32_t)k.size(1); s.Nq = (int32_t)q.size(2);
    s.Nk = (int32_t)k.size(2); s.d = (int32_t)q.size(3);
    set(q, s.q_sb, s.q_sh, s.q_sn);
    set(k, s.k_sb, s.k_sh, s.k_sn);
    set(dk, s.d_sb, s.d_sh, s.d_sn);
  }
};

void cross_check(const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& lengths) {
  const std::pair<const char*, const Tensor*> named[] = {{"q", &q}, {"k", &k}, {"v", &v}};
  for (const auto& [name, t] : named) {
    TORCH_CHECK_VALUE(t->is_cuda(), name, " must live on the GPU: the operator has no CPU path");
    TORCH_CHECK_VALUE(t->scalar_type() == at::kBFloat16 && t->dim() == 4, name, " must be a bf16 [B, H, N, d] view");
    TORCH_CHECK_VALUE(t->stride(3) == 1, "the head dimension must be contiguous");
  }
  TORCH_CHECK_VALUE(v.sizes() == k.sizes(), "k and v share one shape");
  TORCH_CHECK_VALUE(k.size(0) == q.size(0) && k.size(3) == q.size(3), "q and k share batch and head dimension");
  TORCH_CHECK_VALUE(k.size(1) > 0 && q.size(1) % k.size(1) == 0, "the number of query heads is a multiple of that of key heads");
  TORCH_CHECK_VALUE(k.device() == q.device() && v.device() == q.device(), "q, k and v live on one GPU");
  TORCH_CHECK_VALUE(!lengths.defined() || (lengths.scalar_type() == at::kInt && lengths.dim() == 1 && lengths.size(0) == q.size(0) &&
                                           lengths.is_contiguous() && lengths.device() == q.device()),
                    "lengths are int32 [B] on the device of q");
}

Tensor copy_of(const Tensor& x) {
  const Tensor y = dense_like(x, x.scalar_type());
  y.copy_(x);
  return y;
}
// One layout for a query tensor and all that is shaped like it: q itself where it has no gaps, else a copy without them.
Tensor without_gaps(const Tensor& q) { return q.is_non_overlapping_and_dense() ? q : copy_of(q); }

struct CrossResult { Tensor q, k, v, o, o_res, lse; };       // (q, k and v in the layouts that the kernels took)
CrossResult cross_call(const Tensor& q_in, const Tensor& k_in, const Tensor& v_in, const Tensor& lengths, double scale, bool training) {
  const c10::DeviceGuard device(q_in.device());
  const bool one_layout = strides_of(k_in) == strides_of(v_in);
  CrossResult r;
  r.q = without_gaps(q_in);
  r.k = one_layout ? k_in : copy_of(k_in);
  r.v = one_layout ? v_in : in_order(v_in, r.k);
  const CrossShape c(r.q, r.k, r.k);
  r.o = like(r.q);
  if (training && r.k.size(2) > 64) r.o_res = like(r.q);       // (up to 64 keys the backward pass takes D without O)
  // one scratch buffer; a log-sum-exp that nobody reads lies behind the workspace
  const int64_t need = (int64_t)spa2_cross_fwd_workspace_bytes(&c.s), at = (need + 255) & ~(int64_t)255;
  const int64_t rows = r.q.size(0) * r.q.size(1) * r.q.size(2);
  if (training) r.lse = at::empty({r.q.size(0), r.q.size(1), r.q.size(2)}, r.q.options().dtype(at::kFloat));
  const Tensor ws = !training || need ? bytes(training ? need : at + 4 * rows, r.q) : Tensor();
  float* lse = training ? (float*)r.lse.data_ptr() : (float*)((char*)ws.data_ptr() + at);
  check(spa2_cross_fwd(r.q.data_ptr(), r.k.data_ptr(), r.v.data_ptr(), (const int32_t*)ptr(lengths), &c.s, (float)scale,
                       r.o.data_ptr(), (void*)ptr(r.o_res), lse, (void*)ptr(ws), (size_t)need, stream_of(r.q)), "spa2_cross_fwd");
  return r;
}

struct CrossAttention : torch::autograd::Function<CrossAttention> {
  static Tensor forward(AutogradContext* ctx, const Tensor& q, const Tensor& k, const Tensor& v, const OptTensor& lengths_,
                        double scale) {
    const Tensor lengths = or_none(lengths_);
    const CrossResult r = cross_call(q, k, v, lengths, scale, true);
    ctx->save_for_backward({r.q, r.k, r.v, r.o, r.o_res, r.lse, lengths});
    ctx->saved_data["keys"] = r.k.sizes().vec();
    ctx->saved_data["scale"] = scale;
    return r.o;
  }

  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    const bool graph = at::GradMode::is_enabled();
    const at::NoGradGuard no_graph;
    const variable_list s = ctx->get_saved_variables();
    const Tensor &q = s[0], &k = s[1], &v = s[2], &o = s[3], &o_res = s[4], &lse = s[5], &lengths = s[6];
    // (saved-tensor hooks may bring something else back)
    cross_check(q, k, v, lengths);
    TORCH_CHECK_VALUE(k.sizes().vec() == ctx->saved_data["keys"].toIntVector() && strides_of(k) == strides_of(v),
                      "saved k and v come back in their shape and one layout");
    TORCH_CHECK_VALUE(grads[0].sizes() == q.sizes() && grads[0].device() == q.device(), "saved q comes back in its shape on its GPU");
    same_layout(q, {&o});
    if (o_res.defined()) same_layout(q, {&o_res});
    TORCH_CHECK_VALUE(lse.device() == q.device() && lse.scalar_type() == at::kFloat && lse.is_contiguous() &&
                      lse.numel() == q.size(0) * q.size(1) * q.size(2), "the log-sum-exp comes back as B * H * N contiguous fp32 numbers");
    const c10::DeviceGuard device(q.device());
    const Tensor d_o = in_order(grads[0].to(at::kBFloat16), q);
    const Tensor dq = like(q), dk = dense_like(k, k.scalar_type()), dv = dense_like(k, k.scalar_type());
    const CrossShape c(q, k, dk);
    const int64_t need = (int64_t)spa2_cross_bwd_workspace_bytes(&c.s);
    const Tensor ws = bytes(need, q);
    check(spa2_cross_bwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), (const int32_t*)ptr(lengths), o.data_ptr(), (void*)ptr(o_res),
                         d_o.data_ptr(), (const float*)lse.data_ptr(), &c.s, (float)ctx->saved_data["scale"].toDouble(),
                         dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), ws.data_ptr(), (size_t)need, stream_of(q)),
          "spa2_cross_bwd");
    return once({dq, dk, dv, Variable(), Variable()}, graph, "cross_attention");
  }
};

Tensor cross_attention(const Tensor& q, const Tensor& k, const Tensor& v, const OptTensor& lengths, double scale) {
  cross_check(q, k, v, or_none(lengths));
  if (!differentiated({&q, &k, &v})) return cross_call(q, k, v, or_none(lengths), scale, false).o;
  capture_check(q, {q, k, v});
  return CrossAttention::apply(q, k, v, lengths, scale);
}

// x as the elementwise kernels take it: contiguous from a 16-byte boundary.
Tensor packed(const Tensor& x) {
  const Tensor y = x.contiguous();
  return aligned(y) ? y : y.clone();
}

void seed_check(const Tensor& s, const Tensor& x) {
  TORCH_CHECK_VALUE(!s.defined() || (s.scalar_type() == at::kLong && s.numel() == 2 && s.is_contiguous() && s.device() == x.device()),
                    "a seed on the device is two int64 numbers, seed and offset, on the device of x");
}

Tensor dropout_call(const Tensor& x_in, const Tensor& residual_in, double p, int64_t seed, int64_t offset, const Tensor& so) {
  const c10::DeviceGuard device(x_in.device());
  const Tensor x = packed(x_in), residual = residual_in.defined() ? packed(residual_in) : Tensor();
  const Tensor y = at::empty_like(residual.defined() ? residual : x);
  check(spa2_dropout_add(x.data_ptr(), ptr(residual), x.numel(), dtype_of(x), dtype_of(y), p, (uint64_t)seed,
                         (uint64_t)offset, (const int64_t*)ptr(so), y.data_ptr(), stream_of(x)), "spa2_dropout_add");
  return y;
}

struct DropoutAdd : torch::autograd::Function<DropoutAdd> {
  static Tensor forward(AutogradContext* ctx, const Tensor& x, const OptTensor& residual_in, double p, int64_t seed,
                        int64_t offset, const OptTensor& seed_offset) {
    const Tensor residual = or_none(residual_in), so = or_none(seed_offset);
    const Tensor y = dropout_call(x, residual, p, seed, offset, so);
    ctx->save_for_backward({so});
    ctx->saved_data["p"] = p;
    ctx->saved_data["seed"] = seed;
    ctx->saved_data["offset"] = offset;
    ctx->saved_data["bf16"] = x.scalar_type() == at::kBFloat16;
    ctx->saved_data["residual"] = residual.defined();
    return y;
  }

  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    const bool graph = at::GradMode::is_enabled();
    const at::NoGradGuard no_graph;
    const Tensor so = ctx->get_saved_variables()[0];
    const Tensor dy = packed(grads[0]);
    seed_check(so, dy);
    const c10::DeviceGuard device(dy.device());
    const Tensor dx = at::empty(dy.sizes(), dy.options().dtype(ctx->saved_data["bf16"].toBool() ? at::kBFloat16 : at::kFloat));
    check(spa2_dropout_bwd(dy.data_ptr(), dy.numel(), dtype_of(dy), dtype_of(dx), ctx->saved_data["p"].toDouble(),
                           (uint64_t)ctx->saved_data["seed"].toInt(), (uint64_t)ctx->saved_data["offset"].toInt(),
                           (const int64_t*)ptr(so), dx.data_ptr(), stream_of(dy)), "spa2_dropout_bwd");
    const variable_list first = once({dx}, graph, "dropout_add");
    return {first[0], ctx->saved_data["residual"].toBool() ? grads[0] : Variable(), Variable(), Variable(), Variable(), Variable()};
  }
};

Tensor dropout_add(const Tensor& x, const OptTensor& residual, double p, int64_t seed, int64_t offset, const OptTensor& seed_offset) {
  TORCH_CHECK_VALUE(x.is_cuda(), "x must live on the GPU: the operator has no CPU path");
  TORCH_CHECK_VALUE(float_kind(x), "x is bf16 or fp32");
  if (residual)
    TORCH_CHECK_VALUE(residual->sizes() == x.sizes() && residual->device() == x.device() &&
                      (residual->scalar_type() == x.scalar_type() || residual->scalar_type() == at::kFloat),
                      "the residual has the shape and device of x and its type, or fp32");
  seed_check(or_none(seed_offset), x);
  const Tensor r = or_none(residual);
  if (!differentiated({&x, &r})) return dropout_call(x, r, p, seed, offset, or_none(seed_offset));
  capture_check(x, {x, r});
  return DropoutAdd::apply(x, residual, p, seed, offset, seed_offset);
}

}  // namespace

PYBIND11_MODULE(TORCH_EXTENSION_NAME, m) {
  m.def("attention", &attention, py::call_guard<py::gil_scoped_release>());
  m.def("norm_rotate", &norm_rotate, py::call_guard<py::gil_scoped_release>());
  m.def("cross_attention", &cross_attention, py::call_guard<py::gil_scoped_release>());
  m.def("dropout_add", &dropout_add, py::call_guard<py::gil_scoped_release>());
  m.def("velocity_loss", &velocity_loss, py::call_guard<py::gil_scoped_release>());
}
