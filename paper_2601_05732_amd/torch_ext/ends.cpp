// The calls of paper_2601_05732_amd/ends.py in C++, for tensors that the library reads as they are: the same allocations and the same call
// into libmhcl in half of the time and less (us a call, Python / this: mhcl_embed of 16 tokens 11.3 / 5.0, mhcl_streams_norm of one
// 10.1 / 4.4).  A call with any other tensor returns None, and ends.py copies or refuses.  What the library itself refuses is raised as its status.
#include <c10/hip/HIPFunctions.h>

#include <optional>
#include <tuple>

#include "native.h"

namespace native {
namespace {

// A plain tensor of the current GPU that lies dense in memory, its first byte at a multiple of `align`
bool ready(const Tensor &t, int device, uintptr_t align) {
  return t.defined() && t.is_cuda() && t.get_device() == device && t.layout() == at::kStrided && t.is_contiguous() && !t.is_neg() && !t.is_conj() &&
         !t.key_set().has_any(c10::DispatchKeySet({c10::DispatchKey::Python, c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::FuncTorchGradWrapper,
                                                   c10::DispatchKey::Functionalize})) &&
         (t.numel() == 0 || reinterpret_cast<uintptr_t>(t.data_ptr()) % align == 0);
}

std::optional<int32_t> type_of(at::ScalarType t) {
  if (t == at::kBFloat16) return MHCL_BF16;
  if (t == at::kFloat) return MHCL_F32;
  return std::nullopt;
}
bool ids_ready(const Tensor &ids, int device) {
  return (ids.scalar_type() == at::kLong || ids.scalar_type() == at::kInt) && ready(ids, device, ids.element_size());
}
bool fits(int64_t v) { return v >= 0 && v <= 0x7fffffff; }

mhcl_ends_desc describe(int64_t n, int64_t C, int64_t T, int64_t V, int32_t io, int32_t w, const Tensor *ids, double scale, double eps) {
  mhcl_ends_desc d{};
  d.n = static_cast<int32_t>(n);
  d.C = static_cast<int32_t>(C);
  d.T = T;
  d.V = static_cast<int32_t>(V);
  d.io_dtype = io;
  d.w_dtype = w;
  d.id_dtype = ids && ids->scalar_type() == at::kInt ? MHCL_I32 : MHCL_I64;
  d.scale = static_cast<float>(scale);
  d.eps = static_cast<float>(eps);
  return d;
}

Tensor workspace_of(const mhcl_ends_desc &d, int op, const Tensor &like) {
  return at::empty({static_cast<int64_t>(mhcl_ends_workspace_bytes(&d, op))}, like.options().dtype(at::kByte));
}

std::optional<Tensor> embed(const Tensor &table, const Tensor &ids, int64_t n, double scale, at::ScalarType dtype) {
  const int device = c10::hip::current_device();
  const auto io = type_of(dtype), w = type_of(table.scalar_type());
  if (!io || !w || table.dim() != 2 || ids.dim() != 1 || !ready(table, device, 16) || !ids_ready(ids, device) || !fits(n) ||
      !fits(table.size(0)) || !fits(table.size(1)))
    return std::nullopt;
  const mhcl_ends_desc d = describe(n, table.size(1), ids.size(0), table.size(0), *io, *w, &ids, scale, 0.);
  const Tensor x = empty_stream(at::empty({0}, table.options().dtype(dtype)), {d.T, n, table.size(1)}, 0);
  check(mhcl_embed(&d, ptr(table), ptr(ids), ptr(x), stream()), "mhcl_embed");
  return x;
}

std::optional<Tensor> embed_grad(const Tensor &ids, const Tensor &g_x, int64_t V, double scale, at::ScalarType dtype, const std::optional<Tensor> &into) {
  const int device = c10::hip::current_device();
  const auto io = type_of(g_x.scalar_type()), w = type_of(into ? into->scalar_type() : dtype);
  if (!io || !w || g_x.dim() != 3 || ids.dim() != 1 || ids.size(0) != g_x.size(0) || !ready(g_x, device, 16) || !ids_ready(ids, device) || !fits(V) ||
      !fits(g_x.size(1)) || !fits(g_x.size(2)))
    return std::nullopt;
  if (into && (into->dim() != 2 || into->size(0) != V || into->size(1) != g_x.size(2) || !ready(*into, device, 16))) return std::nullopt;
  const mhcl_ends_desc d = describe(g_x.size(1), g_x.size(2), ids.size(0), V, *io, *w, &ids, scale, 0.);
  const Tensor g_table = into ? *into : at::empty({V, g_x.size(2)}, g_x.options().dtype(dtype));
  const Tensor ws = workspace_of(d, MHCL_OP_EMBED_BWD, g_x);
  check(mhcl_embed_bwd(&d, ptr(ids), ptr(g_x), ptr(g_table), into ? 1 : 0, ws.data_ptr(), ws.nbytes(), stream()), "mhcl_embed_bwd");
  return g_table;
}

bool norm_ready(const Tensor &x, const Tensor &gain, int device) {
  return type_of(x.scalar_type()) && x.dim() == 3 && gain.dim() == 1 && gain.size(0) == x.size(2) && gain.scalar_type() == at::kFloat &&
         ready(x, device, 16) && ready(gain, device, 16) && fits(x.size(1)) && fits(x.size(2));
}

std::optional<Tensor> norm(const Tensor &x, const Tensor &gain, double eps) {
  if (!norm_ready(x, gain, c10::hip::current_device())) return std::nullopt;
  const mhcl_ends_desc d = describe(x.size(1), x.size(2), x.size(0), 1, *type_of(x.scalar_type()), MHCL_F32, nullptr, 1., eps);
  const Tensor h = at::empty({x.size(0), x.size(2)}, x.options());
  check(mhcl_streams_norm(&d, ptr(x), ptr<float>(gain), ptr(h), stream()), "mhcl_streams_norm");
  return h;
}

std::optional<std::tuple<Tensor, Tensor>> norm_grad(const Tensor &x, const Tensor &gain, const Tensor &g_h, double eps) {
  const int device = c10::hip::current_device();
  if (!norm_ready(x, gain, device) || g_h.dim() != 2 || g_h.size(0) != x.size(0) || g_h.size(1) != x.size(2) ||
      g_h.scalar_type() != x.scalar_type() || !ready(g_h, device, 16))
    return std::nullopt;
  const mhcl_ends_desc d = describe(x.size(1), x.size(2), x.size(0), 1, *type_of(x.scalar_type()), MHCL_F32, nullptr, 1., eps);
  const Tensor g_x = empty_stream(x, x.sizes(), 512), g_gain = floats(x, gain.sizes());
  const Tensor ws = workspace_of(d, MHCL_OP_STREAMS_NORM_BWD, x);
  check(mhcl_streams_norm_bwd(&d, ptr(x), ptr<float>(gain), ptr(g_h), ptr(g_x), ptr<float>(g_gain), ws.data_ptr(), ws.nbytes(), stream()),
        "mhcl_streams_norm_bwd");
  return std::make_tuple(g_x, g_gain);
}

bool head_ready(const Tensor &h, const Tensor &W, const Tensor &targets, int device) {
  return type_of(h.scalar_type()) && type_of(W.scalar_type()) && h.dim() == 2 && W.dim() == 2 && targets.dim() == 1 && h.size(1) == W.size(1) &&
         h.size(0) == targets.size(0) && ready(h, device, 16) && ready(W, device, 16) && ids_ready(targets, device) && fits(W.size(0)) &&
         fits(W.size(1));
}

std::optional<std::tuple<Tensor, Tensor>> head(const Tensor &h, const Tensor &W, const Tensor &targets) {
  if (!head_ready(h, W, targets, c10::hip::current_device())) return std::nullopt;
  const mhcl_ends_desc d =
      describe(1, h.size(1), h.size(0), W.size(0), *type_of(h.scalar_type()), *type_of(W.scalar_type()), &targets, 1., 0.);
  const Tensor loss = floats(h, {d.T}), lse = floats(h, {d.T}), ws = workspace_of(d, MHCL_OP_HEAD_LOSS, h);
  check(mhcl_head_loss(&d, ptr(h), ptr(W), ptr(targets), ptr<float>(loss), ptr<float>(lse), ws.data_ptr(), ws.nbytes(), stream()),
        "mhcl_head_loss");
  return std::make_tuple(loss, lse);
}

std::optional<std::tuple<Tensor, Tensor, Tensor, Tensor>> head_grad(const Tensor &h, const Tensor &W, const Tensor &targets,
                                                                    const std::optional<Tensor> &weight, at::ScalarType dtype) {
  const int device = c10::hip::current_device();
  if (!head_ready(h, W, targets, device)) return std::nullopt;
  const bool unrounded = dtype == at::kFloat && h.scalar_type() != at::kFloat;
  if (!unrounded && dtype != h.scalar_type()) return std::nullopt;
  if (weight && (weight->dim() != 1 || weight->size(0) != h.size(0) || weight->scalar_type() != at::kFloat || !ready(*weight, device, 4)))
    return std::nullopt;
  const mhcl_ends_desc d =
      describe(1, h.size(1), h.size(0), W.size(0), *type_of(h.scalar_type()), *type_of(W.scalar_type()), &targets, 1., 0.);
  const Tensor loss = floats(h, {d.T}), lse = floats(h, {d.T}), g_h = at::empty(h.sizes(), h.options().dtype(dtype)), g_W = at::empty(W.sizes(), W.options().dtype(unrounded ? dtype : W.scalar_type()));
  const Tensor ws = workspace_of(d, MHCL_OP_HEAD_LOSS_GRAD, h);
  const float *const weights = weight ? ptr<float>(*weight) : nullptr;
  if (unrounded)
    check(mhcl_head_loss_grad_unrounded(&d, ptr(h), ptr(W), ptr(targets), weights, ptr<float>(loss), ptr<float>(lse), ptr<float>(g_h), ptr<float>(g_W),
                                        ws.data_ptr(), ws.nbytes(), stream()),
          "mhcl_head_loss_grad_unrounded");
  else
    check(mhcl_head_loss_grad(&d, ptr(h), ptr(W), ptr(targets), weights, ptr<float>(loss), ptr<float>(lse), ptr(g_h), ptr(g_W), ws.data_ptr(),
                              ws.nbytes(), stream()),
          "mhcl_head_loss_grad");
  return std::make_tuple(loss, lse, g_h, g_W);
}

}  // namespace

void bind_ends(py::module &m) {
  const auto wrap = [](auto f) { return torch::wrap_pybind_function_no_gil(f); };
  m.def("embed", wrap(&embed));
  m.def("embed_grad", wrap(&embed_grad));
  m.def("norm", wrap(&norm));
  m.def("norm_grad", wrap(&norm_grad));
  m.def("head", wrap(&head));
  m.def("head_grad", wrap(&head_grad));
}

}  // namespace native
