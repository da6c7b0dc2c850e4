// Marshalling of the training-step operators for torch tensors: argument checks, outputs and workspaces from torch's
// allocator, the current stream. All the work is behind the C ABI (ones_train.h). Small calls are bound by what the host
// does before the launch: the same in Python takes 9 us of a layer norm's 13.
#include "ones_torch.h"

namespace {

// A tensor [..][cols] as rows that can be read, and the distance of two rows in values. align: 8 for rows that have to
// start on 16-byte boundaries (16-bit types).
struct Rows {
    Tensor t;
    int64_t n, c, ld;
    int rc = 0;  // of a copy
};
Rows rows_of(const Tensor& x, int64_t align = 0) {
    Rows r{x.dim() == 2 ? x : x.reshape({-1, x.size(-1)}), 0, 0, 0};
    r.n = r.t.size(0), r.c = r.t.size(1);
    r.ld = r.t.stride(0);
    TORCH_CHECK_VALUE(r.n <= INT32_MAX && r.c <= INT32_MAX, "more than 2^31 - 1 rows or columns");
    const int64_t least = std::max<int64_t>(r.c, 1);
    if (r.n <= 1) r.ld = align ? (least + align - 1) / align * align : least;  // there is no second row
    if ((r.t.stride(1) != 1 && r.c > 1) || r.ld < r.c) {
        r.t = r.t.contiguous();
        r.ld = r.c;
    }
    if (align && (r.ld % align || reinterpret_cast<uintptr_t>(r.t.data_ptr()) % 16)) {
        const int64_t ld = (r.c + 63) / 64 * 64;  // on 128-byte lines, which are loaded faster than 16-byte blocks (587 x 769: 102 -> 92 us)
        Tensor wide = fresh({r.n, ld}, r.t, r.t.scalar_type());
        r.rc = ones_align_rows(r.t.data_ptr(), r.ld, (int)r.n, (int)r.c, kind_of(r.t.scalar_type()), wide.data_ptr(), ld, stream());
        r.t = wide, r.ld = ld;
    }
    return r;
}

bool is_param(const MaybeTensor& t, int64_t cols, const Tensor& x) {
    return !t || (t->dim() == 1 && t->size(0) == cols && t->device() == x.device() && t->is_contiguous() &&
                  (t->scalar_type() == at::kFloat || t->scalar_type() == x.scalar_type()));
}

py::object layer_norm(const Tensor& x, const MaybeTensor& weight, const MaybeTensor& bias, double eps) {
    no_graph({&x, given(weight, x), given(bias, x)});
    const int kind = kind_of(x.scalar_type());
    TORCH_CHECK_VALUE(x.is_cuda() && kind >= 0 && x.dim() >= 1, "x: a float32, bfloat16 or float16 CUDA tensor is needed");
    const int64_t cols = x.size(-1);
    TORCH_CHECK_VALUE(is_param(weight, cols, x) && is_param(bias, cols, x) && (!weight || !bias || weight->scalar_type() == bias->scalar_type()),
                      "weight, bias: contiguous vectors of x's columns, device and one type, x's or float32, are needed");
    const int wkind = weight ? kind_of(weight->scalar_type()) : bias ? kind_of(bias->scalar_type()) : ONES_F32;
    const at::NoGradGuard no_grad;
    const c10::cuda::CUDAGuard guard(x.device());
    const Rows r = rows_of(x);
    const auto lead = x.sizes().slice(0, x.dim() - 1);
    Tensor y = fresh(x.sizes(), x, x.scalar_type()), mean = fresh(lead, x, at::kFloat), rstd = fresh(lead, x, at::kFloat);
    const int rc = ones_layer_norm(r.t.data_ptr(), r.ld, ptr(weight), ptr(bias), (int)r.n, (int)r.c, (float)eps, kind, wkind, y.data_ptr(),
                                   r.c, mean.data_ptr<float>(), rstd.data_ptr<float>(), stream());
    return result(rc, py::make_tuple(y, mean, rstd));
}

py::object layer_norm_backward(const Tensor& dy, const Tensor& x, const Tensor& mean, const Tensor& rstd, const MaybeTensor& weight,
                               bool parameters) {
    no_graph({&dy, &x, &mean, &rstd, given(weight, x)});
    const int kind = kind_of(x.scalar_type());
    TORCH_CHECK_VALUE(x.is_cuda() && kind >= 0 && x.dim() >= 1, "x: a float32, bfloat16 or float16 CUDA tensor is needed");
    TORCH_CHECK_VALUE(dy.sizes() == x.sizes() && dy.scalar_type() == x.scalar_type() && dy.device() == x.device(),
                      "dy needs x's shape, type and device");
    const int64_t cols = x.size(-1);
    TORCH_CHECK_VALUE(is_param(weight, cols, x), "weight: a contiguous vector of x's columns and device, of x's type or float32, is needed");
    for (const Tensor* s : {&mean, &rstd})
        TORCH_CHECK_VALUE(s->scalar_type() == at::kFloat && s->device() == x.device() && s->sizes() == x.sizes().slice(0, x.dim() - 1) &&
                              s->is_contiguous(),
                          "mean, rstd: what layer_norm returned is needed");
    const at::NoGradGuard no_grad;
    const c10::cuda::CUDAGuard guard(x.device());
    const at::ScalarType wt = weight ? weight->scalar_type() : at::kFloat;
    const Rows r = rows_of(x), q = rows_of(dy);
    Tensor dx = fresh(x.sizes(), x, x.scalar_type());
    MaybeTensor dw, db, space;
    size_t nbytes = 0;
    if (parameters) {
        dw = fresh({cols}, x, wt), db = fresh({cols}, x, wt);
        nbytes = ones_layer_norm_workspace_bytes((int)r.n, (int)r.c);
        space = bytes(nbytes, x);
    }
    const int rc = ones_layer_norm_backward(q.t.data_ptr(), q.ld, r.t.data_ptr(), r.ld, mean.data_ptr<float>(), rstd.data_ptr<float>(),
                                            ptr(weight), (int)r.n, (int)r.c, kind, kind_of(wt), dx.data_ptr(), r.c, ptr(dw), ptr(db),
                                            ptr(space), nbytes, stream());
    return result(rc, py::make_tuple(dx, dw, db));
}

void check_loss(const Tensor& hidden, const Tensor& weight, const Tensor& target) {
    TORCH_CHECK_VALUE(hidden.is_cuda() && (hidden.scalar_type() == at::kBFloat16 || hidden.scalar_type() == at::kHalf) && hidden.dim() >= 1,
                      "hidden: a bfloat16 or float16 CUDA tensor is needed");
    TORCH_CHECK_VALUE(weight.dim() == 2 && weight.scalar_type() == hidden.scalar_type() && weight.device() == hidden.device() &&
                          weight.size(1) == hidden.size(-1),
                      "weight: [vocab][cols] of hidden's type and device is needed");
    TORCH_CHECK_VALUE(target.scalar_type() == at::kLong && target.device() == hidden.device() &&
                          target.sizes() == hidden.sizes().slice(0, hidden.dim() - 1),
                      "target: int64 with hidden's leading dimensions is needed");
}

py::object linear_cross_entropy(const Tensor& hidden, const Tensor& weight, const Tensor& target) {
    no_graph({&hidden, &weight});
    check_loss(hidden, weight, target);
    const at::NoGradGuard no_grad;
    const c10::cuda::CUDAGuard guard(hidden.device());
    const Rows h = rows_of(hidden, 8), w = rows_of(weight, 8);
    if (h.rc || w.rc) return py::int_(h.rc ? h.rc : w.rc);
    const Tensor t = target.contiguous();
    Tensor loss = fresh(target.sizes(), hidden, at::kFloat), lse = fresh(target.sizes(), hidden, at::kFloat);
    const size_t nbytes = ones_linear_ce_workspace_bytes((int)h.n, (int)w.n);
    Tensor space = bytes(nbytes, hidden);
    const int rc = ones_linear_ce(h.t.data_ptr(), h.ld, w.t.data_ptr(), w.ld, t.data_ptr<int64_t>(), (int)h.n, (int)h.c, (int)w.n,
                                  kind_of(hidden.scalar_type()), loss.data_ptr<float>(), lse.data_ptr<float>(), space.data_ptr(), nbytes, stream());
    return result(rc, py::make_tuple(loss, lse));
}

py::object linear_cross_entropy_backward(const Tensor& dloss, const Tensor& hidden, const Tensor& weight, const Tensor& target, const Tensor& lse,
                                         bool weight_gradient_f32, int64_t piece) {
    no_graph({&dloss, &hidden, &weight, &lse});
    check_loss(hidden, weight, target);
    for (const Tensor* s : {&dloss, &lse})
        TORCH_CHECK_VALUE(s->scalar_type() == at::kFloat && s->device() == hidden.device() && s->sizes() == target.sizes(),
                          "dloss, lse: float32 with target's shape is needed");
    const at::NoGradGuard no_grad;
    const c10::cuda::CUDAGuard guard(hidden.device());
    const at::ScalarType wt = weight_gradient_f32 ? at::kFloat : weight.scalar_type();
    const Rows h = rows_of(hidden), w = rows_of(weight, 8);
    if (w.rc) return py::int_(w.rc);
    const Tensor t = target.contiguous(), g = dloss.contiguous(), l = lse.contiguous();
    Tensor dh = fresh(hidden.sizes(), hidden, hidden.scalar_type()), dw = fresh(weight.sizes(), weight, wt);
    const int32_t entries = piece < 0 || piece > INT32_MAX ? -1 : (int32_t)piece;
    const size_t nbytes = ones_linear_ce_backward_workspace_bytes((int)h.n, (int)h.c, (int)w.n, entries);
    Tensor space = bytes(nbytes, hidden);
    const int rc = ones_linear_ce_backward(g.data_ptr<float>(), h.t.data_ptr(), h.ld, w.t.data_ptr(), w.ld, t.data_ptr<int64_t>(),
                                           l.data_ptr<float>(), (int)h.n, (int)h.c, (int)w.n, kind_of(hidden.scalar_type()), kind_of(wt), entries,
                                           dh.data_ptr(), h.c, dw.data_ptr(), h.c, space.data_ptr(), nbytes, stream());
    return result(rc, py::make_tuple(dh, dw));
}

py::object orthogonalize(const Tensor& g, int64_t steps, double a, double b, double c, double eps) {
    no_graph({&g});
    const int kind = kind_of(g.scalar_type());
    TORCH_CHECK_VALUE(g.is_cuda() && kind >= 0 && (g.dim() == 2 || g.dim() == 3), "g: a float32, bfloat16 or float16 CUDA matrix is needed, or several");
    const at::NoGradGuard no_grad;
    const c10::cuda::CUDAGuard guard(g.device());
    Tensor s = g.dim() == 3 ? g : g.unsqueeze(0);
    const int64_t count = s.size(0), m = s.size(1), n = s.size(2);
    if ((s.stride(2) != 1 && n > 1) || (s.stride(1) < n && m > 1)) s = s.contiguous();
    Tensor out = fresh(g.sizes(), g, at::kBFloat16);
    if (out.numel() == 0) return py::cast(out);
    if (count > INT32_MAX || m > INT32_MAX || n > INT32_MAX || steps < 1 || steps > INT32_MAX) return py::int_((int)ONES_ERR_BAD_PARAM);
    const size_t nbytes = ones_orthogonalize_workspace_bytes((int)count, (int)m, (int)n);
    if (nbytes == 0) return py::int_((int)ONES_ERR_BAD_PARAM);
    Tensor space = bytes(nbytes, g);
    const int rc = ones_orthogonalize(s.data_ptr(), m > 1 ? s.stride(1) : n, s.stride(0), (int)count, (int)m, (int)n, kind, (int)steps, (float)a,
                                      (float)b, (float)c, (float)eps, out.data_ptr(), space.data_ptr(), nbytes, stream());
    return result(rc, py::cast(out));
}

}  // namespace

PYBIND11_MODULE(_train_torch, m) {
    m.def("layer_norm", &layer_norm);
    m.def("layer_norm_backward", &layer_norm_backward);
    m.def("linear_cross_entropy", &linear_cross_entropy);
    m.def("linear_cross_entropy_backward", &linear_cross_entropy_backward);
    m.def("orthogonalize", &orthogonalize);
    add_attention(m);
}
