// Marshalling of the attention layer's operators for torch tensors.
#include "ones_attention.h"

#include <algorithm>
#include <cmath>
#include <utility>
#include <vector>

#include "ones_torch.h"

namespace {

// A tensor [..][heads][dim] as vectors of values that lie side by side.
ones_heads heads_of(const Tensor& t) {
    return {t.data_ptr(), t.stride(0), t.stride(1), (int32_t)t.size(1)};
}
// tensor memory that heads share or that has gaps within a vector cannot be given on as it is
bool plain(const Tensor& t) {
    return (t.stride(2) == 1 || t.size(2) == 1) && (t.size(1) == 1 || t.stride(1) >= t.size(2)) && (t.size(0) == 1 || t.stride(0) >= 1);
}
Tensor flat(const Tensor& t) { return t.dim() == 3 ? t : t.flatten(0, t.dim() - 3); }
Tensor readable(const Tensor& t) {
    const Tensor f = flat(t);
    return f.numel() == 0 || plain(f) ? f : f.contiguous();
}
// The same with every vector on a 16-byte boundary; rc of a copy.
Tensor aligned_heads(const Tensor& t, int& rc) {
    Tensor f = readable(t);
    const int64_t n = f.size(0), h = f.size(1), d = f.size(2);
    if (f.numel() == 0 || (reinterpret_cast<uintptr_t>(f.data_ptr()) % 16 == 0 && (h == 1 || f.stride(1) % 8 == 0) && (n == 1 || f.stride(0) % 8 == 0)))
        return f;
    Tensor wide = fresh({n, h, (d + 7) / 8 * 8}, f, f.scalar_type());
    const int64_t row = h > 1 ? f.stride(1) : n > 1 ? f.stride(0) : d;
    if (row >= d && (h == 1 || n == 1 || f.stride(0) == h * row) && n * h <= INT32_MAX) {  // vectors at one distance
        rc = ones_align_rows(f.data_ptr(), row, (int)(n * h), (int)d, kind_of(f.scalar_type()), wide.data_ptr(), wide.size(2), stream());
        return wide.narrow(2, 0, d);
    }
    wide = wide.narrow(2, 0, d);
    wide.copy_(f);
    return wide;
}

bool is_weight(const MaybeTensor& t, int64_t dim, const Tensor& x) {
    return !t || (t->dim() == 1 && t->size(0) == dim && t->device() == x.device() && t->is_contiguous() &&
                  (t->scalar_type() == at::kFloat || t->scalar_type() == x.scalar_type()));
}

struct Norm {
    Tensor q, k, positions, frequencies;
    int kind, wkind;
    at::ScalarType wtype;
};
Norm check_norm(const Tensor& q, const Tensor& k, const Tensor& positions, const Tensor& frequencies, const MaybeTensor& q_weight,
                const MaybeTensor& k_weight) {
    const int kind = kind_of(q.scalar_type());
    TORCH_CHECK_VALUE(q.is_cuda() && kind >= 0 && q.dim() >= 3, "q: a float32, bfloat16 or float16 CUDA tensor [..][heads][dim] is needed");
    const int64_t dim = q.size(-1);
    TORCH_CHECK_VALUE(k.device() == q.device() && k.scalar_type() == q.scalar_type() && k.dim() == q.dim() && k.size(-1) == dim &&
                          k.sizes().slice(0, k.dim() - 2) == q.sizes().slice(0, q.dim() - 2),
                      "k needs q's shape but for the heads, its type and device");
    TORCH_CHECK_VALUE(positions.scalar_type() == at::kLong && positions.device() == q.device() && positions.sizes() == q.sizes().slice(0, q.dim() - 2),
                      "positions: int64 with q's leading dimensions is needed");
    TORCH_CHECK_VALUE(frequencies.scalar_type() == at::kDouble && frequencies.device() == q.device() && frequencies.dim() == 1 &&
                          frequencies.size(0) <= dim / 2,
                      "frequencies: a float64 vector of at most dim / 2 values on q's device is needed");
    TORCH_CHECK_VALUE(dim <= ONES_QK_NORM_MAX_DIM && q.size(-2) <= ONES_MAX_HEADS && k.size(-2) <= ONES_MAX_HEADS,
                      "heads of at most 256 values, and at most 1024 of them, are possible");
    TORCH_CHECK_VALUE(is_weight(q_weight, dim, q) && is_weight(k_weight, dim, q) &&
                          (!q_weight || !k_weight || q_weight->scalar_type() == k_weight->scalar_type()),
                      "q_weight, k_weight: contiguous vectors of dim values on q's device and of one type, q's or float32, are needed");
    Norm n{readable(q), readable(k), positions.contiguous(), frequencies.contiguous(), kind, ONES_F32, at::kFloat};
    TORCH_CHECK_VALUE(n.q.size(0) <= INT32_MAX, "more than 2^31 - 1 tokens");
    if (q_weight || k_weight) n.wtype = (q_weight ? q_weight : k_weight)->scalar_type(), n.wkind = kind_of(n.wtype);
    return n;
}

py::object qk_norm(const Tensor& q, const Tensor& k, const Tensor& positions, const Tensor& frequencies, const MaybeTensor& q_weight,
                   const MaybeTensor& k_weight, double eps, bool interleaved) {
    no_graph({&q, &k, &frequencies, given(q_weight, q), given(k_weight, q)});
    const at::NoGradGuard no_grad;
    const c10::cuda::OptionalCUDAGuard guard(q.is_cuda() ? std::optional<at::Device>(q.device()) : std::nullopt);
    const Norm n = check_norm(q, k, positions, frequencies, q_weight, k_weight);
    Tensor qo = fresh(q.sizes(), q, q.scalar_type()), ko = fresh(k.sizes(), k, k.scalar_type());
    const ones_heads qi = heads_of(n.q), ki = heads_of(n.k), qh = heads_of(flat(qo)), kh = heads_of(flat(ko));
    const int rc = ones_qk_norm(&qi, &ki, n.positions.data_ptr<int64_t>(), n.frequencies.data_ptr<double>(), ptr(q_weight), ptr(k_weight),
                                (int)n.q.size(0), (int)q.size(-1), (int)(2 * n.frequencies.size(0)), interleaved, (float)eps, n.kind, n.wkind, &qh, &kh,
                                stream());
    return result(rc, py::make_tuple(qo, ko));
}

py::object qk_norm_backward(const Tensor& dq, const Tensor& dk, const Tensor& q, const Tensor& k, const Tensor& positions, const Tensor& frequencies,
                            const MaybeTensor& q_weight, const MaybeTensor& k_weight, double eps, bool interleaved, bool parameters) {
    no_graph({&dq, &dk, &q, &k, &frequencies, given(q_weight, q), given(k_weight, q)});
    const at::NoGradGuard no_grad;
    const c10::cuda::OptionalCUDAGuard guard(q.is_cuda() ? std::optional<at::Device>(q.device()) : std::nullopt);
    const Norm n = check_norm(q, k, positions, frequencies, q_weight, k_weight);
    TORCH_CHECK_VALUE(dq.sizes() == q.sizes() && dk.sizes() == k.sizes() && dq.scalar_type() == q.scalar_type() && dk.scalar_type() == q.scalar_type() &&
                          dq.device() == q.device() && dk.device() == q.device(),
                      "dq, dk need the shapes, type and device of q, k");
    const Tensor gq = readable(dq), gk = readable(dk);
    Tensor qo = fresh(q.sizes(), q, q.scalar_type()), ko = fresh(k.sizes(), k, k.scalar_type());
    MaybeTensor qw, kw, space;
    size_t nbytes = 0;
    if (parameters) {
        qw = fresh({q.size(-1)}, q, n.wtype), kw = fresh({q.size(-1)}, q, n.wtype);
        nbytes = ones_qk_norm_workspace_bytes((int)q.size(-1));
        space = bytes(nbytes, q);
    }
    const ones_heads yq = heads_of(gq), yk = heads_of(gk), qi = heads_of(n.q), ki = heads_of(n.k), qh = heads_of(flat(qo)), kh = heads_of(flat(ko));
    const int rc = ones_qk_norm_backward(&yq, &yk, &qi, &ki, n.positions.data_ptr<int64_t>(), n.frequencies.data_ptr<double>(), ptr(q_weight),
                                         ptr(k_weight), (int)n.q.size(0), (int)q.size(-1), (int)(2 * n.frequencies.size(0)), interleaved, (float)eps,
                                         n.kind, n.wkind, &qh, &kh, ptr(qw), ptr(kw), ptr(space), nbytes, stream());
    return result(rc, py::make_tuple(qo, ko, qw, kw));
}

// Tokens and sequences of an attention call.
struct Packed {
    int32_t tokens, sequences;
    MaybeTensor offsets;
    const int64_t* at() const { return offsets ? offsets->data_ptr<int64_t>() : nullptr; }
};
Packed check_attention(const Tensor& q, const Tensor& k, const Tensor& v, const MaybeTensor& offsets) {
    TORCH_CHECK_VALUE(q.is_cuda() && (q.scalar_type() == at::kBFloat16 || q.scalar_type() == at::kHalf) && (q.dim() == 3 || q.dim() == 4),
                      "q: a bfloat16 or float16 CUDA tensor [tokens][heads][dim] or [batch][tokens][heads][dim] is needed");
    for (const Tensor* t : {&k, &v})
        TORCH_CHECK_VALUE(t->device() == q.device() && t->scalar_type() == q.scalar_type() && t->dim() == q.dim() && t->size(-1) == q.size(-1) &&
                              t->sizes().slice(0, q.dim() - 2) == q.sizes().slice(0, q.dim() - 2) && t->size(-2) == k.size(-2),
                          "k, v need q's shape but for the heads, its type and device");
    const int64_t heads = q.size(-2), kv = k.size(-2), dim = q.size(-1), tokens = q.dim() == 3 ? q.size(0) : q.size(0) * q.size(1);
    TORCH_CHECK_VALUE(heads >= 1 && heads <= ONES_MAX_HEADS && kv >= 1 && heads % kv == 0 && heads / kv <= 128,
                      "heads: a multiple of the keys' heads, at most 128 times and at most 1024, is needed");
    TORCH_CHECK_VALUE(dim >= 1 && dim <= ONES_ATTENTION_MAX_DIM, "dim: 1 to 128 values of a head are possible");
    TORCH_CHECK_VALUE(tokens < 1 << 30, "at most 2^30 - 1 tokens are possible");
    if (offsets) {
        TORCH_CHECK_VALUE(q.dim() == 3 && offsets->scalar_type() == at::kLong && offsets->device() == q.device() && offsets->dim() == 1 &&
                              offsets->size(0) >= 1 && offsets->size(0) <= (1 << 22) + 1,
                          "offsets: an int64 vector on q's device, of one value more than sequences, and q [tokens][heads][dim], are needed");
        return {(int32_t)tokens, (int32_t)offsets->size(0) - 1, offsets->contiguous()};
    }
    TORCH_CHECK_VALUE(q.dim() == 3 || q.size(0) <= 1 << 22, "at most 2^22 sequences are possible");
    return {(int32_t)tokens, q.dim() == 3 ? 1 : (int32_t)q.size(0), std::nullopt};
}
float scale_of(const std::optional<double>& scale, const Tensor& q) { return (float)(scale ? *scale : 1.0 / std::sqrt((double)q.size(-1))); }

py::object attention(const Tensor& q, const Tensor& k, const Tensor& v, const MaybeTensor& offsets, std::optional<double> scale) {
    no_graph({&q, &k, &v});
    const at::NoGradGuard no_grad;
    const c10::cuda::OptionalCUDAGuard guard(q.is_cuda() ? std::optional<at::Device>(q.device()) : std::nullopt);
    const Packed p = check_attention(q, k, v, offsets);
    int rc = 0;
    const Tensor qa = aligned_heads(q, rc), ka = aligned_heads(k, rc), va = aligned_heads(v, rc);
    if (rc) return py::int_(rc);
    Tensor out = fresh(q.sizes(), q, q.scalar_type()), lse = fresh(q.sizes().slice(0, q.dim() - 1), q, at::kFloat);
    const size_t nbytes = ones_attention_workspace_bytes(p.tokens, p.sequences, (int)q.size(-2), (int)k.size(-2));
    Tensor space = bytes(nbytes, q);
    const ones_heads qh = heads_of(qa), kh = heads_of(ka), vh = heads_of(va), oh = heads_of(flat(out));
    rc = ones_attention(&qh, &kh, &vh, p.at(), p.tokens, p.sequences, (int)q.size(-1), scale_of(scale, q), kind_of(q.scalar_type()), &oh,
                        lse.data_ptr<float>(), space.data_ptr(), nbytes, stream());
    return result(rc, py::make_tuple(out, lse));
}

py::object attention_backward(const Tensor& dout, const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& out, const Tensor& lse,
                              const MaybeTensor& offsets, std::optional<double> scale) {
    no_graph({&dout, &q, &k, &v, &out, &lse});
    const at::NoGradGuard no_grad;
    const c10::cuda::OptionalCUDAGuard guard(q.is_cuda() ? std::optional<at::Device>(q.device()) : std::nullopt);
    const Packed p = check_attention(q, k, v, offsets);
    for (const Tensor* t : {&dout, &out})
        TORCH_CHECK_VALUE(t->sizes() == q.sizes() && t->scalar_type() == q.scalar_type() && t->device() == q.device(),
                          "dout, out need q's shape, type and device");
    TORCH_CHECK_VALUE(lse.scalar_type() == at::kFloat && lse.device() == q.device() && lse.sizes() == q.sizes().slice(0, q.dim() - 1) && lse.is_contiguous(),
                      "lse: what attention returned is needed");
    int rc = 0;
    const Tensor ga = aligned_heads(dout, rc), qa = aligned_heads(q, rc), ka = aligned_heads(k, rc), va = aligned_heads(v, rc),
                 oa = aligned_heads(out, rc);  // read faster so, though it need not be
    if (rc) return py::int_(rc);
    Tensor dq = fresh(q.sizes(), q, q.scalar_type()), dk = fresh(k.sizes(), q, q.scalar_type()), dv = fresh(v.sizes(), q, q.scalar_type());
    const size_t nbytes = ones_attention_backward_workspace_bytes(p.tokens, p.sequences, (int)q.size(-2), (int)k.size(-2), (int)q.size(-1));
    Tensor space = bytes(nbytes, q);
    const ones_heads gh = heads_of(ga), qh = heads_of(qa), kh = heads_of(ka), vh = heads_of(va), oh = heads_of(oa), dqh = heads_of(flat(dq)),
                     dkh = heads_of(flat(dk)), dvh = heads_of(flat(dv));
    rc = ones_attention_backward(&gh, &qh, &kh, &vh, &oh, lse.data_ptr<float>(), p.at(), p.tokens, p.sequences, (int)q.size(-1), scale_of(scale, q),
                                 kind_of(q.scalar_type()), &dqh, &dkh, &dvh, space.data_ptr(), nbytes, stream());
    return result(rc, py::make_tuple(dq, dk, dv));
}

// Addresses, sizes and types of tensors whose values lie without gaps, in whatever order.
struct Listed {
    std::vector<void*> at;
    std::vector<int64_t> size;
    std::vector<int32_t> type;
};
Listed list_of(const std::vector<Tensor>& ts) {
    Listed l;
    l.at.reserve(ts.size()), l.size.reserve(ts.size()), l.type.reserve(ts.size());
    for (const Tensor& t : ts) {
        const int kind = kind_of(t.scalar_type());
        TORCH_CHECK_VALUE(t.is_cuda() && t.device() == ts[0].device() && kind >= 0 && t.is_non_overlapping_and_dense(),
                          "gradients: float32, bfloat16 or float16 CUDA tensors without gaps, on one device, are needed");
        l.at.push_back(t.data_ptr()), l.size.push_back(t.numel()), l.type.push_back(kind);
    }
    return l;
}
void no_overlap(const Listed& in, const Listed& out) {
    std::vector<std::pair<const char*, const char*>> spans;
    for (size_t i = 0; i < in.at.size(); ++i) {
        const int64_t n = in.size[i] * (in.type[i] == ONES_F32 ? 4 : 2);
        if (!n) continue;
        spans.emplace_back((const char*)in.at[i], (const char*)in.at[i] + n);
        if (out.at[i] != in.at[i]) spans.emplace_back((const char*)out.at[i], (const char*)out.at[i] + n);
    }
    if (!std::is_sorted(spans.begin(), spans.end())) std::sort(spans.begin(), spans.end());
    for (size_t i = 1; i < spans.size(); ++i)
        TORCH_CHECK_VALUE(spans[i - 1].second <= spans[i].first, "gradients: two of the tensors share memory");
}

py::object clip(const std::vector<Tensor>& gradients, const std::optional<std::vector<Tensor>>& out, std::optional<double> max_norm, double eps) {
    for (const Tensor& t : gradients) no_graph({&t});
    const at::NoGradGuard no_grad;
    const Listed in = list_of(gradients);
    const c10::cuda::OptionalCUDAGuard guard(gradients.empty() ? std::nullopt : std::optional<at::Device>(gradients[0].device()));
    const auto options = at::TensorOptions().dtype(at::kFloat).device(at::Device(at::kCUDA, c10::cuda::current_device()));
    Listed to = in;
    if (out) {
        TORCH_CHECK_VALUE(out->size() == gradients.size(), "out: a tensor for each gradient is needed");
        for (const Tensor& t : *out) no_graph({&t});
        to = list_of(*out);
        for (size_t i = 0; i < out->size(); ++i)
            TORCH_CHECK_VALUE((*out)[i].sizes() == gradients[i].sizes() && (*out)[i].strides() == gradients[i].strides() &&
                                  (*out)[i].scalar_type() == gradients[i].scalar_type() && (*out)[i].device() == gradients[0].device(),
                              "out needs the gradients' shapes, strides, types and device");
    }
    if (max_norm) no_overlap(in, to);
    Tensor norm = at::empty({}, options);
    const int count = (int)std::min<size_t>(gradients.size(), INT32_MAX);
    const size_t nbytes = ones_gradient_norm_workspace_bytes(count);
    Tensor space = bytes(nbytes, norm);
    int rc;
    if (max_norm) {
        for (const Tensor& t : out ? *out : gradients) t.unsafeGetTensorImpl()->bump_version();
        rc = ones_clip_gradients(in.at.data(), to.at.data(), in.size.data(), in.type.data(), count, *max_norm, eps, norm.data_ptr<float>(),
                                 space.data_ptr(), nbytes, stream());
    } else {
        rc = ones_gradient_norm(in.at.data(), in.size.data(), in.type.data(), count, norm.data_ptr<float>(), space.data_ptr(), nbytes, stream());
    }
    return result(rc, py::cast(norm));
}

}  // namespace

void add_attention(py::module_& m) {
    m.def("qk_norm", &qk_norm);
    m.def("qk_norm_backward", &qk_norm_backward);
    m.def("attention", &attention);
    m.def("attention_backward", &attention_backward);
    m.def("clip", &clip);
}
