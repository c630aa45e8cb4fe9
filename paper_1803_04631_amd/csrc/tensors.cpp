// The operators' calls on torch tensors: argument checks, outputs, workspaces, and one call of the C ABI each (include/mlda.h), on
// torch's current stream of the tensors' device.  operators.py is what a user imports, and says what each call does.
//
// This is compiled code because small calls are spent here: layer norm of one document takes the GPU 2.8 us, and
// took 12 us to call through ctypes.
#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/pybind.h>

#include <optional>
#include <string>
#include <tuple>
#include <vector>

#include "../../include/mlda.h"

namespace {

using at::Tensor;
typedef std::optional<Tensor> Maybe;

// An argument that is to be a tensor, and one that may be None.
const Tensor& tensor(py::handle h, const char* name) {
    TORCH_CHECK_VALUE(THPVariable_Check(h.ptr()), name, " must be a tensor");
    return THPVariable_Unpack(h.ptr());
}
Maybe maybe(py::handle h, const char* name) { return h.is_none() ? Maybe() : Maybe(tensor(h, name)); }

std::vector<Tensor> tensors_of(py::handle h, const char* name) {
    const py::object list = py::reinterpret_steal<py::object>(PySequence_Fast(h.ptr(), "a list of tensors is wanted"));
    if (!list) throw py::error_already_set();
    std::vector<Tensor> all((size_t)PySequence_Fast_GET_SIZE(list.ptr()));
    for (size_t i = 0; i < all.size(); ++i) all[i] = tensor(PySequence_Fast_GET_ITEM(list.ptr(), (Py_ssize_t)i), name);
    return all;
}

int type_code(const Tensor& t) {
    switch (t.scalar_type()) {
    case at::kFloat: return MLDA_FP32;
    case at::kBFloat16: return MLDA_BF16;
    case at::kHalf: return MLDA_FP16;
    default: return -1;
    }
}

// An error of the library as the binding's MldaError.
void check(int rc) {
    if (rc == MLDA_OK) return;
    const std::string message = mlda_last_error();
    const py::object type = py::module_::import("paper_1803_04631_amd").attr("MldaError");
    PyErr_SetObject(type.ptr(), type(rc, message).ptr());
    throw py::error_already_set();
}

// A matrix's rows of consecutive columns.
struct Rows {
    int64_t rows, stride;
    int32_t cols;
    int kind;
    void* at;
    at::Device device = at::kCPU;
};

Rows rows_of(const Tensor& t, const char* name) {
    TORCH_CHECK_VALUE(t.defined() && t.is_cuda(), name, " must be a tensor on a GPU: there is no CPU path");
    const int kind = type_code(t);
    TORCH_CHECK_VALUE(kind >= 0, name, " must be fp32, bf16 or fp16");
    TORCH_CHECK_VALUE(t.dim() == 2 && t.size(1) >= 1 && t.size(1) <= INT32_MAX, name, " must be a matrix with at least one column");
    const int64_t rows = t.size(0), cols = t.size(1);
    TORCH_CHECK_VALUE((t.stride(1) == 1 || cols == 1) && (rows <= 1 || t.stride(0) >= cols), name,
                      " must have consecutive columns and rows that do not overlap");
    return Rows{rows, t.stride(0), (int32_t)cols, kind, t.data_ptr(), t.device()};
}

// Rows of the shape, type and device of others'.
Rows rows_like(const Tensor& t, const char* name, const Rows& like) {
    const Rows r = rows_of(t, name);
    TORCH_CHECK_VALUE(r.rows == like.rows && r.cols == like.cols && r.kind == like.kind && r.device == like.device, name,
                      " must have the shape, type and device of the input");
    return r;
}

// The address of a contiguous tensor of that shape, type and device.
void* at_of(const Tensor& t, const char* name, at::IntArrayRef shape, at::ScalarType type, at::Device device) {
    TORCH_CHECK_VALUE(t.defined() && t.sizes() == shape && t.scalar_type() == type && t.device() == device && t.is_contiguous(), name,
                      " must be a contiguous ", type, " tensor of shape ", shape, " on ", device);
    return t.data_ptr();
}

Tensor empty(at::IntArrayRef shape, at::ScalarType type, at::Device device) { return at::empty(shape, at::TensorOptions(device).dtype(type)); }
Tensor fp32(at::IntArrayRef shape, at::Device device) { return empty(shape, at::kFloat, device); }
// A number for each token: the library writes all of them, but without rows it has nothing to do.
Tensor of_tokens(int64_t n, int64_t rows, at::Device device) {
    const Tensor t = empty({n}, at::kFloat, device);
    return rows ? t : t.zero_();
}

Tensor out_for(const Maybe& out, const Tensor& like, const Rows& rows, Rows& r) {
    const Tensor t = out ? *out : empty(like.sizes(), like.scalar_type(), rows.device);
    r = rows_like(t, "out", rows);
    return t;
}

// Tells torch that a tensor of the caller's has been written, as its own operations in place do: a backward pass that has saved it can
// see that.  (Tensors of inference mode have no versions.)
void written(const Tensor& t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
void written(const Maybe& out) {
    if (out) written(*out);
}

struct Workspace {
    Tensor held;
    void* at = nullptr;
    size_t bytes;
    Workspace(size_t n, at::Device device) : bytes(n) {
        if (!n) return;
        held = empty({(int64_t)n}, at::kByte, device);
        at = held.data_ptr();
    }
};

void* stream_of(at::Device device) { return c10::hip::getCurrentHIPStream(device.index()).stream(); }

// The addresses of weight and bias, and their type code.
struct Columns {
    void* weight = nullptr;
    void* bias = nullptr;
    int kind;
    Columns(const Maybe& w, const Maybe& b, const Tensor& x, const Rows& r) : kind(r.kind) {
        const Tensor* first = w ? &*w : b ? &*b : nullptr;
        if (!first) return;
        kind = first->defined() ? type_code(*first) : -1;
        TORCH_CHECK_VALUE(kind == r.kind || kind == MLDA_FP32, "weight and bias must have the type of x, or be fp32");
        if (w) weight = at_of(*w, "weight", {r.cols}, first->scalar_type(), r.device);
        if (b) bias = at_of(*b, "bias", {r.cols}, first->scalar_type(), r.device);
    }
};

std::tuple<Tensor, Tensor, Tensor> layer_norm(const Tensor& x, const Maybe& weight, const Maybe& bias, double eps, const Maybe& out) {
    const Rows r = rows_of(x, "x");
    const Columns c(weight, bias, x, r);
    Rows ry;
    const Tensor y = out_for(out, x, r, ry);
    const Tensor mean = fp32({r.rows}, r.device), rstd = fp32({r.rows}, r.device);
    const c10::DeviceGuard guard(r.device);
    check(mlda_layer_norm(r.at, r.stride, c.weight, c.bias, ry.at, ry.stride, mean.data_ptr<float>(), rstd.data_ptr<float>(), r.rows, r.cols,
                          eps, r.kind, c.kind, stream_of(r.device)));
    written(out);
    return {y, mean, rstd};
}

std::tuple<Tensor, Tensor, Tensor> layer_norm_backward(const Tensor& grad_y, const Tensor& x, const Tensor& mean, const Tensor& rstd,
                                                       const Maybe& weight, const Maybe& out) {
    const Rows r = rows_of(x, "x"), rg = rows_like(grad_y, "grad_y", r);
    const Columns c(weight, std::nullopt, x, r);
    void* at_mean = at_of(mean, "mean", {r.rows}, at::kFloat, r.device);
    void* at_rstd = at_of(rstd, "rstd", {r.rows}, at::kFloat, r.device);
    Rows rx;
    const Tensor grad_x = out_for(out, x, r, rx);
    const at::ScalarType type = weight ? weight->scalar_type() : x.scalar_type();
    const Tensor grad_weight = empty({r.cols}, type, r.device), grad_bias = empty({r.cols}, type, r.device);
    size_t bytes = 0;
    check(mlda_layer_norm_workspace_bytes(r.rows, r.cols, &bytes));
    const Workspace w(bytes, r.device);
    const c10::DeviceGuard guard(r.device);
    check(mlda_layer_norm_backward(rg.at, rg.stride, r.at, r.stride, (const float*)at_mean, (const float*)at_rstd, c.weight, rx.at, rx.stride,
                                   grad_weight.data_ptr(), grad_bias.data_ptr(), r.rows, r.cols, r.kind, c.kind, w.at, w.bytes, stream_of(r.device)));
    written(out);
    return {grad_x, grad_weight, grad_bias};
}

struct Documents {
    Rows r;
    int64_t n;
    const int32_t* tokens;
    const int64_t* row_ptr = nullptr;
    Documents(const Tensor& logits, const Tensor& t, const Maybe& bounds) : r(rows_of(logits, "logits")) {
        n = t.defined() ? t.numel() : -1;
        tokens = (const int32_t*)at_of(t, "tokens", {n}, at::kInt, r.device);
        if (bounds) row_ptr = (const int64_t*)at_of(*bounds, "row_ptr", {r.rows + 1}, at::kLong, r.device);
        else TORCH_CHECK_VALUE(n == r.rows, "without row_ptr there must be one token to a row");
    }
    size_t workspace(int32_t alternatives) const {
        size_t bytes = 0;
        check(mlda_token_logprobs_workspace_bytes(r.rows, r.cols, alternatives, r.kind, &bytes));
        return bytes;
    }
};

std::tuple<Tensor, Tensor, Maybe, Maybe, Maybe> token_logprobs(const Tensor& logits, const Tensor& tokens, const Maybe& row_ptr,
                                                               int64_t alternatives, bool entropy) {
    const Documents d(logits, tokens, row_ptr);
    const Rows& r = d.r;
    TORCH_CHECK_VALUE(alternatives >= 0 && alternatives <= MLDA_MAX_ALTERNATIVES && alternatives <= r.cols,
                      "alternatives must be in 0 .. ", MLDA_MAX_ALTERNATIVES, ", and no more than there are words");
    const Tensor logprobs = of_tokens(d.n, r.rows, r.device), stats = fp32({r.rows, 2}, r.device);
    Maybe entropies, ids, top;
    if (entropy) entropies = fp32({r.rows}, r.device);
    if (alternatives) {
        ids = empty({r.rows, alternatives}, at::kInt, r.device);
        top = fp32({r.rows, alternatives}, r.device);
    }
    const Workspace w(d.workspace((int32_t)alternatives), r.device);
    const c10::DeviceGuard guard(r.device);
    check(mlda_token_logprobs(r.at, r.stride, r.rows, r.cols, r.kind, d.tokens, d.row_ptr, d.n, (int32_t)alternatives, logprobs.data_ptr<float>(),
                              stats.data_ptr<float>(), entropy ? entropies->data_ptr<float>() : nullptr, ids ? ids->data_ptr<int32_t>() : nullptr,
                              top ? top->data_ptr<float>() : nullptr, w.at, w.bytes, stream_of(r.device)));
    return {logprobs, stats, entropies, ids, top};
}

Tensor token_logprobs_backward(const Tensor& grad_logprobs, const Tensor& logits, const Tensor& tokens, const Tensor& stats, const Maybe& row_ptr,
                               const Maybe& grad_entropy, const Maybe& entropy, const Maybe& out) {
    const Documents d(logits, tokens, row_ptr);
    const Rows& r = d.r;
    void* at_grad = at_of(grad_logprobs, "grad_logprobs", {d.n}, at::kFloat, r.device);
    void* at_stats = at_of(stats, "stats", {r.rows, 2}, at::kFloat, r.device);
    void* at_h = nullptr;
    void* at_entropy = nullptr;
    if (grad_entropy) {
        TORCH_CHECK_VALUE(entropy, "a gradient of the entropy needs the entropy");
        at_h = at_of(*grad_entropy, "grad_entropy", {r.rows}, at::kFloat, r.device);
        at_entropy = at_of(*entropy, "entropy", {r.rows}, at::kFloat, r.device);
    }
    Rows ro;
    const Tensor grad = out_for(out, logits, r, ro);
    const c10::DeviceGuard guard(r.device);
    check(mlda_token_logprobs_backward(r.at, r.stride, r.rows, r.cols, r.kind, d.tokens, d.row_ptr, d.n, (const float*)at_stats, (const float*)at_grad,
                                       (const float*)at_entropy, (const float*)at_h, ro.at, ro.stride, stream_of(r.device)));
    written(out);
    return grad;
}

std::tuple<Tensor, Tensor> token_logprobs_grad(const Tensor& logits, const Tensor& tokens, const Tensor& weights, const Maybe& row_ptr, const Maybe& out) {
    const Documents d(logits, tokens, row_ptr);
    const Rows& r = d.r;
    void* at_weights = at_of(weights, "weights", {d.n}, at::kFloat, r.device);
    const Tensor logprobs = of_tokens(d.n, r.rows, r.device);
    Rows ro;
    const Tensor grad = out_for(out, logits, r, ro);
    const Workspace w(d.workspace(0), r.device);
    const c10::DeviceGuard guard(r.device);
    check(mlda_token_logprobs_grad(r.at, r.stride, r.rows, r.cols, r.kind, d.tokens, d.row_ptr, d.n, (const float*)at_weights,
                                   logprobs.data_ptr<float>(), ro.at, ro.stride, w.at, w.bytes, stream_of(r.device)));
    written(out);
    return {logprobs, grad};
}

// The norm of the tensors; with `most` they are scaled, into `out` or in place.
Tensor clip_grads(const std::vector<Tensor>& tensors, std::optional<double> most, const std::optional<std::vector<Tensor>>& out) {
    TORCH_CHECK_VALUE(!tensors.empty(), "there must be at least one tensor");
    TORCH_CHECK_VALUE(tensors[0].defined() && tensors[0].is_cuda(), "tensors must be on a GPU: there is no CPU path");
    const size_t n = tensors.size();
    const at::Device device = tensors[0].device();
    TORCH_CHECK_VALUE(n <= INT32_MAX && (!out || out->size() == n), "out must have as many tensors");
    std::vector<const void*> in(n);
    std::vector<void*> to(n);
    std::vector<int64_t> sizes(n);
    std::vector<int32_t> types(n);
    for (size_t i = 0; i < n; ++i) {
        const Tensor& t = tensors[i];
        TORCH_CHECK_VALUE(t.defined() && t.is_contiguous() && t.device() == device && type_code(t) >= 0,
                          "tensors must be contiguous fp32, bf16 or fp16 tensors on one GPU");
        in[i] = to[i] = t.data_ptr();
        sizes[i] = t.numel();
        types[i] = type_code(t);
        if (out) {
            const Tensor& o = (*out)[i];
            TORCH_CHECK_VALUE(o.defined() && o.is_contiguous() && o.device() == device && o.scalar_type() == t.scalar_type() && o.sizes() == t.sizes(),
                              "out must have a contiguous tensor of the shape, type and device of each of tensors");
            to[i] = o.data_ptr();
        }
    }
    const Tensor norm = fp32({}, device);
    size_t bytes = 0;
    check(mlda_grad_norm_workspace_bytes((int32_t)n, &bytes));
    const Workspace w(bytes, device);
    const c10::DeviceGuard guard(device);
    if (most) {
        check(mlda_clip_grads(in.data(), to.data(), sizes.data(), types.data(), (int32_t)n, *most, norm.data_ptr<float>(), w.at, w.bytes, stream_of(device)));
        for (const Tensor& t : out ? *out : tensors) written(t);
    } else {
        check(mlda_grad_norm(in.data(), sizes.data(), types.data(), (int32_t)n, norm.data_ptr<float>(), w.at, w.bytes, stream_of(device)));
    }
    return norm;
}

}  // namespace

PYBIND11_MODULE(_tensors, m) {
    typedef py::handle H;
    m.def("layer_norm", [](H x, H weight, H bias, double eps, H out) {
        return layer_norm(tensor(x, "x"), maybe(weight, "weight"), maybe(bias, "bias"), eps, maybe(out, "out"));
    });
    m.def("layer_norm_backward", [](H grad_y, H x, H mean, H rstd, H weight, H out) {
        return layer_norm_backward(tensor(grad_y, "grad_y"), tensor(x, "x"), tensor(mean, "mean"), tensor(rstd, "rstd"), maybe(weight, "weight"),
                                   maybe(out, "out"));
    });
    m.def("token_logprobs", [](H logits, H tokens, H row_ptr, int64_t alternatives, bool entropy) {
        return token_logprobs(tensor(logits, "logits"), tensor(tokens, "tokens"), maybe(row_ptr, "row_ptr"), alternatives, entropy);
    });
    m.def("token_logprobs_backward", [](H grad_logprobs, H logits, H tokens, H stats, H row_ptr, H grad_entropy, H entropy, H out) {
        return token_logprobs_backward(tensor(grad_logprobs, "grad_logprobs"), tensor(logits, "logits"), tensor(tokens, "tokens"),
                                       tensor(stats, "stats"), maybe(row_ptr, "row_ptr"), maybe(grad_entropy, "grad_entropy"),
                                       maybe(entropy, "entropy"), maybe(out, "out"));
    });
    m.def("token_logprobs_grad", [](H logits, H tokens, H weights, H row_ptr, H out) {
        return token_logprobs_grad(tensor(logits, "logits"), tensor(tokens, "tokens"), tensor(weights, "weights"), maybe(row_ptr, "row_ptr"),
                                   maybe(out, "out"));
    });
    m.def("grad_norm", [](H tensors) { return clip_grads(tensors_of(tensors, "every one of tensors"), std::nullopt, std::nullopt); });
    m.def("clip_grads", [](H tensors, std::optional<double> most, H out) {
        TORCH_CHECK_VALUE(most, "max_norm must be a number: grad_norm gives the norm alone");
        return clip_grads(tensors_of(tensors, "every one of tensors"), most,
                          out.is_none() ? std::nullopt : std::optional<std::vector<Tensor>>(tensors_of(out, "every one of out")));
    });
}
