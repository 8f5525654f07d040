// Python binding of the calls that a training step makes, as a native module: argument checks, output and scratch tensors,
// stream lookup and the autograd nodes (GELU + Linear, gated linear, rotary positions) in C++, on top of the C ABI in include/dropit.h.  A layer call is tens
// of microseconds of GPU time, less than what marshalling the same calls through ctypes takes on the host.
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGraphsC10Utils.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/saved_variable.h>
#include <torch/extension.h>

#include <algorithm>
#include <cstdlib>
#include <mutex>
#include <tuple>
#include <vector>

#include "dropit.h"
#include "layer_ops.h"

namespace {

using at::Tensor;

py::object* g_error_class = nullptr;

// A status that is not OK becomes the package's DropITError.  It travels as a python_error, which is a std::exception: the autograd
// engine hands those from the thread of a backward pass to the caller, anything else that leaves a node ends the process.
void check(dropit_status s, const char* where) {
    if (s == DROPIT_OK) return;
    py::gil_scoped_acquire gil;
    PyErr_SetObject(g_error_class ? g_error_class->ptr() : PyExc_RuntimeError, py::make_tuple((int)s, where).ptr());
    python_error error;
    error.persist();
    throw error;
}

std::string type_name(const Tensor& t) { return "torch." + c10::getDtypeNames(t.scalar_type()).first; }
dropit_dtype dtype_code(const Tensor& t, const char* name) {
    if (t.scalar_type() == at::kBFloat16) return DROPIT_BF16;
    if (t.scalar_type() == at::kFloat) return DROPIT_F32;
    throw py::type_error(std::string(name) + ": dtype " + type_name(t) + " is not supported (bf16 or fp32)");
}
dropit_dtype require_cuda(const Tensor& t, const char* name) {
    if (!t.is_cuda()) throw py::value_error(std::string(name) + " must be a CUDA tensor (there is no CPU path)");
    if (!t.is_contiguous()) throw py::value_error(std::string(name) + " must be contiguous");
    return dtype_code(t, name);
}
void require_bf16(const Tensor& t, const char* where) {
    if (t.scalar_type() != at::kBFloat16) throw py::type_error(std::string(where) + " takes bf16 tensors");
}

Tensor empty1(int64_t n, at::ScalarType type, const Tensor& like) {
    return at::detail::empty_cuda({n}, type, like.device(), c10::nullopt);
}
void* ptr(const Tensor& t) { return t.defined() && t.numel() ? t.data_ptr() : nullptr; }
void* table_ptr(const c10::optional<Tensor>& t) { return t.has_value() ? ptr(*t) : nullptr; }
void* current_stream(const Tensor& t) { return c10::cuda::getCurrentCUDAStream(t.device().index()).stream(); }

// One status word per device, which every kernel's bounded waits report to.
Tensor status_word(int64_t device) {
    static std::mutex lock;
    static auto* words = new std::vector<Tensor>();      // never destroyed: the CUDA context may be gone by then
    std::lock_guard<std::mutex> guard(lock);
    if ((int64_t)words->size() <= device) words->resize(device + 1);
    Tensor& w = (*words)[device];
    if (!w.defined()) w = at::zeros({4}, at::TensorOptions().dtype(at::kInt).device(at::kCUDA, (c10::DeviceIndex)device));
    return w;
}
int32_t* status_ptr(const Tensor& like) { return status_word(like.device().index()).data_ptr<int32_t>(); }

// The caller's scratch if it is large enough, else a new one.
Tensor scratch(const c10::optional<Tensor>& given, size_t bytes, const Tensor& like) {
    if (given.has_value() && given->defined() && (size_t)given->numel() >= bytes) return *given;
    return empty1(bytes > 16 ? (int64_t)bytes : 16, at::kByte, like);
}

struct CacheParts {
    Tensor values, meta, offsets;
    int64_t k;
    size_t workspace;
};
CacheParts make_cache(const Tensor& x, dropit_dtype dt, double gamma, int fmt) {
    size_t vb, mb, ob, wb;
    const int64_t n = x.numel();
    check(dropit_cache_sizes(n, gamma, dt, (dropit_format)fmt, &vb, &mb, &ob, &wb), "dropit_cache_sizes");
    CacheParts c;
    c.k = dropit_keep_count(n, gamma);
    c.values = empty1((int64_t)(vb / (dt == DROPIT_BF16 ? 2 : 4)), x.scalar_type(), x);
    c.meta = empty1((int64_t)(mb / 4), at::kInt, x);
    c.offsets = empty1((int64_t)(ob / 4), at::kInt, x);
    c.workspace = wb;
    return c;
}

using CacheTuple = std::tuple<Tensor, Tensor, Tensor, int64_t>;

CacheTuple compress(const Tensor& x, double gamma, int fmt, const c10::optional<Tensor>& workspace) {
    const dropit_dtype dt = require_cuda(x, "x");
    c10::cuda::CUDAGuard guard(x.device());
    CacheParts c = make_cache(x, dt, gamma, fmt);
    const Tensor ws = scratch(workspace, c.workspace, x);
    check(dropit_compress(ptr(x), x.numel(), gamma, dt, (dropit_format)fmt, ptr(c.values), ptr(c.meta), (uint32_t*)ptr(c.offsets),
                          ptr(ws), (size_t)ws.numel(), status_ptr(x), current_stream(x)), "dropit_compress");
    return {c.values, c.meta, c.offsets, c.k};
}

std::tuple<Tensor, Tensor> produce(const Tensor& x, double gamma, int act, const c10::optional<Tensor>& table, bool want_y) {
    require_cuda(x, "x");
    require_bf16(x, "dropit_produce");
    c10::cuda::CUDAGuard guard(x.device());
    size_t bytes;
    check(dropit_produce_workspace(x.numel(), &bytes), "dropit_produce_workspace");
    Tensor y;
    if (want_y) y = at::empty_like(x);
    Tensor prep = empty1(bytes > 16 ? (int64_t)bytes : 16, at::kByte, x);
    check(dropit_produce(ptr(x), x.numel(), gamma, (dropit_activation)act, table.has_value() ? (const uint16_t*)ptr(*table) : nullptr,
                         ptr(y), ptr(prep), (size_t)prep.numel(), current_stream(x)), "dropit_produce");
    return {y, prep};
}

CacheTuple compress_prepared(const Tensor& y, double gamma, const Tensor& prep, int fmt, const c10::optional<Tensor>& workspace) {
    require_cuda(y, "y");
    require_bf16(y, "dropit_compress_prepared");
    c10::cuda::CUDAGuard guard(y.device());
    CacheParts c = make_cache(y, DROPIT_BF16, gamma, fmt);
    const Tensor ws = scratch(workspace, c.workspace, y);
    check(dropit_compress_prepared(ptr(y), y.numel(), gamma, (dropit_format)fmt, ptr(c.values), ptr(c.meta), (uint32_t*)ptr(c.offsets),
                                   ptr(prep), (size_t)prep.numel(), ptr(ws), (size_t)ws.numel(), status_ptr(y), current_stream(y)),
          "dropit_compress_prepared");
    return {c.values, c.meta, c.offsets, c.k};
}

std::string mismatch(const Tensor& dy, const Tensor& values) {
    return "dy dtype " + type_name(dy) + " != cache dtype " + type_name(values);
}

// `offsets` may be absent: a coordinate cache can do without its seek table.
Tensor weight_grad(const Tensor& dy, const Tensor& values, const Tensor& meta, const c10::optional<Tensor>& offsets, int64_t n, int64_t Ca,
                   int64_t k, int fmt, const c10::optional<Tensor>& out, bool accumulate, const c10::optional<Tensor>& workspace, bool no_scratch) {
    const dropit_dtype dt = require_cuda(dy, "dy");
    if (dy.scalar_type() != values.scalar_type()) throw py::type_error(mismatch(dy, values));
    const int64_t M = Ca ? n / Ca : 0, Cz = dy.size(-1);
    if (dy.numel() != M * Cz)
        throw py::value_error("dy has " + std::to_string(dy.numel()) + " elements, expected " + std::to_string(M) + " x " + std::to_string(Cz));
    if (!out.has_value() && accumulate) throw py::value_error("accumulate=True needs out");
    c10::cuda::CUDAGuard guard(dy.device());
    const Tensor dw = out.has_value() ? *out : Tensor(at::detail::empty_cuda({Cz, Ca}, at::kFloat, dy.device(), c10::nullopt));
    size_t bytes;
    check(dropit_weight_grad_workspace(M, Ca, Cz, dt, (dropit_format)fmt, &bytes), "dropit_weight_grad_workspace");
    const Tensor ws = scratch(workspace, bytes, dy);
    auto fn = no_scratch ? dropit_weight_grad_fused : dropit_weight_grad;
    check(fn(ptr(dy), ptr(values), ptr(meta), (const uint32_t*)table_ptr(offsets), M, Ca, Cz, k, dt, (dropit_format)fmt, (float*)ptr(dw),
             accumulate ? 1 : 0, ptr(ws), (size_t)ws.numel(), status_ptr(dy), current_stream(dy)),
          no_scratch ? "dropit_weight_grad_fused" : "dropit_weight_grad");
    return dw;
}

Tensor conv_weight_grad(const Tensor& dy, const Tensor& values, const Tensor& meta, const c10::optional<Tensor>& offsets, int B, int Ca, int H,
                        int W, int R, int S, int stride, int pad, int dilation, int64_t k, int fmt, const c10::optional<Tensor>& out,
                        bool accumulate, const c10::optional<Tensor>& workspace) {
    const dropit_dtype dt = require_cuda(dy, "dy");
    if (dy.scalar_type() != values.scalar_type()) throw py::type_error(mismatch(dy, values));
    const int Cz = (int)dy.size(1);
    if (!out.has_value() && accumulate) throw py::value_error("accumulate=True needs out");
    c10::cuda::CUDAGuard guard(dy.device());
    const Tensor dw = out.has_value() ? *out : Tensor(at::detail::empty_cuda({Cz, Ca, R, S}, at::kFloat, dy.device(), c10::nullopt));
    size_t bytes;
    check(dropit_conv_weight_grad_workspace(B, Ca, H, W, Cz, R, S, stride, pad, dt, (dropit_format)fmt, &bytes),
          "dropit_conv_weight_grad_workspace");
    const Tensor ws = scratch(workspace, bytes, dy);
    check(dropit_conv_weight_grad(ptr(dy), ptr(values), ptr(meta), (const uint32_t*)table_ptr(offsets), B, Ca, H, W, Cz, R, S, stride, pad,
                                  dilation, k, dt, (dropit_format)fmt, (float*)ptr(dw), accumulate ? 1 : 0, ptr(ws),
                                  (size_t)ws.numel(), status_ptr(dy), current_stream(dy)), "dropit_conv_weight_grad");
    return dw;
}

// z = GELU(x) W^T + b for bf16 tensors, with the GELU written by the library's producer kernel so that the selection statistics
// of GELU(x), the tensor the Linear caches, are taken while it is written (Sec. 3.5: the activation keeps its own cache x; only
// the Linear's cache is replaced by D(GELU(x))).
struct GeluLinear : public torch::autograd::Function<GeluLinear> {
    static Tensor forward(torch::autograd::AutogradContext* ctx, const Tensor& x, const Tensor& weight, const c10::optional<Tensor>& bias,
                          double gamma, int64_t fmt, const Tensor& table) {
        const Tensor x2 = x.reshape({-1, x.size(-1)}).contiguous();
        Tensor y, prep;
        std::tie(y, prep) = produce(x2, gamma, DROPIT_ACT_TABLE, table, true);
        std::vector<int64_t> shape = x.sizes().vec();
        shape.back() = weight.size(0);
        Tensor z = at::linear(y, weight, bias).reshape(shape);
        Tensor values, meta, offsets;
        int64_t k;
        std::tie(values, meta, offsets, k) = compress_prepared(y, gamma, prep, (int)fmt, c10::nullopt);
        ctx->save_for_backward({x2, weight, values, meta, offsets});
        ctx->saved_data["cache"] = std::vector<int64_t>{y.numel(), y.size(1), k, fmt};
        ctx->saved_data["shape"] = x.sizes().vec();
        ctx->saved_data["bias"] = bias.has_value() && bias->defined();
        return z;
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
        const auto saved = ctx->get_saved_variables();
        const Tensor &x2 = saved[0], &weight = saved[1], &values = saved[2];
        const auto cache = ctx->saved_data["cache"].toIntVector();
        const Tensor dz2 = grads[0].reshape({-1, grads[0].size(-1)}).contiguous();
        const bool bias = ctx->saved_data["bias"].toBool() && ctx->needs_input_grad(2);
        // With create_graph the gradients are to be differentiated again: what can be is then formed by operations that autograd knows.
        const bool graph = at::GradMode::is_enabled();
        Tensor dx, dw, db;
        if (ctx->needs_input_grad(0)) {                                  // Eq. 3: exact, needs theta only; the activation's cache is x
            const Tensor dy = at::matmul(dz2, weight);
            if (!graph && dy.scalar_type() == at::kBFloat16 && x2.scalar_type() == at::kBFloat16 && dy.is_contiguous() &&
                reinterpret_cast<uintptr_t>(x2.data_ptr()) % 16 == 0) {
                c10::cuda::CUDAGuard guard(dy.device());
                dx = at::empty_like(x2);
                check(dropit::gelu_backward_bf16(ptr(dy), ptr(x2), ptr(dx), x2.numel(), current_stream(dy)), "gelu_backward");
            } else {
                dx = at::gelu_backward(dy, x2);
            }
            dx = dx.reshape(ctx->saved_data["shape"].toIntVector());
        }
        const bool own = !graph && weight.scalar_type() == at::kBFloat16 && dz2.scalar_type() == at::kBFloat16 && dz2.size(1) % 8 == 0 &&
                         dz2.numel() != 0 && reinterpret_cast<uintptr_t>(dz2.data_ptr()) % 16 == 0;
        if (ctx->needs_input_grad(1)) {                                  // Eq. 6
            const Tensor full = weight_grad(dz2.to(values.scalar_type()), values, saved[3], saved[4], cache[0], cache[1], cache[2],
                                            (int)cache[3], c10::nullopt, false, c10::nullopt, false);
            if (own) {                                                   // rounded to the parameter's type together with the bias gradient
                c10::cuda::CUDAGuard guard(dz2.device());
                dw = at::detail::empty_cuda(full.sizes(), at::kBFloat16, full.device(), c10::nullopt);
                if (bias) db = empty1(dz2.size(1), at::kBFloat16, dz2);
                check(dropit::finish_linear_backward((const float*)ptr(full), ptr(dw), full.numel(), ptr(dz2), dz2.size(0), dz2.size(1),
                                                     bias ? ptr(db) : nullptr, current_stream(dz2)), "finish_linear_backward");
            } else {
                dw = full.to(weight.scalar_type());
            }
        }
        if (bias && !db.defined()) db = dz2.sum(0);
        return {dx, dw, db, Tensor(), Tensor(), Tensor()};
    }
};

Tensor gelu_linear(const Tensor& x, const Tensor& weight, const c10::optional<Tensor>& bias, double gamma, int64_t fmt, const Tensor& table) {
    return GeluLinear::apply(x, weight, bias, gamma, fmt, table);
}

// The nodes below compute no forward-mode derivatives, and results without a tangent would pass for constants.
bool has_tangent(const Tensor& t) { return t.defined() && t._fw_grad(/*level=*/0).defined(); }
bool has_tangent(const c10::optional<Tensor>& t) { return t.has_value() && has_tangent(*t); }
template <typename... T>
void refuse_tangents(const char* name, const T&... inputs) {
    TORCH_CHECK_NOT_IMPLEMENTED(!(has_tangent(inputs) || ...), name, " has no forward-mode derivative");
}

// ---- gated linear: h = f(x Wg^T + bg) * (x Wu^T + bu) ----

// The library takes 16-byte aligned buffers; a slice may start anywhere.
Tensor aligned(const Tensor& t) {
    const Tensor c = t.contiguous();
    return reinterpret_cast<uintptr_t>(c.data_ptr()) % 16 ? c.clone() : c;
}
void require_like(const Tensor& t, const Tensor& x, const char* name, const char* of) {
    if (t.device() != x.device()) throw py::value_error(std::string(name) + " is on another device than " + of);
    if (t.scalar_type() != x.scalar_type())
        throw py::type_error(std::string(name) + " dtype " + type_name(t) + " != " + of + " dtype " + type_name(x));
}
struct GatedSizes {
    int64_t M, C, H;
    dropit_dtype dtype;
};
GatedSizes gated_sizes(const Tensor& x, const Tensor& weight, const c10::optional<Tensor>& bias) {
    if (!x.is_cuda()) throw py::value_error("x must be a CUDA tensor (there is no CPU path)");
    GatedSizes s;
    s.dtype = dtype_code(x, "x");
    if (weight.dim() != 2 || weight.size(0) % 2 || weight.size(0) == 0 || weight.size(1) == 0)
        throw py::value_error("weight must be [2 * hidden, channels]: the gate's rows, then the other half");
    s.C = weight.size(1);
    s.H = weight.size(0) / 2;
    if (x.dim() < 1 || x.size(-1) != s.C) throw py::value_error("x must have " + std::to_string(s.C) + " channels in its last dimension");
    s.M = x.numel() / s.C;
    require_like(weight, x, "weight", "x");
    if (bias.has_value() && bias->defined()) {
        require_like(*bias, x, "bias", "x");
        if (bias->dim() != 1 || bias->numel() != 2 * s.H) throw py::value_error("bias must have " + std::to_string(2 * s.H) + " elements");
    }
    return s;
}

std::vector<int64_t> with_last(const Tensor& x, int64_t last) {
    std::vector<int64_t> shape = x.sizes().vec();
    shape.back() = last;
    return shape;
}
// h and, with keep, gu = a | u, in x's leading dimensions; x is laid out densely and aligned.
std::tuple<Tensor, Tensor> gated_products(const Tensor& x, const Tensor& weight, const c10::optional<Tensor>& bias, const GatedSizes& s, int64_t gate,
                                          bool keep) {
    c10::cuda::CUDAGuard guard(x.device());
    const Tensor w = aligned(weight);
    Tensor b;
    if (bias.has_value() && bias->defined()) b = aligned(*bias);
    Tensor h = at::detail::empty_cuda(with_last(x, s.H), x.scalar_type(), x.device(), c10::nullopt), gu;
    if (keep) gu = at::detail::empty_cuda(with_last(x, 2 * s.H), x.scalar_type(), x.device(), c10::nullopt);
    check(dropit_gated_linear(ptr(x), ptr(w), b.defined() ? ptr(b) : nullptr, s.M, s.C, s.H, s.dtype, (dropit_gate)gate, ptr(h),
                              keep ? ptr(gu) : nullptr, status_ptr(x), current_stream(x)), "dropit_gated_linear");
    return {h, gu};
}

std::tuple<Tensor, c10::optional<Tensor>> gated_linear(const Tensor& x, const Tensor& weight, const c10::optional<Tensor>& bias, int64_t gate, bool keep) {
    refuse_tangents("the gated linear", x, weight, bias);
    const GatedSizes s = gated_sizes(x, weight, bias);
    Tensor h, gu;
    std::tie(h, gu) = gated_products(aligned(x), weight, bias, s, gate, keep);
    c10::optional<Tensor> kept;
    if (keep) kept = gu;
    return {h, kept};
}

// h outside of training, unless a derivative is asked for or the kernels have no form for x: nothing then.
c10::optional<Tensor> gated_inference(const Tensor& x, const Tensor& weight, const c10::optional<Tensor>& bias, int64_t gate) {
    if (!x.is_cuda() || (x.scalar_type() != at::kBFloat16 && x.scalar_type() != at::kFloat)) return c10::nullopt;
    if (at::GradMode::is_enabled() && (x.requires_grad() || weight.requires_grad() || (bias.has_value() && bias->requires_grad()))) return c10::nullopt;
    if (has_tangent(x) || has_tangent(weight) || has_tangent(bias)) return c10::nullopt;
    const GatedSizes s = gated_sizes(x, weight, bias);
    const int64_t limit = (int64_t)1 << 31;
    if (s.M >= limit || s.M * std::max(s.C, 2 * s.H) >= limit) return c10::nullopt;
    return std::get<0>(gated_products(aligned(x), weight, bias, s, gate, false));
}

std::tuple<Tensor, c10::optional<Tensor>> gated_linear_backward(const Tensor& dh, const Tensor& gu, int64_t gate, bool want_db) {
    refuse_tangents("the gated linear's gradient", dh, gu);
    if (!dh.is_cuda()) throw py::value_error("dh must be a CUDA tensor (there is no CPU path)");
    const dropit_dtype dt = dtype_code(dh, "dh");
    require_like(gu, dh, "gu", "dh");
    if (dh.dim() < 1 || dh.size(-1) == 0 || gu.sizes().vec() != with_last(dh, 2 * dh.size(-1)))
        throw py::value_error("gu must have dh's shape with twice its last dimension");
    c10::cuda::CUDAGuard guard(dh.device());
    const int64_t H = dh.size(-1), M = dh.numel() / H;
    const Tensor d = aligned(dh), k = aligned(gu);
    Tensor dgu = at::detail::empty_cuda(gu.sizes(), gu.scalar_type(), gu.device(), c10::nullopt);
    c10::optional<Tensor> db;
    Tensor ws;
    if (want_db) {
        size_t bytes;
        check(dropit_gated_linear_backward_workspace(M, H, dt, &bytes), "dropit_gated_linear_backward_workspace");
        db = empty1(2 * H, dh.scalar_type(), dh);
        ws = empty1(bytes > 16 ? (int64_t)bytes : 16, at::kByte, dh);
    }
    check(dropit_gated_linear_backward(ptr(d), ptr(k), M, H, dt, (dropit_gate)gate, ptr(dgu), want_db ? ptr(*db) : nullptr, want_db ? ptr(ws) : nullptr,
                                       want_db ? (size_t)ws.numel() : 0, current_stream(dh)), "dropit_gated_linear_backward");
    return {dgu, db};
}

Tensor gated_input_grad(const Tensor& dgu, const Tensor& weight) {
    refuse_tangents("the gated linear's gradient", dgu, weight);
    if (!dgu.is_cuda()) throw py::value_error("dgu must be a CUDA tensor (there is no CPU path)");
    const dropit_dtype dt = dtype_code(dgu, "dgu");
    require_like(weight, dgu, "weight", "dgu");
    if (weight.dim() != 2 || weight.size(0) % 2 || dgu.dim() < 1 || dgu.size(-1) != weight.size(0) || weight.numel() == 0)
        throw py::value_error("dgu's last dimension must be weight's first, 2 * hidden");
    c10::cuda::CUDAGuard guard(dgu.device());
    const int64_t K = weight.size(0), C = weight.size(1), M = dgu.numel() / K;
    const Tensor d = aligned(dgu), w = aligned(weight);
    Tensor dx = at::detail::empty_cuda(with_last(dgu, C), dgu.scalar_type(), dgu.device(), c10::nullopt);
    check(dropit_gated_input_grad(ptr(d), ptr(w), M, C, K / 2, dt, ptr(dx), status_ptr(dgu), current_stream(dgu)), "dropit_gated_input_grad");
    return dx;
}

bool wants(const Tensor& t) { return t.defined() && t.requires_grad(); }
// A node that takes gradients of these tensors (made without the templates of autograd::Function, whose bookkeeping takes longer than the kernels
// of a small layer).
template <typename Node>
std::shared_ptr<Node> make_node(const torch::autograd::variable_list& inputs) {
    std::shared_ptr<Node> node(new Node(), torch::autograd::deleteNode);
    node->set_next_edges(torch::autograd::collect_next_edges(inputs));
    return node;
}

// The layer: x is cached as D(x) for the weight gradient (Sec. 3.2), a and u as the gate's own cache (Sec. 3.5).
struct GatedLinearNode : public torch::autograd::Node {
    torch::autograd::SavedVariable weight_, gu_, values_, meta_, offsets_;
    std::vector<int64_t> shape;              // of x
    int64_t k = 0, fmt = 0, gate = 0;
    std::string name() const override { return "DropITGatedLinear"; }
    void release_variables() override {
        std::lock_guard<std::mutex> lock(mutex_);
        for (auto* v : {&weight_, &gu_, &values_, &meta_, &offsets_}) v->reset_data();
    }
    torch::autograd::variable_list apply(torch::autograd::variable_list&& grads) override {
        std::lock_guard<std::mutex> lock(mutex_);
        torch::autograd::variable_list out(3);
        if (!grads[0].defined()) return out;
        refuse_tangents("the gated linear's gradient", grads[0]);
        const Tensor weight = weight_.unpack(), gu = gu_.unpack();          // an error, if they have been released
        const bool want_x = task_should_compute_output(0), want_w = task_should_compute_output(1), want_b = task_should_compute_output(2);
        {
            at::AutoGradMode no_graph(false);
            c10::cuda::CUDAGuard guard(gu.device());
            const Tensor dh = aligned(grads[0].scalar_type() == gu.scalar_type() ? grads[0] : grads[0].to(gu.scalar_type()));
            const int64_t H = gu.size(-1) / 2, M = gu.numel() / (2 * H);
            const dropit_dtype dt = dtype_code(gu, "gu");
            const Tensor dgu = at::detail::empty_cuda({M, 2 * H}, gu.scalar_type(), gu.device(), c10::nullopt);
            const int64_t chunks = want_b ? dropit::gated_backward_chunks(M, H, dt) : 0;
            Tensor partial, full;
            if (want_b) partial = empty1(chunks * 2 * H, at::kFloat, gu);
            if (want_b || M)
                check(dropit::gated_backward_sums(ptr(dh), ptr(gu), M, H, dt, (dropit_gate)gate, ptr(dgu), want_b ? (float*)ptr(partial) : nullptr,
                                                  current_stream(gu)), "dropit_gated_linear_backward");
            if (want_x) {
                const Tensor w = aligned(weight);
                out[0] = at::detail::empty_cuda(shape, gu.scalar_type(), gu.device(), c10::nullopt);
                check(dropit_gated_input_grad(ptr(dgu), ptr(w), M, weight.size(1), H, dt, ptr(out[0]), status_ptr(gu), current_stream(gu)),
                      "dropit_gated_input_grad");
            }
            if (want_w) {
                full = weight_grad(dgu, values_.unpack(), meta_.unpack(), offsets_.unpack(), M * weight.size(1), weight.size(1), k, (int)fmt, c10::nullopt, false, c10::nullopt, false);
                out[1] = dt == DROPIT_F32 ? full : Tensor(at::detail::empty_cuda(full.sizes(), gu.scalar_type(), gu.device(), c10::nullopt));
            }
            if (want_b) out[2] = empty1(2 * H, gu.scalar_type(), gu);
            // the bias gradient and the rounding of the weight gradient to the parameter's type
            const bool rounds = want_w && dt == DROPIT_BF16;
            check(dropit::gated_finish(want_b ? (const float*)ptr(partial) : nullptr, chunks, 2 * H, dt, want_b ? ptr(out[2]) : nullptr,
                                       rounds ? (const float*)ptr(full) : nullptr, rounds ? ptr(out[1]) : nullptr, rounds ? full.numel() : 0, current_stream(gu)),
                  "dropit_gated_linear_backward");
        }
        if (at::GradMode::is_enabled()) {       // a and u depend on x and W: what is kept of them cannot be differentiated again
            torch::autograd::variable_list given;
            std::vector<size_t> at_place;
            for (size_t i = 0; i < 3; ++i)
                if (out[i].defined()) given.push_back(out[i].requires_grad_(true)), at_place.push_back(i);
            auto error = std::make_shared<torch::autograd::DelayedError>("the gradients of DropITGatedLinear cannot be differentiated again",
                                                                         (int64_t)given.size());
            const auto guarded = (*error)(std::move(given));
            for (size_t i = 0; i < guarded.size(); ++i) out[at_place[i]] = guarded[i];
        }
        return out;
    }
};
Tensor gated_layer(const Tensor& x, const Tensor& weight, const c10::optional<Tensor>& bias, double gamma, int64_t fmt, int64_t gate) {
    refuse_tangents("the gated linear", x, weight, bias);
    const Tensor b = bias.has_value() ? *bias : Tensor();
    const GatedSizes s = gated_sizes(x, weight, bias);
    const bool records = at::GradMode::is_enabled() && (wants(x) || wants(weight) || wants(b));
    std::shared_ptr<GatedLinearNode> node;
    Tensor h;
    {
        at::AutoGradMode no_graph(false);
        const Tensor dense = aligned(x);
        Tensor gu;
        std::tie(h, gu) = gated_products(dense, weight, bias, s, gate, records);
        if (records) {
            node = make_node<GatedLinearNode>({x, weight, b});
            node->weight_ = torch::autograd::SavedVariable(weight, false);
            node->gu_ = torch::autograd::SavedVariable(gu, false);
            node->shape = x.sizes().vec();
            node->fmt = fmt;
            node->gate = gate;
            if (weight.requires_grad()) {
                const CacheTuple cache = compress(dense, gamma, (int)fmt, c10::nullopt);
                node->values_ = torch::autograd::SavedVariable(std::get<0>(cache), false);
                node->meta_ = torch::autograd::SavedVariable(std::get<1>(cache), false);
                node->offsets_ = torch::autograd::SavedVariable(std::get<2>(cache), false);
                node->k = std::get<3>(cache);
            }
        }
    }
    if (records) torch::autograd::set_history(h, node);
    return h;
}

// ---- rotary positions ----

// A plan travels as the bytes of the C structure in a CPU tensor.
Tensor rotary_plan(int64_t head_dim, const std::vector<int64_t>& sections, double theta, bool shared, bool interleaved) {
    std::vector<int> s(sections.begin(), sections.end());
    Tensor t = at::zeros({(int64_t)sizeof(dropit_rotary_plan)}, at::kByte);
    check(dropit_rotary_make_plan((int)head_dim, s.data(), (int)s.size(), theta, shared, interleaved, (dropit_rotary_plan*)t.data_ptr()),
          "dropit_rotary_make_plan");
    return t;
}
const dropit_rotary_plan* plan_of(const Tensor& t) {
    if (t.device().type() != at::kCPU || t.scalar_type() != at::kByte || t.numel() != (int64_t)sizeof(dropit_rotary_plan) || !t.is_contiguous())
        throw py::value_error("plan must be what dropit_rotary_plan returned");
    return (const dropit_rotary_plan*)t.data_ptr();
}

// [.., length, heads, head_dim] with a batch dimension or without
dropit_rotary_tensor rotary_tensor(const Tensor& in, Tensor& out, const dropit_rotary_plan* plan, const char* name) {
    if ((in.dim() != 3 && in.dim() != 4) || in.size(-1) != plan->head_dim)
        throw py::value_error(std::string(name) + " must be [batch, length, heads, " + std::to_string(plan->head_dim) + "] or [length, heads, " +
                              std::to_string(plan->head_dim) + "]");
    const bool batched = in.dim() == 4;
    dropit_rotary_tensor t;
    t.in = in.numel() ? in.data_ptr() : nullptr;
    t.out = out.numel() ? out.data_ptr() : nullptr;
    t.in_batch = batched ? in.stride(0) : 0;
    t.in_token = in.stride(-3);
    t.in_head = in.stride(-2);
    t.out_batch = batched ? out.stride(0) : 0;
    t.out_token = out.stride(-3);
    t.out_head = out.stride(-2);
    t.heads = (int32_t)in.size(-2);
    return t;
}
Tensor rotary_input(const Tensor& t) { return t.dim() && t.stride(-1) != 1 ? t.contiguous() : t; }

// Writing in place: do two (token, head)s have channels in common?  Rows of `size(-1)` channels lie at multiples of the other dimensions' strides.
// Of one tensor: no, if every stride passes all that the smaller ones reach (any permutation of a slice of a dense tensor).
bool has_places_of_its_own(const Tensor& t) {
    std::vector<std::pair<int64_t, int64_t>> dims;
    for (int64_t d = 0; d + 1 < t.dim(); ++d)
        if (t.size(d) > 1) dims.emplace_back(t.stride(d), t.size(d));
    std::sort(dims.begin(), dims.end());
    int64_t reach = t.dim() ? t.size(-1) : 1;
    for (const auto& [stride, size] : dims) {
        if (stride < reach) return t.numel() == 0;
        reach += (size - 1) * stride;
    }
    return true;
}
// Of two: is there a choice of steps whose sum comes within a row's width of the distance between the tensors?  A dimension that both have with the
// same stride counts once, by the difference of its indices.  Larger strides first: what the smaller ones reach leaves one to three choices for each.
struct Steps {
    int64_t stride, low, high;
};
bool meets(const std::vector<Steps>& steps, const std::vector<int64_t>& reach, size_t at, int64_t left, int& tries) {
    if (--tries < 0) return true;                                   // strides that are not worth the search
    if (at == steps.size()) return std::abs(left) <= reach[at];
    const Steps& s = steps[at];
    const auto quotient = [&](int64_t n) { return n / s.stride - (n % s.stride < 0); };     // rounded down
    const int64_t first = std::max(s.low, quotient(left - reach[at + 1] + s.stride - 1)), last = std::min(s.high, quotient(left + reach[at + 1]));
    for (int64_t i = first; i <= last; ++i)
        if (meets(steps, reach, at + 1, left - i * s.stride, tries)) return true;
    return false;
}
bool share_channels(const Tensor& q, const Tensor& k) {
    if (q.numel() == 0 || k.numel() == 0 || q.scalar_type() != k.scalar_type()) return false;
    const int64_t size = q.element_size(), bytes = (const char*)k.data_ptr() - (const char*)q.data_ptr();
    std::vector<Steps> steps;
    for (int64_t d = 0; d + 1 < q.dim(); ++d)
        if (q.size(d) > 1) steps.push_back({q.stride(d), 0, q.size(d) - 1});
    for (int64_t d = 0; d + 1 < k.dim(); ++d) {
        if (k.size(d) <= 1) continue;
        auto same = std::find_if(steps.begin(), steps.end(), [&](const Steps& s) { return s.stride == k.stride(d) && s.low == 0; });
        if (same != steps.end()) same->low = 1 - k.size(d);
        else steps.push_back({k.stride(d), 1 - k.size(d), 0});
    }
    std::sort(steps.begin(), steps.end(), [](const Steps& a, const Steps& b) { return a.stride > b.stride; });
    std::vector<int64_t> reach(steps.size() + 1);
    reach[steps.size()] = std::max(q.size(-1), k.size(-1)) - 1;
    for (size_t i = steps.size(); i-- > 0;) reach[i] = reach[i + 1] + std::max(-steps[i].low, steps[i].high) * steps[i].stride;
    int tries = 1 << 14;
    return meets(steps, reach, 0, bytes / size, tries);             // (both are aligned to their values)
}

std::tuple<Tensor, c10::optional<Tensor>> rotary(const Tensor& q_in, const c10::optional<Tensor>& k_in, const Tensor& positions, const Tensor& plan_bytes,
                                                 bool inverse, bool in_place) {
    refuse_tangents("the rotation", q_in, k_in, positions);
    const dropit_rotary_plan* plan = plan_of(plan_bytes);
    const bool has_k = k_in.has_value() && k_in->defined();
    if (in_place) {
        for (const Tensor& t : {q_in, has_k ? *k_in : q_in}) {
            if (t.dim() && t.stride(-1) != 1) throw py::value_error("in place: the channels of a head must lie together");
            if (!has_places_of_its_own(t)) throw py::value_error("in place: every head of a token must have a place of its own");
        }
        if (has_k && share_channels(q_in, *k_in)) throw py::value_error("in place: q and k share values");
        // what is written over would pass for the result of the operation that q and k came from
        TORCH_CHECK(!at::GradMode::is_enabled() || !(q_in.requires_grad() || (has_k && k_in->requires_grad())),
                    "in place: q or k requires a gradient, which the rotation would not be part of");
    }
    if (!q_in.is_cuda()) throw py::value_error("q must be a CUDA tensor (there is no CPU path)");
    const dropit_dtype dt = dtype_code(q_in, "q");
    const Tensor q = rotary_input(q_in), k = has_k ? rotary_input(*k_in) : Tensor();
    c10::cuda::CUDAGuard guard(q.device());
    Tensor q_out = in_place ? q : Tensor(at::detail::empty_cuda(q.sizes(), q.scalar_type(), q.device(), c10::nullopt)), k_out;
    const dropit_rotary_tensor tq = rotary_tensor(q, q_out, plan, "q");
    dropit_rotary_tensor tk;
    if (has_k) {
        require_like(k, q, "k", "q");
        k_out = in_place ? k : Tensor(at::detail::empty_cuda(k.sizes(), k.scalar_type(), k.device(), c10::nullopt));
        tk = rotary_tensor(k, k_out, plan, "k");
        if (k.dim() != q.dim() || k.size(-3) != q.size(-3) || (q.dim() == 4 && k.size(0) != q.size(0)))
            throw py::value_error("k must have q's batch and length");
    }
    const int64_t batch = q.dim() == 4 ? q.size(0) : 1, length = q.size(-3);
    if (positions.device() != q.device()) throw py::value_error("positions is on another device than q");
    dropit_position_type type;
    if (positions.scalar_type() == at::kInt) type = DROPIT_POSITION_I32;
    else if (positions.scalar_type() == at::kLong) type = DROPIT_POSITION_I64;
    else if (positions.scalar_type() == at::kFloat) type = DROPIT_POSITION_F32;
    else throw py::type_error("positions: dtype " + type_name(positions) + " is not supported (int32, int64 or fp32)");
    const bool each = positions.dim() == 3 && q.dim() == 4;
    if ((positions.dim() != 2 && !each) || positions.size(-1) != plan->axes || positions.size(-2) != length ||
        (each && positions.size(0) != batch && positions.size(0) != 1))
        throw py::value_error("positions must be [length, " + std::to_string(plan->axes) + "] or [batch, length, " + std::to_string(plan->axes) +
                              "] with q's length and batch");
    const int64_t pos_batch = each && positions.size(0) != 1 ? positions.stride(0) : 0;
    if (in_place) {         // an error for tensors of inference mode outside of it, before they change
        q_out.unsafeGetTensorImpl()->bump_version();
        if (has_k) k_out.unsafeGetTensorImpl()->bump_version();
    }
    check(dropit_rotary(plan, batch, length, &tq, has_k ? &tk : nullptr, positions.numel() ? positions.data_ptr() : nullptr, type, pos_batch,
                        positions.stride(-2), positions.stride(-1), dt, inverse, current_stream(q)), "dropit_rotary");
    c10::optional<Tensor> second;
    if (has_k) second = k_out;
    return {q_out, second};
}

std::tuple<Tensor, c10::optional<Tensor>> rotary_layer(const Tensor& q, const c10::optional<Tensor>& k, const Tensor& positions, const Tensor& plan, bool inverse);

// The gradient of a rotation is the inverse rotation, which can be differentiated again.
struct RotaryNode : public torch::autograd::Node {
    torch::autograd::SavedVariable positions_;
    Tensor plan;
    bool inverse = false, has_k = false;
    std::string name() const override { return "DropITRotary"; }
    void release_variables() override {
        std::lock_guard<std::mutex> lock(mutex_);
        positions_.reset_data();
    }
    torch::autograd::variable_list apply(torch::autograd::variable_list&& grads) override {
        std::lock_guard<std::mutex> lock(mutex_);
        torch::autograd::variable_list out(2);
        const bool q = grads[0].defined() && task_should_compute_output(0), k = has_k && grads[1].defined() && task_should_compute_output(1);
        if (!q && !k) return out;
        const Tensor positions = positions_.unpack();    // an error, if it has been released or changed in place
        c10::optional<Tensor> second;
        if (q && k) second = grads[1];
        Tensor first;
        std::tie(first, second) = rotary_layer(q ? grads[0] : grads[1], second, positions, plan, !inverse);
        out[q ? 0 : 1] = first;
        if (q && k) out[1] = *second;
        return out;
    }
};
std::tuple<Tensor, c10::optional<Tensor>> rotary_layer(const Tensor& q, const c10::optional<Tensor>& k, const Tensor& positions, const Tensor& plan,
                                                       bool inverse) {
    const bool has_k = k.has_value() && k->defined();
    const Tensor key = has_k ? *k : Tensor();
    TORCH_CHECK(!at::GradMode::is_enabled() || !positions.requires_grad(), "positions require a gradient, which the rotation does not have");
    if (!at::GradMode::is_enabled() || !(wants(q) || wants(key))) return rotary(q, k, positions, plan, inverse, false);
    Tensor q_out;
    c10::optional<Tensor> k_out;
    {
        at::AutoGradMode no_graph(false);
        std::tie(q_out, k_out) = rotary(q, k, positions, plan, inverse, false);
    }
    auto node = make_node<RotaryNode>({q, key});
    node->positions_ = torch::autograd::SavedVariable(positions, false);
    node->plan = plan;
    node->inverse = inverse;
    node->has_k = has_k;
    torch::autograd::set_history(q_out, node);
    if (has_k) torch::autograd::set_history(*k_out, node);
    return {q_out, k_out};
}

// ---- AdamW ----

// The parameters that an optimizer steps, where their moments lie, and which group's settings hold for them.
struct AdamWParams {
    std::vector<Tensor> params;
    std::vector<int64_t> first_block, group;
    std::vector<std::vector<int64_t>> sizes, strides;       // as they were when the moments were laid out
    std::vector<at::ScalarType> types;
};
using AdamWGroupTuple = std::tuple<double, c10::optional<Tensor>, double, double, double, double>;     // lr, lr on the device, decay, betas, eps

// One call of the library for each combination of types and of betas and eps among the parameters that have a gradient.  True if the step is captured.
bool adamw_step(const AdamWParams& all, const std::vector<AdamWGroupTuple>& settings, int64_t state_bits, bool dither, int64_t seed, const Tensor& exp_avg,
                const Tensor& exp_avg_sq, const c10::optional<Tensor>& exp_avg_scale, const c10::optional<Tensor>& exp_avg_sq_scale,
                const c10::optional<Tensor>& master, const Tensor& steps, const Tensor& ticket, const c10::optional<Tensor>& grad_factor) {
    struct Call {
        dropit_adamw_options options;
        std::vector<dropit_adamw_tensor> tensors;
    };
    std::vector<Call> calls;
    std::vector<Tensor> held;               // gradients laid out again
    c10::cuda::CUDAGuard guard(exp_avg.device());
    for (size_t i = 0; i < all.params.size(); ++i) {
        const Tensor& p = all.params[i];
        Tensor g = p.grad();
        if (!g.defined()) continue;
        if (g.layout() != at::kStrided) throw py::type_error("sparse gradients are not supported");
        const dropit_dtype pt = dtype_code(p, "parameter"), gt = dtype_code(g, "gradient");
        if (p.device() != exp_avg.device()) throw py::value_error("a parameter has moved to another device than its moments");
        if (p.sizes() != all.sizes[i] || p.strides() != all.strides[i]) throw py::value_error("a parameter's shape or strides have changed since its moments were laid out");
        // bf16 parameters have an fp32 copy, fp32 ones zeros in its place
        if (master.has_value() && p.scalar_type() != all.types[i]) throw py::value_error("a parameter's type has changed since its copy in fp32 was made");
        if (g.device() != p.device() || g.sizes() != p.sizes()) throw py::value_error("a gradient differs from its parameter in shape or device");
        if (!(p.is_contiguous() && g.is_contiguous()) && g.strides() != p.strides()) {
            Tensor same = at::empty_strided(p.sizes(), p.strides(), g.options());
            same.copy_(g);
            held.push_back(same);
            g = same;
        }
        double lr, decay, beta1, beta2, eps;
        c10::optional<Tensor> lr_device;
        std::tie(lr, lr_device, decay, beta1, beta2, eps) = settings[all.group[i]];
        Call* call = nullptr;
        for (Call& c : calls)
            if (c.options.param_dtype == pt && c.options.grad_dtype == gt && c.options.beta1 == beta1 && c.options.beta2 == beta2 && c.options.eps == eps)
                call = &c;
        if (!call) {
            calls.push_back({{pt, gt, (int32_t)state_bits, dither ? 1 : 0, beta1, beta2, eps, (uint32_t)seed}, {}});
            call = &calls.back();
            call->tensors.reserve(all.params.size());
        }
        call->tensors.push_back({p.data_ptr(), g.data_ptr(), lr_device.has_value() ? lr_device->data_ptr<float>() : nullptr, p.numel(),
                                 all.first_block[i], (int32_t)i, (float)lr, (float)decay});
    }
    auto words = [](const c10::optional<Tensor>& t) { return t.has_value() ? t->data_ptr<float>() : nullptr; };
    for (size_t i = 0; i < all.params.size(); ++i)          // autograd sees that they change
        if (all.params[i].grad().defined()) all.params[i].unsafeGetTensorImpl()->bump_version();
    for (Call& c : calls) {
        const dropit_adamw_state state = {exp_avg.data_ptr(), exp_avg_sq.data_ptr(), words(exp_avg_scale), words(exp_avg_sq_scale),
                                          c.options.param_dtype == DROPIT_BF16 ? words(master) : nullptr, steps.data_ptr<int32_t>(),
                                          (uint32_t*)ticket.data_ptr(), words(grad_factor)};
        check(dropit_adamw_step(c.tensors.data(), (int)c.tensors.size(), &c.options, &state, current_stream(exp_avg)), "dropit_adamw_step");
    }
    return !calls.empty() && c10::cuda::currentStreamCaptureStatusMayInitCtx() != c10::cuda::CaptureStatus::None;
}

}  // namespace

PYBIND11_MODULE(_native, m) {
    py::register_exception_translator([](std::exception_ptr p) {
        try {
            if (p) std::rethrow_exception(p);
        } catch (python_error& e) {
            e.restore();
        }
    });
    m.def("set_error_class", [](py::object cls) { g_error_class = new py::object(cls); });
    // Without the interpreter's lock, as a call through ctypes is: a launch can wait for room in the stream's queue.
    m.def("status_word", torch::wrap_pybind_function_no_gil(status_word));
    m.def("compress", torch::wrap_pybind_function_no_gil(compress));
    m.def("produce", torch::wrap_pybind_function_no_gil(produce));
    m.def("compress_prepared", torch::wrap_pybind_function_no_gil(compress_prepared));
    m.def("weight_grad", torch::wrap_pybind_function_no_gil(weight_grad));
    m.def("conv_weight_grad", torch::wrap_pybind_function_no_gil(conv_weight_grad));
    m.def("gelu_linear", torch::wrap_pybind_function_no_gil(gelu_linear));
    m.def("gated_linear", torch::wrap_pybind_function_no_gil(gated_linear));
    m.def("gated_inference", torch::wrap_pybind_function_no_gil(gated_inference));
    m.def("gated_linear_backward", torch::wrap_pybind_function_no_gil(gated_linear_backward));
    m.def("gated_input_grad", torch::wrap_pybind_function_no_gil(gated_input_grad));
    m.def("gated_layer", torch::wrap_pybind_function_no_gil(gated_layer));
    m.def("rotary_plan", torch::wrap_pybind_function_no_gil(rotary_plan));
    m.def("rotary", torch::wrap_pybind_function_no_gil(rotary));
    m.def("rotary_layer", torch::wrap_pybind_function_no_gil(rotary_layer));
    py::class_<AdamWParams>(m, "AdamWParams").def(py::init([](std::vector<Tensor> params, std::vector<int64_t> first_block, std::vector<int64_t> group) {
        AdamWParams all{std::move(params), std::move(first_block), std::move(group), {}, {}, {}};
        for (const Tensor& p : all.params)
            all.sizes.push_back(p.sizes().vec()), all.strides.push_back(p.strides().vec()), all.types.push_back(p.scalar_type());
        return all;
    }));
    m.def("adamw_step", torch::wrap_pybind_function_no_gil(adamw_step));
}
