// Tensors to aet_ops.h: checks that the tensors of a call agree, allocates its outputs and its workspace with PyTorch and
// hands pointers and strides over.  Marshalling only, compiled because it is most of a small call's time: a linear layer of
// one row takes 4.9 us of the host this way, of which 3.6 are the C call with its launch, and took 8.9 in Python with ctypes.
#include <c10/core/StreamGuard.h>
#include <torch/extension.h>

#include "aet_ops.h"

namespace py = pybind11;
using at::Tensor;
using OptTensor = std::optional<Tensor>;

namespace {

[[noreturn]] void value_error(const std::string &what) { throw py::value_error(what); }

std::string text(at::ScalarType type, const Tensor &t) { return std::string(c10::toString(type)) + " on " + t.device().str(); }
std::string text(const Tensor &t) { return text(t.scalar_type(), t); }

// A call's type, device and stream, by its first tensor.
struct Call {
    const Tensor &x;
    at::ScalarType type;
    int dtype;
    void *handle;
    c10::DeviceGuard guard;
    // Not the current stream: what is allocated belongs to it (memory that the current stream has given back may still
    // be in use there) and is kept for the current one too; what is handed over is kept for it.
    std::optional<c10::StreamGuard> other;
    const Tensor *places[4];   // outputs' that the caller gave
    int count = 0;

    Call(const Tensor &first, int64_t handle_, const std::optional<std::tuple<int64_t, int64_t, int64_t>> &stream)
        : Call(first, first.scalar_type(), handle_, stream) {}
    // The call's type is another than its first tensor's.
    Call(const Tensor &first, at::ScalarType type_, int64_t handle_, const std::optional<std::tuple<int64_t, int64_t, int64_t>> &stream)
        : x(first), type(type_), dtype(type_ == at::kBFloat16 ? AET_BF16 : AET_F32), handle((void *)handle_), guard(checked(first, type_)) {
        if (!stream) return;
        if (std::get<1>(*stream) != x.device().index())
            value_error("the stream is one of device " + std::to_string(std::get<1>(*stream)) + ", the tensors are " + text(x));
        other.emplace(c10::Stream::unpack3(std::get<0>(*stream), (c10::DeviceIndex)std::get<1>(*stream), (c10::DeviceType)std::get<2>(*stream)));
    }
    static c10::Device checked(const Tensor &t, at::ScalarType type) {
        if ((type != at::kFloat && type != at::kBFloat16) || !t.is_cuda())
            value_error("float32 or bfloat16 on a GPU is wanted, got " + text(type, t));
        return t.device();
    }
    void *use(const Tensor &t) {
        if (other) t.record_stream(other->current_stream());
        return t.data_ptr();
    }
    // Nothing is recorded for automatic differentiation: its gradient would be lost without a word.
    static void no_graph(const char *name, const Tensor &t) {
        if (t.requires_grad() && at::GradMode::is_enabled())
            value_error(std::string(name) + " requires a gradient, which the operators do not record: call them under torch.no_grad() or with "
                                            "detached tensors, and the _backward calls for gradients");
    }
    // The tensor's type, device, shape and last stride are as they have to be.
    void agree(const char *name, const Tensor &t, at::IntArrayRef shape) { agree(name, t, shape, type); }
    void agree(const char *name, const Tensor &t, at::IntArrayRef shape, at::ScalarType want) {
        no_graph(name, t);
        if (t.scalar_type() != want || t.device() != x.device())
            value_error(std::string(name) + " is " + text(t) + ", wanted is " + text(want, x));
        if (t.sizes() != shape) {
            std::ostringstream o;
            o << name << " has shape " << t.sizes() << ", expected " << shape;
            value_error(o.str());
        }
        if (shape.back() > 1 && t.strides().back() != 1)
            value_error(std::string(name) + ": the last axis has stride " + std::to_string(t.strides().back()) + ", 1 is wanted");
    }
    // A matrix per client (three axes), or one (two); `shared`: two axes are one for all clients
    template <class M>
    void mat(M &to, const char *name, const OptTensor &t, at::IntArrayRef shape, bool shared = false) { mat(to, name, t, shape, shared, type); }
    template <class M>
    void mat(M &to, const char *name, const OptTensor &t, at::IntArrayRef shape, bool shared, at::ScalarType want) {
        if (!t) return;
        agree(name, *t, shape, want);
        const auto st = t->strides();
        to.p = use(*t);
        to.client = st.size() == 3 ? st[0] : shared ? 0 : shape[0] * st[0];
        to.row = st[st.size() - 2];
    }
    template <class M>
    void vec(M &to, const char *name, const OptTensor &t, int64_t n, int64_t cols) {
        if (!t) return;
        if (t->dim() == 2) agree(name, *t, {n, cols});
        else agree(name, *t, {cols});
        to.p = use(*t);
        to.client = t->dim() == 2 ? t->stride(0) : 0;
    }
    template <class M>
    void maps(M &to, const char *name, const OptTensor &t, at::IntArrayRef shape) {
        if (!t) return;
        agree(name, *t, shape);
        const auto st = t->strides();
        const size_t d = st.size();
        to.p = use(*t);
        to.client = d == 4 ? st[0] : shape[0] * st[0];
        to.sample = st[d - 3];
        to.row = st[d - 2];
    }
    Tensor made(at::IntArrayRef shape, at::ScalarType type) {
        const Tensor t = at::empty(shape, x.options().dtype(type));
        if (other) t.record_stream(other->original_stream());
        return t;
    }
    OptTensor out(const OptTensor &given, bool wanted, at::IntArrayRef shape) {
        if (given) places[count++] = &*given;
        return given ? given : wanted ? OptTensor(made(shape, type)) : std::nullopt;
    }
    template <class A>
    void run(aet_status (*fn)(const A *, void *, size_t, void *), size_t (*bytes)(const A *), const A &a) {
        const size_t need = bytes(&a);
        Tensor ws;
        if (need) ws = at::empty({(int64_t)need}, x.options().dtype(at::kByte));
        done(fn(&a, need ? use(ws) : nullptr, need, handle));
    }
    // Written to, a tensor has another version: automatic differentiation that has kept it for a gradient finds out.
    void done(aet_status rc) {
        for (int i = 0; i < count; ++i)
            if (!places[i]->is_inference()) places[i]->unsafeGetTensorImpl()->bump_version();
        if (rc == AET_OK) return;
        const py::object type = py::module_::import("paper_2112_13935_amd.binding").attr("AetError");
        PyErr_SetObject(type.ptr(), type((int)rc, std::string(aet_ops_last_error())).ptr());
        throw py::error_already_set();
    }
};

typedef std::optional<std::tuple<int64_t, int64_t, int64_t>> Stream;
typedef std::tuple<OptTensor, OptTensor, OptTensor> Three;

int32_t size32(int64_t v) {
    if (v > INT32_MAX) value_error("a size is over 2^31 - 1");
    return (int32_t)v;
}

// n, rows, columns of a tensor with or without an axis of clients
struct Axes {
    int32_t n, rows, cols;
    Axes(const Tensor &x) {
        if (x.dim() != 2 && x.dim() != 3) value_error("a tensor of 2 or 3 axes is wanted");
        n = x.dim() == 3 ? size32(x.size(0)) : 1;
        rows = size32(x.size(-2));
        cols = size32(x.size(-1));
    }
};

std::tuple<Tensor, OptTensor> linear_forward(const Tensor &x, const Tensor &w, const OptTensor &bias, const OptTensor &residual, int act, double p,
                                             uint64_t seed, int64_t first_row, bool keep_pre, const OptTensor &out, int64_t handle, const Stream &stream) {
    Call c(x, handle, stream);
    const Axes s(x);
    if (w.dim() != 2 && w.dim() != 3) value_error("w: [n, out, in] or [out, in] is wanted");
    const int64_t outs = w.size(-2);
    aet_linear a = {c.dtype, act, s.n, s.rows, s.cols, size32(outs), p, seed, first_row};
    const std::array<int64_t, 3> xs = {s.n, s.rows, s.cols}, ys = {s.n, s.rows, outs}, wsh = {s.n, outs, s.cols};
    const size_t skip = 3 - x.dim();
    const at::IntArrayRef shape = at::IntArrayRef(ys).slice(skip);
    c.mat(a.x, "x", x, at::IntArrayRef(xs).slice(skip));
    c.mat(a.w, "w", w, at::IntArrayRef(wsh).slice(3 - w.dim()), true);
    c.vec(a.bias, "bias", bias, s.n, outs);
    c.mat(a.residual, "residual", residual, shape);
    const OptTensor y = c.out(out, true, shape), pre = c.out(std::nullopt, keep_pre, shape);
    c.mat(a.y, "out", y, shape);
    c.mat(a.pre, "pre", pre, shape);
    c.run(aet_linear_forward, aet_linear_workspace_bytes, a);
    return {*y, pre};
}

Three linear_backward(const Tensor &dy, const Tensor &x, const Tensor &w, const OptTensor &pre, int act, double p, uint64_t seed, int64_t first_row,
                      std::array<bool, 3> need, const Three &out, int64_t handle, const Stream &stream) {
    Call c(x, handle, stream);
    const Axes s(x);
    if (w.dim() != 2 && w.dim() != 3) value_error("w: [n, out, in] or [out, in] is wanted");
    if (act != AET_ACT_NONE && !pre) value_error("pre, as the forward call gave it, is wanted where there is an activation");
    const int64_t outs = w.size(-2);
    aet_linear_grad a = {c.dtype, act, s.n, s.rows, s.cols, size32(outs), p, seed, first_row};
    const std::array<int64_t, 3> xsh = {s.n, s.rows, s.cols}, ysh = {s.n, s.rows, outs}, wsh = {s.n, outs, s.cols};
    const size_t skip = 3 - x.dim();
    const at::IntArrayRef xs = at::IntArrayRef(xsh).slice(skip), ys = at::IntArrayRef(ysh).slice(skip), ws = at::IntArrayRef(wsh).slice(3 - w.dim());
    c.mat(a.dy, "dy", dy, ys);
    c.mat(a.x, "x", x, xs);
    c.mat(a.w, "w", w, ws, true);
    c.mat(a.pre, "pre", pre, ys);
    const Three made = {c.out(std::get<0>(out), need[0], xs), c.out(std::get<1>(out), need[1], ws), c.out(std::get<2>(out), need[2], ws.slice(0, ws.size() - 1))};
    c.mat(a.dx, "dx", std::get<0>(made), xs);
    c.mat(a.dw, "dw", std::get<1>(made), ws, true);
    c.vec(a.db, "db", std::get<2>(made), s.n, outs);
    c.run(aet_linear_backward, aet_linear_backward_workspace_bytes, a);
    return made;
}

// n, batch, positions, groups and width of maps with or without an axis of clients
struct MapAxes {
    int32_t n, batch, positions, groups, width;
    MapAxes(const Tensor &x, int64_t groups_) {
        if (x.dim() != 3 && x.dim() != 4) value_error("a tensor of 3 or 4 axes is wanted");
        n = x.dim() == 4 ? size32(x.size(0)) : 1;
        batch = size32(x.size(-3));
        positions = size32(x.size(-2));
        if (groups_ < 1 || x.size(-1) % groups_)
            value_error(std::to_string(x.size(-1)) + " channels cannot be parted into " + std::to_string(groups_) + " groups");
        groups = size32(groups_);
        width = size32(x.size(-1) / groups_);
    }
    std::array<int64_t, 3> stats() const { return {n, batch, groups}; }
};

// The statistics of a normalisation, as the forward call gave them
void statistics(Call &c, const Tensor &mean, const Tensor &rstd, at::IntArrayRef shape, const char *axes) {
    for (const auto &[name, t] : {std::pair<const char *, const Tensor &>("mean", mean), {"rstd", rstd}}) {
        c.no_graph(name, t);
        if (t.scalar_type() != at::kFloat || t.device() != c.x.device() || t.sizes() != shape || !t.is_contiguous())
            value_error(std::string(name) + " has to be as the forward call gave it: float32, contiguous, " + axes);
    }
}

std::tuple<Tensor, Tensor, Tensor> group_norm_forward(const Tensor &x, int64_t groups, const OptTensor &gamma, const OptTensor &beta, double eps, int act,
                                                      const OptTensor &out, int64_t handle, const Stream &stream) {
    const MapAxes s(x, groups);
    Call c(x, handle, stream);
    aet_group_norm a = {c.dtype, act, s.n, s.batch, s.positions, s.groups, s.width, (float)eps};
    const auto all = s.stats();
    const at::IntArrayRef stats = at::IntArrayRef(all).slice(4 - x.dim());
    c.maps(a.x, "x", x, x.sizes());
    c.vec(a.gamma, "gamma", gamma, s.n, x.size(-1));
    c.vec(a.beta, "beta", beta, s.n, x.size(-1));
    const OptTensor y = c.out(out, true, x.sizes());
    c.maps(a.y, "out", y, x.sizes());
    const Tensor mean = c.made(stats, at::kFloat), rstd = c.made(stats, at::kFloat);
    a.mean = (float *)c.use(mean);
    a.rstd = (float *)c.use(rstd);
    c.run(aet_group_norm_forward, aet_group_norm_workspace_bytes, a);
    return {*y, mean, rstd};
}

Three group_norm_backward(const Tensor &dy, const Tensor &x, const Tensor &mean, const Tensor &rstd, const OptTensor &gamma, const OptTensor &beta, int act,
                          std::array<bool, 2> need, const Three &out, int64_t handle, const Stream &stream) {
    const MapAxes s(x, mean.dim() ? mean.size(-1) : 0);
    Call c(x, handle, stream);
    if (gamma && beta && gamma->dim() != beta->dim()) value_error("gamma and beta: either both or none have an axis of clients");
    const auto all = s.stats();
    const at::IntArrayRef stats = at::IntArrayRef(all).slice(4 - x.dim());
    statistics(c, mean, rstd, stats, "[n, batch, groups]");
    aet_group_norm_grad a = {c.dtype, act, s.n, s.batch, s.positions, s.groups, s.width};
    const int64_t channels = x.size(-1);
    c.maps(a.dy, "dy", dy, x.sizes());
    c.maps(a.x, "x", x, x.sizes());
    a.mean = (const float *)c.use(mean);
    a.rstd = (const float *)c.use(rstd);
    c.vec(a.gamma, "gamma", gamma, s.n, channels);
    c.vec(a.beta, "beta", beta, s.n, channels);
    const Three made = {c.out(std::get<0>(out), need[0], x.sizes()), gamma ? c.out(std::get<1>(out), need[1], gamma->sizes()) : std::nullopt,
                        beta ? c.out(std::get<2>(out), need[1], beta->sizes()) : std::nullopt};
    c.maps(a.dx, "dx", std::get<0>(made), x.sizes());
    c.vec(a.dgamma, "dgamma", std::get<1>(made), s.n, channels);
    c.vec(a.dbeta, "dbeta", std::get<2>(made), s.n, channels);
    c.run(aet_group_norm_backward, aet_group_norm_backward_workspace_bytes, a);
    return made;
}

Tensor dropout(bool back, const Tensor &x, double p, uint64_t seed, int64_t first_row, const OptTensor &residual, const OptTensor &out, int64_t handle,
               const Stream &stream) {
    Call c(x, handle, stream);
    const Axes s(x);
    aet_dropout a = {c.dtype, s.n, s.rows, s.cols, p, seed, first_row};
    const OptTensor y = c.out(out, true, x.sizes());
    c.mat(a.x, "x", x, x.sizes());
    c.mat(a.residual, "residual", residual, x.sizes());
    c.mat(a.y, "out", y, x.sizes());
    c.done(back ? aet_dropout_backward(&a, c.handle) : aet_dropout_forward(&a, c.handle));
    return *y;
}

std::tuple<Tensor, OptTensor, Tensor, Tensor> layer_norm_forward(const Tensor &x, const OptTensor &gamma, const OptTensor &beta, const OptTensor &residual,
                                                                 double eps, const std::tuple<OptTensor, OptTensor> &out, int64_t handle, const Stream &stream) {
    Call c(x, handle, stream);
    const Axes s(x);
    aet_layer_norm a = {c.dtype, s.n, s.rows, s.cols, (float)eps};
    const at::IntArrayRef stats = x.sizes().slice(0, x.dim() - 1);
    c.mat(a.x, "x", x, x.sizes());
    c.mat(a.residual, "residual", residual, x.sizes());
    c.vec(a.gamma, "gamma", gamma, s.n, s.cols);
    c.vec(a.beta, "beta", beta, s.n, s.cols);
    if (std::get<1>(out) && !residual) value_error("h is x where there is no residual: a place for it is not wanted");
    const OptTensor y = c.out(std::get<0>(out), true, x.sizes()), h = c.out(std::get<1>(out), residual.has_value(), x.sizes());
    c.mat(a.y, "out", y, x.sizes());
    c.mat(a.h, "out", h, x.sizes());
    const Tensor mean = c.made(stats, at::kFloat), rstd = c.made(stats, at::kFloat);
    a.mean = (float *)c.use(mean);
    a.rstd = (float *)c.use(rstd);
    c.done(aet_layer_norm_forward(&a, c.handle));
    return {*y, h, mean, rstd};
}

Three layer_norm_backward(const Tensor &dy, const Tensor &x, const Tensor &mean, const Tensor &rstd, const OptTensor &gamma, const OptTensor &dh,
                          std::array<bool, 2> need, const Three &out, int64_t handle, const Stream &stream) {
    Call c(x, handle, stream);
    const Axes s(x);
    statistics(c, mean, rstd, x.sizes().slice(0, x.dim() - 1), "[n, rows]");
    aet_layer_norm_grad a = {c.dtype, s.n, s.rows, s.cols};
    c.mat(a.dy, "dy", dy, x.sizes());
    c.mat(a.x, "x", x, x.sizes());
    c.mat(a.dh, "dh", dh, x.sizes());
    c.vec(a.gamma, "gamma", gamma, s.n, s.cols);
    a.mean = (const float *)c.use(mean);
    a.rstd = (const float *)c.use(rstd);
    const bool params = need[1] && gamma;
    const Three made = {c.out(std::get<0>(out), need[0], x.sizes()), c.out(std::get<1>(out), params, gamma ? gamma->sizes() : at::IntArrayRef()),
                        c.out(std::get<2>(out), params, gamma ? gamma->sizes() : at::IntArrayRef())};
    const OptTensor &dgamma = std::get<1>(made), &dbeta = std::get<2>(made);
    if (dgamma && dbeta && dgamma->dim() != dbeta->dim()) value_error("dgamma and dbeta: either both or none have an axis of clients");
    c.mat(a.dx, "dx", std::get<0>(made), x.sizes());
    c.vec(a.dgamma, "dgamma", dgamma, s.n, s.cols);
    c.vec(a.dbeta, "dbeta", dbeta, s.n, s.cols);
    c.run(aet_layer_norm_backward, aet_layer_norm_backward_workspace_bytes, a);
    return made;
}

Tensor orthogonalise(const Tensor &g, int64_t steps, std::tuple<double, double, double> polynomial, double eps, const OptTensor &w, double keep, double scale,
                     const OptTensor &out, int64_t handle, const Stream &stream) {
    Call c(g, handle, stream);
    const Axes s(g);
    aet_orthogonal a = {c.dtype, s.n, s.rows, s.cols, size32(steps), std::get<0>(polynomial), std::get<1>(polynomial), std::get<2>(polynomial), eps, keep, scale};
    const OptTensor y = c.out(out, true, g.sizes());
    c.mat(a.g, "g", g, g.sizes());
    c.mat(a.w, "w", w, g.sizes());
    c.mat(a.y, "out", y, g.sizes());
    c.run(aet_orthogonalise, aet_orthogonalise_workspace_bytes, a);
    return *y;
}

// Codes and scales of a tensor of this shape (its last axis: cols)
struct HeldShape {
    std::vector<int64_t> codes, scales;
    HeldShape(at::IntArrayRef shape) : codes(shape.vec()), scales(shape.vec()) {
        codes.back() = (shape.back() + 1) / 2;
        scales.back() = (shape.back() + 31) / 32;
    }
};

std::tuple<Tensor, Tensor> mx4_quantise(const Tensor &x, const std::tuple<OptTensor, OptTensor> &out, int64_t handle, const Stream &stream) {
    Call c(x, handle, stream);
    const Axes s(x);
    aet_mx4_values a = {c.dtype, s.n, s.rows, s.cols};
    const HeldShape held(x.sizes());
    c.mat(a.x, "x", x, x.sizes());
    const auto place = [&](const OptTensor &given, at::IntArrayRef shape) {
        if (given) c.places[c.count++] = &*given;
        return given ? *given : c.made(shape, at::kByte);
    };
    const Tensor codes = place(std::get<0>(out), held.codes), scales = place(std::get<1>(out), held.scales);
    c.mat(a.codes, "codes", codes, held.codes, false, at::kByte);
    c.mat(a.scales, "scales", scales, held.scales, false, at::kByte);
    c.done(aet_mx4_quantise(&a, c.handle));
    return {codes, scales};
}

// The number of columns that codes stand for
int64_t held_cols(const Tensor &codes, std::optional<int64_t> cols) {
    if (codes.dim() != 2 && codes.dim() != 3) value_error("codes: a tensor of 2 or 3 axes is wanted");
    const int64_t all = cols ? *cols : 2 * codes.size(-1);
    if (all < 0 || (all + 1) / 2 != codes.size(-1))
        value_error(std::to_string(codes.size(-1)) + " bytes of codes do not stand for " + std::to_string(all) + " columns");
    return all;
}
std::vector<int64_t> held_shape(const Tensor &codes, int64_t cols) {
    std::vector<int64_t> shape = codes.sizes().vec();
    shape.back() = cols;
    return shape;
}

Tensor mx4_dequantise(const Tensor &codes, const Tensor &scales, std::optional<int64_t> cols, bool bf16, const OptTensor &out, int64_t handle, const Stream &stream) {
    const std::vector<int64_t> shape = held_shape(codes, held_cols(codes, cols));
    const HeldShape held(shape);
    Call c(codes, bf16 ? at::kBFloat16 : at::kFloat, handle, stream);
    const Axes s(codes);
    aet_mx4_codes a = {c.dtype, s.n, s.rows, size32(shape.back())};
    c.mat(a.codes, "codes", codes, held.codes, false, at::kByte);
    c.mat(a.scales, "scales", scales, held.scales, false, at::kByte);
    const OptTensor y = c.out(out, true, shape);
    c.mat(a.y, "out", y, shape);
    c.done(aet_mx4_dequantise(&a, c.handle));
    return *y;
}

std::tuple<Tensor, OptTensor> mx4_linear_forward(const Tensor &x, const Tensor &x_scales, const Tensor &w, const Tensor &w_scales, const OptTensor &bias,
                                                 std::optional<int64_t> cols, const OptTensor &residual, int act, double p, uint64_t seed, int64_t first_row,
                                                 bool keep_pre, bool bf16, const OptTensor &out, int64_t handle, const Stream &stream) {
    const std::vector<int64_t> xs = held_shape(x, held_cols(x, cols));
    Call c(x, bf16 ? at::kBFloat16 : at::kFloat, handle, stream);
    const Axes s(x);
    if (w.dim() != 2 && w.dim() != 3) value_error("w: [n, out, bytes] or [out, bytes] is wanted");
    const int64_t outs = w.size(-2);
    aet_mx4_linear a = {c.dtype, act, s.n, s.rows, size32(xs.back()), size32(outs), p, seed, first_row};
    const std::array<int64_t, 3> ysh = {s.n, s.rows, outs}, wsh = {s.n, outs, xs.back()};
    const at::IntArrayRef shape = at::IntArrayRef(ysh).slice(3 - x.dim());
    const HeldShape hx(xs), hw(at::IntArrayRef(wsh).slice(3 - w.dim()));
    c.mat(a.x, "x", x, hx.codes, false, at::kByte);
    c.mat(a.x_scales, "x_scales", x_scales, hx.scales, false, at::kByte);
    c.mat(a.w, "w", w, hw.codes, true, at::kByte);
    c.mat(a.w_scales, "w_scales", w_scales, hw.scales, true, at::kByte);
    c.vec(a.bias, "bias", bias, s.n, outs);
    c.mat(a.residual, "residual", residual, shape);
    const OptTensor y = c.out(out, true, shape), pre = c.out(std::nullopt, keep_pre, shape);
    c.mat(a.y, "out", y, shape);
    c.mat(a.pre, "pre", pre, shape);
    c.run(aet_mx4_linear_forward, aet_mx4_linear_workspace_bytes, a);
    return {*y, pre};
}

Three mx4_linear_backward(const Tensor &dy, const Tensor &x, const Tensor &x_scales, const Tensor &w, const Tensor &w_scales, const OptTensor &pre,
                          std::optional<int64_t> cols, int act, double p, uint64_t seed, int64_t first_row, std::array<bool, 3> need, const Three &out,
                          int64_t handle, const Stream &stream) {
    const std::vector<int64_t> xsh = held_shape(x, held_cols(x, cols));
    Call c(dy, handle, stream);
    const Axes s(x);
    if (w.dim() != 2 && w.dim() != 3) value_error("w: [n, out, bytes] or [out, bytes] is wanted");
    if (act != AET_ACT_NONE && !pre) value_error("pre, as the forward call gave it, is wanted where there is an activation");
    const int64_t outs = w.size(-2);
    aet_mx4_linear_grad a = {c.dtype, act, s.n, s.rows, size32(xsh.back()), size32(outs), p, seed, first_row};
    const std::array<int64_t, 3> ysh = {s.n, s.rows, outs}, wsh = {s.n, outs, xsh.back()};
    const at::IntArrayRef xs = xsh, ys = at::IntArrayRef(ysh).slice(3 - x.dim()), ws = at::IntArrayRef(wsh).slice(3 - w.dim());
    const HeldShape hx(xs), hw(ws);
    c.mat(a.dy, "dy", dy, ys);
    c.mat(a.x, "x", x, hx.codes, false, at::kByte);
    c.mat(a.x_scales, "x_scales", x_scales, hx.scales, false, at::kByte);
    c.mat(a.w, "w", w, hw.codes, true, at::kByte);
    c.mat(a.w_scales, "w_scales", w_scales, hw.scales, true, at::kByte);
    c.mat(a.pre, "pre", pre, ys);
    const Three made = {c.out(std::get<0>(out), need[0], xs), c.out(std::get<1>(out), need[1], ws), c.out(std::get<2>(out), need[2], ws.slice(0, ws.size() - 1))};
    c.mat(a.dx, "dx", std::get<0>(made), xs);
    c.mat(a.dw, "dw", std::get<1>(made), ws, true);
    c.vec(a.db, "db", std::get<2>(made), s.n, outs);
    c.run(aet_mx4_linear_backward, aet_mx4_linear_backward_workspace_bytes, a);
    return made;
}

}  // namespace

PYBIND11_MODULE(_ops_torch, m) {
    m.def("linear_forward", &linear_forward);
    m.def("linear_backward", &linear_backward);
    m.def("group_norm_forward", &group_norm_forward);
    m.def("group_norm_backward", &group_norm_backward);
    m.def("dropout", &dropout);
    m.def("layer_norm_forward", &layer_norm_forward);
    m.def("layer_norm_backward", &layer_norm_backward);
    m.def("orthogonalise", &orthogonalise);
    m.def("mx4_quantise", &mx4_quantise);
    m.def("mx4_dequantise", &mx4_dequantise);
    m.def("mx4_linear_forward", &mx4_linear_forward);
    m.def("mx4_linear_backward", &mx4_linear_backward);
}
