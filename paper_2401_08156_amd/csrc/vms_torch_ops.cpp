// The operators of include/vms_ops.h for PyTorch tensors, with their gradients: checks of arguments, outputs and
// workspaces from PyTorch's allocator, the current stream, autograd nodes.  Host code only; the kernels are in
// libvmsreplay.so.  Written against PyTorch's C++ interface because a step of a small model is a chain of such
// calls: a node in Python took 23 us of the host's time forward and 27 us backward on a thread that autograd wakes for
// it, the kernels 8 us.
#include <c10/core/DeviceGuard.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/VariableTypeUtils.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/jit/frontend/tracer.h>
#include <torch/extension.h>

#include "../../include/vms_ops.h"

namespace {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

py::handle vms_error;               // binding.VmsError, held by the module

// A call of the library that did not return VMS_OK
struct LibraryError : std::exception {
    int code;
    const char *name;
    std::string text;
    LibraryError(int c, const char *n) : code(c), name(n), text(std::string(n) + ": " + vms_strerror(c) + " (" + std::to_string(c) + ")") {}
    const char *what() const noexcept override { return text.c_str(); }
};

[[noreturn]] void refuse(const std::string &why) { throw py::value_error(why); }

void *stream_of(const Tensor &x) { return c10::hip::getCurrentHIPStream(x.get_device()).stream(); }

template <class A>
void call(int (*f)(const A *, void *), const char *name, const A &a, const Tensor &x)
{
    const c10::OptionalDeviceGuard guard(x.device());
    const int rc = f(&a, stream_of(x));
    if (rc != VMS_OK) throw LibraryError(rc, name);
}

uint32_t type_of(const Tensor &x)
{
    switch (x.scalar_type()) {
    case at::kFloat: return VMS_F32;
    case at::kHalf: return VMS_F16;
    case at::kBFloat16: return VMS_BF16;
    default: refuse(std::string("float32, float16 or bfloat16 tensors, got ") + c10::toString(x.scalar_type()));
    }
}

// The kernels are called past PyTorch's dispatcher: a trace would hold an output that nothing fills, and a tangent would end here.
void refuse_followers(std::initializer_list<const Tensor *> tensors)
{
    using c10::impl::TorchDispatchModeTLS;
    if (torch::jit::tracer::isTracing() || TorchDispatchModeTLS::get_mode(c10::impl::TorchDispatchModeKey::PROXY) ||
        c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::PreDispatch))
        refuse("these operators cannot be traced");
    for (const Tensor *t : tensors)
        if (t->defined() && t->_fw_grad(0).defined()) refuse("these operators have no forward-mode gradients");
}

// every other tensor has x's type and device
void same(const Tensor &x, std::initializer_list<const Tensor *> others)
{
    refuse_followers({ &x });
    refuse_followers(others);
    type_of(x);
    if (!x.is_cuda()) refuse("tensors on a GPU, got one on " + x.device().str());
    for (const Tensor *t : others)
        if (t->defined() && (t->scalar_type() != x.scalar_type() || t->device() != x.device()))
            refuse(std::string("all tensors have one type and device, got ") + c10::toString(t->scalar_type()) + " on " + t->device().str() +
                   " beside " + c10::toString(x.scalar_type()) + " on " + x.device().str());
}

// a tensor as rows of its last dimension; a copy where its strides do not allow that, or rows are `far` elements apart
// (what the library's entry points refuse)
const uint64_t FAR = 1ull << 31, LOWRANK_FAR = 1ull << 23;
const int64_t MOST = 65535;         // adapters and requests of a call
struct Matrix {
    Tensor t;
    uint64_t ld = 0;
    const void *ptr() const { return t.defined() ? t.const_data_ptr() : nullptr; }
};

// (what lies in the memory of a negative view, as of a conjugate's imaginary part, is not its values)
Tensor flat(const Tensor &t) { return t.defined() ? t.resolve_neg().contiguous() : t; }

Matrix matrix(const Tensor &t, uint64_t far = FAR)
{
    if (!t.defined()) return {};
    if (t.is_neg()) return matrix(flat(t), far);
    const int64_t n = t.dim(), cols = t.size(-1);
    if (t.is_contiguous()) return { t, (uint64_t)cols };
    if (t.stride(-1) == 1 || cols == 1) {
        int64_t stride = -1, wanted = 0;        // of the rows; that of the next dimension outwards if all is evenly spaced
        bool even = true;
        for (int64_t i = n - 2; i >= 0; i--) {
            if (t.size(i) == 1) continue;
            if (stride < 0)
                stride = t.stride(i);
            else if (t.stride(i) != wanted)
                even = false;
            wanted = t.stride(i) * t.size(i);
        }
        if (even && (stride < 0 || (uint64_t)stride < far)) return { t, (uint64_t)(stride < 0 ? cols : stride) };
    }
    return { t.contiguous(), (uint64_t)cols };
}

uint64_t columns(const Tensor &t) { return (uint64_t)t.size(-1); }
uint64_t rows(const Tensor &t) { return t.size(-1) ? (uint64_t)(t.numel() / t.size(-1)) : 0; }

Tensor like(const Tensor &x) { return at::empty(x.sizes(), x.options().requires_grad(false)); }
Tensor bytes(uint64_t n, const Tensor &x) { return at::empty({ (int64_t)n }, x.options().dtype(at::kByte).requires_grad(false)); }
void *ptr(const Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }

bool wanted(std::initializer_list<const Tensor *> tensors)
{
    if (!at::GradMode::is_enabled()) return false;
    for (const Tensor *t : tensors)
        if (t->defined() && t->requires_grad()) return true;
    return false;
}

// Gradients of gradients: where they are asked for (create_graph), what a backward pass returns goes on from a node that refuses,
// as a function of the gradients that arrived and of those inputs of the operator that it varies with (`by`: a bit for each
// input, for each gradient).
struct FirstOrder : torch::autograd::Node {
    variable_list apply(variable_list &&) override { TORCH_CHECK(false, "these operators have gradients of first order only"); }
};

variable_list first_order(variable_list grads, const variable_list &from, std::initializer_list<uint32_t> by)
{
    if (!at::GradMode::is_enabled()) return grads;
    const auto here = torch::autograd::get_current_node();
    for (size_t i = 0; i < by.size(); i++) {
        if (!grads[i].defined()) continue;
        torch::autograd::edge_list edges;
        for (const Tensor &f : from)
            if (f.defined() && f.requires_grad()) edges.push_back(torch::autograd::impl::gradient_edge(f));
        for (uint32_t k = 0; k < here->num_outputs(); k++)
            if ((by.begin()[i] >> k & 1) && here->next_edge(k).is_valid()) edges.push_back(here->next_edge(k));
        if (edges.empty()) continue;
        const std::shared_ptr<FirstOrder> node(new FirstOrder, torch::autograd::deleteNode);       // (long graphs are taken down without recursion)
        node->set_next_edges(std::move(edges));
        grads[i] = grads[i].detach();
        torch::autograd::set_history(grads[i], node);
    }
    return grads;
}

// (Tensors that are not there reach a node as an empty option, those without a gradient inside a structure: a node takes
// every Tensor among its arguments for an input of its own.)
typedef std::optional<Tensor> Maybe;
Maybe maybe(const Tensor &t) { return t.defined() ? Maybe(t) : Maybe(); }

struct Seed {
    uint64_t number = 0;
    Tensor tensor;
};

vms_dropout_mask mask_of(double p, const Seed &s, uint64_t call)
{
    return { p, s.number, s.tensor.defined() ? (const uint64_t *)s.tensor.const_data_ptr() : nullptr, call };
}

uint64_t word(const py::handle &v, const char *what)
{
    const py::object n = py::reinterpret_steal<py::object>(PyNumber_Index(v.ptr()));        // int, numpy's integers
    const unsigned long long w = n ? PyLong_AsUnsignedLongLong(n.ptr()) : 0;
    if (PyErr_Occurred()) {
        PyErr_Clear();
        refuse(std::string(what) + " is a number of 64 bits, got " + py::cast<std::string>(py::repr(v)));
    }
    return w;
}

Seed seed_of(const py::handle &v, const Tensor &x)
{
    if (!THPVariable_Check(v.ptr())) return { word(v, "seed"), {} };
    const Tensor t = py::cast<Tensor>(v);
    if (t.scalar_type() != at::kLong || t.numel() != 1 || t.device() != x.device()) refuse("a seed tensor is one int64 on the input's device");
    return { 0, flat(t) };
}

void check_share(double p)
{
    if (!(p >= 0.0 && p <= 1.0)) refuse("p is a share from 0 to 1, got " + std::to_string(p));
}

// ---- dropout ---------------------------------------------------------------------------------------------------------

Tensor run_dropout(const Tensor &x, const Tensor &residual, const vms_dropout_mask &mask)
{
    Tensor y = like(x);
    const Matrix m = matrix(x), r = matrix(residual);
    const uint64_t cols = columns(x);
    const vms_dropout_args a = { sizeof a, type_of(x), rows(x), cols, m.ptr(), r.ptr(), y.data_ptr(), m.ld, r.ld, cols, mask };
    call(vms_dropout, "vms_dropout", a, x);
    return y;
}

struct Dropout : torch::autograd::Function<Dropout> {
    static Tensor forward(AutogradContext *ctx, const Tensor &x, const Maybe &residual, double p, const Seed &seed, uint64_t call)
    {
        ctx->save_for_backward({ seed.tensor });        // so that a seed changed before the backward pass is noticed
        ctx->saved_data["p"] = p;
        ctx->saved_data["seed"] = (int64_t)seed.number;
        ctx->saved_data["call"] = (int64_t)call;
        ctx->saved_data["residual"] = residual.has_value();
        return run_dropout(x, residual.value_or(Tensor()), mask_of(p, seed, call));
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        const Tensor &dy = grads[0];
        const Seed seed = { (uint64_t)ctx->saved_data["seed"].toInt(), ctx->get_saved_variables()[0] };
        const vms_dropout_mask mask = mask_of(ctx->saved_data["p"].toDouble(), seed, (uint64_t)ctx->saved_data["call"].toInt());
        Tensor dx;
        if (ctx->needs_input_grad(0)) {
            const at::NoGradGuard none;
            dx = run_dropout(dy, {}, mask);
        }
        const bool residual = ctx->saved_data["residual"].toBool() && ctx->needs_input_grad(1);
        return first_order({ dx, residual ? dy : Tensor(), {}, {}, {} }, grads, { 0, 0 });
    }
};

Tensor dropout(const Tensor &x, double p, const py::object &seed, const py::object &call, const std::optional<Tensor> &given)
{
    const Tensor residual = given.value_or(Tensor());
    same(x, { &residual });
    if (!x.dim()) refuse("x has no dimension");
    if (residual.defined() && residual.sizes() != x.sizes()) refuse("residual and x have different shapes");
    check_share(p);
    const Seed s = seed_of(seed, x);
    const uint64_t number = word(call, "call");
    const py::gil_scoped_release go;
    if (wanted({ &x, &residual })) return Dropout::apply(x, maybe(residual), p, s, number);
    return run_dropout(x, residual, mask_of(p, s, number));
}

// ---- layer norm ------------------------------------------------------------------------------------------------------

struct Normed {
    Tensor y, s, stats;
};

Normed run_norm(const Tensor &x, const Tensor &weight, const Tensor &bias, double eps, const Tensor &residual, const vms_dropout_mask &mask, bool backward)
{
    Normed o;
    const uint64_t n = rows(x), cols = columns(x);
    o.y = like(x);
    if (residual.defined()) o.s = like(x);
    if (backward) o.stats = at::empty({ (int64_t)n, 2 }, x.options().dtype(at::kFloat).requires_grad(false));
    const Matrix m = matrix(x), r = matrix(residual);
    const Tensor w = flat(weight), b = flat(bias);
    const vms_layernorm_args a = { sizeof a, type_of(x), n, cols, m.ptr(), r.ptr(), ptr(w), ptr(b), o.y.data_ptr(), ptr(o.s),
                                   (float *)ptr(o.stats), m.ld, r.ld, cols, cols, eps, mask };
    call(vms_layernorm, "vms_layernorm", a, x);
    return o;
}

struct LayerNorm : torch::autograd::Function<LayerNorm> {
    static variable_list forward(AutogradContext *ctx, const Tensor &x, const Maybe &weight_, const Maybe &bias, const Maybe &residual, double eps,
                                 double p, const Seed &seed, uint64_t call)
    {
        const Tensor weight = weight_.value_or(Tensor());
        const Normed o = run_norm(x, weight, bias.value_or(Tensor()), eps, residual.value_or(Tensor()), mask_of(p, seed, call), true);
        // (an alias of s: where a hook on saved tensors ends the pass here, as recomputation's does, the output itself would keep
        // this node alive and the node the output)
        ctx->save_for_backward({ o.s.defined() ? o.s.detach() : x, o.stats, weight, seed.tensor });
        ctx->saved_data["p"] = p;
        ctx->saved_data["seed"] = (int64_t)seed.number;
        ctx->saved_data["call"] = (int64_t)call;
        ctx->saved_data["there"] = (int64_t)(weight_.has_value() | bias.has_value() << 1 | residual.has_value() << 2);
        ctx->set_materialize_grads(false);
        return o.s.defined() ? variable_list{ o.y, o.s } : variable_list{ o.y };
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        variable_list none(8);
        const Tensor &dy = grads[0];
        const Tensor ds = grads.size() > 1 ? grads[1] : Tensor();
        if (!dy.defined() && !ds.defined()) return none;
        const auto saved = ctx->get_saved_variables();
        const Tensor &s = saved[0], &weight = saved[2];
        Tensor dres, dx, dweight, dbias;
        const double p = ctx->saved_data["p"].toDouble();
        const int64_t there = ctx->saved_data["there"].toInt();
        size_t input = 1;               // inputs are numbered without those that are not there
        const auto need = [&](int64_t bit) { return (there & bit) && ctx->needs_input_grad(input++); };
        const bool need_x = ctx->needs_input_grad(0), need_w = need(1), need_b = need(2), need_r = need(4);
        const auto options = s.options().requires_grad(false);
        const Seed seed = { (uint64_t)ctx->saved_data["seed"].toInt(), saved[3] };
        const vms_dropout_mask mask = mask_of(p, seed, (uint64_t)ctx->saved_data["call"].toInt());
        if (!dy.defined()) {            // only s is used: rows without a norm have this gradient all the same
            if (need_x) {
                const at::NoGradGuard guard;
                none[0] = p > 0.0 ? run_dropout(ds, {}, mask) : ds;
            }
            if (need_w) none[1] = at::zeros({ (int64_t)columns(s) }, options);
            if (need_b) none[2] = at::zeros({ (int64_t)columns(s) }, options);
            if (need_r) none[3] = ds;
            return first_order(none, grads, { 0, 0, 0, 0 });
        }
        {
            const at::NoGradGuard guard;
            const uint64_t n = rows(s), cols = columns(s);
            dres = like(s);
            if (p > 0.0 && need_x) dx = like(s);
            if (need_w) dweight = at::empty({ (int64_t)cols }, options);
            if (need_b) dbias = at::empty({ (int64_t)cols }, options);
            const Matrix m = matrix(dy), e = matrix(ds), k = matrix(s);
            const Tensor w = flat(weight);
            vms_layernorm_backward_args a = { sizeof a, type_of(s), n, cols, m.ptr(), e.ptr(), k.ptr(), ptr(w), (const float *)ptr(saved[1]), dres.data_ptr(),
                                              ptr(dx), ptr(dweight), ptr(dbias), m.ld, e.ld, k.ld, cols, cols,
                                              mask, nullptr, 0 };
            Tensor workspace;
            a.workspace_bytes = vms_layernorm_backward_workspace_bytes(&a);
            if (a.workspace_bytes) {
                workspace = bytes(a.workspace_bytes, s);
                a.d_workspace = workspace.data_ptr();
            }
            call(vms_layernorm_backward, "vms_layernorm_backward", a, s);
        }
        none[0] = !need_x ? Tensor() : p > 0.0 ? dx : dres;
        none[1] = dweight;
        none[2] = dbias;
        if (need_r) none[3] = dres;
        const uint32_t sum = 1 | (there & 4 ? 1u << (input - 1) : 0), all = sum | (there & 1 ? 2 : 0);     // inputs that make up s, and with the weight
        return first_order(none, grads, { all, sum, 0, all });
    }
};

py::object layer_norm(const Tensor &x, const std::optional<Tensor> &weight_, const std::optional<Tensor> &bias_, double eps, const std::optional<Tensor> &residual_,
                      double p, const py::object &seed, const py::object &call)
{
    const Tensor weight = weight_.value_or(Tensor()), bias = bias_.value_or(Tensor()), residual = residual_.value_or(Tensor());
    same(x, { &weight, &bias, &residual });
    if (!x.dim() || !x.size(-1)) refuse("x has no columns");
    for (const Tensor *t : { &weight, &bias })
        if (t->defined() && (t->dim() != 1 || t->size(0) != x.size(-1))) refuse("weight and bias have one element for each of the " + std::to_string(x.size(-1)) + " columns");
    if (residual.defined() && residual.sizes() != x.sizes()) refuse("residual and x have different shapes");
    check_share(p);
    if (!residual.defined() && p != 0.0) refuse("dropout is applied on the way to the residual sum: p needs a residual");
    if (!(eps >= 0.0)) refuse("eps is not negative, got " + std::to_string(eps));
    const Seed s = seed_of(seed, x);
    const uint64_t number = word(call, "call");
    variable_list out;
    {
        const py::gil_scoped_release go;
        if (wanted({ &x, &weight, &bias, &residual })) {
            out = LayerNorm::apply(x, maybe(weight), maybe(bias), maybe(residual), eps, p, s, number);
        } else {
            const Normed o = run_norm(x, weight, bias, eps, residual, mask_of(p, s, number), false);
            out = { o.y, o.s };
        }
    }
    return residual.defined() ? py::cast(std::make_tuple(out[0], out[1])) : py::cast(out[0]);
}

// ---- low-rank adapters -----------------------------------------------------------------------------------------------

struct Batch {
    double scale = 0.0;
    Tensor scales, starts, which;
};

vms_lowrank_args lowrank_args(const Matrix &x, const Tensor &a, const Tensor &b, const Batch &batch)
{
    const bool many = a.dim() == 3;
    vms_lowrank_args f = {};
    f.struct_size = sizeof f;
    f.dtype = type_of(x.t);
    f.rows = rows(x.t);
    f.in = (uint64_t)a.size(-1);
    f.out = (uint64_t)b.size(-2);
    f.rank = (uint32_t)a.size(-2);
    f.n_adapters = many ? (uint32_t)a.size(0) : 1;
    f.n_requests = batch.starts.defined() ? (uint32_t)(batch.starts.numel() - 1) : 0;
    f.scale = (float)batch.scale;
    f.d_scales = (const float *)ptr(batch.scales);
    f.d_x = x.ptr();
    f.d_a = a.const_data_ptr();
    f.d_b = b.const_data_ptr();
    f.d_starts = (const int32_t *)ptr(batch.starts);
    f.d_which = (const int32_t *)ptr(batch.which);
    f.ldx = x.ld;
    return f;
}

// -> y + ..., and what the backward pass reads
std::pair<Tensor, Tensor> run_low_rank(const Tensor &y, const Tensor &x, const Tensor &a, const Tensor &b, const Batch &batch, bool inplace)
{
    const Matrix m = matrix(x, LOWRANK_FAR), base = matrix(y, LOWRANK_FAR);
    vms_lowrank_args f = lowrank_args(m, a, b, batch);
    Tensor out = inplace ? y : like(y);
    f.d_y = base.ptr();
    f.ldy = base.ld;
    f.d_out = out.data_ptr();
    f.ldo = inplace ? base.ld : columns(y);
    f.hidden_bytes = vms_lowrank_hidden_bytes(&f);
    const Tensor hidden = bytes(f.hidden_bytes, x);
    f.d_hidden = hidden.data_ptr();
    call(vms_lowrank, "vms_lowrank", f, x);
    return { out, hidden };
}

// May an element of t lie in the memory of y, a matrix of rows of its own?  Columns of one matrix beside each other may not.
bool shares(const Tensor &y, const Tensor &t)
{
    if (!t.defined() || !y.numel() || !t.numel()) return false;
    const auto begin = [](const Tensor &v) { return (uintptr_t)v.const_data_ptr(); };
    const auto size = [](const Tensor &v) {         // bytes from the first element to behind the last
        int64_t last = 0;
        for (int64_t i = 0; i < v.dim(); i++) last += (v.size(i) - 1) * v.stride(i);
        return (uintptr_t)(last + 1) * v.element_size();
    };
    if (begin(t) >= begin(y) + size(y) || begin(y) >= begin(t) + size(t)) return false;
    const Matrix m = matrix(y), k = matrix(t);
    if (!k.t.is_same(t) || k.ld != m.ld || t.element_size() != y.element_size()) return true;
    const uint64_t row = m.ld * y.element_size();
    const uint64_t at = begin(t) >= begin(y) ? (begin(t) - begin(y)) % row : (row - (begin(y) - begin(t)) % row) % row;     // in a row of y
    return at < columns(y) * y.element_size() || at + columns(t) * t.element_size() > row;
}

struct LowRankAdd : torch::autograd::Function<LowRankAdd> {
    static Tensor forward(AutogradContext *ctx, const Tensor &y, const Tensor &x, const Tensor &a, const Tensor &b, const Batch &batch, bool inplace)
    {
        const auto [out, hidden] = run_low_rank(y, x, a, b, batch, inplace);
        if (inplace) ctx->mark_dirty({ y });
        ctx->save_for_backward({ x, a, b, hidden, batch.starts, batch.which, batch.scales });
        ctx->saved_data["scale"] = batch.scale;
        return out;
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        const Tensor &dout = grads[0];
        const auto saved = ctx->get_saved_variables();
        const Tensor &x = saved[0], &a = saved[1], &b = saved[2];
        const bool need_y = ctx->needs_input_grad(0), need_x = ctx->needs_input_grad(1), need_a = ctx->needs_input_grad(2), need_b = ctx->needs_input_grad(3);
        Tensor dx, da, db;
        if (need_x || need_a || need_b) {
            const at::NoGradGuard guard;
            const Matrix m = matrix(x, LOWRANK_FAR), d = matrix(dout, LOWRANK_FAR);
            if (need_x) dx = like(x);
            if (need_a) da = like(a);
            if (need_b) db = like(b);
            vms_lowrank_backward_args g = {};
            g.struct_size = sizeof g;
            g.f = lowrank_args(m, a, b, { ctx->saved_data["scale"].toDouble(), saved[6], saved[4], saved[5] });
            g.f.d_hidden = saved[3].data_ptr();
            g.f.hidden_bytes = (uint64_t)saved[3].numel();
            g.d_dout = d.ptr();
            g.lddout = d.ld;
            g.d_dx = ptr(dx);
            g.d_da = ptr(da);
            g.d_db = ptr(db);
            g.lddx = columns(x);
            g.workspace_bytes = vms_lowrank_backward_workspace_bytes(&g);
            const Tensor workspace = bytes(g.workspace_bytes, x);
            g.d_workspace = workspace.data_ptr();
            call(vms_lowrank_backward, "vms_lowrank_backward", g, x);
        }
        return first_order({ need_y ? dout : Tensor(), dx, da, db, {}, {} }, grads, { 0, 0xC, 0xA, 0x6 });
    }
};

Tensor low_rank_add(const Tensor &y, const Tensor &x_, const Tensor &a_, const Tensor &b_, const py::object &scale, const std::optional<Tensor> &starts_,
                    const std::optional<Tensor> &which_, bool inplace)
{
    const Tensor starts = starts_.value_or(Tensor()), which = which_.value_or(Tensor());
    same(x_, { &y, &a_, &b_ });
    if (!x_.dim() || x_.dim() != y.dim() || x_.sizes().slice(0, x_.dim() - 1) != y.sizes().slice(0, y.dim() - 1)) refuse("x and y have different rows");
    if (a_.dim() != b_.dim() || (a_.dim() != 2 && a_.dim() != 3)) refuse("a is [rank, in] and b [out, rank], or both with the adapters in front");
    const int64_t rank = a_.size(-2), adapters = a_.dim() == 3 ? a_.size(0) : 1;
    if ((a_.dim() == 3 && b_.size(0) != adapters) || rank != b_.size(-1) || a_.size(-1) != x_.size(-1) || b_.size(-2) != y.size(-1))
        refuse("a and b do not lead from " + std::to_string(x_.size(-1)) + " to " + std::to_string(y.size(-1)) + " features by the same rank and adapters");
    if (rank < 1 || rank > VMS_LOWRANK_MAX_RANK) refuse("ranks from 1 to " + std::to_string(VMS_LOWRANK_MAX_RANK) + ", got " + std::to_string(rank));
    if (adapters > MOST || (which.defined() && which.numel() > MOST))       // (before they are counted in 32 bits)
        refuse("up to " + std::to_string(MOST) + " adapters and requests, got " + std::to_string(adapters) + " and " + std::to_string(which.defined() ? which.numel() : 1));
    if (starts.defined() != which.defined()) refuse("starts and which come together");
    if (!starts.defined() && adapters != 1) refuse("several adapters need starts and which");
    for (const Tensor *t : { &starts, &which })
        if (t->defined() && (t->scalar_type() != at::kInt || t->device() != x_.device() || t->dim() != 1 || !t->is_contiguous()))
            refuse("starts and which are contiguous int32 vectors on the input's device");
    if (starts.defined() && starts.numel() != which.numel() + 1)
        refuse(std::to_string(which.numel()) + " requests have one start more, not " + std::to_string(starts.numel()));
    double factor = 0.0;
    Tensor scales;
    if (THPVariable_Check(scale.ptr())) {
        scales = py::cast<Tensor>(scale);
        if (scales.scalar_type() != at::kFloat || scales.device() != x_.device() || scales.dim() != 1 || scales.size(0) != adapters || !scales.is_contiguous())
            refuse("a scale tensor is a contiguous float32 vector with one number for each adapter");
        refuse_followers({ &scales });
        if (scales.requires_grad()) refuse("scales have no gradient");
    } else {
        factor = PyFloat_AsDouble(scale.ptr());
        if (PyErr_Occurred()) {
            PyErr_Clear();
            refuse("scale is a number or a tensor, got " + py::cast<std::string>(py::repr(scale)));
        }
    }
    if (inplace && !matrix(y, LOWRANK_FAR).t.is_same(y)) refuse("y's strides do not allow the sum in place");
    if (inplace && at::GradMode::is_enabled() && y.requires_grad() && y.is_leaf()) refuse("the sum in place of a leaf that requires a gradient");
    if (inplace) {          // what autograd would refuse when the sum is made already
        const bool node = wanted({ &y, &x_, &a_, &b_ });
        if (y.is_inference() && !c10::InferenceMode::is_enabled()) refuse("the sum in place of an inference tensor outside inference mode");
        for (const Tensor *t : std::initializer_list<const Tensor *>{ &x_, &a_, &b_, &scales, &starts, &which })
            if (node && t->defined() && t->is_inference()) refuse("inference tensors are not kept for a backward pass");
        torch::autograd::check_inplace(y, node);
    }
    const py::gil_scoped_release go;
    // What lies in the memory that the sum goes to is read from a copy: workgroups write columns of a row whose x others still read
    const auto apart = [&](const Tensor &t) { return inplace && shares(y, t) ? t.clone() : t; };
    const Tensor x = apart(x_), a = flat(apart(a_)), b = flat(apart(b_));
    const Batch batch = { factor, flat(apart(scales)), flat(apart(starts)), flat(apart(which)) };
    if (wanted({ &y, &x, &a, &b })) return LowRankAdd::apply(y, x, a, b, batch, inplace);
    const Tensor out = run_low_rank(y, x, a, b, batch, inplace).first;
    if (inplace) y.unsafeGetTensorImpl()->bump_version();       // as a node's mark_dirty does: what was saved of y is noticed
    return out;
}

}  // namespace

PYBIND11_MODULE(_vms_torch, m)
{
    m.def("raise_as", [](py::object cls) { vms_error = cls.release(); }, "the exception for calls of the library that fail: cls(code, name)");
    py::register_exception_translator([](std::exception_ptr p) {
        try {
            if (p) std::rethrow_exception(p);
        } catch (const LibraryError &e) {
            if (vms_error.ptr()) {
                const py::object error = vms_error(e.code, e.name);
                PyErr_SetObject(vms_error.ptr(), error.ptr());
            } else {
                PyErr_SetString(PyExc_RuntimeError, e.what());
            }
        }
    });
    m.def("dropout", &dropout, py::arg("x"), py::arg("p"), py::arg("seed"), py::arg("call"), py::arg("residual"));
    m.def("layer_norm", &layer_norm, py::arg("x"), py::arg("weight"), py::arg("bias"), py::arg("eps"), py::arg("residual"), py::arg("p"), py::arg("seed"), py::arg("call"));
    m.def("low_rank_add", &low_rank_add, py::arg("y"), py::arg("x"), py::arg("a"), py::arg("b"), py::arg("scale"), py::arg("starts"), py::arg("which"), py::arg("inplace"));
    m.def("matrix", [](const Tensor &t) {
        const Matrix k = matrix(t);
        return std::make_tuple(k.t, k.ld);
    }, "(tensor, row stride) of a tensor as rows of its last dimension");
}
