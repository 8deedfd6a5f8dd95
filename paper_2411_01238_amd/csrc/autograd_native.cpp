// Autograd nodes of the transformer operators (arxiv 2411.01238, Section 4.2) in C++: no arithmetic, only the C ABI's calls.
//
// The backward pass of a GPU graph runs on a thread of its own, where every microsecond of Python costs two or three (a cold core and
// the interpreter's lock): a layer norm's forward and backward on 64 x 256 took 132 us of host time as Python nodes, a
// library's own 65.  Calls run on the device of their tensors and on its current stream; workspaces come from torch's allocator.
#include <torch/extension.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include "sdrop.h"

namespace {

using torch::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;
using OptTensor = std::optional<Tensor>;

struct Failure : std::runtime_error {
    int code;
    const char *call;
    Failure(int rc, const char *name) : std::runtime_error(name), code(rc), call(name) {}
};
void check(int rc, const char *what)
{
    if (rc != SDROP_OK) throw Failure(rc, what);
}
void require(bool ok, const char *what)
{
    if (!ok) throw std::invalid_argument(what);
}
// (the graph's thread knows no Python exceptions)
void check_backward(int rc, const char *what)
{
    TORCH_CHECK(rc == SDROP_OK, what, " failed in the backward pass: ", sdrop_strerror(rc), " (code ", rc, ")");
}

void *stream_of(const Tensor &t) { return static_cast<void *>(c10::hip::getCurrentHIPStream(t.get_device()).stream()); }

int type_code(const Tensor &t, const char *what)
{
    switch (t.scalar_type()) {
    case torch::kHalf: return SDROP_F16;
    case torch::kBFloat16: return SDROP_BF16;
    case torch::kFloat: return SDROP_F32;
    default: throw Failure(SDROP_EDTYPE, what);
    }
}

// t [.., N] as M rows, ld elements apart (at most 2^24): a matrix with contiguous rows as it is, any other tensor that lies in one piece, else
// a copy.
struct Rows {
    Tensor t;
    int64_t M, N, ld;
    explicit Rows(const Tensor &x) : t(x)
    {
        require(x.is_cuda() && x.dim() >= 1, "a GPU tensor is needed");
        N = x.size(-1);
        M = N ? x.numel() / N : 0;
        ld = N;
        if (x.dim() == 2 && (N == 1 || x.stride(1) == 1) && (M <= 1 || (x.stride(0) >= N && x.stride(0) <= int64_t(1) << 24))) {
            if (M > 1) ld = x.stride(0);
        } else if (!x.is_contiguous()) {
            t = x.contiguous();
        }
    }
    void *ptr() const { return t.data_ptr(); }
};

// A gradient cannot be differentiated once more: where a graph of it is asked for, the error waits between it and the tensors `of`
// that it was computed from.
variable_list once(variable_list &&out, const variable_list &of)
{
    if (!at::GradMode::is_enabled()) return std::move(out);
    const size_t n = out.size();
    out.insert(out.end(), of.begin(), of.end());
    auto node = std::make_shared<torch::autograd::DelayedError>("libsdrop's operators can be differentiated once", (int)out.size());
    node->set_next_edges(torch::autograd::edge_list());
    variable_list res = (*node)(std::move(out));
    res.resize(n);
    return res;
}
variable_list joined(variable_list a, const variable_list &b)
{
    a.insert(a.end(), b.begin(), b.end());
    return a;
}

uint64_t bits(const c10::IValue &v) { return (uint64_t)v.toInt(); }

// (The C ABI's sizes are positive.  Tensors with nothing in them have results with nothing in them, as torch's operators do; other arguments are
// checked all the same.)
Tensor drop(const Rows &x, const Rows *r, double p, uint64_t seed, uint64_t stream, int &rc)
{
    Tensor y = torch::empty(x.t.sizes(), x.t.options());
    const int dtype = type_code(x.t, "sdrop_dropout");
    if (!x.t.numel()) {
        rc = p >= 0.0 && p <= 1.0 ? SDROP_OK : SDROP_EINVAL;
        return y;
    }
    rc = sdrop_dropout(x.ptr(), r ? r->ptr() : nullptr, y.data_ptr(), x.M, x.N, p, seed, stream, dtype, x.ld,
                       r ? r->ld : 0, 0, stream_of(x.t));
    return y;
}

struct Dropout : torch::autograd::Function<Dropout> {
    static Tensor forward(AutogradContext *ctx, const Tensor &x, const OptTensor &residual, double p, int64_t seed, int64_t stream)
    {
        at::AutoDispatchBelowADInplaceOrView guard;
        const c10::DeviceGuard on(x.device());
        const Rows m(x);
        std::optional<Rows> r;
        if (residual) {
            require(residual->sizes() == x.sizes() && residual->scalar_type() == x.scalar_type() && residual->device() == x.device(),
                    "residual must have x's shape, dtype and device");
            r.emplace(*residual);
        }
        ctx->saved_data["p"] = p;
        ctx->saved_data["seed"] = seed;
        ctx->saved_data["stream"] = stream;
        ctx->saved_data["residual"] = residual.has_value();
        int rc;
        Tensor y = drop(m, r ? &*r : nullptr, p, (uint64_t)seed, (uint64_t)stream, rc);
        check(rc, "sdrop_dropout");
        return y;
    }
    static variable_list backward(AutogradContext *ctx, variable_list g)
    {
        Tensor dx;
        if (ctx->needs_input_grad(0)) {
            at::AutoDispatchBelowADInplaceOrView guard;
            int rc;
            dx = drop(Rows(g[0]), nullptr, ctx->saved_data["p"].toDouble(), bits(ctx->saved_data["seed"]), bits(ctx->saved_data["stream"]), rc);
            check_backward(rc, "sdrop_dropout");
        }
        return once({dx, ctx->saved_data["residual"].toBool() ? g[0] : Tensor(), Tensor(), Tensor(), Tensor()}, g);
    }
};

void check_weights(const Tensor &x, const Tensor &w, const OptTensor &b)
{
    const int64_t N = x.size(-1);
    for (const Tensor *t : {&w, b ? &*b : &w})
        require(t->is_cuda() && t->dim() == 1 && t->size(0) == N && t->is_contiguous() && t->device() == x.device() &&
                    (t->scalar_type() == x.scalar_type() || t->scalar_type() == torch::kFloat) && t->scalar_type() == w.scalar_type(),
                "weight and bias must have one value per column, of x's dtype or fp32, both of the same");
}

// The norm's forward pass; `r` and p as for sdrop_layer_norm.  stats: [2, M].
void norm_forward(const Rows &x, const Rows *r, const Tensor &w, const OptTensor &b, double p, double eps, uint64_t seed, uint64_t stream,
                  Tensor &y, Tensor &h, Tensor &stats)
{
    y = torch::empty(x.t.sizes(), x.t.options());
    if (r || p != 0.0) h = torch::empty(x.t.sizes(), x.t.options());
    stats = torch::empty({2, x.M}, x.t.options().dtype(torch::kFloat));
    if (!x.t.numel()) {
        type_code(x.t, "sdrop_layer_norm");
        return check(p >= 0.0 && p <= 1.0 && eps >= 0.0 && eps < INFINITY ? SDROP_OK : SDROP_EINVAL, "sdrop_layer_norm");
    }
    float *const s = stats.data_ptr<float>();
    check(sdrop_layer_norm(x.ptr(), r ? r->ptr() : nullptr, w.data_ptr(), b ? b->data_ptr() : nullptr, h.defined() ? h.data_ptr() : nullptr,
                           y.data_ptr(), s, s + x.M, x.M, x.N, eps, p, seed, stream, type_code(x.t, "sdrop_layer_norm"),
                           type_code(w, "sdrop_layer_norm"), x.ld, r ? r->ld : 0, 0, 0, stream_of(x.t)), "sdrop_layer_norm");
}

// (dx, dr, dweight, dbias); with p = 0, dx is dr
void norm_backward(const Tensor &gy, const Tensor &gh, const Tensor &h, const Tensor &w, const Tensor &stats, double p, uint64_t seed,
                   uint64_t stream, bool need_x, bool need_r, bool need_w, bool need_b, Tensor (&out)[4])
{
    const Rows dy(gy), hs(h);
    std::optional<Rows> dh;
    if (gh.defined()) dh.emplace(gh);
    const bool drops = p != 0.0;
    Tensor dr, dx, dg, db, ws;
    if (need_r || (need_x && !drops)) dr = torch::empty(gy.sizes(), gy.options());
    if (need_x && drops) dx = torch::empty(gy.sizes(), gy.options());
    const bool none = !gy.numel();
    if (need_w) dg = none ? torch::zeros(w.sizes(), w.options()) : torch::empty(w.sizes(), w.options());
    if (need_b) db = none ? torch::zeros(w.sizes(), w.options()) : torch::empty(w.sizes(), w.options());
    size_t need = 0;
    if (!none && (need_w || need_b)) {
        need = sdrop_layer_norm_bwd_workspace_bytes(dy.M, dy.N);
        ws = torch::empty({(int64_t)need}, w.options().dtype(torch::kByte));
    }
    auto at = [](const Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; };
    const float *const s = stats.data_ptr<float>();
    if (!none)
        check_backward(sdrop_layer_norm_bwd(dy.ptr(), dh ? dh->ptr() : nullptr, hs.ptr(), w.data_ptr(), s, s + dy.M, at(dr), at(dx), at(dg), at(db),
                                            dy.M, dy.N, p, seed, stream, type_code(gy, "sdrop_layer_norm_bwd"), type_code(w, "sdrop_layer_norm_bwd"),
                                            dy.ld, dh ? dh->ld : 0, hs.ld, 0, 0, at(ws), need, stream_of(gy)), "sdrop_layer_norm_bwd");
    out[0] = drops ? dx : need_x ? dr : Tensor();
    out[1] = need_r ? dr : Tensor();
    out[2] = dg;
    out[3] = db;
}

struct LayerNorm : torch::autograd::Function<LayerNorm> {
    static Tensor forward(AutogradContext *ctx, const Tensor &x, const Tensor &w, const OptTensor &b, double eps)
    {
        at::AutoDispatchBelowADInplaceOrView guard;
        const c10::DeviceGuard on(x.device());
        const Rows m(x);
        check_weights(x, w, b);
        Tensor y, h, stats;
        norm_forward(m, nullptr, w, b, 0.0, eps, 0, 0, y, h, stats);
        ctx->save_for_backward({m.t, w, stats});
        ctx->saved_data["bias"] = b.has_value();
        return y;
    }
    static variable_list backward(AutogradContext *ctx, variable_list g)
    {
        const variable_list s = ctx->get_saved_variables();
        const bool has_b = ctx->saved_data["bias"].toBool(), nx = ctx->needs_input_grad(0), nw = ctx->needs_input_grad(1), nb = has_b && ctx->needs_input_grad(2);
        Tensor out[4];
        if (nx || nw || nb) {
            at::AutoDispatchBelowADInplaceOrView guard;
            norm_backward(g[0], Tensor(), s[0], s[1], s[2], 0.0, 0, 0, nx, false, nw, nb, out);
        }
        return once({out[0], out[2], out[3], Tensor()}, joined(g, s));
    }
};

struct DropoutAddNorm : torch::autograd::Function<DropoutAddNorm> {
    static variable_list forward(AutogradContext *ctx, const Tensor &x, const Tensor &residual, const Tensor &w, const OptTensor &b, double p,
                                 double eps, int64_t seed, int64_t stream)
    {
        at::AutoDispatchBelowADInplaceOrView guard;
        const c10::DeviceGuard on(x.device());
        require(residual.sizes() == x.sizes() && residual.scalar_type() == x.scalar_type() && residual.device() == x.device(),
                "residual must have x's shape, dtype and device");
        const Rows m(x), r(residual);
        check_weights(x, w, b);
        Tensor y, h, stats;
        norm_forward(m, &r, w, b, p, eps, (uint64_t)seed, (uint64_t)stream, y, h, stats);
        ctx->set_materialize_grads(false);
        ctx->save_for_backward({h, w, stats});
        ctx->saved_data["p"] = p;
        ctx->saved_data["seed"] = seed;
        ctx->saved_data["stream"] = stream;
        ctx->saved_data["bias"] = b.has_value();
        return {y, h};
    }
    static variable_list backward(AutogradContext *ctx, variable_list g)
    {
        const variable_list s = ctx->get_saved_variables();
        const bool has_b = ctx->saved_data["bias"].toBool(), nx = ctx->needs_input_grad(0), nr = ctx->needs_input_grad(1), nw = ctx->needs_input_grad(2),
                   nb = has_b && ctx->needs_input_grad(3);
        const double p = ctx->saved_data["p"].toDouble();
        const uint64_t seed = bits(ctx->saved_data["seed"]), stream = bits(ctx->saved_data["stream"]);
        Tensor out[4];
        {
            at::AutoDispatchBelowADInplaceOrView guard;
            if (g[0].defined()) {
                if (nx || nr || nw || nb) norm_backward(g[0], g[1], s[0], s[1], s[2], p, seed, stream, nx, nr, nw, nb, out);
            } else if (g[1].defined()) {        // only the residual stream is used further on
                if (nx && p != 0.0) {
                    int rc;
                    out[0] = drop(Rows(g[1]), nullptr, p, seed, stream, rc);
                    check_backward(rc, "sdrop_dropout");
                } else if (nx) {
                    out[0] = g[1];
                }
                if (nr) out[1] = g[1];
            }
        }
        return once({out[0], out[1], out[2], out[3], Tensor(), Tensor(), Tensor(), Tensor()}, joined(g, s));
    }
};

// ---- attention ----

// What the kernels take in place (contiguous heads, 16-byte steps and addresses, tokens at most 2^24 elements apart), else a copy: of a tensor
// in one piece too, which may begin anywhere (a gradient that comes back through a concatenation).
Tensor in_place(const Tensor &t)
{
    if (!t.is_cuda() || t.dim() < 3) return t;          // (refused where the call is described)
    bool ok = (t.stride(-1) == 1 || t.size(-1) == 1) && reinterpret_cast<uintptr_t>(t.data_ptr()) % 16 == 0;
    for (int64_t d = 0; ok && d < t.dim() - 1; ++d)
        ok = t.size(d) == 1 || (t.stride(d) > 0 && t.stride(d) % 8 == 0 && t.stride(d) <= int64_t(1) << (d == t.dim() - 3 ? 24 : 50));
    return ok ? t : t.clone(at::MemoryFormat::Contiguous);
}

void strides(const Tensor &t, int64_t &b, int64_t &tok, int64_t &h)
{
    const int64_t n = t.dim();
    b = n == 4 && t.size(0) > 1 ? t.stride(0) : 0;
    tok = t.size(n - 3) > 1 ? t.stride(n - 3) : 0;
    h = t.size(n - 2) > 1 ? t.stride(n - 2) : 0;
}

struct AttnArgs {
    bool causal;
    double scale;               // 0: D ** -0.5
    OptTensor cu_q, cu_k, k_len;
    int64_t max_q, max_k;
    bool train = false;         // a graph is wanted of this call (inside a node's forward pass gradients are off)
};

// The description of a call on [B, T, H, D] or packed [tokens, H, D] tensors.
sdrop_attn_t describe(const Tensor &q, const Tensor &k, const Tensor &v, const AttnArgs &a)
{
    const bool pq = a.cu_q.has_value(), pk = a.cu_k.has_value();
    require(q.is_cuda() && q.dim() == (pq ? 3 : 4) && k.dim() == (pk ? 3 : 4) && v.sizes() == k.sizes(),
            "q, k and v are GPU tensors [B, tokens, heads, D], or [tokens, heads, D] where their offsets are given");
    require(k.scalar_type() == q.scalar_type() && v.scalar_type() == q.scalar_type() && k.device() == q.device() && v.device() == q.device(),
            "q, k and v must have the same dtype and device");
    sdrop_attn_t d = {};
    d.dtype = type_code(q, "attention");
    d.Hq = q.size(-2);
    d.Hkv = k.size(-2);
    d.D = q.size(-1);
    require(k.size(-1) == d.D, "q, k and v must have the same head size");
    d.B = pq ? a.cu_q->size(0) - 1 : q.size(0);
    require(pk || k.size(0) == d.B, "q and k must have the same number of sequences");
    d.max_q = pq ? a.max_q : q.size(1);
    d.max_k = pk ? a.max_k : k.size(1);
    d.total_q = pq ? q.size(0) : 0;
    d.total_k = pk ? k.size(0) : 0;
    auto index = [&](const OptTensor &t, int64_t n) -> const int32_t * {
        if (!t) return nullptr;
        require(t->is_cuda() && t->scalar_type() == torch::kInt && t->dim() == 1 && t->size(0) == n && t->is_contiguous() && t->device() == q.device(),
                "offsets are int32 [B + 1] and lengths int32 [B], on the tensors' device");
        return t->data_ptr<int32_t>();
    };
    d.cu_q = index(a.cu_q, d.B + 1);
    d.cu_k = index(a.cu_k, d.B + 1);
    d.k_len = index(a.k_len, d.B);
    d.scale = a.scale != 0.0 ? a.scale : 1.0 / std::sqrt((double)d.D);
    d.causal = a.causal;
    strides(q, d.q_b, d.q_t, d.q_h);
    strides(k, d.k_b, d.k_t, d.k_h);
    strides(v, d.v_b, d.v_t, d.v_h);
    return d;
}

// A result like t.  With offsets or lengths not every row is written: those behind the last packed sequence, and those of a sequence whose
// values do not fit the call, are 0.
bool some_left(const AttnArgs &a) { return a.cu_q || a.cu_k || a.k_len; }
Tensor like(const Tensor &t, const AttnArgs &a) { return some_left(a) ? torch::zeros(t.sizes(), t.options()) : torch::empty(t.sizes(), t.options()); }

// No queries, no keys or no sequences: there is nothing to launch, and what the description says of the heads is checked here.
bool nothing(const Tensor &q, const Tensor &k, const sdrop_attn_t &d)
{
    if (q.numel() && k.numel() && d.B) return false;
    sdrop_attn_t one = {};
    one.B = one.max_q = one.max_k = 1;
    one.Hq = d.Hq;
    one.Hkv = d.Hkv;
    one.o_h = one.do_h = one.dq_h = one.dk_h = one.dv_h = one.D = d.D;
    one.scale = d.scale;
    one.causal = d.causal;
    one.dtype = d.dtype;
    check(sdrop_attn_bwd_workspace_bytes(&one) ? SDROP_OK : SDROP_ESHAPE, "sdrop_attn");
    return true;
}

// o; for_backward: also lse and what o's rounding took
Tensor attn_forward(const Tensor &q, const Tensor &k, const Tensor &v, const AttnArgs &a, bool for_backward, Tensor &lse, Tensor &rest)
{
    sdrop_attn_t d = describe(q, k, v, a);
    Tensor o = like(q, a);
    strides(o, d.o_b, d.o_t, d.o_h);
    if (for_backward) {
        const auto f = q.options().dtype(torch::kFloat);
        lse = a.cu_q ? torch::empty({d.Hq, d.total_q}, f) : torch::empty({d.B, d.Hq, d.max_q}, f);
        rest = torch::empty(q.sizes(), q.options());
    }
    if (nothing(q, k, d)) return o.zero_();
    const size_t need = sdrop_attn_workspace_bytes(&d);
    Tensor ws;
    if (need) ws = torch::empty({(int64_t)need}, q.options().dtype(torch::kByte));
    check(sdrop_attn(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), for_backward ? rest.data_ptr() : nullptr,
                     for_backward ? lse.data_ptr<float>() : nullptr, &d, need ? ws.data_ptr() : nullptr, need, stream_of(q)), "sdrop_attn");
    return o;
}

// into dq, dk and dv (contiguous or slices)
void attn_backward(const Tensor &grad, const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &o, const Tensor &lse, const Tensor &rest,
                   const AttnArgs &a, const Tensor &dq, const Tensor &dk, const Tensor &dv)
{
    const Tensor g = in_place(grad);
    sdrop_attn_t d = describe(q, k, v, a);
    if (nothing(q, k, d)) {
        for (const Tensor &t : {dq, dk, dv}) t.zero_();
        return;
    }
    strides(o, d.o_b, d.o_t, d.o_h);
    strides(g, d.do_b, d.do_t, d.do_h);
    strides(dq, d.dq_b, d.dq_t, d.dq_h);
    strides(dk, d.dk_b, d.dk_t, d.dk_h);
    strides(dv, d.dv_b, d.dv_t, d.dv_h);
    const size_t need = sdrop_attn_bwd_workspace_bytes(&d);
    const Tensor ws = torch::empty({(int64_t)need}, q.options().dtype(torch::kByte));
    check_backward(sdrop_attn_bwd(g.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), rest.data_ptr(), lse.data_ptr<float>(),
                                  dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), &d, ws.data_ptr(), need, stream_of(q)), "sdrop_attn_bwd");
}

void keep(AutogradContext *ctx, const AttnArgs &a)
{
    ctx->saved_data["causal"] = a.causal;
    ctx->saved_data["scale"] = a.scale;
    ctx->saved_data["max_q"] = a.max_q;
    ctx->saved_data["max_k"] = a.max_k;
}
AttnArgs kept(AutogradContext *ctx, const Tensor &cu_q, const Tensor &cu_k, const Tensor &k_len)
{
    auto opt = [](const Tensor &t) { return t.defined() ? OptTensor(t) : OptTensor(); };
    return AttnArgs{ctx->saved_data["causal"].toBool(), ctx->saved_data["scale"].toDouble(), opt(cu_q), opt(cu_k), opt(k_len),
                    ctx->saved_data["max_q"].toInt(), ctx->saved_data["max_k"].toInt()};
}
Tensor or_none(const OptTensor &t) { return t ? *t : Tensor(); }

struct Attention : torch::autograd::Function<Attention> {
    static Tensor forward(AutogradContext *ctx, const Tensor &q0, const Tensor &k0, const Tensor &v0, const AttnArgs &a)
    {
        at::AutoDispatchBelowADInplaceOrView guard;
        const c10::DeviceGuard on(q0.device());
        const Tensor q = in_place(q0), k = in_place(k0), v = in_place(v0);
        Tensor lse, rest;
        Tensor o = attn_forward(q, k, v, a, a.train, lse, rest);
        if (a.train) {
            ctx->save_for_backward({q, k, v, o, lse, rest, or_none(a.cu_q), or_none(a.cu_k), or_none(a.k_len)});
            keep(ctx, a);
        }
        return o;
    }
    static variable_list backward(AutogradContext *ctx, variable_list g)
    {
        const variable_list s = ctx->get_saved_variables();
        const AttnArgs a = kept(ctx, s[6], s[7], s[8]);
        Tensor dq, dk, dv;
        {
            at::AutoDispatchBelowADInplaceOrView guard;
            dq = like(s[0], a);
            dk = like(s[1], a);
            dv = like(s[2], a);
            attn_backward(g[0], s[0], s[1], s[2], s[3], s[4], s[5], a, dq, dk, dv);
        }
        return once({dq, dk, dv, Tensor()}, joined(g, s));
    }
};

// The same on one tensor [.., Hq + 2 Hkv, D]: query, key and value heads of a token side by side, as one projection writes them.  Its
// gradient is one tensor too, written in place of three that autograd would have to put together.
struct QkvAttention : torch::autograd::Function<QkvAttention> {
    static Tensor forward(AutogradContext *ctx, const Tensor &qkv0, int64_t hkv, const AttnArgs &a)
    {
        at::AutoDispatchBelowADInplaceOrView guard;
        const c10::DeviceGuard on(qkv0.device());
        require(qkv0.is_cuda() && (qkv0.dim() == 3 || qkv0.dim() == 4) && hkv >= 1 && qkv0.size(-2) > 2 * hkv, "qkv is a GPU tensor [.., Hq + 2 Hkv, D]");
        const Tensor qkv = in_place(qkv0);
        const int64_t hq = qkv.size(-2) - 2 * hkv;
        Tensor lse, rest;
        Tensor o = attn_forward(qkv.narrow(-2, 0, hq), qkv.narrow(-2, hq, hkv), qkv.narrow(-2, hq + hkv, hkv), a, a.train, lse, rest);
        if (a.train) {
            ctx->save_for_backward({qkv, o, lse, rest, or_none(a.cu_q), or_none(a.k_len)});
            keep(ctx, a);
            ctx->saved_data["hkv"] = hkv;
        }
        return o;
    }
    static variable_list backward(AutogradContext *ctx, variable_list g)
    {
        const variable_list s = ctx->get_saved_variables();
        const AttnArgs a = kept(ctx, s[4], s[4], s[5]);
        const int64_t hkv = ctx->saved_data["hkv"].toInt(), hq = s[0].size(-2) - 2 * hkv;
        Tensor d;
        {
            at::AutoDispatchBelowADInplaceOrView guard;
            d = like(s[0], a);
            auto part = [&](const Tensor &t, int i) { return i == 0 ? t.narrow(-2, 0, hq) : t.narrow(-2, hq + (i - 1) * hkv, hkv); };
            attn_backward(g[0], part(s[0], 0), part(s[0], 1), part(s[0], 2), s[1], s[2], s[3], a, part(d, 0), part(d, 1), part(d, 2));
        }
        return once({d, Tensor(), Tensor()}, joined(g, s));
    }
};

}  // namespace

PYBIND11_MODULE(_native, m)
{
    m.doc() = "Autograd nodes of libsdrop's transformer operators";
    pybind11::register_exception_translator([](std::exception_ptr e) {
        try {
            if (e) std::rethrow_exception(e);
        } catch (const Failure &f) {
            pybind11::object cls = pybind11::module_::import("paper_2411_01238_amd.sdrop").attr("SdropError");
            PyErr_SetObject(cls.ptr(), cls(f.code, f.call).ptr());
        }
    });
    m.def("dropout", [](const Tensor &x, const OptTensor &residual, double p, uint64_t seed, uint64_t stream) {
        return Dropout::apply(x, residual, p, (int64_t)seed, (int64_t)stream);
    });
    m.def("layer_norm", [](const Tensor &x, const Tensor &w, const OptTensor &b, double eps) { return LayerNorm::apply(x, w, b, eps); });
    m.def("dropout_add_norm", [](const Tensor &x, const Tensor &r, const Tensor &w, const OptTensor &b, double p, double eps, uint64_t seed, uint64_t stream) {
        const variable_list o = DropoutAddNorm::apply(x, r, w, b, p, eps, (int64_t)seed, (int64_t)stream);
        return std::make_pair(o[0], o[1]);
    });
    m.def("attention", [](const Tensor &q, const Tensor &k, const Tensor &v, bool causal, double scale, const OptTensor &cu_q, const OptTensor &cu_k,
                          int64_t max_q, int64_t max_k, const OptTensor &k_len) {
        const bool train = at::GradMode::is_enabled() && (q.requires_grad() || k.requires_grad() || v.requires_grad());
        return Attention::apply(q, k, v, AttnArgs{causal, scale, cu_q, cu_k, k_len, max_q, max_k, train});
    });
    m.def("qkv_attention", [](const Tensor &qkv, int64_t hkv, bool causal, double scale, const OptTensor &cu, int64_t max_len, const OptTensor &k_len) {
        const bool train = at::GradMode::is_enabled() && qkv.requires_grad();
        return QkvAttention::apply(qkv, hkv, AttnArgs{causal, scale, cu, cu, k_len, max_len, max_len, train});
    });
}
