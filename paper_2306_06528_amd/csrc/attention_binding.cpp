// What a call of attention.py needs before the library can be called, as layers_binding.cpp does it for layers.py.
#include "binding_common.hpp"

#include "../../include/svgd_attention.h"

namespace {

const char *const kNoHeads = "%s must be a CUDA tensor (particles, batch, tokens, heads, dim) of float32, bfloat16 or float16";

// Activations with heads.
struct HeadsOf {
    at::Tensor t;
    int64_t size(int d) const { return t.size(d); }
    int dtype() const { return dtype_of(t.scalar_type()); }
    svgd_heads desc() const { return {t.data_ptr(), t.stride(0), t.stride(1), t.stride(2), t.stride(3)}; }
};

void same_kind(const at::Tensor &t, const at::Tensor &like, const char *name)
{
    if (t.scalar_type() != like.scalar_type() || t.device() != like.device()) fail(PyExc_ValueError, "%s must have the type and device of the other activations", name);
}

HeadsOf heads(PyObject *obj, const char *name, const HeadsOf *like = nullptr)
{
    if (!THPVariable_Check(obj)) fail(PyExc_TypeError, kNoHeads, name);
    HeadsOf h{THPVariable_Unpack(obj)};
    if (!h.t.is_cuda() || dtype_of(h.t.scalar_type()) < 0 || h.t.dim() != 5) fail(PyExc_TypeError, kNoHeads, name);
    if (like) same_kind(h.t, like->t, name);
    if (h.t.size(4) != 1 && h.t.stride(4) != 1 && h.t.numel()) fail(PyExc_TypeError, "%s must have contiguous heads", name);
    return h;
}

void shaped(const HeadsOf &h, at::IntArrayRef shape, const char *name)
{
    if (h.t.sizes() == shape) return;
    std::ostringstream text;
    text << "%s must have the shape " << shape << ", not " << h.t.sizes();
    fail(PyExc_ValueError, text.str().c_str(), name);
}

// Attention's kernels reach so far from token to token and head to head; beyond that a copy.
HeadsOf near_heads(PyObject *obj, const char *name, const HeadsOf *like = nullptr)
{
    HeadsOf h = heads(obj, name, like);
    const int64_t most = SVGD_ATTENTION_MAX_STRIDE, count = h.t.size(3);
    if ((h.t.size(2) > 1 && h.t.stride(2) >= most) || (count > 1 && h.t.stride(3) >= most / count)) {
        const at::NoGradGuard no_grad;
        h.t = h.t.contiguous();
    }
    return h;
}

at::Tensor new_heads(const HeadsOf &h) { return at::empty(h.t.sizes(), h.t.options().memory_format(c10::nullopt)); }
svgd_heads desc(const at::Tensor &t) { return t.defined() ? svgd_heads{t.data_ptr(), t.stride(0), t.stride(1), t.stride(2), t.stride(3)} : svgd_heads{nullptr, 0, 0, 0, 0}; }

// param and current_stream look at an activation's device (and its particles)
Act act_of(const HeadsOf &h) { return Act{h.t, h.t}; }

int small(int64_t v) { return v > INT32_MAX ? INT32_MAX : (int)v; } // (refused by the library)

// A contiguous tensor of whole numbers (or doubles) on the activations' device; None: undefined.
at::Tensor numbers(PyObject *obj, const char *name, at::ScalarType type, const at::Tensor &like, const char *what)
{
    if (obj == Py_None) return {};
    if (!THPVariable_Check(obj)) fail(PyExc_TypeError, what, name);
    const at::Tensor &t = THPVariable_Unpack(obj);
    if (t.scalar_type() != type || t.device() != like.device() || !t.is_contiguous()) fail(PyExc_TypeError, what, name);
    return t;
}

int activation_of(PyObject *obj)
{
    const char *const name = PyUnicode_Check(obj) ? PyUnicode_AsUTF8(obj) : "";
    if (!name) throw Failed{};
    const int a = !strcmp(name, "none")   ? SVGD_NO_ACTIVATION
                  : !strcmp(name, "silu") ? SVGD_SILU
                  : !strcmp(name, "gelu") ? SVGD_GELU
                  : !strcmp(name, "relu") ? SVGD_RELU
                  : !strcmp(name, "tanh") ? SVGD_TANH
                                          : -1;
    if (a < 0) fail(PyExc_ValueError, "activation must be one of %s", "('none', 'silu', 'gelu', 'relu', 'tanh')");
    return a;
}

// A linear map's weight, (particles, out, width).
struct Linear {
    int activation;
    int64_t out;
    Param weight;
};
Linear linear_of(const Act &x, PyObject *weight, PyObject *activation)
{
    Linear l;
    l.activation = activation_of(activation);
    if (!THPVariable_Check(weight) || THPVariable_Unpack(weight).dim() != 3) fail(PyExc_TypeError, "%s must be a float32 CUDA tensor (particles, out, width)", "weight");
    l.out = THPVariable_Unpack(weight).size(1);
    l.weight = param(weight, "weight", {x.n(), l.out, x.width()}, x);
    return l;
}

// Activations like x's with `out` values in a row.
Act out_act(PyObject *obj, const char *name, const Act &x, int64_t out)
{
    const Act a = act(obj, name);
    auto want = x.given.sizes().vec();
    want.back() = out;
    if (a.given.sizes() != at::IntArrayRef(want)) {
        std::ostringstream text;
        text << "%s must have the shape " << at::IntArrayRef(want) << ", not " << a.given.sizes();
        fail(PyExc_ValueError, text.str().c_str(), name);
    }
    same_kind(a.given, x.given, name);
    return a;
}

const svgd_rows kNoRows{nullptr, 0, 0};

// What both passes of the rotation take.  a: q_weight, k_weight, frequencies, positions, layout, eps
struct Rotary {
    svgd_rotary p{};
    Param q_weight, k_weight;
    at::Tensor frequencies, positions;
};
Rotary rotary_of(const HeadsOf &q, const HeadsOf &k, PyObject *const *a)
{
    Rotary r;
    const Act x = act_of(q);
    if (k.size(0) != q.size(0) || k.size(1) != q.size(1) || k.size(2) != q.size(2) || k.size(4) != q.size(4)) shaped(k, {q.size(0), q.size(1), q.size(2), k.size(3), q.size(4)}, "k");
    r.q_weight = param(a[0], "q_weight", {q.size(0), q.size(4)}, x, true);
    r.k_weight = param(a[1], "k_weight", {q.size(0), q.size(4)}, x, true);
    if (!r.q_weight.t != !r.k_weight.t) fail(PyExc_ValueError, "%s must be given together, or neither", "q_weight and k_weight");
    r.frequencies = numbers(a[2], "frequencies", at::kDouble, q.t, "%s must be a contiguous float64 tensor (pairs,) on the device of q");
    r.positions = numbers(a[3], "positions", at::kLong, q.t, "%s must be a contiguous int64 tensor (tokens,) or (batch, tokens) on the device of q");
    if (r.frequencies.defined() != r.positions.defined()) fail(PyExc_ValueError, "%s must be given together, or neither", "frequencies and positions");
    const char *const layout = PyUnicode_Check(a[4]) ? PyUnicode_AsUTF8(a[4]) : "";
    if (!layout) throw Failed{};
    if (strcmp(layout, "half") && strcmp(layout, "interleaved")) fail(PyExc_ValueError, "layout must be one of %s", "('half', 'interleaved')");
    svgd_rotary &p = r.p;
    p.n = small(q.size(0));
    p.batch = q.size(1);
    p.length = q.size(2);
    p.heads = small(q.size(3));
    p.kv_heads = small(k.size(3));
    p.dim = small(q.size(4));
    p.interleaved = !strcmp(layout, "interleaved");
    p.eps = number(a[5]);
    if (r.frequencies.defined()) {
        if (r.frequencies.dim() != 1 || 2 * r.frequencies.size(0) > q.size(4)) fail(PyExc_ValueError, "%s must be a float64 tensor (pairs,), two values of a head for each pair", "frequencies");
        const at::Tensor &t = r.positions;
        if (!(t.dim() == 1 && t.size(0) == p.length) && !(t.dim() == 2 && t.size(0) == p.batch && t.size(1) == p.length))
            fail(PyExc_ValueError, "%s must have the shape (tokens,) or (batch, tokens)", "positions");
        p.pairs = small(r.frequencies.size(0));
        p.positions_stride = t.dim() == 2 ? p.length : 0;
    }
    return r;
}
void set_pointers(Rotary &r) // last, behind everything that can run other code
{
    r.p.q_weight = r.q_weight.p();
    r.p.q_weight_stride = r.q_weight.stride;
    r.p.k_weight = r.k_weight.p();
    r.p.k_weight_stride = r.k_weight.stride;
    r.p.frequencies = r.frequencies.defined() ? (const double *)r.frequencies.data_ptr() : nullptr;
    r.p.positions = r.positions.defined() ? (const int64_t *)r.positions.data_ptr() : nullptr;
}

// What both passes of attention take.  a: causal, cap, slopes, scale (None: 1 / sqrt(dim)), starts, lengths, documents, prefix
struct Attention {
    svgd_attention p{};
    Param slopes;
    at::Tensor starts, lengths, documents, prefix;
};
Attention attention_of(const HeadsOf &q, const HeadsOf &k, const HeadsOf &v, PyObject *const *a)
{
    Attention r;
    const int64_t n = q.size(0), batch = q.size(1), d = q.size(4);
    if (k.size(0) != n || k.size(1) != batch || k.size(4) != d) shaped(k, {n, batch, k.size(2), k.size(3), d}, "k");
    shaped(v, k.t.sizes(), "v");
    if (k.size(3) < 1 || q.size(3) % k.size(3)) fail(PyExc_ValueError, "%s must be a multiple of those of k", "the heads of q");
    svgd_attention &p = r.p;
    p.n = small(n);
    p.batch = batch;
    p.length = q.size(2);
    p.keys = k.size(2);
    p.heads = small(q.size(3));
    p.kv_heads = small(k.size(3));
    p.dim = small(d);
    p.causal = truth(a[0]);
    p.cap = number(a[1]);
    r.slopes = param(a[2], "slopes", {n, q.size(3)}, act_of(q), true);
    p.scale = a[3] == Py_None ? 1.0 / std::sqrt((double)(d < 1 ? 1 : d)) : number(a[3]);
    const char *const each = "%s must be a contiguous int32 tensor (batch,) on the device of q", *const keys = "%s must be a contiguous int32 tensor (batch, keys) on the device of q";
    r.starts = numbers(a[4], "starts", at::kInt, q.t, each);
    r.lengths = numbers(a[5], "lengths", at::kInt, q.t, each);
    r.documents = numbers(a[6], "documents", at::kInt, q.t, keys);
    r.prefix = numbers(a[7], "prefix", at::kInt, q.t, each);
    const std::pair<const at::Tensor *, const char *> lists[3] = {{&r.starts, "starts"}, {&r.lengths, "lengths"}, {&r.prefix, "prefix"}};
    for (const auto &l : lists)
        if (l.first->defined() && (l.first->dim() != 1 || l.first->size(0) != batch)) fail(PyExc_TypeError, each, l.second);
    if (r.documents.defined() && (r.documents.dim() != 2 || r.documents.size(0) != batch || r.documents.size(1) != p.keys)) fail(PyExc_TypeError, keys, "documents");
    return r;
}
const int32_t *ints(const at::Tensor &t) { return t.defined() ? (const int32_t *)t.data_ptr() : nullptr; }
void set_pointers(Attention &r)
{
    r.p.slopes = r.slopes.p();
    r.p.slopes_stride = r.slopes.stride;
    r.p.starts = ints(r.starts);
    r.p.lengths = ints(r.lengths);
    r.p.documents = ints(r.documents);
    r.p.prefix = ints(r.prefix);
}

} // namespace

// linear_forward(current_device, stream_of, x, weight, bias, activation, residual, save) -> (y, saved)
PyObject *linear_forward(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    return guarded(na, 8, [&]() -> PyObject * {
        const Act x = act(a[2], "x");
        const Linear l = linear_of(x, a[3], a[5]);
        const Param b = param(a[4], "bias", {x.n(), l.out}, x, true);
        Act residual;
        if (a[6] != Py_None) residual = out_act(a[6], "residual", x, l.out);
        const bool save = truth(a[7]) && l.activation != SVGD_NO_ACTIVATION;
        void *stream;
        if (!current_stream(x, a, stream)) Py_RETURN_NONE;
        auto shape = x.given.sizes().vec();
        shape.back() = l.out;
        const at::Tensor y = at::empty(shape, x.given.options());
        const size_t z_need = save ? svgd_linear_saved(x.particles(), x.rows(), l.out) : 0, need = svgd_linear_forward_scratch(x.particles(), x.rows(), x.width(), l.out);
        at::Tensor z, scratch;
        if (save) z = at::empty({(int64_t)(z_need / 4)}, x.given.options().dtype(at::kFloat));
        if (need) scratch = bytes(need, x);
        const int rc = unlocked([&] {
            return svgd_linear_forward(x.dtype(), l.activation, x.particles(), x.rows(), x.width(), l.out, x.desc(), l.weight.p(), l.weight.stride, b.p(), b.stride,
                                       residual.t.defined() ? residual.desc() : kNoRows, svgd_rows{y.data_ptr(), x.rows() * l.out, l.out}, z_need ? z.data_ptr() : nullptr, z_need,
                                       need ? scratch.data_ptr() : nullptr, need, stream);
        });
        return result(rc, {&y, &z});
    });
}

// linear_backward(current_device, stream_of, dy, x, weight, saved, dweight, dbias, activation, accumulate, want_dx) -> (dx,)
PyObject *linear_backward(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    return guarded(na, 11, [&]() -> PyObject * {
        const Act x = act(a[3], "x");
        const Linear l = linear_of(x, a[4], a[8]);
        const Act dy = out_act(a[2], "dy", x, l.out);
        const Param dw = param(a[6], "dweight", {x.n(), l.out, x.width()}, x, true), db = param(a[7], "dbias", {x.n(), l.out}, x, true);
        const size_t z_need = l.activation == SVGD_NO_ACTIVATION ? 0 : svgd_linear_saved(x.particles(), x.rows(), l.out);
        at::Tensor z;
        if (l.activation != SVGD_NO_ACTIVATION) {
            const char *const what = "%s must be what linear_forward returned for x with save=True";
            if (!THPVariable_Check(a[5])) fail(PyExc_TypeError, what, "saved");
            z = THPVariable_Unpack(a[5]);
            if (z.scalar_type() != at::kFloat || (size_t)z.numel() * 4 != z_need || z.device() != x.given.device() || !z.is_contiguous()) fail(PyExc_TypeError, what, "saved");
        }
        const bool accumulate = truth(a[9]), want_dx = truth(a[10]);
        void *stream;
        if (!current_stream(x, a, stream)) Py_RETURN_NONE;
        at::Tensor dx;
        if (want_dx) dx = new_like(x);
        const size_t all = svgd_linear_scratch(x.particles(), x.rows(), x.width(), l.out);
        const size_t need = all && l.activation == SVGD_NO_ACTIVATION ? all - svgd_linear_saved(x.particles(), x.rows(), l.out) : all;
        const at::Tensor scratch = bytes(need, x);
        const int rc = unlocked([&] {
            return svgd_linear_backward(x.dtype(), l.activation, x.particles(), x.rows(), x.width(), l.out, dy.desc(), x.desc(), l.weight.p(), l.weight.stride,
                                        z_need ? z.data_ptr() : nullptr, z_need, want_dx ? dense(dx, x) : kNoRows, dw.p(), dw.stride, db.p(), db.stride, accumulate,
                                        scratch.data_ptr(), need, stream);
        });
        return result(rc, {&dx});
    });
}

// qk_norm_rotary_forward(current_device, stream_of, q, k, q_weight, k_weight, frequencies, positions, layout, eps) -> (q, k)
PyObject *qk_norm_rotary_forward(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    return guarded(na, 10, [&]() -> PyObject * {
        const HeadsOf q = heads(a[2], "q"), k = heads(a[3], "k", &q);
        Rotary r = rotary_of(q, k, a + 4);
        void *stream;
        if (!current_stream(act_of(q), a, stream)) Py_RETURN_NONE;
        const at::Tensor qo = new_heads(q), ko = new_heads(k);
        set_pointers(r);
        const int rc = unlocked([&] { return svgd_qk_norm_rotary_forward(q.dtype(), &r.p, q.desc(), k.desc(), desc(qo), desc(ko), stream); });
        return result(rc, {&qo, &ko});
    });
}

// qk_norm_rotary_backward(current_device, stream_of, dq_out, dk_out, q, k, q_weight, k_weight, frequencies, positions, layout, eps,
// dq_weight, dk_weight, accumulate) -> (dq, dk)
PyObject *qk_norm_rotary_backward(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    return guarded(na, 15, [&]() -> PyObject * {
        const HeadsOf q = heads(a[4], "q"), k = heads(a[5], "k", &q), dqo = heads(a[2], "dq", &q), dko = heads(a[3], "dk", &q);
        Rotary r = rotary_of(q, k, a + 6);
        shaped(dqo, q.t.sizes(), "dq");
        shaped(dko, k.t.sizes(), "dk");
        const Act x = act_of(q);
        const Param dqw = param(a[12], "dq_weight", {q.size(0), q.size(4)}, x, true), dkw = param(a[13], "dk_weight", {q.size(0), q.size(4)}, x, true);
        if ((dqw.t || dkw.t) && !r.q_weight.t) fail(PyExc_ValueError, "%s need q_weight and k_weight", "dq_weight and dk_weight");
        const bool accumulate = truth(a[14]);
        void *stream;
        if (!current_stream(x, a, stream)) Py_RETURN_NONE;
        const at::Tensor dq = new_heads(q), dk = new_heads(k);
        at::Tensor scratch;
        const size_t need = dqw.t || dkw.t ? svgd_qk_norm_rotary_scratch(&r.p) : 0;
        if (need) scratch = bytes(need, x);
        set_pointers(r);
        const int rc = unlocked([&] {
            return svgd_qk_norm_rotary_backward(q.dtype(), &r.p, dqo.desc(), dko.desc(), q.desc(), k.desc(), desc(dq), desc(dk), dqw.p(), dqw.stride, dkw.p(), dkw.stride, accumulate,
                                                need ? scratch.data_ptr() : nullptr, need, stream);
        });
        return result(rc, {&dq, &dk});
    });
}

// attention_forward(current_device, stream_of, q, k, v, causal, cap, slopes, scale, starts, lengths, documents, prefix) -> (o, lse)
PyObject *attention_forward(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    return guarded(na, 13, [&]() -> PyObject * {
        const HeadsOf q = near_heads(a[2], "q"), k = near_heads(a[3], "k", &q), v = near_heads(a[4], "v", &q);
        Attention r = attention_of(q, k, v, a + 5);
        const Act x = act_of(q);
        void *stream;
        if (!current_stream(x, a, stream)) Py_RETURN_NONE;
        const at::Tensor o = new_heads(q), lse = at::empty({q.size(0), q.size(1), q.size(3), q.size(2)}, q.t.options().dtype(at::kFloat));
        set_pointers(r);
        const size_t need = svgd_attention_forward_scratch(&r.p);
        at::Tensor scratch;
        if (need) scratch = bytes(need, x);
        const int rc = unlocked([&] {
            return svgd_attention_forward(q.dtype(), &r.p, q.desc(), k.desc(), v.desc(), desc(o), (float *)lse.data_ptr(), need ? scratch.data_ptr() : nullptr, need, stream);
        });
        return result(rc, {&o, &lse});
    });
}

// attention_backward(current_device, stream_of, do, q, k, v, o, lse, causal, cap, slopes, scale, starts, lengths, documents, prefix,
// dslopes, accumulate, want_dq, want_dkv) -> (dq, dk, dv)
PyObject *attention_backward(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    return guarded(na, 20, [&]() -> PyObject * {
        const HeadsOf q = near_heads(a[3], "q"), k = near_heads(a[4], "k", &q), v = near_heads(a[5], "v", &q), d_o = near_heads(a[2], "do", &q), o = heads(a[6], "o", &q);
        Attention r = attention_of(q, k, v, a + 8);
        shaped(d_o, q.t.sizes(), "do");
        shaped(o, q.t.sizes(), "o");
        const Act x = act_of(q);
        const char *const what = "%s must be what attention_forward returned for q, k and v";
        if (!THPVariable_Check(a[7])) fail(PyExc_TypeError, what, "lse");
        const at::Tensor lse = THPVariable_Unpack(a[7]);
        if (lse.scalar_type() != at::kFloat || lse.device() != q.t.device() || !lse.is_contiguous() || lse.sizes() != at::IntArrayRef({q.size(0), q.size(1), q.size(3), q.size(2)}))
            fail(PyExc_TypeError, what, "lse");
        const Param ds = param(a[16], "dslopes", {q.size(0), q.size(3)}, x, true);
        if (ds.t && !r.slopes.t) fail(PyExc_ValueError, "%s need slopes", "dslopes");
        const bool accumulate = truth(a[17]), want_dq = truth(a[18]), want_dkv = truth(a[19]);
        void *stream;
        if (!current_stream(x, a, stream)) Py_RETURN_NONE;
        at::Tensor dq, dk, dv;
        if (want_dq) dq = new_heads(q);
        if (want_dkv) {
            dk = new_heads(k);
            dv = new_heads(v);
        }
        set_pointers(r);
        const size_t need = svgd_attention_scratch(&r.p);
        const at::Tensor scratch = bytes(need, x);
        const int rc = unlocked([&] {
            return svgd_attention_backward(q.dtype(), &r.p, d_o.desc(), q.desc(), k.desc(), v.desc(), o.desc(), (const float *)lse.data_ptr(), desc(dq), desc(dk), desc(dv), ds.p(),
                                           ds.stride, accumulate, scratch.data_ptr(), need, stream);
        });
        return result(rc, {&dq, &dk, &dv});
    });
}
