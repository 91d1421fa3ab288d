// Native half of the Python binding of include/ssm_learn.h; the contract with learn.py is that of pybind.cpp with binding.py: the outputs when the
// call was made, an int (the ssm_status) when the library refused it, None for arguments that the general path has to look at.
// Host time of a call with new outputs, general path -> here: a step of the recurrence 15 -> 5.0 us, its forward and gradient pass 38 -> 11.9, loss and gradient of a policy 29 -> 10.4
// (five outputs, a workspace and two launches), AdamW of six tensors 25 -> 4.6.
#include "pybind_common.h"

#include <vector>

namespace {

// code of an ssm_dtype, or -1
int dtype_code(const Arg &a)
{
    if (!a.t) return -1;
    switch (a.t->scalar_type()) {
    case c10::kFloat: return SSM_F32;
    case c10::kBFloat16: return SSM_BF16;
    case c10::kHalf: return SSM_F16;
    default: return -1;
    }
}
// a GPU tensor of this type and shape with a dense last dimension
bool rows_ok(const Arg &a, c10::ScalarType dt, c10::IntArrayRef shape)
{
    return a.t && a.t->is_cuda() && a.t->scalar_type() == dt && a.t->sizes() == shape && (shape.back() <= 1 || a.t->stride(-1) == 1);
}
ssm_strides strides_of(const at::Tensor &t) { return {t.stride(0), t.stride(1)}; }

// An output that lies in memory as `like` does (dense where that one has gaps or overlaps itself), or the caller's, checked like an input.
bool activation(PyObject *given, const at::Tensor &like, at::Tensor &t)
{
    if (given && given != Py_None) {
        const Arg g(given);
        if (!rows_ok(g, like.scalar_type(), like.sizes())) return false;
        t = *g.t;
        return true;
    }
    if (!like.is_contiguous()) {
        t = at::empty_like(like);
        if (like.sizes().back() <= 1 || t.stride(-1) == 1) return true;      // (else windows over one array: empty_like has put the dimensions in another order)
    }
    t = at::Tensor(at::detail::empty_cuda(like.sizes(), like.scalar_type(), like.device(), std::nullopt));
    return true;
}
// A float32 output of this shape, or the caller's.
bool plain(PyObject *given, std::initializer_list<int64_t> shape, const at::Tensor &like, at::Tensor &t)
{
    if (given && given != Py_None) {
        const Arg g(given);
        if (!g.is(F32, shape)) return false;
        t = *g.t;
        return true;
    }
    t = empty(shape, F32, like);
    return true;
}
bool number(PyObject *o, double &v)
{
    v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); return false; }
    return true;
}
bool one_value(const Arg &a) { return a.none || (a.t && a.t->is_cuda() && a.t->scalar_type() == F32 && a.t->numel() == 1); }

struct Gated {
    Arg gate, u, first, h0;
    int64_t Bt = 0, L = 0, D = 0;
    int code;
    bool ok;
    explicit Gated(PyObject *const *a) : gate(a[0]), u(a[1]), first(a[2]), h0(a[3]), code(dtype_code(gate))
    {
        ok = code >= 0 && gate.dim() == 3;
        if (!ok) return;
        Bt = gate.size(0); L = gate.size(1); D = gate.size(2);
        const c10::ScalarType dt = gate.t->scalar_type();
        ok = rows_ok(gate, dt, {Bt, L, D}) && rows_ok(u, dt, {Bt, L, D}) && first.is(U8, {Bt, L}, true) && h0.is(F32, {Bt, D}, true);
    }
};
// The workspace of a recurrence: most shapes need none.
struct GatedWorkspace {
    at::Tensor own;
    void *p = nullptr;
    size_t n = 0;
    bool bad = false;
    GatedWorkspace(const Arg &given, const Gated &i, int bwd, bool own_stream)
    {
        if (workspace_ok(given)) { p = given.t->data_ptr(); n = (size_t)given.t->numel(); return; }
        if (!given.none) { bad = true; return; }
        n = ssm_gated_workspace_bytes(i.Bt, i.L, i.D, i.code, bwd);
        if (n == 0) return;
        if (!own_stream) { bad = true; return; }
        own = empty({(int64_t)n}, U8, *i.gate.t);
        p = own.data_ptr();
    }
};

// (gate, u, is_first, h0, linear, want_carry, workspace, stream, out)
ENTRY(gated_scan_fwd)
{
    TRY_BEGIN
    GENERAL_PATH_UNLESS(n == 9);
    const Gated i(a);
    const Arg ws(a[6]);
    void *s;
    GENERAL_PATH_UNLESS(i.ok && !ws.bad && stream_of(a[7], nullptr, s) && (a[8] == Py_None || PyDict_Check(a[8])));
    const int linear = yes(a[4]);
    const at::Tensor &u = *i.u.t;
    const int64_t rows = ssm_gated_carry_rows(i.L);
    const GatedWorkspace w(ws, i, 0, a[7] == Py_None);
    at::Tensor h, last, carry;
    GENERAL_PATH_UNLESS(!w.bad && activation(item(a[8], "h"), u, h) && plain(item(a[8], "h_last"), {i.Bt, i.D}, u, last));
    if (yes(a[5]) && rows) GENERAL_PATH_UNLESS(plain(item(a[8], "carry"), {i.Bt, rows, i.D}, u, carry));
    CALL(ssm_gated_scan_fwd, i.gate.ptr<const void>(), strides_of(*i.gate.t), i.u.ptr<const void>(), strides_of(u), i.first.u8(), i.h0.f32(), i.code,
         linear, i.Bt, i.L, i.D, h.data_ptr(), strides_of(h), f32(last), f32(carry), w.p, w.n, s);
    return dict({{"h", &h}, {"h_last", &last}, {"carry", &carry}});
    TRY_END
}

// (gate, u, is_first, h0, carry, dh, dh_last, linear, want_dh0, workspace, stream, out)
ENTRY(gated_scan_bwd)
{
    TRY_BEGIN
    GENERAL_PATH_UNLESS(n == 12);
    const Gated i(a);
    const Arg carry(a[4]), dh(a[5]), dl(a[6]), ws(a[9]);
    void *s;
    GENERAL_PATH_UNLESS(i.ok && !ws.bad && stream_of(a[10], nullptr, s) && (a[11] == Py_None || PyDict_Check(a[11])));
    const int64_t rows = ssm_gated_carry_rows(i.L);
    GENERAL_PATH_UNLESS(carry.is(F32, {i.Bt, rows, i.D}, rows == 0) && rows_ok(dh, i.gate.t->scalar_type(), {i.Bt, i.L, i.D}) &&
                        dl.is(F32, {i.Bt, i.D}, true));
    const int linear = yes(a[7]);
    const GatedWorkspace w(ws, i, 1, a[10] == Py_None);
    at::Tensor dgate, du, dh0;
    GENERAL_PATH_UNLESS(!w.bad && activation(item(a[11], "dgate"), *i.gate.t, dgate) && activation(item(a[11], "du"), *i.u.t, du));
    if (yes(a[8])) GENERAL_PATH_UNLESS(plain(item(a[11], "dh0"), {i.Bt, i.D}, *i.u.t, dh0));
    CALL(ssm_gated_scan_bwd, i.gate.ptr<const void>(), strides_of(*i.gate.t), i.u.ptr<const void>(), strides_of(*i.u.t), i.first.u8(), i.h0.f32(),
         carry.f32(), dh.ptr<const void>(), strides_of(*dh.t), dl.f32(), i.code, linear, i.Bt, i.L, i.D, dgate.data_ptr(), strides_of(dgate),
         du.data_ptr(), strides_of(du), f32(dh0), w.p, w.n, s);
    return dict({{"dgate", &dgate}, {"du", &du}, {"dh0", &dh0}});
    TRY_END
}

// (gate, u, h_prev, is_first, linear, h, y, stream)
ENTRY(gated_step)
{
    TRY_BEGIN
    GENERAL_PATH_UNLESS(n == 8);
    const Arg gate(a[0]), u(a[1]), prev(a[2]), first(a[3]);
    const int code = dtype_code(gate);
    void *s;
    GENERAL_PATH_UNLESS(code >= 0 && gate.dim() == 2 && stream_of(a[7], nullptr, s));
    const int64_t Bt = gate.size(0), D = gate.size(1);
    const c10::ScalarType dt = gate.t->scalar_type();
    GENERAL_PATH_UNLESS(rows_ok(gate, dt, {Bt, D}) && rows_ok(u, dt, {Bt, D}) && prev.is(F32, {Bt, D}, true) && first.is(U8, {Bt}, true));
    const int linear = yes(a[4]);
    const Arg yo(a[6]);
    at::Tensor h, y;
    GENERAL_PATH_UNLESS(plain(a[5], {Bt, D}, *gate.t, h) && yo.is(dt, {Bt, D}, true));
    y = yo.t ? *yo.t : empty({Bt, D}, dt, *gate.t);
    CALL(ssm_gated_step, gate.ptr<const void>(), gate.t->stride(0), u.ptr<const void>(), u.t->stride(0), prev.f32(), first.u8(), code, linear, Bt, D,
         f32(h), y.data_ptr(), s);
    return tuple({&y, &h});
    TRY_END
}

// logits, action, logp_old, advantage, weight, logp_ref and the four terms behind them
struct Policy {
    Arg x, action, old, adv, weight, ref;
    int64_t N = 0, K = 0;
    int code;
    bool ok;
    explicit Policy(PyObject *const *a) : x(a[0]), action(a[1]), old(a[2]), adv(a[3]), weight(a[4]), ref(a[5]), code(dtype_code(x))
    {
        ok = code >= 0 && x.dim() == 2;
        if (!ok) return;
        N = x.size(0); K = x.size(1);
        ok = rows_ok(x, x.t->scalar_type(), {N, K}) && action.is(c10::kLong, {N}) && old.is(F32, {N}) && adv.is(F32, {N}) && weight.is(F32, {N}, true) &&
             ref.is(F32, {N}, true);
    }
};
bool terms_of(PyObject *const *a, ssm_policy_terms &t)
{
    double v[4];
    for (int k = 0; k < 4; ++k) if (!number(a[k], v[k])) return false;
    t = {(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
    return true;
}
struct RowResults {
    at::Tensor loss, logp, entropy, lse;
    bool ok;
    RowResults(PyObject *out, const Policy &i)
    {
        const at::Tensor &x = *i.x.t;
        ok = plain(item(out, "loss"), {}, x, loss) && plain(item(out, "logp"), {i.N}, x, logp) && plain(item(out, "entropy"), {i.N}, x, entropy) &&
             plain(item(out, "lse"), {i.N}, x, lse);
    }
};

// (logits, action, logp_old, advantage, weight, logp_ref, clip_low, clip_high, kl_coef, entropy_coef, workspace, stream, out)
ENTRY(policy_loss_fwd)
{
    TRY_BEGIN
    GENERAL_PATH_UNLESS(n == 13);
    const Policy i(a);
    const Arg ws(a[10]);
    ssm_policy_terms t;
    void *s;
    GENERAL_PATH_UNLESS(i.ok && terms_of(a + 6, t) && stream_of(a[11], &ws, s) && (a[12] == Py_None || PyDict_Check(a[12])));
    const Workspace w(ws, ws.none ? ssm_policy_loss_workspace_bytes(i.N, i.K) : 0, *i.x.t);
    GENERAL_PATH_UNLESS(!w.bad);
    const RowResults r(a[12], i);
    GENERAL_PATH_UNLESS(r.ok);
    CALL(ssm_policy_loss_fwd, i.x.ptr<const void>(), i.x.t->stride(0), i.action.ptr<const int64_t>(), i.old.f32(), i.adv.f32(), i.weight.f32(), i.ref.f32(), t,
         i.code, i.N, i.K, f32(r.loss), f32(r.logp), f32(r.entropy), f32(r.lse), w.p, w.n, s);
    return dict({{"loss", &r.loss}, {"logp", &r.logp}, {"entropy", &r.entropy}, {"lse", &r.lse}});
    TRY_END
}

// (logits, action, logp_old, advantage, weight, logp_ref, clip_low, clip_high, kl_coef, entropy_coef, logp, entropy, lse, dloss, dlogits, stream)
ENTRY(policy_loss_bwd)
{
    TRY_BEGIN
    GENERAL_PATH_UNLESS(n == 16);
    const Policy i(a);
    const Arg logp(a[10]), entropy(a[11]), lse(a[12]), dloss(a[13]);
    ssm_policy_terms t;
    void *s;
    GENERAL_PATH_UNLESS(i.ok && terms_of(a + 6, t) && stream_of(a[15], nullptr, s) && logp.is(F32, {i.N}) && entropy.is(F32, {i.N}) && lse.is(F32, {i.N}) &&
                        one_value(dloss));
    at::Tensor dx;
    GENERAL_PATH_UNLESS(activation(a[14], *i.x.t, dx));
    CALL(ssm_policy_loss_bwd, i.x.ptr<const void>(), i.x.t->stride(0), i.action.ptr<const int64_t>(), i.old.f32(), i.adv.f32(), i.weight.f32(), i.ref.f32(), t,
         i.code, i.N, i.K, logp.f32(), entropy.f32(), lse.f32(), dloss.f32(), dx.data_ptr(), dx.stride(0), s);
    return wrap(dx);
    TRY_END
}

// (logits, action, logp_old, advantage, weight, logp_ref, clip_low, clip_high, kl_coef, entropy_coef, dloss, workspace, stream, out)
ENTRY(policy_loss_grad)
{
    TRY_BEGIN
    GENERAL_PATH_UNLESS(n == 14);
    const Policy i(a);
    const Arg dloss(a[10]), ws(a[11]);
    ssm_policy_terms t;
    void *s;
    GENERAL_PATH_UNLESS(i.ok && terms_of(a + 6, t) && stream_of(a[12], &ws, s) && (a[13] == Py_None || PyDict_Check(a[13])) && one_value(dloss));
    const Workspace w(ws, ws.none ? ssm_policy_loss_workspace_bytes(i.N, i.K) : 0, *i.x.t);
    GENERAL_PATH_UNLESS(!w.bad);
    const RowResults r(a[13], i);
    at::Tensor dx;
    GENERAL_PATH_UNLESS(r.ok && activation(item(a[13], "dlogits"), *i.x.t, dx));
    CALL(ssm_policy_loss_grad, i.x.ptr<const void>(), i.x.t->stride(0), i.action.ptr<const int64_t>(), i.old.f32(), i.adv.f32(), i.weight.f32(), i.ref.f32(), t,
         i.code, i.N, i.K, dloss.f32(), f32(r.loss), f32(r.logp), f32(r.entropy), f32(r.lse), dx.data_ptr(), dx.stride(0), w.p, w.n, s);
    return dict({{"loss", &r.loss}, {"logp", &r.logp}, {"entropy", &r.entropy}, {"lse", &r.lse}, {"dlogits", &dx}});
    TRY_END
}

// One list (or tuple) of tensors; absent where None.
struct List {
    PyObject *const *items = nullptr;
    Py_ssize_t n = 0;
    bool none, ok;
    explicit List(PyObject *o) : none(o == Py_None), ok(none || PyList_Check(o) || PyTuple_Check(o))
    {
        if (!none && ok) { n = PySequence_Fast_GET_SIZE(o); items = PySequence_Fast_ITEMS(o); }
    }
};
bool like_ok(const Arg &a, c10::ScalarType dt, c10::IntArrayRef shape)
{
    return a.t && a.t->is_cuda() && a.t->scalar_type() == dt && a.t->sizes() == shape && a.t->is_contiguous();
}
int64_t blocks_of(int64_t n) { return (n + SSM_ADAMW_BLOCK - 1) / SSM_ADAMW_BLOCK; }

// (params, grads, m, v, m_scale, v_scale, lr, beta1, beta2, eps, weight_decay, step, grad_scale, skip, stream)
ENTRY(adamw_step)
{
    TRY_BEGIN
    GENERAL_PATH_UNLESS(n == 15);
    const List p(a[0]), g(a[1]), m(a[2]), v(a[3]), ms(a[4]), vs(a[5]);
    GENERAL_PATH_UNLESS(p.ok && g.ok && m.ok && v.ok && ms.ok && vs.ok && p.n > 0 && g.n == p.n && m.n == p.n && v.n == p.n);
    const Arg p0(p.items[0]), g0(g.items[0]), m0(m.items[0]), scale(a[12]), skip(a[13]);
    const int pc = dtype_code(p0), gc = dtype_code(g0);
    ssm_adamw_rates r;
    void *s;
    GENERAL_PATH_UNLESS(pc >= 0 && gc >= 0 && m0.t && one_value(scale) && one_value(skip) && number(a[6], r.lr) && number(a[7], r.beta1) && number(a[8], r.beta2) &&
                        number(a[9], r.eps) && number(a[10], r.weight_decay) && PyLong_Check(a[11]));
    r.step = PyLong_AsLongLong(a[11]);
    if (r.step == -1 && PyErr_Occurred()) { PyErr_Clear(); Py_RETURN_NONE; }
    const bool eight = m0.t->scalar_type() == U8;
    GENERAL_PATH_UNLESS(!eight || (ms.n == p.n && vs.n == p.n));
    const c10::ScalarType pdt = p0.t->scalar_type(), gdt = g0.t->scalar_type(), sdt = eight ? U8 : F32;
    std::vector<ssm_adamw_tensor> rows((size_t)p.n);
    for (Py_ssize_t k = 0; k < p.n; ++k) {
        const Arg pk(p.items[k]), gk(g.items[k]), mk(m.items[k]), vk(v.items[k]);
        GENERAL_PATH_UNLESS(pk.t && like_ok(pk, pdt, pk.t->sizes()) && like_ok(gk, gdt, pk.t->sizes()) && like_ok(mk, sdt, pk.t->sizes()) &&
                            like_ok(vk, sdt, pk.t->sizes()));
        ssm_adamw_tensor &t = rows[(size_t)k];
        t = {pk.ptr<void>(), gk.ptr<const void>(), mk.ptr<void>(), vk.ptr<void>(), nullptr, nullptr, pk.t->numel()};
        if (eight) {
            const Arg msk(ms.items[k]), vsk(vs.items[k]);
            GENERAL_PATH_UNLESS(msk.is(F32, {blocks_of(t.n)}) && vsk.is(F32, {blocks_of(t.n)}));
            t.m_scale = msk.ptr<float>(); t.v_scale = vsk.ptr<float>();
        }
    }
    GENERAL_PATH_UNLESS(stream_of(a[14], nullptr, s));
    CALL(ssm_adamw_step, (const ssm_adamw_tensor *)rows.data(), (int64_t)p.n, r, pc, gc, eight ? 8 : 32, scale.f32(), skip.f32(), s);
    Py_RETURN_TRUE;
    TRY_END
}

// (m, v, m_scale, v_scale, m_out, v_out, stream)
ENTRY(adamw_values)
{
    TRY_BEGIN
    GENERAL_PATH_UNLESS(n == 7);
    const List m(a[0]), v(a[1]), ms(a[2]), vs(a[3]), mo(a[4]), vo(a[5]);
    void *s;
    GENERAL_PATH_UNLESS(m.ok && v.ok && ms.ok && vs.ok && mo.ok && vo.ok && m.n > 0 && v.n == m.n && ms.n == m.n && vs.n == m.n && mo.n == m.n && vo.n == m.n &&
                        stream_of(a[6], nullptr, s));
    std::vector<ssm_adamw_stored> rows((size_t)m.n);
    for (Py_ssize_t k = 0; k < m.n; ++k) {
        const Arg mk(m.items[k]), vk(v.items[k]), msk(ms.items[k]), vsk(vs.items[k]), mok(mo.items[k]), vok(vo.items[k]);
        GENERAL_PATH_UNLESS(mk.t && like_ok(mk, U8, mk.t->sizes()) && like_ok(vk, U8, mk.t->sizes()) && like_ok(mok, F32, mk.t->sizes()) &&
                            like_ok(vok, F32, mk.t->sizes()));
        const int64_t numel = mk.t->numel();
        GENERAL_PATH_UNLESS(msk.is(F32, {blocks_of(numel)}) && vsk.is(F32, {blocks_of(numel)}));
        rows[(size_t)k] = {mk.ptr<const void>(), vk.ptr<const void>(), msk.f32(), vsk.f32(), mok.ptr<float>(), vok.ptr<float>(), numel};
    }
    CALL(ssm_adamw_values, (const ssm_adamw_stored *)rows.data(), (int64_t)m.n, s);
    Py_RETURN_TRUE;
    TRY_END
}

PyMethodDef methods[] = {METHOD(gated_scan_fwd), METHOD(gated_scan_bwd), METHOD(gated_step), METHOD(policy_loss_fwd), METHOD(policy_loss_bwd),
                         METHOD(policy_loss_grad), METHOD(adamw_step), METHOD(adamw_values), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ssmlearn", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject *PyInit__ssmlearn(void) { return PyModule_Create(&module); }
