// Extension module _native_losses: the losses on logits (losses.py), from Python to the library, with autograd's node and outputs from torch's allocator.
// In Python a step, loss and gradient, cost 160 to 210 us of the host.
#define PY_SSIZE_T_CLEAN
#include "zf_py_tensors.h"

namespace {

struct {                               // the library's calls (addresses given by losses.py)
    int (*distill)(const zf_distill_args *, void *, int64_t, int32_t, void *);
    int (*distill_back)(const zf_distill_args *, const float *, int32_t, void *, int64_t, int32_t, void *);
    int (*policy)(const zf_policy_args *, void *, int64_t, int32_t, void *);
    int (*policy_back)(const zf_policy_args *, const float *, int32_t, void *, int64_t, int32_t, void *);
    int (*preference)(const zf_preference_args *, int32_t, void *);
    int (*preference_back)(const zf_preference_args *, const float *, void *, int64_t, int32_t, void *);
    const char *(*last_error)(void);
} L;

enum Kind { DISTILL, POLICY, PREFERENCE };
const char *const NAMES[] = {"distill_loss", "policy_loss", "preference_loss"};
struct Numbers {
    double temperature = 1.0, clip_low = 0.0, clip_high = 0.0, kl_weight = 0.0, entropy_weight = 0.0, beta = 0.0, label_smoothing = 0.0;
    bool rest = false, entropy = false, average = false;
};
// What a loss reads beside the logits; which of them are there depends on the loss.
struct Inputs {
    Tensor logits, mask, weight, ids, values, old_logprobs, advantages, ref, offsets;          // ids: the teacher's, or the tokens
};
struct Results { Tensor loss, losses, logprobs, entropy, chosen, rejected, stats, slopes; };

float *f32(const Tensor &t) { return t.defined() ? t.data_ptr<float>() : nullptr; }
int id_bytes(const Tensor &t) { return t.scalar_type() == at::kLong ? 8 : 4; }
zf_loss_rows rows_of(const Inputs &in, const Numbers &n, const Results &r) {
    zf_loss_rows a{};
    a.logits = in.logits.data_ptr(); a.dtype = logit_type(in.logits); a.V = (int32_t)in.logits.size(1); a.rows = in.logits.size(0); a.row_stride_elems = row_stride(in.logits);
    a.mask = in.mask.defined() ? (const uint32_t *)in.mask.data_ptr() : nullptr;
    a.weight = f32(in.weight); a.temperature = n.temperature; a.loss = f32(r.loss); a.losses = f32(r.losses);
    return a;
}
zf_distill_args distill_args(const Inputs &in, const Numbers &n, const Results &r) {
    zf_distill_args a{};
    a.r = rows_of(in, n, r);
    a.ids = in.ids.data_ptr(); a.values = in.values.data_ptr(); a.id_bytes = id_bytes(in.ids); a.values_dtype = logit_type(in.values); a.n_listed = (int32_t)in.ids.size(1); a.rest = n.rest;
    return a;
}
zf_policy_args policy_args(const Inputs &in, const Numbers &n, const Results &r) {
    zf_policy_args a{};
    a.r = rows_of(in, n, r);
    a.tokens = in.ids.data_ptr(); a.token_bytes = id_bytes(in.ids); a.old_logprobs = f32(in.old_logprobs); a.advantages = f32(in.advantages); a.ref_logprobs = f32(in.ref);
    a.clip_low = n.clip_low; a.clip_high = n.clip_high; a.kl_weight = n.kl_weight; a.entropy_weight = n.entropy_weight; a.logprobs = f32(r.logprobs); a.entropy = f32(r.entropy);
    return a;
}
zf_preference_args preference_args(const Inputs &in, const Numbers &n, const Results &r) {
    zf_preference_args a{};
    a.r = rows_of(in, n, r);
    a.tokens = in.ids.data_ptr(); a.token_bytes = id_bytes(in.ids); a.offsets = in.offsets.data_ptr(); a.offset_bytes = id_bytes(in.offsets); a.ref_logprobs = f32(in.ref);
    a.pairs = in.offsets.size(0) / 2; a.beta = n.beta; a.label_smoothing = n.label_smoothing; a.average = n.average;
    a.chosen = f32(r.chosen); a.rejected = f32(r.rejected); a.stats = f32(r.stats); a.slopes = f32(r.slopes);
    return a;
}
Results results_of(int kind, const Inputs &in, const Numbers &n) {
    auto of = [&](c10::IntArrayRef size) { return fresh(size, at::kFloat, in.logits); };
    const int64_t rows = in.logits.size(0), items = kind == PREFERENCE ? in.offsets.size(0) / 2 : rows;
    Results r;
    r.loss = of({}); r.losses = of({items});
    if (kind == POLICY) r.logprobs = of({rows});
    if (n.entropy) r.entropy = of({rows});
    if (kind == PREFERENCE) { r.chosen = of({items}); r.rejected = of({items}); r.stats = of({rows, 4}); r.slopes = of({2 * items}); }
    return r;
}
int call(int kind, const Inputs &in, const Numbers &n, const Results &r, void *grad) {
    const int32_t device = in.logits.get_device();
    void *const s = stream_of(in.logits);
    const int64_t V = in.logits.size(1);
    if (kind == DISTILL) { const auto a = distill_args(in, n, r); return L.distill(&a, grad, V, device, s); }
    if (kind == POLICY) { const auto a = policy_args(in, n, r); return L.policy(&a, grad, V, device, s); }
    const auto a = preference_args(in, n, r);
    return L.preference(&a, device, s);
}
int call_back(int kind, const Inputs &in, const Numbers &n, const Results &r, const float *g, bool held, void *grad) {
    const int32_t device = in.logits.get_device();
    void *const s = stream_of(in.logits);
    const int64_t V = in.logits.size(1);
    if (kind == DISTILL) { const auto a = distill_args(in, n, r); return L.distill_back(&a, g, held, grad, V, device, s); }
    if (kind == POLICY) { const auto a = policy_args(in, n, r); return L.policy_back(&a, g, held, grad, V, device, s); }
    const auto a = preference_args(in, n, r);
    return L.preference_back(&a, g, grad, V, device, s);
}
bool capturing(const Tensor &with) {
    hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
    return hipStreamIsCapturing((hipStream_t)stream_of(with), &status) != hipSuccess || status != hipStreamCaptureStatusNone;
}

// What a backward pass is given beside what was saved: shapes as they were.
struct Shapes : torch::CustomClassHolder {
    int kind;
    Numbers n;
    std::vector<int64_t> logits;
    int64_t listed, offsets;
    at::ScalarType dtype, id_type, value_type, offset_type;
    Tensor held;                       // the gradient for a factor of one; handed out once, to the pass that may find no other
};

struct LossOf : public torch::autograd::Function<LossOf> {
    // saved: logits, mask, weight, ids, values, old_logprobs, advantages, ref, offsets, then of a preference stats, slopes
    static torch::autograd::variable_list forward(torch::autograd::AutogradContext *ctx, const Tensor &logits, const Inputs &in, int64_t kind, const Numbers &n) {
        const Results r = results_of((int)kind, in, n);
        auto like = c10::make_intrusive<Shapes>();
        like->kind = (int)kind; like->n = n; like->logits = logits.sizes().vec(); like->dtype = logits.scalar_type(); like->id_type = in.ids.scalar_type();
        like->listed = kind == DISTILL ? in.ids.size(1) : 0;
        like->offsets = kind == PREFERENCE ? in.offsets.size(0) : 0;
        like->value_type = kind == DISTILL ? in.values.scalar_type() : at::kFloat;
        like->offset_type = kind == PREFERENCE ? in.offsets.scalar_type() : at::kLong;
        if (kind != PREFERENCE && !capturing(logits)) like->held = fresh(logits.sizes(), logits.scalar_type(), logits);
        must(call((int)kind, in, n, r, like->held.defined() ? like->held.data_ptr() : nullptr));
        ctx->save_for_backward({logits, in.mask, in.weight, in.ids, in.values, in.old_logprobs, in.advantages, in.ref, in.offsets, r.stats, r.slopes});
        ctx->saved_data["shapes"] = c10::IValue::make_capsule(std::move(like));
        ctx->set_materialize_grads(false);
        torch::autograd::variable_list out, constant;
        for (const Tensor *t : {&r.loss, &r.losses, &r.logprobs, &r.entropy, &r.chosen, &r.rejected}) if (t && t->defined()) out.push_back(*t);
        constant.assign(out.begin() + 1, out.end());
        ctx->mark_non_differentiable(constant);
        return out;
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext *ctx, torch::autograd::variable_list grads) {
        const auto saved = ctx->get_saved_variables();       // (raises where one of them was written since)
        if (!grads[0].defined()) return {Tensor(), Tensor(), Tensor(), Tensor()};
        const auto like = c10::static_intrusive_pointer_cast<Shapes>(ctx->saved_data["shapes"].toCapsule());
        const int kind = like->kind;
        const char *const name = NAMES[kind];
        const int64_t rows = like->logits[0], V = like->logits[1], items = kind == PREFERENCE ? like->offsets / 2 : rows;
        Inputs in;
        in.logits = kept(name, saved[0], "logits", saved[0], like->dtype, like->logits, true);
        auto some = [&](int i, const char *what, at::ScalarType type, c10::IntArrayRef size) { return saved[i].defined() ? kept(name, saved[i], what, in.logits, type, size) : Tensor(); };
        const int64_t of_ids[] = {rows, like->listed};
        const c10::IntArrayRef ids(of_ids, kind == DISTILL ? 2 : 1);
        in.mask = some(1, "mask", at::kInt, {rows, (V + 31) / 32});
        in.weight = some(2, "weight", at::kFloat, {items});
        in.ids = some(3, "ids", like->id_type, ids);
        in.values = some(4, "values", like->value_type, ids);
        in.old_logprobs = some(5, "old_logprobs", at::kFloat, {rows});
        in.advantages = some(6, "advantages", at::kFloat, {rows});
        in.ref = some(7, "ref_logprobs", at::kFloat, {rows});
        in.offsets = some(8, "offsets", like->offset_type, {like->offsets});
        const Tensor g = kept(name, grads[0].scalar_type() == at::kFloat ? grads[0] : grads[0].detach().to(at::kFloat), "gradient", in.logits, at::kFloat, {});
        Results r;                                           // none is written: the addresses only say that they are there
        r.loss = r.losses = r.logprobs = r.chosen = r.rejected = g;
        if (like->n.entropy) r.entropy = g;
        if (kind == PREFERENCE) { r.stats = some(9, "stats", at::kFloat, {rows, 4}); r.slopes = some(10, "slopes", at::kFloat, {2 * items}); }
        // The gradient for a factor of one is handed out once: whoever has it may write it.  What a capture records may run again under another factor.
        Tensor grad;
        bool held = false;
        if (!capturing(in.logits)) { grad = std::move(like->held); like->held.reset(); held = grad.defined(); }
        if (!held) grad = fresh(like->logits, like->dtype, in.logits);
        const int rc = call_back(kind, in, like->n, r, g.data_ptr<float>(), held, grad.data_ptr());
        TORCH_CHECK(rc == ZF_OK, "zapformat error ", rc, ": ", L.last_error());
        if (at::GradMode::is_enabled())            // a graph of the gradient is made: it ends here, with an error for whoever follows it
            grad = torch::autograd::DelayedError(std::string(name) + ": its gradient cannot be differentiated again", 1)({grad.requires_grad_()})[0];
        return {grad, Tensor(), Tensor(), Tensor()};
    }
};

// ---- arguments ----
bool number(PyObject *o, double *out) { if (!PyFloat_CheckExact(o)) return false; *out = PyFloat_AS_DOUBLE(o); return true; }
bool truth(PyObject *o, bool *out) { if (!PyBool_Check(o)) return false; *out = o == Py_True; return true; }
bool tensor(PyObject *o, Tensor *out, bool needed) {
    std::optional<Tensor> t;
    if (!tensor_or_none(o, &t) || (needed && !t)) return false;
    if (t) *out = std::move(*t);
    return true;
}
bool logits_fit(const Inputs &in) {
    const Tensor &x = in.logits;
    return matrix(x) && logit_type(x) >= 0 && x.size(0) >= 1 && x.size(1) >= 1 && x.size(1) <= INT32_MAX && rows_without_gaps(x) &&
           (!in.mask.defined() || mask_fits(in.mask, x.size(0), x.size(1), x));
}
bool constant_fits(const Tensor &t, const Tensor &with, c10::IntArrayRef size) {
    return plain(t) && t.device() == with.device() && t.sizes() == size && t.is_contiguous() && !(at::GradMode::is_enabled() && t.requires_grad());
}
bool floats_fit(const Tensor &t, const Tensor &with, int64_t n) { return !t.defined() || (t.scalar_type() == at::kFloat && constant_fits(t, with, {n})); }
bool is_id(const Tensor &t) { return t.scalar_type() == at::kLong || t.scalar_type() == at::kInt; }

// The results in order, None for those that are not there; `loss` first.
PyObject *run(Kind kind, const Inputs &in, const Numbers &n, int n_out) {
    torch::autograd::variable_list out;
    if (at::GradMode::is_enabled() && in.logits.requires_grad()) out = LossOf::apply(in.logits, in, (int64_t)kind, n);
    else {
        const Results r = results_of(kind, in, n);
        must(call(kind, in, n, r, nullptr));
        for (const Tensor *t : {&r.loss, &r.losses, &r.logprobs, &r.entropy, &r.chosen, &r.rejected}) if (t && t->defined()) out.push_back(*t);
    }
    PyObject *t = PyTuple_New(n_out);
    if (!t) return nullptr;
    for (int i = 0; i < n_out; i++) {
        PyObject *o = i < (int)out.size() ? THPVariable_Wrap(out[i]) : Py_NewRef(Py_None);
        if (!o) { Py_DECREF(t); return nullptr; }
        PyTuple_SET_ITEM(t, i, o);
    }
    return t;
}

PyObject *distill_loss(PyObject *const *args, Py_ssize_t n) {          // (logits, ids, values, mask, temperature, rest, weight)
    Inputs in;
    Numbers o;
    if (n != 7 || !tensor(args[0], &in.logits, true) || !tensor(args[1], &in.ids, true) || !tensor(args[2], &in.values, true) || !tensor(args[3], &in.mask, false) || !number(args[4], &o.temperature) ||
        !truth(args[5], &o.rest) || !tensor(args[6], &in.weight, false) || !logits_fit(in)) return nullptr;
    const int64_t rows = in.logits.size(0);
    if (in.ids.dim() != 2 || in.ids.size(1) < 1 || in.ids.size(1) > 1024 || !is_id(in.ids) || logit_type(in.values) < 0) return nullptr;
    const int64_t shape[] = {rows, in.ids.size(1)};
    if (!constant_fits(in.ids, in.logits, shape) || !constant_fits(in.values, in.logits, shape) || !floats_fit(in.weight, in.logits, rows)) return nullptr;
    return run(DISTILL, in, o, 2);
}

PyObject *policy_loss(PyObject *const *args, Py_ssize_t n) {           // (logits, tokens, old_logprobs, advantages, mask, ref_logprobs, temperature, clip_low, clip_high, kl_weight, entropy or not, entropy_weight, weight)
    Inputs in;
    Numbers o;
    if (n != 13 || !tensor(args[0], &in.logits, true) || !tensor(args[1], &in.ids, true) || !tensor(args[2], &in.old_logprobs, true) || !tensor(args[3], &in.advantages, true) || !tensor(args[4], &in.mask, false) ||
        !tensor(args[5], &in.ref, false) || !number(args[6], &o.temperature) || !number(args[7], &o.clip_low) || !number(args[8], &o.clip_high) || !number(args[9], &o.kl_weight) || !truth(args[10], &o.entropy) ||
        !number(args[11], &o.entropy_weight) || !tensor(args[12], &in.weight, false) || !logits_fit(in)) return nullptr;
    const int64_t rows = in.logits.size(0);
    if (!is_id(in.ids) || !constant_fits(in.ids, in.logits, {rows}) || !floats_fit(in.old_logprobs, in.logits, rows) || !floats_fit(in.advantages, in.logits, rows) || !floats_fit(in.ref, in.logits, rows) ||
        !floats_fit(in.weight, in.logits, rows) || (!in.ref.defined() && o.kl_weight != 0.0)) return nullptr;
    return run(POLICY, in, o, 4);
}

PyObject *preference_loss(PyObject *const *args, Py_ssize_t n) {       // (logits, tokens, offsets, ref_logprobs, mask, beta, label_smoothing, average, temperature, weight)
    Inputs in;
    Numbers o;
    if (n != 10 || !tensor(args[0], &in.logits, true) || !tensor(args[1], &in.ids, true) || !tensor(args[2], &in.offsets, true) || !tensor(args[3], &in.ref, false) || !tensor(args[4], &in.mask, false) ||
        !number(args[5], &o.beta) || !number(args[6], &o.label_smoothing) || !truth(args[7], &o.average) || !number(args[8], &o.temperature) || !tensor(args[9], &in.weight, false) || !logits_fit(in)) return nullptr;
    const int64_t rows = in.logits.size(0);
    if (!is_id(in.ids) || !is_id(in.offsets) || in.offsets.dim() != 1 || in.offsets.size(0) % 2 == 0 || in.offsets.size(0) < 3 || !constant_fits(in.ids, in.logits, {rows}) ||
        !constant_fits(in.offsets, in.logits, in.offsets.sizes()) || !floats_fit(in.ref, in.logits, rows) || !floats_fit(in.weight, in.logits, in.offsets.size(0) / 2)) return nullptr;
    return run(PREFERENCE, in, o, 4);
}

PyObject *bind(PyObject *, PyObject *args) {                    // ({name: address}, _check)
    PyObject *addr, *chk;
    if (!PyArg_ParseTuple(args, "O!O", &PyDict_Type, &addr, &chk)) return nullptr;
    auto take = [&](const char *name, void **to) {
        PyObject *v = PyDict_GetItemString(addr, name);
        *to = v ? PyLong_AsVoidPtr(v) : nullptr;
        if (!*to && !PyErr_Occurred()) PyErr_Format(PyExc_RuntimeError, "no address of %s", name);
        return *to != nullptr;
    };
    if (!take("zf_distill_loss", (void **)&L.distill) || !take("zf_distill_loss_backward", (void **)&L.distill_back) || !take("zf_policy_loss", (void **)&L.policy) ||
        !take("zf_policy_loss_backward", (void **)&L.policy_back) || !take("zf_preference_loss", (void **)&L.preference) || !take("zf_preference_loss_backward", (void **)&L.preference_back) ||
        !take("zf_last_error", (void **)&L.last_error)) return nullptr;
    Py_INCREF(chk); Py_XSETREF(check_py, chk);
    Py_RETURN_NONE;
}

#define FAST(f) (PyCFunction)(void (*)(void))guarded<f>, METH_FASTCALL
PyMethodDef methods[] = {
    {"distill_loss", FAST(distill_loss), nullptr}, {"policy_loss", FAST(policy_loss), nullptr}, {"preference_loss", FAST(preference_loss), nullptr},
    {"bind", bind, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_native_losses", "The losses on logits, from Python to the library.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native_losses(void) { return PyModule_Create(&module_def); }
