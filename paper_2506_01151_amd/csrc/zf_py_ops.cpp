// Extension module _native_ops: the calls at the two ends of a step's logits (operators.py), from Python to the library, with outputs and
// workspace from torch's allocator.  In Python a call cost 13 us of checks and marshalling, and one with a gradient 70.
#define PY_SSIZE_T_CLEAN
#include "zf_py_tensors.h"

namespace {

struct {                               // the library's calls (addresses given by binding.py)
    int (*quantize_blocks)(const void *, int32_t, int64_t, int32_t, int64_t, int32_t, uint8_t *, float *, int32_t, void *);
    int (*head_logits)(const uint8_t *, int64_t, const float *, const uint8_t *, int64_t, const float *, int32_t, int32_t, int32_t, const uint32_t *, void *, int32_t, int64_t, int32_t, void *);
    int64_t (*workspace)(const zf_logprobs_args *);
    int (*token_logprobs)(const zf_logprobs_args *, void *, int64_t, int32_t, void *);
    int (*backward)(const zf_logprobs_args *, const float *, const float *, const float *, void *, int64_t, int32_t, void *);
    const char *(*last_error)(void);
} L;

const int64_t BLOCK = 128;

// ---- the calls ----
PyObject *quantize_blocks(PyObject *const *args, Py_ssize_t n) {       // (x, block_rows)
    std::optional<Tensor> x;
    if (n != 2 || !tensor_or_none(args[0], &x) || !x || !PyLong_CheckExact(args[1])) return nullptr;
    const long tall = PyLong_AsLong(args[1]);
    if ((tall != 1 && tall != BLOCK) || !matrix(*x) || logit_type(*x) < 0 || !rows_without_gaps(*x) || x->size(1) < 1 || x->size(0) < 1) { PyErr_Clear(); return nullptr; }
    const int64_t rows = x->size(0), cols = x->size(1), blocks = (cols + BLOCK - 1) / BLOCK;
    const Tensor q = fresh({rows, blocks * BLOCK}, at::kFloat8_e4m3fn, *x), scale = fresh({(rows + tall - 1) / tall, blocks}, at::kFloat, *x);
    if (cols > INT32_MAX) return nullptr;
    must(L.quantize_blocks(x->data_ptr(), logit_type(*x), rows, (int32_t)cols, row_stride(*x), (int32_t)tall, (uint8_t *)q.data_ptr(), scale.data_ptr<float>(), x->get_device(), stream_of(*x)));
    return Py_BuildValue("(NN)", THPVariable_Wrap(q), THPVariable_Wrap(scale));
}

PyObject *head_logits(PyObject *const *args, Py_ssize_t n) {           // (q, q_scale, weight, weight_scale, mask, type of the result)
    std::optional<Tensor> q, qs, w, ws, mask;
    if (n != 6 || !tensor_or_none(args[0], &q) || !tensor_or_none(args[1], &qs) || !tensor_or_none(args[2], &w) || !tensor_or_none(args[3], &ws) ||
        !tensor_or_none(args[4], &mask) || !q || !qs || !w || !ws || !PyLong_CheckExact(args[5])) return nullptr;
    const long type = PyLong_AsLong(args[5]);
    if (!matrix(*q) || !matrix(*w) || !matrix(*qs) || !matrix(*ws) || q->scalar_type() != at::kFloat8_e4m3fn || w->scalar_type() != at::kFloat8_e4m3fn || qs->scalar_type() != at::kFloat ||
        ws->scalar_type() != at::kFloat || (type != 0 && type != 1)) { PyErr_Clear(); return nullptr; }
    const int64_t batch = q->size(0), K = q->size(1), V = w->size(0), k = K / BLOCK;
    if (batch < 1 || V < 1 || V > INT32_MAX || K < BLOCK || K % BLOCK || K > INT32_MAX || batch > INT32_MAX || w->size(1) != K || !rows_without_gaps(*q) || !rows_without_gaps(*w) || !qs->is_contiguous() || !ws->is_contiguous() ||
        qs->size(0) != batch || qs->size(1) != k || ws->size(0) != (V + BLOCK - 1) / BLOCK || ws->size(1) != k || w->device() != q->device() || qs->device() != q->device() ||
        ws->device() != q->device() || !mask_fits(mask, batch, V, *q) ||
        (at::GradMode::is_enabled() && (q->requires_grad() || qs->requires_grad() || w->requires_grad() || ws->requires_grad()))) return nullptr;
    const Tensor out = fresh({batch, V}, type == 0 ? at::kFloat : at::kBFloat16, *q);
    must(L.head_logits((const uint8_t *)q->data_ptr(), row_stride(*q), qs->data_ptr<float>(), (const uint8_t *)w->data_ptr(), row_stride(*w), ws->data_ptr<float>(), (int32_t)batch, (int32_t)V, (int32_t)K,
                       mask ? (const uint32_t *)mask->data_ptr() : nullptr, out.data_ptr(), (int32_t)type, V, q->get_device(), stream_of(*q)));
    return THPVariable_Wrap(out);
}

zf_logprobs_args args_of(const Tensor &logits, const std::optional<Tensor> &tokens, const std::optional<Tensor> &mask, double temperature, int64_t top) {
    zf_logprobs_args a{};
    a.logits = logits.data_ptr(); a.dtype = logit_type(logits); a.V = (int32_t)logits.size(1); a.rows = logits.size(0); a.row_stride_elems = row_stride(logits);
    a.mask = mask ? (const uint32_t *)mask->data_ptr() : nullptr;
    if (tokens) { a.tokens = tokens->data_ptr(); a.token_bytes = tokens->scalar_type() == at::kLong ? 8 : 4; a.n_tokens = tokens->dim() == 2 ? (int32_t)tokens->size(1) : 1; }
    a.temperature = (float)temperature; a.top = (int32_t)top;
    return a;
}
struct Results { std::optional<Tensor> logprobs, entropy, ids, top, stats; };
void point(zf_logprobs_args *a, const Results &r) {
    a->logprobs = r.logprobs ? r.logprobs->data_ptr<float>() : nullptr;
    a->entropy = r.entropy ? r.entropy->data_ptr<float>() : nullptr;
    a->top_ids = r.ids ? r.ids->data_ptr<int32_t>() : nullptr;
    a->top_logprobs = r.top ? r.top->data_ptr<float>() : nullptr;
    a->stats = r.stats ? r.stats->data_ptr<float>() : nullptr;
}
Results forward(const Tensor &logits, const std::optional<Tensor> &tokens, const std::optional<Tensor> &mask, double temperature, bool entropy, int64_t top, bool stats) {
    zf_logprobs_args a = args_of(logits, tokens, mask, temperature, top);
    Results r;
    const int64_t rows = logits.size(0);
    if (tokens) r.logprobs = fresh(tokens->sizes(), at::kFloat, logits);
    if (entropy) r.entropy = fresh({rows}, at::kFloat, logits);
    if (top) { r.ids = fresh({rows, top}, at::kInt, logits); r.top = fresh({rows, top}, at::kFloat, logits); }
    if (stats) r.stats = fresh({rows, 2}, at::kFloat, logits);
    point(&a, r);
    const int64_t size = L.workspace(&a);
    if (size < 0) throw Failed{(int)size};
    const Tensor work = size ? fresh({size}, at::kByte, logits) : Tensor();
    must(L.token_logprobs(&a, size ? work.data_ptr() : nullptr, size, logits.get_device(), stream_of(logits)));
    return r;
}

struct TokenLogprobs : public torch::autograd::Function<TokenLogprobs> {
    static torch::autograd::variable_list forward(torch::autograd::AutogradContext *ctx, const Tensor &logits, const std::optional<Tensor> &tokens, const std::optional<Tensor> &mask,
                                                  double temperature, bool entropy, int64_t top) {
        const Results r = ::forward(logits, tokens, mask, temperature, entropy, top, true);
        auto of = [](const std::optional<Tensor> &t) { return t ? *t : Tensor(); };
        ctx->save_for_backward({logits, of(tokens), of(mask), of(r.logprobs), of(r.entropy), of(r.ids), of(r.top), of(r.stats)});
        ctx->saved_data["temperature"] = temperature;
        ctx->set_materialize_grads(false);
        torch::autograd::variable_list out;
        for (const auto *t : {&r.logprobs, &r.entropy, &r.ids, &r.top}) if (*t) out.push_back(**t);
        if (r.ids) ctx->mark_non_differentiable({*r.ids});
        return out;
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext *ctx, torch::autograd::variable_list grads) {
        const auto saved = ctx->get_saved_variables();
        const Tensor logits = kept("token_logprobs", saved[0], "logits", saved[0], saved[0].scalar_type(), saved[0].sizes(), true);
        TORCH_CHECK(logits.dim() == 2 && logit_type(logits) >= 0, "token_logprobs: saved logits came back as others");
        const int64_t rows = logits.size(0), V = logits.size(1);
        auto some = [&](int i, const char *what, at::ScalarType type, c10::IntArrayRef size) { return saved[i].defined() ? std::optional<Tensor>(kept("token_logprobs", saved[i], what, logits, type, size)) : std::nullopt; };
        auto width = [&](int i) { return saved[i].defined() && saved[i].dim() == 2 ? saved[i].size(1) : 0; };
        const int64_t of_rows[] = {rows, width(3)}, of_top[] = {rows, width(5)};
        const c10::IntArrayRef given(of_rows, saved[3].defined() && saved[3].dim() == 2 ? 2 : 1);
        const std::optional<Tensor> tokens = some(1, "tokens", saved[1].defined() && saved[1].scalar_type() == at::kInt ? at::kInt : at::kLong, given), mask = some(2, "mask", at::kInt, {rows, (V + 31) / 32});
        const Results r{some(3, "logprobs", at::kFloat, given), some(4, "entropy", at::kFloat, {rows}), some(5, "top_ids", at::kInt, of_top), some(6, "top_logprobs", at::kFloat, of_top), some(7, "stats", at::kFloat, {rows, 2})};
        const double temperature = ctx->saved_data["temperature"].toDouble();
        size_t at = 0;
        auto next = [&](const std::optional<Tensor> &of) {
            const Tensor g = of ? grads[at++] : Tensor();
            return g.defined() ? kept("token_logprobs", g.scalar_type() == at::kFloat ? g : g.detach().to(at::kFloat), "gradient", logits, at::kFloat, of->sizes()) : g;
        };
        const Tensor g_lp = next(r.logprobs), g_H = next(r.entropy);
        (void)next(r.ids);
        const Tensor g_top = next(r.top);
        zf_logprobs_args a = args_of(logits, tokens, mask, temperature, r.ids ? r.ids->size(1) : 0);
        point(&a, r);
        auto ptr = [](const Tensor &t) { return t.defined() ? t.data_ptr<float>() : nullptr; };
        Tensor grad = fresh(logits.sizes(), logits.scalar_type(), logits);
        const int rc = L.backward(&a, ptr(g_lp), ptr(g_H), ptr(g_top), grad.data_ptr(), logits.size(1), logits.get_device(), stream_of(logits));
        TORCH_CHECK(rc == ZF_OK, "zapformat error ", rc, ": ", L.last_error());
        if (at::GradMode::is_enabled())            // a graph of the gradient is made: it ends here, with an error for whoever follows it
            grad = torch::autograd::DelayedError("token_logprobs: its gradient cannot be differentiated again", 1)({grad.requires_grad_()})[0];
        return {grad, Tensor(), Tensor(), Tensor(), Tensor(), Tensor()};
    }
};

PyObject *token_logprobs(PyObject *const *args, Py_ssize_t n) {        // (logits, tokens, mask, temperature, entropy, top) -> (logprobs, entropy, top_ids, top_logprobs)
    std::optional<Tensor> logits, tokens, mask;
    if (n != 6 || !tensor_or_none(args[0], &logits) || !tensor_or_none(args[1], &tokens) || !tensor_or_none(args[2], &mask) || !logits || !PyFloat_CheckExact(args[3]) || !PyBool_Check(args[4]) || !PyLong_CheckExact(args[5])) return nullptr;
    const double temperature = PyFloat_AS_DOUBLE(args[3]);
    const bool entropy = args[4] == Py_True;
    const long top = PyLong_AsLong(args[5]);
    if (!matrix(*logits) || logit_type(*logits) < 0 || logits->size(0) < 1 || logits->size(1) < 1 || logits->size(1) > INT32_MAX || !rows_without_gaps(*logits) || top < 0 || top > 64 ||
        !mask_fits(mask, logits->size(0), logits->size(1), *logits)) { PyErr_Clear(); return nullptr; }
    if (tokens && (!plain(*tokens) || (tokens->scalar_type() != at::kLong && tokens->scalar_type() != at::kInt) || tokens->dim() < 1 || tokens->dim() > 2 || tokens->size(0) != logits->size(0) ||
                   !tokens->is_contiguous() || tokens->device() != logits->device() || (tokens->dim() == 2 && tokens->size(1) > INT32_MAX))) return nullptr;
    std::optional<Tensor> out[4];
    if (at::GradMode::is_enabled() && logits->requires_grad()) {
        const auto r = TokenLogprobs::apply(*logits, tokens, mask, temperature, entropy, (int64_t)top);
        size_t at = 0;
        if (tokens) out[0] = r[at++];
        if (entropy) out[1] = r[at++];
        if (top) { out[2] = r[at++]; out[3] = r[at++]; }
    } else {
        Results r = forward(*logits, tokens, mask, temperature, entropy, top, false);
        out[0] = r.logprobs; out[1] = r.entropy; out[2] = r.ids; out[3] = r.top;
    }
    PyObject *t = PyTuple_New(4);
    if (!t) return nullptr;
    for (int i = 0; i < 4; i++) {
        PyObject *o = out[i] ? THPVariable_Wrap(*out[i]) : Py_NewRef(Py_None);
        if (!o) { Py_DECREF(t); return nullptr; }
        PyTuple_SET_ITEM(t, i, o);
    }
    return t;
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
    if (!take("zf_quantize_blocks", (void **)&L.quantize_blocks) || !take("zf_head_logits", (void **)&L.head_logits) || !take("zf_token_logprobs_workspace", (void **)&L.workspace) ||
        !take("zf_token_logprobs", (void **)&L.token_logprobs) || !take("zf_token_logprobs_backward", (void **)&L.backward) || !take("zf_last_error", (void **)&L.last_error)) return nullptr;
    Py_INCREF(chk); Py_XSETREF(check_py, chk);
    Py_RETURN_NONE;
}

#define FAST(f) (PyCFunction)(void (*)(void))guarded<f>, METH_FASTCALL
PyMethodDef methods[] = {
    {"quantize_blocks", FAST(quantize_blocks), nullptr}, {"head_logits", FAST(head_logits), nullptr}, {"token_logprobs", FAST(token_logprobs), nullptr},
    {"bind", bind, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_native_ops", "The calls at the two ends of a step's logits, from Python to the library.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native_ops(void) { return PyModule_Create(&module_def); }
