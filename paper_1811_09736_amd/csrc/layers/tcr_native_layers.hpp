// binding.py's calls of linear attention and of the root-mean-square norm in their ordinary form (part of tcr_native.cpp, whose rules hold here: a
// function returns None, before it has done anything, where binding.py has to look itself).  us a call, through Python / native, at sizes whose
// kernels take less: a step of attention 16 / 5.1, a norm in 8 bits 15 / 6.8.
#pragma once

decltype(&tcr_linear_attention) g_linear_attention;
decltype(&tcr_linear_attention_step) g_linear_attention_step;
decltype(&tcr_linear_attention_backward) g_linear_attention_backward;
decltype(&tcr_rms_norm) g_rms_norm;
decltype(&tcr_rms_norm_quantized) g_rms_norm_quantized;
decltype(&tcr_rms_norm_backward) g_rms_norm_backward;

// A tensor in this process's GPU memory and nothing more special than that; its elements of the last dimension consecutive.
const at::Tensor* rows(PyObject* o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    constexpr c10::DispatchKeySet usual({c10::DispatchKey::CUDA, c10::DispatchKey::ADInplaceOrView, c10::DispatchKey::AutogradCUDA, c10::DispatchKey::AutocastCUDA});
    const c10::DispatchKeySet keys = t.key_set();
    if (!keys.has(c10::DispatchKey::CUDA) || (keys.raw_repr() & ~usual.raw_repr()) != 0 || t.dim() < 1 || t.stride(-1) != 1) return nullptr;
    return &t;
}
// The first of a call's: on the current device; no mode wants to see what is called.
const at::Tensor* leading(PyObject* o) {
    const at::Tensor* x = rows(o);
    if (x == nullptr || at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set()) return nullptr;
    c10::DeviceIndex device = -1;
    if (c10::hip::GetDevice(&device) != hipSuccess || device != x->device().index()) return nullptr;
    return x;
}
// One like x: of its type, dimensions and device.
const at::Tensor* beside(PyObject* o, const at::Tensor& x) {
    const at::Tensor* t = rows(o);
    return t != nullptr && t->scalar_type() == x.scalar_type() && t->dim() == x.dim() && t->device() == x.device() ? t : nullptr;
}
// A contiguous one of these sizes.
const at::Tensor* whole(PyObject* o, at::ScalarType type, at::IntArrayRef sizes, const at::Tensor& x) {
    const at::Tensor* t = plain(o, type);
    return t != nullptr && t->sizes() == sizes && t->device() == x.device() ? t : nullptr;
}
bool real(PyObject* o, double& v) {
    if (!PyFloat_CheckExact(o)) return false;
    v = PyFloat_AS_DOUBLE(o);
    return true;
}
uint32_t type_of(at::ScalarType t) { return t == at::kHalf ? TCR_F16 : t == at::kBFloat16 ? TCR_BF16 : TCR_F32; }
PyObject* wrapped(const at::Tensor& t) { return THPVariable_Wrap(t); }
c10::TensorOptions options_of(const at::Tensor& x, at::ScalarType t) { return x.options().dtype(t).requires_grad(false); }
void* data_of(const at::Tensor* t) { return t != nullptr ? t->data_ptr() : nullptr; }
// A tensor of the caller's that a call has written through its pointer: autograd is to notice where it has kept it.
void written(const at::Tensor* t) {
    if (t != nullptr && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}

// ------------------------------------------------------------------------------------------------ attention
struct Attention {
    tcr_attention shape = {};
    const at::Tensor *q = nullptr, *k = nullptr, *v = nullptr;
    int64_t states[4] = {};

    // q, k, v, log_decay, scale, offsets; `step`: one token a sequence, [sequence, head, element]
    bool set(PyObject* const* args, bool step) {
        q = leading(args[0]);
        if (q == nullptr || (q->scalar_type() != at::kHalf && q->scalar_type() != at::kBFloat16)) return false;
        k = beside(args[1], *q);
        v = k != nullptr ? beside(args[2], *q) : nullptr;
        if (v == nullptr) return false;
        const bool packed = args[5] != Py_None;
        const int64_t dims = packed || step ? 3 : 4;
        if (q->dim() != dims) return false;
        const int64_t heads = q->size(-2), kv = k->size(-2), dk = q->size(-1), dv = v->size(-1);
        for (int64_t d = 0; d + 2 < dims; ++d)
            if (k->size(d) != q->size(d) || v->size(d) != q->size(d)) return false;
        if (kv < 1 || heads < 1 || heads % kv != 0 || v->size(-2) != kv || k->size(-1) != dk || heads > 65535 || dk > 65535 || dv > 65535) return false;
        const at::Tensor* decay = whole(args[3], at::kFloat, {heads}, *q);
        if (decay == nullptr) return false;
        double scale = 1.0 / std::sqrt((double)dk);
        if (args[4] != Py_None && !real(args[4], scale)) return false;
        shape.sequences = (uint64_t)q->size(0);
        shape.tokens = step ? 1 : (uint64_t)(packed ? q->size(0) : q->size(1));
        if (packed) {
            const at::Tensor* offsets = entries(args[5], *q);
            if (offsets == nullptr) return false;
            shape.offsets = static_cast<const uint64_t*>(offsets->data_ptr());
            shape.sequences = (uint64_t)offsets->numel() - 1;
        }
        shape.dtype = type_of(q->scalar_type());
        shape.heads = (uint32_t)heads;
        shape.kv_heads = (uint32_t)kv;
        shape.dk = (uint32_t)dk;
        shape.dv = (uint32_t)dv;
        shape.log_decay = static_cast<const float*>(decay->data_ptr());
        shape.scale = (float)scale;
        strides(*q, shape.q_stride, step);
        strides(*k, shape.k_stride, step);
        strides(*v, shape.v_stride, step);
        states[0] = (int64_t)shape.sequences;
        states[1] = heads;
        states[2] = dk;
        states[3] = dv;
        return true;
    }
    static void strides(const at::Tensor& t, int64_t (&to)[3], bool step) {
        const int64_t d = t.dim();
        to[0] = d == 4 ? t.stride(0) : step ? t.stride(0) : 0;
        to[1] = d == 4 ? t.stride(1) : step ? 0 : t.stride(0);
        to[2] = t.stride(d - 2);
    }
    // out (or its gradient): given, or to be made
    bool output(PyObject* o, const at::Tensor** given, bool step) {
        *given = nullptr;
        if (o == Py_None) return true;
        const at::Tensor* t = beside(o, *q);
        if (t == nullptr || t->size(-1) != (int64_t)shape.dv) return false;
        for (int64_t d = 0; d + 1 < q->dim(); ++d)
            if (t->size(d) != q->size(d)) return false;
        strides(*t, shape.o_stride, step);
        *given = t;
        return true;
    }
    at::Tensor make_output(bool step) {
        c10::SmallVector<int64_t, 4> sizes(q->sizes().begin(), q->sizes().end());
        sizes.back() = (int64_t)shape.dv;
        at::Tensor made = at::empty(sizes, options_of(*q, q->scalar_type()));
        strides(made, shape.o_stride, step);
        return made;
    }
    // states: given or not
    bool state(PyObject* o, const at::Tensor** t) const {
        *t = nullptr;
        if (o == Py_None) return true;
        *t = whole(o, at::kFloat, at::IntArrayRef(states, 4), *q);
        return *t != nullptr;
    }
};

// linear_attention(q, k, v, log_decay, scale, offsets, state, final_state, out)
PyObject* linear_attention(PyObject*, PyObject* const* args, Py_ssize_t count) {
    HANDLE_TH_ERRORS
    Attention a;
    const at::Tensor *state, *given;
    if (count != 9 || !a.set(args, false) || !a.state(args[6], &state) || !a.output(args[8], &given, false)) Py_RETURN_NONE;
    if (args[7] != Py_True && args[7] != Py_False) Py_RETURN_NONE;
    at::Tensor out, last;
    void* const stream = stream_of(*a.q);
    TCR_CALL((out = given != nullptr ? *given : a.make_output(false),
              last = args[7] == Py_True ? at::empty(at::IntArrayRef(a.states, 4), options_of(*a.q, at::kFloat)) : at::Tensor()),
             g_linear_attention(&a.shape, a.q->data_ptr(), a.k->data_ptr(), a.v->data_ptr(), out.data_ptr(), static_cast<const float*>(data_of(state)),
                                last.defined() ? static_cast<float*>(last.data_ptr()) : nullptr, stream))
    if (st != TCR_OK) return failed(st, "tcr_linear_attention");
    written(given);
    return last.defined() ? Py_BuildValue("NN", wrapped(out), wrapped(last)) : wrapped(out);
    END_HANDLE_TH_ERRORS
}

// linear_attention_step(q, k, v, log_decay, scale, None, state, new_state, out)
PyObject* linear_attention_step(PyObject*, PyObject* const* args, Py_ssize_t count) {
    HANDLE_TH_ERRORS
    Attention a;
    const at::Tensor *state, *next, *given;
    if (count != 9 || args[5] != Py_None || !a.set(args, true) || !a.state(args[6], &state) || state == nullptr || !a.state(args[7], &next) ||
        !a.output(args[8], &given, true))
        Py_RETURN_NONE;
    at::Tensor out;
    float* const to = static_cast<float*>(data_of(next != nullptr ? next : state));
    void* const stream = stream_of(*a.q);
    TCR_CALL((out = given != nullptr ? *given : a.make_output(true)),
             g_linear_attention_step(&a.shape, a.q->data_ptr(), a.k->data_ptr(), a.v->data_ptr(), out.data_ptr(),
                                     static_cast<const float*>(state->data_ptr()), to, stream))
    if (st != TCR_OK) return failed(st, "tcr_linear_attention_step");
    written(next != nullptr ? next : state);
    written(given);
    return wrapped(out);
    END_HANDLE_TH_ERRORS
}

// linear_attention_backward(q, k, v, log_decay, scale, offsets, state, dfinal, dout)
PyObject* linear_attention_backward(PyObject*, PyObject* const* args, Py_ssize_t count) {
    HANDLE_TH_ERRORS
    Attention a;
    const at::Tensor *state, *dfinal, *dout;
    if (count != 9 || !a.set(args, false) || !a.state(args[6], &state) || !a.state(args[7], &dfinal) || !a.output(args[8], &dout, false) || dout == nullptr)
        Py_RETURN_NONE;
    at::Tensor dq, dk, dv, dstate;
    void* const stream = stream_of(*a.q);
    const auto like = options_of(*a.q, a.q->scalar_type());
    TCR_CALL((dq = at::empty(a.q->sizes(), like), dk = at::empty(a.k->sizes(), like), dv = at::empty(a.v->sizes(), like),
              dstate = state != nullptr ? at::empty(state->sizes(), options_of(*a.q, at::kFloat)) : at::Tensor()),
             g_linear_attention_backward(&a.shape, dout->data_ptr(), a.q->data_ptr(), a.k->data_ptr(), a.v->data_ptr(), dq.data_ptr(), dk.data_ptr(),
                                         dv.data_ptr(), static_cast<const float*>(data_of(state)), static_cast<const float*>(data_of(dfinal)),
                                         dstate.defined() ? static_cast<float*>(dstate.data_ptr()) : nullptr, stream))
    if (st != TCR_OK) return failed(st, "tcr_linear_attention_backward");
    PyObject* ds = Py_None;
    if (dstate.defined()) ds = wrapped(dstate);
    else Py_INCREF(ds);
    return Py_BuildValue("NNNN", wrapped(dq), wrapped(dk), wrapped(dv), ds);
    END_HANDLE_TH_ERRORS
}

// ------------------------------------------------------------------------------------------------ norm
struct NormRows {
    const at::Tensor *x = nullptr, *weight = nullptr, *residual = nullptr;
    uint64_t rows_ = 0, cols = 0;
    uint32_t dtype = 0, weight_dtype = 0;
    // contiguous rows; binding.py sees to others
    bool set(PyObject* first, PyObject* w, PyObject* second) {
        x = leading(first);
        if (x == nullptr || !x->is_contiguous() || x->size(-1) < 1) return false;
        const at::ScalarType t = x->scalar_type();
        if (t != at::kHalf && t != at::kBFloat16 && t != at::kFloat) return false;
        cols = (uint64_t)x->size(-1);
        rows_ = (uint64_t)x->numel() / cols;
        weight = whole(w, t, {(int64_t)cols}, *x);
        if (weight == nullptr && t != at::kFloat) weight = whole(w, at::kFloat, {(int64_t)cols}, *x);
        if (weight == nullptr) return false;
        dtype = type_of(t);
        weight_dtype = type_of(weight->scalar_type());
        return like(second, &residual);
    }
    bool like(PyObject* o, const at::Tensor** t) const {
        *t = nullptr;
        if (o == Py_None) return true;
        *t = whole(o, x->scalar_type(), x->sizes(), *x);
        return *t != nullptr;
    }
    at::Tensor make(at::ScalarType t) const { return at::empty(x->sizes(), options_of(*x, t)); }
};

// rms_norm(x, weight, residual, eps, rstd)
PyObject* rms_norm(PyObject*, PyObject* const* args, Py_ssize_t count) {
    HANDLE_TH_ERRORS
    NormRows n;
    double eps = 0;
    if (count != 5 || !n.set(args[0], args[1], args[2]) || !real(args[3], eps) || (args[4] != Py_True && args[4] != Py_False)) Py_RETURN_NONE;
    const bool want = args[4] == Py_True;
    at::Tensor out, total, rstd;
    void* const stream = stream_of(*n.x);
    TCR_CALL((out = n.make(n.x->scalar_type()), total = n.residual != nullptr ? n.make(n.x->scalar_type()) : at::Tensor(),
              rstd = want ? at::empty(n.x->sizes().slice(0, n.x->dim() - 1), options_of(*n.x, at::kFloat)) : at::Tensor()),
             g_rms_norm(n.x->data_ptr(), data_of(n.residual), n.weight->data_ptr(), out.data_ptr(), total.defined() ? total.data_ptr() : nullptr,
                        want ? static_cast<float*>(rstd.data_ptr()) : nullptr, n.rows_, n.cols, (int64_t)n.cols, (int64_t)n.cols, (float)eps, n.dtype,
                        n.weight_dtype, stream))
    if (st != TCR_OK) return failed(st, "tcr_rms_norm");
    if (!want && n.residual == nullptr) return wrapped(out);
    if (!want) return Py_BuildValue("NN", wrapped(out), wrapped(total));
    if (n.residual == nullptr) return Py_BuildValue("NN", wrapped(out), wrapped(rstd));
    return Py_BuildValue("NNN", wrapped(out), wrapped(total), wrapped(rstd));
    END_HANDLE_TH_ERRORS
}

// rms_norm_quantized(x, weight, residual, eps, whole numbers, group)
PyObject* rms_norm_quantized(PyObject*, PyObject* const* args, Py_ssize_t count) {
    HANDLE_TH_ERRORS
    NormRows n;
    double eps = 0;
    uint64_t group = 0;
    if (count != 6 || !n.set(args[0], args[1], args[2]) || !real(args[3], eps) || (args[4] != Py_True && args[4] != Py_False) ||
        !number(args[5], 0, 128, group))
        Py_RETURN_NONE;
    const bool numbers = args[4] == Py_True;
    at::Tensor codes, scales, total;
    c10::SmallVector<int64_t, 4> sizes(n.x->sizes().begin(), n.x->sizes().end());
    sizes.back() = group != 0 ? (int64_t)((n.cols + group - 1) / group) : 1;
    void* const stream = stream_of(*n.x);
    TCR_CALL((codes = n.make(numbers ? at::kChar : at::kFloat8_e4m3fn), scales = at::empty(sizes, options_of(*n.x, at::kFloat)),
              total = n.residual != nullptr ? n.make(n.x->scalar_type()) : at::Tensor()),
             g_rms_norm_quantized(n.x->data_ptr(), data_of(n.residual), n.weight->data_ptr(), codes.data_ptr(), static_cast<float*>(scales.data_ptr()),
                                  total.defined() ? total.data_ptr() : nullptr, n.rows_, n.cols, (int64_t)n.cols, (int64_t)n.cols, (float)eps, n.dtype,
                                  n.weight_dtype, numbers ? TCR_I8 : TCR_E4M3, (uint32_t)group, stream))
    if (st != TCR_OK) return failed(st, "tcr_rms_norm_quantized");
    return n.residual == nullptr ? Py_BuildValue("NN", wrapped(codes), wrapped(scales)) : Py_BuildValue("NNN", wrapped(codes), wrapped(scales), wrapped(total));
    END_HANDLE_TH_ERRORS
}

// rms_norm_backward(dout, total, weight, rstd, dtotal)
PyObject* rms_norm_backward(PyObject*, PyObject* const* args, Py_ssize_t count) {
    HANDLE_TH_ERRORS
    NormRows n;
    const at::Tensor* dout;
    if (count != 5 || !n.set(args[1], args[2], args[4]) || !n.like(args[0], &dout) || dout == nullptr) Py_RETURN_NONE;
    const at::Tensor* rstd = plain(args[3], at::kFloat);
    if (rstd == nullptr || (uint64_t)rstd->numel() != n.rows_ || rstd->device() != n.x->device()) Py_RETURN_NONE;
    at::Tensor dx, dweight;
    void* const stream = stream_of(*n.x);
    const int64_t step = (int64_t)n.cols;
    TCR_CALL((dx = n.make(n.x->scalar_type()), dweight = at::empty({step}, options_of(*n.x, n.weight->scalar_type()))),
             g_rms_norm_backward(dout->data_ptr(), n.x->data_ptr(), n.weight->data_ptr(), static_cast<const float*>(rstd->data_ptr()), data_of(n.residual),
                                 dx.data_ptr(), dweight.data_ptr(), n.rows_, n.cols, step, step, step, n.dtype, n.weight_dtype, stream))
    return st == TCR_OK ? Py_BuildValue("NN", wrapped(dx), wrapped(dweight)) : failed(st, "tcr_rms_norm_backward");
    END_HANDLE_TH_ERRORS
}

// bind_layers(addresses): in the order of the variables above
PyObject* bind_layers(PyObject*, PyObject* args) {
    unsigned long long a[6];
    if (!PyArg_ParseTuple(args, "KKKKKK", &a[0], &a[1], &a[2], &a[3], &a[4], &a[5])) return nullptr;
    g_linear_attention = reinterpret_cast<decltype(g_linear_attention)>(a[0]);
    g_linear_attention_step = reinterpret_cast<decltype(g_linear_attention_step)>(a[1]);
    g_linear_attention_backward = reinterpret_cast<decltype(g_linear_attention_backward)>(a[2]);
    g_rms_norm = reinterpret_cast<decltype(g_rms_norm)>(a[3]);
    g_rms_norm_quantized = reinterpret_cast<decltype(g_rms_norm_quantized)>(a[4]);
    g_rms_norm_backward = reinterpret_cast<decltype(g_rms_norm_backward)>(a[5]);
    Py_RETURN_NONE;
}
