// binding.py's calls of the convolution, the selective scan and the clipping in their ordinary form (part of tcr_native.cpp, whose rules hold here, with
// tcr_native_layers.hpp's helpers).
#pragma once

decltype(&tcr_causal_conv) g_causal_conv;
decltype(&tcr_causal_conv_step) g_causal_conv_step;
decltype(&tcr_causal_conv_backward) g_causal_conv_backward;
decltype(&tcr_selective_scan) g_selective_scan;
decltype(&tcr_selective_scan_step) g_selective_scan_step;
decltype(&tcr_selective_scan_backward) g_selective_scan_backward;
decltype(&tcr_gradient_norm) g_gradient_norm;
decltype(&tcr_clip_gradients) g_clip_gradients;

bool truth(PyObject* o, bool& v) {
    v = o == Py_True;
    return o == Py_True || o == Py_False;
}
// A tensor of these sizes and x's type whose last dimension is contiguous, or none.
bool row_tensor(PyObject* o, const at::Tensor& x, at::IntArrayRef sizes, const at::Tensor** t) {
    *t = nullptr;
    if (o == Py_None) return true;
    const at::Tensor* got = beside(o, x);
    if (got == nullptr) {                          // (b and c have a dimension more)
        got = rows(o);
        if (got == nullptr || got->scalar_type() != x.scalar_type() || got->device() != x.device()) return false;
    }
    if (got->sizes() != sizes) return false;
    *t = got;
    return true;
}
bool whole_or_none(PyObject* o, at::ScalarType type, at::IntArrayRef sizes, const at::Tensor& x, const at::Tensor** t) {
    *t = nullptr;
    if (o == Py_None) return true;
    *t = whole(o, type, sizes, x);
    return *t != nullptr;
}

// x and what the tokens are: [sequence, token, channel], packed [token, channel], for one token [sequence, channel].
struct Tokens {
    const at::Tensor* x = nullptr;
    const at::Tensor* offsets = nullptr;
    uint64_t sequences = 0, tokens = 0;
    int64_t channels = 0;
    bool packed = false, step = false;
    bool set(PyObject* first, PyObject* bounds, bool one) {
        x = leading(first);
        if (x == nullptr) return false;
        const at::ScalarType t = x->scalar_type();
        if (t != at::kHalf && t != at::kBFloat16 && t != at::kFloat) return false;
        packed = bounds != Py_None;
        step = one;
        if (x->dim() != (packed || step ? 2 : 3) || (channels = x->size(-1)) < 1 || channels > (1 << 24)) return false;
        sequences = (uint64_t)x->size(0);
        tokens = step ? 1 : (uint64_t)(packed ? x->size(0) : x->size(1));
        if (!packed) return true;
        offsets = entries(bounds, *x);
        if (offsets == nullptr) return false;
        sequences = (uint64_t)offsets->numel() - 1;
        return true;
    }
    // (sequence, token), and with `groups` a third
    void strides(const at::Tensor* t, int64_t* to, bool groups = false) const {
        if (t == nullptr) return;
        to[0] = packed ? 0 : t->stride(0);
        to[1] = step ? 0 : t->stride(packed ? 0 : 1);
        if (groups) to[2] = t->stride(-2);
    }
    const uint64_t* bounds() const { return offsets != nullptr ? static_cast<const uint64_t*>(offsets->data_ptr()) : nullptr; }
    at::Tensor made(at::IntArrayRef sizes, at::ScalarType t) const { return at::empty(sizes, options_of(*x, t)); }
    at::Tensor made_like(const at::Tensor* t) const { return t != nullptr ? made(t->sizes(), t->scalar_type()) : at::Tensor(); }
};
PyObject* wrapped_or_none(const at::Tensor& t) {
    if (t.defined()) return wrapped(t);
    Py_RETURN_NONE;
}
void* data_or_null(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

// ------------------------------------------------------------------------------------------------ convolution
struct ConvolutionCall : Tokens {
    tcr_convolution shape = {};
    const at::Tensor *weight = nullptr, *bias = nullptr, *out = nullptr;
    int64_t states[3] = {};
    // x, weight, bias, activation, offsets, out
    bool set(PyObject* const* args, bool one) {
        if (!Tokens::set(args[0], args[4], one)) return false;
        weight = plain(args[1], x->scalar_type());
        if (weight == nullptr || weight->dim() != 2 || weight->size(0) != channels || weight->size(1) < 2 || weight->size(1) > 1024 || weight->device() != x->device()) return false;
        if (!whole_or_none(args[2], x->scalar_type(), {channels}, *x, &bias)) return false;
        if (args[3] != Py_None && !(PyUnicode_CheckExact(args[3]) && PyUnicode_CompareWithASCIIString(args[3], "silu") == 0)) return false;
        if (!row_tensor(args[5], *x, x->sizes(), &out)) return false;
        shape.dtype = type_of(x->scalar_type());
        shape.channels = (uint32_t)channels;
        shape.width = (uint32_t)weight->size(1);
        shape.activation = args[3] != Py_None;
        shape.sequences = sequences;
        shape.tokens = tokens;
        shape.offsets = bounds();
        strides(x, shape.x_stride);
        strides(out, shape.o_stride);
        states[0] = (int64_t)sequences;
        states[1] = weight->size(1) - 1;
        states[2] = channels;
        return true;
    }
    bool state(PyObject* o, const at::Tensor** t) const { return whole_or_none(o, x->scalar_type(), at::IntArrayRef(states, 3), *x, t); }
    at::Tensor result() {
        if (out != nullptr) return *out;
        at::Tensor t = made(x->sizes(), x->scalar_type());
        strides(&t, shape.o_stride);
        return t;
    }
};

// causal_conv(x, weight, bias, activation, offsets, out, state, final_state)
PyObject* causal_conv(PyObject*, PyObject* const* args, Py_ssize_t count) {
    HANDLE_TH_ERRORS
    ConvolutionCall a;
    const at::Tensor* state;
    bool want = false;
    if (count != 8 || !a.set(args, false) || !a.state(args[6], &state) || !truth(args[7], want)) Py_RETURN_NONE;
    at::Tensor out, last;
    void* const stream = stream_of(*a.x);
    TCR_CALL((out = a.result(), last = want ? a.made(at::IntArrayRef(a.states, 3), a.x->scalar_type()) : at::Tensor()),
             g_causal_conv(&a.shape, a.x->data_ptr(), a.weight->data_ptr(), data_of(a.bias), out.data_ptr(), data_of(state), data_or_null(last), stream))
    if (st != TCR_OK) return failed(st, "tcr_causal_conv");
    written(a.out);
    return want ? Py_BuildValue("NN", wrapped(out), wrapped(last)) : wrapped(out);
    END_HANDLE_TH_ERRORS
}

// causal_conv_step(x, weight, bias, activation, None, out, state, new_state)
PyObject* causal_conv_step(PyObject*, PyObject* const* args, Py_ssize_t count) {
    HANDLE_TH_ERRORS
    ConvolutionCall a;
    const at::Tensor *state, *next;
    if (count != 8 || args[4] != Py_None || !a.set(args, true) || !a.state(args[6], &state) || state == nullptr || !a.state(args[7], &next)) Py_RETURN_NONE;
    if (next == nullptr) next = state;
    at::Tensor out;
    void* const stream = stream_of(*a.x);
    TCR_CALL((out = a.result()), g_causal_conv_step(&a.shape, a.x->data_ptr(), a.weight->data_ptr(), data_of(a.bias), out.data_ptr(), state->data_ptr(), next->data_ptr(), stream))
    if (st != TCR_OK) return failed(st, "tcr_causal_conv_step");
    written(next);
    written(a.out);
    return wrapped(out);
    END_HANDLE_TH_ERRORS
}

// causal_conv_backward(x, weight, bias, activation, offsets, dout, state, dfinal)
PyObject* causal_conv_backward(PyObject*, PyObject* const* args, Py_ssize_t count) {
    HANDLE_TH_ERRORS
    ConvolutionCall a;
    const at::Tensor *state, *dfinal;
    if (count != 8 || !a.set(args, false) || a.out == nullptr || !a.state(args[6], &state) || !a.state(args[7], &dfinal)) Py_RETURN_NONE;
    at::Tensor dx, dweight, dbias, dstate;
    void* const stream = stream_of(*a.x);
    TCR_CALL((dx = a.made_like(a.x), dweight = a.made_like(a.weight), dbias = a.made_like(a.bias), dstate = a.made_like(state)),
             g_causal_conv_backward(&a.shape, a.out->data_ptr(), a.x->data_ptr(), a.weight->data_ptr(), data_of(a.bias), dx.data_ptr(), dweight.data_ptr(), data_or_null(dbias),
                                    data_of(state), data_of(dfinal), data_or_null(dstate), stream))
    if (st != TCR_OK) return failed(st, "tcr_causal_conv_backward");
    return Py_BuildValue("NNNN", wrapped(dx), wrapped(dweight), wrapped_or_none(dbias), wrapped_or_none(dstate));
    END_HANDLE_TH_ERRORS
}

// ------------------------------------------------------------------------------------------------ selective scan
struct SelectiveCall : Tokens {
    tcr_selective shape = {};
    const at::Tensor *dt = nullptr, *a = nullptr, *b = nullptr, *c = nullptr, *skip = nullptr, *gate = nullptr, *bias = nullptr, *out = nullptr;
    int64_t states[3] = {};
    // x, dt, a, b, c, skip, gate, dt_bias, softplus, offsets, out
    bool set(PyObject* const* args, bool one) {
        bool soft = false;
        if (!Tokens::set(args[0], args[9], one) || !truth(args[8], soft)) return false;
        a = plain(args[2], at::kFloat);
        if (a == nullptr || a->dim() != 2 || a->size(0) != channels || a->size(1) < 1 || a->size(1) > 65535 || a->device() != x->device()) return false;
        const at::Tensor* first = rows(args[3]);
        if (first == nullptr || first->dim() != x->dim() + 1 || first->size(-2) < 1 || channels % first->size(-2) != 0) return false;
        c10::SmallVector<int64_t, 4> narrow(x->sizes().begin(), x->sizes().end());
        narrow.back() = first->size(-2);
        narrow.push_back(a->size(1));
        if (!row_tensor(args[1], *x, x->sizes(), &dt) || dt == nullptr || !row_tensor(args[3], *x, narrow, &b) || !row_tensor(args[4], *x, narrow, &c) || c == nullptr ||
            !row_tensor(args[6], *x, x->sizes(), &gate) || !row_tensor(args[10], *x, x->sizes(), &out) || !whole_or_none(args[5], at::kFloat, {channels}, *x, &skip) ||
            !whole_or_none(args[7], at::kFloat, {channels}, *x, &bias))
            return false;
        shape.dtype = type_of(x->scalar_type());
        shape.channels = (uint32_t)channels;
        shape.states = (uint32_t)a->size(1);
        shape.groups = (uint32_t)first->size(-2);
        shape.softplus = soft;
        shape.sequences = sequences;
        shape.tokens = tokens;
        shape.offsets = bounds();
        shape.a = static_cast<const float*>(a->data_ptr());
        shape.skip = static_cast<const float*>(data_of(skip));
        shape.dt_bias = static_cast<const float*>(data_of(bias));
        strides(x, shape.x_stride);
        strides(dt, shape.dt_stride);
        strides(gate, shape.gate_stride);
        strides(out, shape.o_stride);
        strides(b, shape.b_stride, true);
        strides(c, shape.c_stride, true);
        states[0] = (int64_t)sequences;
        states[1] = channels;
        states[2] = a->size(1);
        return true;
    }
    bool state(PyObject* o, const at::Tensor** t) const { return whole_or_none(o, at::kFloat, at::IntArrayRef(states, 3), *x, t); }
    at::Tensor result() {
        if (out != nullptr) return *out;
        at::Tensor t = made(x->sizes(), x->scalar_type());
        strides(&t, shape.o_stride);
        return t;
    }
};
const float* floats(const at::Tensor* t) { return static_cast<const float*>(data_of(t)); }
float* floats(const at::Tensor& t) { return static_cast<float*>(data_or_null(t)); }

// selective_scan(x, dt, a, b, c, skip, gate, dt_bias, softplus, offsets, out, state, final_state)
PyObject* selective_scan(PyObject*, PyObject* const* args, Py_ssize_t count) {
    HANDLE_TH_ERRORS
    SelectiveCall a;
    const at::Tensor* state;
    bool want = false;
    if (count != 13 || !a.set(args, false) || !a.state(args[11], &state) || !truth(args[12], want)) Py_RETURN_NONE;
    at::Tensor out, last;
    void* const stream = stream_of(*a.x);
    TCR_CALL((out = a.result(), last = want ? a.made(at::IntArrayRef(a.states, 3), at::kFloat) : at::Tensor()),
             g_selective_scan(&a.shape, a.x->data_ptr(), a.dt->data_ptr(), a.b->data_ptr(), a.c->data_ptr(), data_of(a.gate), out.data_ptr(), floats(state), floats(last), stream))
    if (st != TCR_OK) return failed(st, "tcr_selective_scan");
    written(a.out);
    return want ? Py_BuildValue("NN", wrapped(out), wrapped(last)) : wrapped(out);
    END_HANDLE_TH_ERRORS
}

// selective_scan_step(x, dt, a, b, c, skip, gate, dt_bias, softplus, None, out, state, new_state)
PyObject* selective_scan_step(PyObject*, PyObject* const* args, Py_ssize_t count) {
    HANDLE_TH_ERRORS
    SelectiveCall a;
    const at::Tensor *state, *next;
    if (count != 13 || args[9] != Py_None || !a.set(args, true) || !a.state(args[11], &state) || state == nullptr || !a.state(args[12], &next)) Py_RETURN_NONE;
    if (next == nullptr) next = state;
    at::Tensor out;
    void* const stream = stream_of(*a.x);
    TCR_CALL((out = a.result()), g_selective_scan_step(&a.shape, a.x->data_ptr(), a.dt->data_ptr(), a.b->data_ptr(), a.c->data_ptr(), data_of(a.gate), out.data_ptr(),
                                                       floats(state), const_cast<float*>(floats(next)), stream))
    if (st != TCR_OK) return failed(st, "tcr_selective_scan_step");
    written(next);
    written(a.out);
    return wrapped(out);
    END_HANDLE_TH_ERRORS
}

// selective_scan_backward(x, dt, a, b, c, skip, gate, dt_bias, softplus, offsets, dout, state, dfinal)
PyObject* selective_scan_backward(PyObject*, PyObject* const* args, Py_ssize_t count) {
    HANDLE_TH_ERRORS
    SelectiveCall a;
    const at::Tensor *state, *dfinal;
    if (count != 13 || !a.set(args, false) || a.out == nullptr || !a.state(args[11], &state) || !a.state(args[12], &dfinal)) Py_RETURN_NONE;
    at::Tensor dx, ddt, da, db, dc, dskip, dgate, dbias, dstate;
    void* const stream = stream_of(*a.x);
    TCR_CALL((dx = a.made_like(a.x), ddt = a.made_like(a.dt), da = a.made_like(a.a), db = a.made_like(a.b), dc = a.made_like(a.c), dskip = a.made_like(a.skip),
              dgate = a.made_like(a.gate), dbias = a.made_like(a.bias), dstate = a.made_like(state)),
             g_selective_scan_backward(&a.shape, a.out->data_ptr(), a.x->data_ptr(), a.dt->data_ptr(), a.b->data_ptr(), a.c->data_ptr(), data_of(a.gate), dx.data_ptr(),
                                       ddt.data_ptr(), floats(da), db.data_ptr(), dc.data_ptr(), floats(dskip), data_or_null(dgate), floats(dbias), floats(state),
                                       floats(dfinal), floats(dstate), stream))
    if (st != TCR_OK) return failed(st, "tcr_selective_scan_backward");
    return Py_BuildValue("NNNNNNNNN", wrapped(dx), wrapped(ddt), wrapped(da), wrapped(db), wrapped(dc), wrapped_or_none(dskip), wrapped_or_none(dgate), wrapped_or_none(dbias),
                         wrapped_or_none(dstate));
    END_HANDLE_TH_ERRORS
}

// ------------------------------------------------------------------------------------------------ norm over many tensors, clipping
// Contiguous tensors of the current device, from a list or tuple; other orders of dimensions are binding.py's.
struct TensorList {
    std::vector<tcr_tensor> places;
    std::vector<const at::Tensor*> tensors;
    bool set(PyObject* list) {
        if (!PyList_CheckExact(list) && !PyTuple_CheckExact(list)) return false;
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(list);
        if (n < 1) return false;
        places.reserve((size_t)n);
        tensors.reserve((size_t)n);
        for (Py_ssize_t i = 0; i < n; ++i) {
            PyObject* o = PySequence_Fast_GET_ITEM(list, i);
            if (!THPVariable_CheckExact(o)) return false;
            const at::ScalarType type = THPVariable_Unpack(o).scalar_type();
            if (type != at::kHalf && type != at::kBFloat16 && type != at::kFloat) return false;
            const at::Tensor* t = plain(o, type);
            if (t == nullptr || (i != 0 && t->device() != tensors[0]->device())) return false;
            places.push_back({t->data_ptr(), (uint64_t)t->numel(), type_of(type)});
            tensors.push_back(t);
        }
        c10::DeviceIndex device = -1;
        if (at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set()) return false;
        return c10::hip::GetDevice(&device) == hipSuccess && device == tensors[0]->device().index();
    }
    at::Tensor norm() const { return at::empty({}, options_of(*tensors[0], at::kFloat)); }
};

// gradient_norm(tensors)
PyObject* gradient_norm(PyObject*, PyObject* const* args, Py_ssize_t count) {
    HANDLE_TH_ERRORS
    TensorList a;
    if (count != 1 || !a.set(args[0])) Py_RETURN_NONE;
    at::Tensor norm;
    void* const stream = stream_of(*a.tensors[0]);
    TCR_CALL((norm = a.norm()), g_gradient_norm(a.places.data(), a.places.size(), static_cast<float*>(norm.data_ptr()), stream))
    return st == TCR_OK ? wrapped(norm) : failed(st, "tcr_gradient_norm");
    END_HANDLE_TH_ERRORS
}

// clip_gradients(tensors, max_norm, eps, out)
PyObject* clip_gradients(PyObject*, PyObject* const* args, Py_ssize_t count) {
    HANDLE_TH_ERRORS
    TensorList a, to;
    double limit = 0, eps = 0;
    if (count != 4 || !a.set(args[0]) || !real(args[1], limit) || !real(args[2], eps)) Py_RETURN_NONE;
    std::vector<void*> out;
    if (args[3] != Py_None) {
        if (!to.set(args[3]) || to.tensors.size() != a.tensors.size()) Py_RETURN_NONE;
        out.reserve(a.tensors.size());
        for (size_t i = 0; i < a.tensors.size(); ++i) {
            if (to.places[i].dtype != a.places[i].dtype || to.tensors[i]->sizes() != a.tensors[i]->sizes() || to.tensors[i]->device() != a.tensors[i]->device()) Py_RETURN_NONE;
            out.push_back(to.places[i].data);
        }
    }
    at::Tensor norm;
    void* const stream = stream_of(*a.tensors[0]);
    TCR_CALL((norm = a.norm()), g_clip_gradients(a.places.data(), out.empty() ? nullptr : out.data(), a.places.size(), (float)limit, (float)eps,
                                                 static_cast<float*>(norm.data_ptr()), stream))
    if (st != TCR_OK) return failed(st, "tcr_clip_gradients");
    for (const at::Tensor* t : out.empty() ? a.tensors : to.tensors) written(t);
    return wrapped(norm);
    END_HANDLE_TH_ERRORS
}

// bind_selective(addresses): in the order of the variables above
PyObject* bind_selective(PyObject*, PyObject* args) {
    unsigned long long a[8];
    if (!PyArg_ParseTuple(args, "KKKKKKKK", &a[0], &a[1], &a[2], &a[3], &a[4], &a[5], &a[6], &a[7])) return nullptr;
    g_causal_conv = reinterpret_cast<decltype(g_causal_conv)>(a[0]);
    g_causal_conv_step = reinterpret_cast<decltype(g_causal_conv_step)>(a[1]);
    g_causal_conv_backward = reinterpret_cast<decltype(g_causal_conv_backward)>(a[2]);
    g_selective_scan = reinterpret_cast<decltype(g_selective_scan)>(a[3]);
    g_selective_scan_step = reinterpret_cast<decltype(g_selective_scan_step)>(a[4]);
    g_selective_scan_backward = reinterpret_cast<decltype(g_selective_scan_backward)>(a[5]);
    g_gradient_norm = reinterpret_cast<decltype(g_gradient_norm)>(a[6]);
    g_clip_gradients = reinterpret_cast<decltype(g_clip_gradients)>(a[7]);
    Py_RETURN_NONE;
}
