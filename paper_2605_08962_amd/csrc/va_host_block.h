// The Python binding's usual calls of the operators around attention in native code; part of va_host.cpp, in whose namespace and to
// whose rules it is written: plain tensors on the current device that pass every check, on the current stream, and NotImplemented for
// anything else.  Such a call on 246 tokens runs 3 to 8 us on the GPU and took 17 to 60 us in Python.  Positions, norm and packing with
// results or workspaces of the caller's own (`out` of the norm and `dx` aside), and any call with a `stream`, still go through Python: 10
// to 27 us where the call that allocates takes 5 to 12.
#pragma once

#ifndef VA_CURRENT_DEVICE  // (a test on the CPU sets its own)
#define VA_CURRENT_DEVICE() c10::hip::current_device()
#endif

decltype(&varlen_attn_rotary_positions) rotary_positions_f = nullptr;
decltype(&varlen_attn_rotary_fwd) rotary_fwd_f = nullptr;
decltype(&varlen_attn_rotary_bwd) rotary_bwd_f = nullptr;
decltype(&varlen_attn_act8_pack) act8_pack_f = nullptr;
decltype(&varlen_attn_act8_unpack) act8_unpack_f = nullptr;
decltype(&varlen_attn_bwd_act8_workspace_bytes) bwd_act8_bytes_f = nullptr;
decltype(&varlen_attn_bwd_act8) bwd_act8_f = nullptr;
decltype(&varlen_attn_norm_fwd) norm_fwd_f = nullptr;
decltype(&varlen_attn_norm_bwd_workspace_bytes) norm_bwd_bytes_f = nullptr;
decltype(&varlen_attn_norm_bwd) norm_bwd_f = nullptr;
PyObject* act8_type = nullptr;  // binding.Act8

// bind_block(addresses of the ten library functions, Act8)
PyObject* bind_block(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 11 || !PyType_Check(a[10])) { PyErr_SetString(PyExc_TypeError, "bind_block takes 10 addresses and a type"); return nullptr; }
    void* f[10];
    for (int i = 0; i < 10; ++i) {
        f[i] = PyLong_AsVoidPtr(a[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    rotary_positions_f = (decltype(rotary_positions_f))f[0];
    rotary_fwd_f = (decltype(rotary_fwd_f))f[1];
    rotary_bwd_f = (decltype(rotary_bwd_f))f[2];
    act8_pack_f = (decltype(act8_pack_f))f[3];
    act8_unpack_f = (decltype(act8_unpack_f))f[4];
    bwd_act8_bytes_f = (decltype(bwd_act8_bytes_f))f[5];
    bwd_act8_f = (decltype(bwd_act8_f))f[6];
    norm_fwd_f = (decltype(norm_fwd_f))f[7];
    norm_bwd_bytes_f = (decltype(norm_bwd_bytes_f))f[8];
    norm_bwd_f = (decltype(norm_bwd_f))f[9];
    Py_INCREF(a[10]);
    Py_XDECREF(act8_type);
    act8_type = a[10];
    Py_RETURN_NONE;
}

// The current device, or, where `t` is not on a GPU (nor perhaps is there any), one that nothing is on.
int device_for(const at::Tensor& t) { return t.is_cuda() ? (int)VA_CURRENT_DEVICE() : INT32_MIN; }
bool here(const at::Tensor& t, int device) { return t.is_cuda() && t.device().index() == device; }
bool usable_here(const at::Tensor& t, at::ScalarType type, int device) {
    return here(t, device) && t.scalar_type() == type && t.is_contiguous();
}
// As binding.py's _token_stride.
bool token_stride(const at::Tensor& t, bool rows, int device, int64_t& stride) {
    if (!here(t, device) || t.scalar_type() != at::kBFloat16 || !(t.dim() == 3 || (rows && t.dim() == 2))) return false;
    for (int i = 0; i < t.dim(); ++i) if (!fits(t.size(i))) return false;
    const int64_t c = t.size(-1), h = t.dim() == 3 ? t.size(1) : 1, width = h * c;
    stride = width;
    if (t.numel() == 0) return true;
    if ((c > 1 && t.stride(-1) != 1) || (h > 1 && t.stride(1) != c) || (t.size(0) > 1 && t.stride(0) < width)) return false;
    if (t.size(0) > 1) stride = t.stride(0);
    return true;
}
bool same_or_none(PyObject* o, const at::Tensor& like, int device) {  // contiguous, of like's shape, bf16
    return o == Py_None || (usable_here(THPVariable_Unpack(o), at::kBFloat16, device) && THPVariable_Unpack(o).sizes() == like.sizes());
}
void* ptr_or_null(PyObject* o) { return o == Py_None ? nullptr : THPVariable_Unpack(o).data_ptr(); }
void* current_stream() { return (void*)c10::hip::getCurrentHIPStream().stream(); }
at::Tensor empty_of(at::IntArrayRef sizes, const at::Tensor& like, at::ScalarType type) { return at::empty(sizes, like.options().dtype(type)); }
PyObject* tuple_of(std::initializer_list<const at::Tensor*> ts) {  // (an undefined one: None)
    PyObject* r = PyTuple_New((Py_ssize_t)ts.size());
    Py_ssize_t i = 0;
    for (const at::Tensor* t : ts) {
        if (!r) return nullptr;
        PyObject* o = t->defined() ? THPVariable_Wrap(*t) : (Py_INCREF(Py_None), Py_None);
        if (!o) { Py_DECREF(r); return nullptr; }
        PyTuple_SET_ITEM(r, i++, o);
    }
    return r;
}

at::DimVector scales_shape(const at::Tensor& t) {
    at::DimVector s(t.sizes().begin(), t.sizes().end());
    s.back() = (s.back() + VA_ACT8_BLOCK - 1) / VA_ACT8_BLOCK;
    return s;
}
at::ScalarType code_type(int format) { return format == VA_ACT8_INT8 ? at::kChar : at::kFloat8_e4m3fn; }
// Codes, scales and format of an Act8; false: not one, or not one that the kernels can read.
bool act8_of(PyObject* o, const at::Tensor*& codes, const at::Tensor*& scales, int& format) {
    if (Py_TYPE(o) != (PyTypeObject*)act8_type || PyTuple_GET_SIZE(o) != 2 || !plain(PyTuple_GET_ITEM(o, 0)) || !plain(PyTuple_GET_ITEM(o, 1)))
        return false;
    codes = &THPVariable_Unpack(PyTuple_GET_ITEM(o, 0));
    scales = &THPVariable_Unpack(PyTuple_GET_ITEM(o, 1));
    format = codes->scalar_type() == at::kChar ? VA_ACT8_INT8 : VA_ACT8_E4M3;
    if (codes->dim() != 2 && codes->dim() != 3) return false;
    for (int i = 0; i < codes->dim(); ++i) if (!fits(codes->size(i))) return false;
    const int device = device_for(*codes);
    return usable_here(*codes, code_type(format), device) && usable_here(*scales, at::kFloat, device) &&
           scales->sizes() == at::IntArrayRef(scales_shape(*codes));
}
varlen_attn_act8_tensor act8_tensor(const at::Tensor& values, int64_t stride, const at::Tensor& codes, const at::Tensor& scales) {
    return {values.data_ptr(), codes.data_ptr(), (float*)scales.data_ptr(), (int32_t)codes.size(0),
            codes.dim() == 3 ? (int32_t)codes.size(1) : 1, (int32_t)codes.size(-1), stride};
}

// positions(cu_rows, grids, total_tokens, first, merge) -> positions, a status or NotImplemented
PyObject* rotary_positions(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 5 || !rotary_positions_f) { PyErr_SetString(PyExc_TypeError, "positions takes 5 arguments, after bind_block"); return nullptr; }
    if (!plain(a[0]) || !plain(a[1]) || !plain_or_none(a[3]) || at::impl::torch_function_mode_enabled()) return not_implemented();
    return guarded([&]() -> PyObject* {
        const at::Tensor &cu = THPVariable_Unpack(a[0]), &grids = THPVariable_Unpack(a[1]);
        const long total = PyLong_AsLong(a[2]), merge = PyLong_AsLong(a[4]);
        if (PyErr_Occurred()) { PyErr_Clear(); return not_implemented(); }
        const int device = device_for(cu);
        if (!usable_here(cu, at::kInt, device) || !usable_here(grids, at::kInt, device) || cu.dim() != 1 || cu.size(0) < 1 || !fits(cu.size(0)) ||
            grids.dim() != 2 || grids.size(0) != cu.size(0) - 1 || grids.size(1) != 3 || !fits(total) || !fits(merge) ||
            (a[3] != Py_None && (!usable_here(THPVariable_Unpack(a[3]), at::kInt, device) || THPVariable_Unpack(a[3]).numel() != cu.size(0) - 1)))
            return not_implemented();
        at::Tensor out;
        int status;
        {
            WithoutLock free;
            out = empty_of({3, total}, cu, at::kInt);
            status = rotary_positions_f((int32_t)total, (int32_t)(cu.size(0) - 1), (int32_t)merge, (const int32_t*)cu.data_ptr(),
                                        (const int32_t*)grids.data_ptr(), (const int32_t*)ptr_or_null(a[3]), (int32_t*)out.data_ptr(),
                                        current_stream());
        }
        return status != VA_OK ? PyLong_FromLong(status) : THPVariable_Wrap(out);
    });
}

// rotary(inverse, q, k, v, positions, inv_freq, pair_axis, interleaved, q_out, k_out, v_out) -> (q, k) or (q, k, v), a status or
// NotImplemented
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 11 || !rotary_fwd_f) { PyErr_SetString(PyExc_TypeError, "rotary takes 11 arguments, after bind_block"); return nullptr; }
    for (int i : {1, 2, 4, 5, 6}) if (!plain(a[i])) return not_implemented();
    for (int i : {3, 8, 9, 10}) if (!plain_or_none(a[i])) return not_implemented();
    if (at::impl::torch_function_mode_enabled()) return not_implemented();
    return guarded([&]() -> PyObject* {
        const at::Tensor &q = THPVariable_Unpack(a[1]), &k = THPVariable_Unpack(a[2]), &pos = THPVariable_Unpack(a[4]),
                         &freq = THPVariable_Unpack(a[5]), &axis = THPVariable_Unpack(a[6]);
        const bool has_v = a[3] != Py_None;
        const int device = device_for(q);
        varlen_attn_rotary_params p{};
        if (!token_stride(q, false, device, p.q_stride) || !token_stride(k, false, device, p.k_stride) || k.size(0) != q.size(0) ||
            k.size(2) != q.size(2) || (!has_v && a[10] != Py_None) || !usable_here(pos, at::kInt, device) ||
            !usable_here(freq, at::kFloat, device) || !usable_here(axis, at::kInt, device) || pos.dim() != 2 || pos.size(1) != q.size(0) ||
            !fits(pos.size(0)) || freq.dim() != 1 || !fits(freq.size(0)) || axis.sizes() != freq.sizes())
            return not_implemented();
        if (has_v && (!token_stride(THPVariable_Unpack(a[3]), false, device, p.v_stride) || THPVariable_Unpack(a[3]).sizes() != k.sizes()))
            return not_implemented();
        int64_t* const strides[3] = {&p.q_out_stride, &p.k_out_stride, &p.v_out_stride};
        for (int i = 0; i < (has_v ? 3 : 2); ++i) {
            const at::Tensor& like = i ? k : q;
            *strides[i] = like.size(1) * like.size(2);
            if (a[8 + i] != Py_None && (!token_stride(THPVariable_Unpack(a[8 + i]), false, device, *strides[i]) ||
                                        THPVariable_Unpack(a[8 + i]).sizes() != like.sizes()))
                return not_implemented();
        }
        p.total_tokens = (int32_t)q.size(0);
        p.num_q_heads = (int32_t)q.size(1);
        p.num_kv_heads = (int32_t)k.size(1);
        p.head_dim = (int32_t)q.size(2);
        p.num_pairs = (int32_t)freq.size(0);
        p.num_axes = (int32_t)pos.size(0);
        p.interleaved = a[7] == Py_True;
        at::Tensor out[3];
        int status;
        {
            WithoutLock free;
            for (int i = 0; i < (has_v ? 3 : 2); ++i)
                out[i] = a[8 + i] != Py_None ? THPVariable_Unpack(a[8 + i]) : empty_of((i ? k : q).sizes(), q, at::kBFloat16);
            status = (a[0] == Py_True ? rotary_bwd_f : rotary_fwd_f)(
                &p, q.data_ptr(), k.data_ptr(), ptr_or_null(a[3]), (const int32_t*)pos.data_ptr(), (const float*)freq.data_ptr(),
                (const int32_t*)axis.data_ptr(), out[0].data_ptr(), out[1].data_ptr(), has_v ? out[2].data_ptr() : nullptr, current_stream());
        }
        if (status != VA_OK) return PyLong_FromLong(status);
        PyObject* r = PyTuple_New(has_v ? 3 : 2);
        for (int i = 0; r && i < (has_v ? 3 : 2); ++i) {
            PyObject* o = object_of(a[8 + i], out[i]);
            if (!o) { Py_DECREF(r); return nullptr; }
            PyTuple_SET_ITEM(r, i, o);
        }
        return r;
    });
}

// act8_pack([tensors], format) -> [Act8], a status or NotImplemented
PyObject* act8_pack(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 2 || !act8_pack_f) { PyErr_SetString(PyExc_TypeError, "act8_pack takes 2 arguments, after bind_block"); return nullptr; }
    if (!PyList_CheckExact(a[0]) || at::impl::torch_function_mode_enabled()) return not_implemented();
    const Py_ssize_t count = PyList_GET_SIZE(a[0]);
    if (count < 1 || count > VA_ACT8_MAX_TENSORS) return not_implemented();
    PyObject* given[VA_ACT8_MAX_TENSORS];
    for (Py_ssize_t i = 0; i < count; ++i) if (!plain(given[i] = PyList_GET_ITEM(a[0], i))) return not_implemented();
    return guarded([&]() -> PyObject* {
        const int format = (int)PyLong_AsLong(a[1]), device = device_for(THPVariable_Unpack(given[0]));
        if (PyErr_Occurred()) { PyErr_Clear(); return not_implemented(); }
        at::Tensor values[VA_ACT8_MAX_TENSORS], codes[VA_ACT8_MAX_TENSORS], scales[VA_ACT8_MAX_TENSORS];
        int64_t stride[VA_ACT8_MAX_TENSORS];
        for (Py_ssize_t i = 0; i < count; ++i) {  // (the list may change once the lock is given up)
            values[i] = THPVariable_Unpack(given[i]);
            if (!token_stride(values[i], true, device, stride[i])) return not_implemented();
        }
        varlen_attn_act8_tensor t[VA_ACT8_MAX_TENSORS];
        int status;
        {
            WithoutLock free;
            for (Py_ssize_t i = 0; i < count; ++i) {
                codes[i] = empty_of(values[i].sizes(), values[i], code_type(format));
                scales[i] = empty_of(scales_shape(values[i]), values[i], at::kFloat);
                t[i] = act8_tensor(values[i], stride[i], codes[i], scales[i]);
            }
            status = act8_pack_f(t, (int32_t)count, format, current_stream());
        }
        if (status != VA_OK) return PyLong_FromLong(status);
        PyObject* r = PyList_New(count);
        for (Py_ssize_t i = 0; r && i < count; ++i) {
            PyObject *c = THPVariable_Wrap(codes[i]), *s = c ? THPVariable_Wrap(scales[i]) : nullptr;
            PyObject* x = s ? PyObject_CallFunctionObjArgs(act8_type, c, s, nullptr) : nullptr;
            Py_XDECREF(c);
            Py_XDECREF(s);
            if (!x) { Py_DECREF(r); return nullptr; }
            PyList_SET_ITEM(r, i, x);
        }
        return r;
    });
}

// act8_unpack([Act8]) -> [tensors], a status or NotImplemented
PyObject* act8_unpack(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 1 || !act8_unpack_f) { PyErr_SetString(PyExc_TypeError, "act8_unpack takes 1 argument, after bind_block"); return nullptr; }
    if (!PyList_CheckExact(a[0]) || at::impl::torch_function_mode_enabled()) return not_implemented();
    const Py_ssize_t count = PyList_GET_SIZE(a[0]);
    if (count < 1 || count > VA_ACT8_MAX_TENSORS) return not_implemented();
    return guarded([&]() -> PyObject* {
        at::Tensor codes[VA_ACT8_MAX_TENSORS], scales[VA_ACT8_MAX_TENSORS], out[VA_ACT8_MAX_TENSORS];
        int format = 0;
        for (Py_ssize_t i = 0; i < count; ++i) {
            const at::Tensor *c, *s;
            int f;
            if (!act8_of(PyList_GET_ITEM(a[0], i), c, s, f) || (i && f != format)) return not_implemented();
            codes[i] = *c;
            scales[i] = *s;
            format = f;
        }
        varlen_attn_act8_tensor t[VA_ACT8_MAX_TENSORS];
        int status;
        {
            WithoutLock free;
            for (Py_ssize_t i = 0; i < count; ++i) {
                out[i] = empty_of(codes[i].sizes(), codes[i], at::kBFloat16);
                t[i] = act8_tensor(out[i], codes[i].dim() == 3 ? codes[i].size(1) * codes[i].size(2) : codes[i].size(1), codes[i], scales[i]);
            }
            status = act8_unpack_f(t, (int32_t)count, format, current_stream());
        }
        if (status != VA_OK) return PyLong_FromLong(status);
        PyObject* r = PyList_New(count);
        for (Py_ssize_t i = 0; r && i < count; ++i) {
            PyObject* x = THPVariable_Wrap(out[i]);
            if (!x) { Py_DECREF(r); return nullptr; }
            PyList_SET_ITEM(r, i, x);
        }
        return r;
    });
}

// bwd_act8(dout, q, k, v, out, lse, cu_seqlens, causal, scale, dq, dk, dv, workspace, kv_splits, max_seqlen) -> (dq, dk, dv), a status
// or NotImplemented
PyObject* bwd_act8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 15 || !bwd_act8_f) { PyErr_SetString(PyExc_TypeError, "bwd_act8 takes 15 arguments, after bind_block"); return nullptr; }
    for (int i : {0, 5, 6}) if (!plain(a[i])) return not_implemented();
    for (int i : {9, 10, 11, 12}) if (!plain_or_none(a[i])) return not_implemented();
    if (at::impl::torch_function_mode_enabled()) return not_implemented();
    return guarded([&]() -> PyObject* {
        const at::Tensor &dout = THPVariable_Unpack(a[0]), &lse = THPVariable_Unpack(a[5]), &cu = THPVariable_Unpack(a[6]);
        const double scale = PyFloat_AsDouble(a[8]);
        const long splits = PyLong_AsLong(a[13]), longest = PyLong_AsLong(a[14]);
        if (PyErr_Occurred()) { PyErr_Clear(); return not_implemented(); }
        const int device = device_for(dout);
        const at::Tensor *codes[4], *scales[4];
        int format[4];
        for (int i = 0; i < 4; ++i)
            if (!act8_of(a[1 + i], codes[i], scales[i], format[i]) || format[i] != format[0]) return not_implemented();
        const at::Tensor &q = *codes[0], &k = *codes[1];
        varlen_attn_params p;
        if (!usable_here(dout, at::kBFloat16, device) || !usable_here(cu, at::kInt, device) || !here(lse, device) ||
            !fill(p, q, k, cu, a[7] == Py_True, scale, splits, longest) || dout.sizes() != q.sizes() || codes[3]->sizes() != q.sizes() ||
            codes[2]->sizes() != k.sizes() || k.size(0) != q.size(0) || k.size(2) != q.size(2) ||
            !has_room(lse, at::kFloat, q.size(0) * q.size(1)) || !none_or_room(a[9], at::kBFloat16, q.numel()) ||
            !none_or_room(a[10], at::kBFloat16, k.numel()) || !none_or_room(a[11], at::kBFloat16, k.numel()) || !none_or_scratch(a[12]))
            return not_implemented();
        for (int i = 9; i < 13; ++i) if (a[i] != Py_None && !here(THPVariable_Unpack(a[i]), device)) return not_implemented();
        at::Tensor grads[3];
        int status;
        {
            WithoutLock free;
            for (int i = 0; i < 3; ++i) grads[i] = a[9 + i] != Py_None ? THPVariable_Unpack(a[9 + i]) : empty_of((i ? k : q).sizes(), dout, at::kBFloat16);
            const at::Tensor ws = workspace_of(a[12], a[12] == Py_None ? bwd_act8_bytes_f(&p) : 0, dout);
            status = bwd_act8_f(&p, format[0], dout.data_ptr(), codes[0]->data_ptr(), (const float*)scales[0]->data_ptr(), codes[1]->data_ptr(),
                                (const float*)scales[1]->data_ptr(), codes[2]->data_ptr(), (const float*)scales[2]->data_ptr(),
                                codes[3]->data_ptr(), (const float*)scales[3]->data_ptr(), (const float*)lse.data_ptr(),
                                (const int32_t*)cu.data_ptr(), grads[0].data_ptr(), grads[1].data_ptr(), grads[2].data_ptr(), ws.data_ptr(),
                                (size_t)ws.numel(), current_stream());
        }
        if (status != VA_OK) return PyLong_FromLong(status);
        PyObject* r = PyTuple_New(3);
        for (int i = 0; r && i < 3; ++i) {
            PyObject* g = object_of(a[9 + i], grads[i]);
            if (!g) { Py_DECREF(r); return nullptr; }
            PyTuple_SET_ITEM(r, i, g);
        }
        return r;
    });
}

// weight's (and bias's) type for the library; false where they do not fit rows of c channels.
bool weights_of(PyObject* weight, PyObject* bias, int64_t c, int device, int32_t& type) {
    type = VA_BF16;
    if (weight == Py_None) return bias == Py_None;
    const at::Tensor& w = THPVariable_Unpack(weight);
    type = w.scalar_type() == at::kFloat ? VA_FP32 : VA_BF16;
    for (PyObject* o : {weight, bias}) {
        if (o == Py_None) continue;
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!usable_here(t, type == VA_FP32 ? at::kFloat : at::kBFloat16, device) || t.dim() != 1 || t.size(0) != c) return false;
    }
    return true;
}

// norm_fwd(x, weight, bias, eps, residual, format or None, out) -> (out, mean, rstd, summed, saved), a status or NotImplemented
PyObject* norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 7 || !norm_fwd_f) { PyErr_SetString(PyExc_TypeError, "norm_fwd takes 7 arguments, after bind_block"); return nullptr; }
    if (!plain(a[0])) return not_implemented();
    for (int i : {1, 2, 4, 6}) if (!plain_or_none(a[i])) return not_implemented();
    if (at::impl::torch_function_mode_enabled()) return not_implemented();
    return guarded([&]() -> PyObject* {
        const at::Tensor& x = THPVariable_Unpack(a[0]);
        const double eps = PyFloat_AsDouble(a[3]);
        const bool save = a[5] != Py_None;
        const int format = save ? (int)PyLong_AsLong(a[5]) : 0, device = device_for(x);
        if (PyErr_Occurred()) { PyErr_Clear(); return not_implemented(); }
        varlen_attn_norm_params p{};
        if (!token_stride(x, true, device, p.x_stride) || !weights_of(a[1], a[2], x.size(-1), device, p.weight_type) ||
            !same_or_none(a[4], x, device) || !same_or_none(a[6], x, device))
            return not_implemented();
        p.total_tokens = (int32_t)x.size(0);
        p.rows_per_token = x.dim() == 3 ? (int32_t)x.size(1) : 1;
        p.channels = (int32_t)x.size(-1);
        p.act8_format = format;
        p.eps = (float)eps;
        at::Tensor out, mean, rstd, summed, codes, scales;
        int status;
        {
            WithoutLock free;
            out = a[6] != Py_None ? THPVariable_Unpack(a[6]) : empty_of(x.sizes(), x, at::kBFloat16);
            const at::IntArrayRef rows = x.sizes().slice(0, x.dim() - 1);
            mean = empty_of(rows, x, at::kFloat);
            rstd = empty_of(rows, x, at::kFloat);
            if (a[4] != Py_None) summed = empty_of(x.sizes(), x, at::kBFloat16);
            if (save) {
                codes = empty_of(x.sizes(), x, code_type(format));
                scales = empty_of(scales_shape(x), x, at::kFloat);
            }
            status = norm_fwd_f(&p, x.data_ptr(), ptr_or_null(a[4]), ptr_or_null(a[1]), ptr_or_null(a[2]), out.data_ptr(),
                                summed.defined() ? summed.data_ptr() : nullptr, (float*)mean.data_ptr(), (float*)rstd.data_ptr(),
                                save ? codes.data_ptr() : nullptr, save ? (float*)scales.data_ptr() : nullptr, current_stream());
        }
        if (status != VA_OK) return PyLong_FromLong(status);
        PyObject* r = tuple_of({&out, &mean, &rstd, &summed, &codes});
        if (r && a[6] != Py_None) { Py_INCREF(a[6]); PyTuple_SetItem(r, 0, a[6]); }
        if (r && save) {
            PyObject* s = THPVariable_Wrap(scales);
            PyObject* kept = s ? PyObject_CallFunctionObjArgs(act8_type, PyTuple_GET_ITEM(r, 4), s, nullptr) : nullptr;
            Py_XDECREF(s);
            if (!kept) { Py_DECREF(r); return nullptr; }
            PyTuple_SetItem(r, 4, kept);
        }
        return r;
    });
}

// norm_bwd(dy, x or Act8, mean, rstd, weight, dsummed, dx) -> (dx, dweight, dbias), a status or NotImplemented
PyObject* norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 7 || !norm_bwd_f) { PyErr_SetString(PyExc_TypeError, "norm_bwd takes 7 arguments, after bind_block"); return nullptr; }
    for (int i : {0, 2, 3}) if (!plain(a[i])) return not_implemented();
    for (int i : {4, 5, 6}) if (!plain_or_none(a[i])) return not_implemented();
    if (at::impl::torch_function_mode_enabled()) return not_implemented();
    return guarded([&]() -> PyObject* {
        const at::Tensor &dy = THPVariable_Unpack(a[0]), &mean = THPVariable_Unpack(a[2]), &rstd = THPVariable_Unpack(a[3]);
        const int device = device_for(dy);
        varlen_attn_norm_params p{};
        const at::Tensor *x = nullptr, *scales = nullptr;
        const bool packed = !plain(a[1]);
        int format = 0;
        if (!token_stride(dy, true, device, p.dy_stride)) return not_implemented();
        if (packed) {
            if (!act8_of(a[1], x, scales, format)) return not_implemented();
        } else {
            x = &THPVariable_Unpack(a[1]);
            if (!token_stride(*x, true, device, p.x_stride)) return not_implemented();
        }
        const at::IntArrayRef rows = dy.sizes().slice(0, dy.dim() - 1);
        if (x->sizes() != dy.sizes() || !usable_here(mean, at::kFloat, device) || !usable_here(rstd, at::kFloat, device) || mean.sizes() != rows ||
            rstd.sizes() != rows || !weights_of(a[4], Py_None, dy.size(-1), device, p.weight_type) || !same_or_none(a[5], dy, device))
            return not_implemented();
        p.rows_per_token = dy.dim() == 3 ? (int32_t)dy.size(1) : 1;
        p.dx_stride = p.rows_per_token * dy.size(-1);
        if (a[6] != Py_None && (!token_stride(THPVariable_Unpack(a[6]), true, device, p.dx_stride) || THPVariable_Unpack(a[6]).sizes() != dy.sizes()))
            return not_implemented();
        p.total_tokens = (int32_t)dy.size(0);
        p.channels = (int32_t)dy.size(-1);
        p.act8_format = format;
        at::Tensor dx, dw, db;
        int status;
        {
            WithoutLock free;
            dx = a[6] != Py_None ? THPVariable_Unpack(a[6]) : empty_of(dy.sizes(), dy, at::kBFloat16);
            at::Tensor ws;
            if (a[4] != Py_None) {
                dw = empty_of({dy.size(-1)}, dy, at::kFloat);
                db = empty_of({dy.size(-1)}, dy, at::kFloat);
                ws = workspace_of(Py_None, norm_bwd_bytes_f(&p), dy);
            }
            status = norm_bwd_f(&p, dy.data_ptr(), packed ? nullptr : x->data_ptr(), packed ? x->data_ptr() : nullptr,
                                packed ? (const float*)scales->data_ptr() : nullptr, (const float*)mean.data_ptr(),
                                (const float*)rstd.data_ptr(), ptr_or_null(a[4]), ptr_or_null(a[5]), dx.data_ptr(),
                                dw.defined() ? (float*)dw.data_ptr() : nullptr, db.defined() ? (float*)db.data_ptr() : nullptr,
                                ws.defined() ? ws.data_ptr() : nullptr, ws.defined() ? (size_t)ws.numel() : 0, current_stream());
        }
        if (status != VA_OK) return PyLong_FromLong(status);
        PyObject* r = tuple_of({&dx, &dw, &db});
        if (r && a[6] != Py_None) { Py_INCREF(a[6]); PyTuple_SetItem(r, 0, a[6]); }
        return r;
    });
}
