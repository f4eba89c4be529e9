// The losses' wrappers on arguments that need nothing done to them, in native code: the checks, the outputs and the call of the library.  Small
// calls wait for the host otherwise (the policy loss of 9 tokens 6.5 us on the GPU).
//
// Every function returns the wrapper's result, an integer (the library's status, not 0), or None for arguments that it leaves
// to the wrapper: whatever has to be converted, copied or refused, what is no plain GPU tensor, and tensors of another device than the
// current one.  No device code here.
#include "../calls_common.hpp"

#include <c10/core/impl/DeviceGuardImplInterface.h>

#include "specsteer_alternatives.h"

namespace {

// The library that the binding has loaded.
struct Library {
    decltype(&specsteer_loss_workspace_bytes) workspace_bytes;
    decltype(&specsteer_token_logprobs) token_logprobs;
    decltype(&specsteer_token_logprobs_grad) token_logprobs_grad;
    decltype(&specsteer_policy_loss) policy_loss;
    decltype(&specsteer_preference_loss) preference_loss;
    decltype(&specsteer_token_alternatives_workspace_bytes) alternatives_workspace_bytes;
    decltype(&specsteer_token_alternatives) token_alternatives;
    decltype(&specsteer_token_alternatives_grad) token_alternatives_grad;
} lib;

// The strides of [B, T, V] with the vocabulary contiguous and no row twice, 0 where a size makes one meaningless.
bool strides_of(const at::Tensor& t, int64_t& sb, int64_t& st) {
    const int64_t B = t.size(0), T = t.size(1);
    if (t.stride(2) != 1) return false;
    sb = B > 1 ? t.stride(0) : 0;
    st = T > 1 ? t.stride(1) : 0;
    return (B == 1 || sb != 0) && (T == 1 || st != 0);
}

// Logits [B, T, V] that are not empty, on the current device.
bool describe(const at::Tensor& t, ss_loss_params& p) {
    if (t.dim() != 3 || (t.scalar_type() != at::kFloat && t.scalar_type() != at::kBFloat16)) return false;
    for (int i = 0; i < 3; ++i)
        if (t.size(i) < 1 || t.size(i) > INT32_MAX) return false;
    if (!strides_of(t, p.stride_b, p.stride_t)) return false;
    if (c10::impl::getDeviceGuardImpl(c10::DeviceType::CUDA)->getDevice() != t.device()) return false;
    p.batch = (int32_t)t.size(0);
    p.length = (int32_t)t.size(1);
    p.vocab = (int32_t)t.size(2);
    p.dtype = t.scalar_type() == at::kFloat ? SS_F32 : SS_BF16;
    p.grad_stride_b = p.grad_stride_t = 0;
    p.temperature = p.grad_scale = 1.f;
    return true;
}

bool rows_shape(const at::Tensor& t, const ss_loss_params& p) { return t.dim() == 2 && t.size(0) == p.batch && t.size(1) == p.length; }

// [B, T] of this type; NULL with `ok` unset if it is something else, with `ok` as it is for None where that may be.
const at::Tensor* rows_of(PyObject* o, at::ScalarType type, const at::Tensor& like, const ss_loss_params& p, bool may_miss, bool& ok) {
    if (o == Py_None) {
        ok = ok && may_miss;
        return nullptr;
    }
    const at::Tensor* t = ready(o, type, like);
    ok = ok && t && rows_shape(*t, p);
    return ok ? t : nullptr;
}
const at::Tensor* mask_of(PyObject* o, const at::Tensor& like, const ss_loss_params& p, bool& ok) {
    if (o == Py_None) return nullptr;
    const at::Tensor* t = ready(o, at::kBool, like);
    if (!t) t = ready(o, at::kByte, like);
    ok = ok && t && rows_shape(*t, p);
    return ok ? t : nullptr;
}

// Where the gradient goes: a tensor given for it, of memory of its own or the logits themselves, a new one, or none.
bool gradient_of(PyObject* o, bool want, const at::Tensor& logits, const at::Tensor* ref, ss_loss_params& p, at::Tensor& out) {
    if (o == Py_None) {
        if (want) out = make(logits, logits.sizes(), logits.scalar_type());
        return true;
    }
    const at::Tensor* t = gpu_tensor(o);
    if (!want || !t || t->sizes() != logits.sizes() || t->scalar_type() != logits.scalar_type() || t->device() != logits.device()) return false;
    if (!strides_of(*t, p.grad_stride_b, p.grad_stride_t)) return false;
    const void* const memory = t->storage().data();
    if (memory == logits.storage().data() && (t->data_ptr() != logits.data_ptr() || t->strides() != logits.strides())) return false;
    if (ref && memory == ref->storage().data()) return false;
    out = *t;
    return true;
}

// Autograd learns that a tensor of the caller's was written, which may be one that a backward pass has saved.
void written(PyObject* given, const at::Tensor& t) {
    if (given != Py_None && !t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

bool workspace_of(PyObject* o, const at::Tensor& logits, const ss_loss_params& p, at::Tensor& out) {
    if (o == Py_None) {
        const size_t need = lib.workspace_bytes(&p);
        out = make(logits, {(int64_t)(need > 256 ? need : 256)}, at::kByte);
        return true;
    }
    const at::Tensor* t = gpu_tensor(o);
    if (!t || !t->is_contiguous() || t->device() != logits.device()) return false;
    out = *t;
    return true;
}

const void* data(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
template <typename T>
const T* data_as(const at::Tensor* t) { return static_cast<const T*>(data(t)); }

// The dict of outputs, a null for an undefined tensor; NULL with a Python error set if it cannot be made.
PyObject* result(std::initializer_list<std::pair<const char*, const at::Tensor*>> entries) {
    PyObject* out = PyDict_New();
    for (const auto& e : entries)
        if (out && !put(out, e.first, *e.second)) Py_CLEAR(out);
    return out;
}

// token_logprobs(logits, tokens, mask, temperature, want_stats, workspace)
PyObject* token_logprobs(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 6) Py_RETURN_NONE;
    const at::Tensor* x = gpu_tensor(a[0]);
    ss_loss_params p;
    bool ok = true, want;
    if (!x || !describe(*x, p)) Py_RETURN_NONE;
    const at::Tensor *y = rows_of(a[1], at::kInt, *x, p, false, ok), *mask = mask_of(a[2], *x, p, ok);
    at::Tensor ws;
    if (!ok || !number(a[3], p.temperature) || !truth(a[4], want) || !workspace_of(a[5], *x, p, ws)) Py_RETURN_NONE;
    const at::Tensor lp = make(*x, {p.batch, p.length}, at::kFloat), stats = want ? make(*x, {p.batch, p.length, 2}, at::kFloat) : at::Tensor();
    void* stream;
    if (!stream_of(*x, stream)) return nullptr;
    const ss_status rc = unlocked([&] {
        return lib.token_logprobs(data(x), data_as<int32_t>(y), data_as<uint8_t>(mask), &p, ptr<float>(lp), ptr<float>(stats), ws.data_ptr(), ws.nbytes(), stream);
    });
    if (rc != SS_OK) return PyLong_FromLong(rc);
    return result({{"logprobs", &lp}, {"stats", &stats}});
    END_HANDLE_TH_ERRORS
}

// token_logprobs_grad(logits, tokens, stats, grad_logprobs, mask, temperature, grad_scale, grad_logits)
PyObject* token_logprobs_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 8) Py_RETURN_NONE;
    const at::Tensor* x = gpu_tensor(a[0]);
    ss_loss_params p;
    bool ok = true;
    if (!x || !describe(*x, p)) Py_RETURN_NONE;
    const at::Tensor *y = rows_of(a[1], at::kInt, *x, p, false, ok), *stats = ready(a[2], at::kFloat, *x);
    const at::Tensor *w = rows_of(a[3], at::kFloat, *x, p, false, ok), *mask = mask_of(a[4], *x, p, ok);
    if (!ok || !stats || stats->dim() != 3 || stats->size(0) != p.batch || stats->size(1) != p.length || stats->size(2) != 2) Py_RETURN_NONE;
    at::Tensor grad;
    if (!number(a[5], p.temperature) || !number(a[6], p.grad_scale) || !gradient_of(a[7], true, *x, nullptr, p, grad)) Py_RETURN_NONE;
    void* stream;
    if (!stream_of(*x, stream)) return nullptr;
    const ss_status rc = unlocked([&] {
        return lib.token_logprobs_grad(data(x), data_as<int32_t>(y), data_as<uint8_t>(mask), data_as<float>(stats), data_as<float>(w), &p, grad.data_ptr(), stream);
    });
    if (rc != SS_OK) return PyLong_FromLong(rc);
    written(a[7], grad);
    if (a[7] != Py_None) return Py_NewRef(a[7]);
    return THPVariable_Wrap(grad);
    END_HANDLE_TH_ERRORS
}

// policy_loss(logits, tokens, old_logprobs, advantages, mask, ref_logits, ref_logprobs, clip_low, clip_high, kl_coef, temperature, flags, grad_scale,
//             want_grad, grad_logits, workspace)
PyObject* policy_loss(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 16) Py_RETURN_NONE;
    const at::Tensor *x = gpu_tensor(a[0]), *z = a[5] == Py_None ? nullptr : gpu_tensor(a[5]);
    ss_loss_params p;
    ss_policy_params q;
    bool ok = true, want;
    if (!x || !describe(*x, p) || (a[5] != Py_None && (!z || !same_form(*x, *z)))) Py_RETURN_NONE;
    const at::Tensor *y = rows_of(a[1], at::kInt, *x, p, false, ok), *old = rows_of(a[2], at::kFloat, *x, p, false, ok);
    const at::Tensor *adv = ready(a[3], at::kFloat, *x), *mask = mask_of(a[4], *x, p, ok), *ref = rows_of(a[6], at::kFloat, *x, p, true, ok);
    if (!ok || !adv || (z && ref)) Py_RETURN_NONE;
    const bool each = adv->dim() == 1 && adv->size(0) == p.batch;
    if (!each && !rows_shape(*adv, p)) Py_RETURN_NONE;
    if (!number(a[7], q.clip_low) || !number(a[8], q.clip_high) || !number(a[9], q.kl_coef) || !number(a[10], p.temperature) || !PyLong_CheckExact(a[11]) ||
        !number(a[12], p.grad_scale) || !truth(a[13], want))
        Py_RETURN_NONE;
    if (q.kl_coef != 0.f && !z && !ref) Py_RETURN_NONE;
    q.flags = (uint32_t)PyLong_AsUnsignedLongMask(a[11]) | (each ? SS_LOSS_SEQ_ADVANTAGES : 0u);
    at::Tensor grad, ws;
    if (!gradient_of(a[14], want, *x, z, p, grad) || !workspace_of(a[15], *x, p, ws)) Py_RETURN_NONE;
    const at::Tensor loss = make(*x, {}, at::kFloat), lp = make(*x, {p.batch, p.length}, at::kFloat);
    const at::Tensor kl = z || ref ? make(*x, {p.batch, p.length}, at::kFloat) : at::Tensor();
    void* stream;
    if (!stream_of(*x, stream)) return nullptr;
    const ss_status rc = unlocked([&] {
        return lib.policy_loss(data(x), data(z), data_as<int32_t>(y), data_as<uint8_t>(mask), data_as<float>(old), data_as<float>(ref), data_as<float>(adv), &p, &q,
                               ptr<float>(loss), ptr<float>(lp), ptr<float>(kl), ptr<void>(grad), ws.data_ptr(), ws.nbytes(), stream);
    });
    if (rc != SS_OK) return PyLong_FromLong(rc);
    written(a[14], grad);
    PyObject* out = result({{"loss", &loss}, {"logprobs", &lp}, {"kl", &kl}, {"grad_logits", &grad}});
    if (out && a[14] != Py_None && PyDict_SetItemString(out, "grad_logits", a[14]) != 0) Py_CLEAR(out);
    return out;
    END_HANDLE_TH_ERRORS
}

// preference_loss(logits, tokens, mask, ref_logprobs, beta, label_smoothing, temperature, flags, grad_scale, want_grad, grad_logits, workspace)
PyObject* preference_loss(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 12) Py_RETURN_NONE;
    const at::Tensor* x = gpu_tensor(a[0]);
    ss_loss_params p;
    ss_preference_params q;
    bool ok = true, want;
    if (!x || !describe(*x, p) || (p.batch & 1)) Py_RETURN_NONE;
    const at::Tensor *y = rows_of(a[1], at::kInt, *x, p, false, ok), *mask = mask_of(a[2], *x, p, ok), *ref = rows_of(a[3], at::kFloat, *x, p, true, ok);
    if (!ok || !number(a[4], q.beta) || !number(a[5], q.label_smoothing) || !number(a[6], p.temperature) || !PyLong_CheckExact(a[7]) ||
        !number(a[8], p.grad_scale) || !truth(a[9], want))
        Py_RETURN_NONE;
    q.flags = (uint32_t)PyLong_AsUnsignedLongMask(a[7]);
    at::Tensor grad, ws;
    if (!gradient_of(a[10], want, *x, nullptr, p, grad) || !workspace_of(a[11], *x, p, ws)) Py_RETURN_NONE;
    const at::Tensor loss = make(*x, {}, at::kFloat), pair = make(*x, {p.batch / 2}, at::kFloat), margin = make(*x, {p.batch / 2}, at::kFloat);
    const at::Tensor lp = make(*x, {p.batch, p.length}, at::kFloat);
    void* stream;
    if (!stream_of(*x, stream)) return nullptr;
    const ss_status rc = unlocked([&] {
        return lib.preference_loss(data(x), data_as<int32_t>(y), data_as<uint8_t>(mask), data_as<float>(ref), &p, &q, ptr<float>(loss), ptr<float>(pair),
                                   ptr<float>(margin), ptr<float>(lp), ptr<void>(grad), ws.data_ptr(), ws.nbytes(), stream);
    });
    if (rc != SS_OK) return PyLong_FromLong(rc);
    written(a[10], grad);
    PyObject* out = result({{"loss", &loss}, {"pair_loss", &pair}, {"margin", &margin}, {"logprobs", &lp}, {"grad_logits", &grad}});
    if (out && a[10] != Py_None && PyDict_SetItemString(out, "grad_logits", a[10]) != 0) Py_CLEAR(out);
    return out;
    END_HANDLE_TH_ERRORS
}

// token_alternatives(logits, tokens, topk, mask, temperature, want_stats, workspace)
PyObject* token_alternatives(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 7) Py_RETURN_NONE;
    const at::Tensor* x = gpu_tensor(a[0]);
    ss_loss_params p;
    bool ok = true, want;
    if (!x || !describe(*x, p) || !PyLong_CheckExact(a[2])) Py_RETURN_NONE;
    const at::Tensor *y = rows_of(a[1], at::kInt, *x, p, true, ok), *mask = mask_of(a[3], *x, p, ok);
    int over = 0;
    const long topk = PyLong_AsLongAndOverflow(a[2], &over);
    if (!ok || over || topk < 0 || topk > SS_MAX_TOPK || !number(a[4], p.temperature) || !truth(a[5], want)) Py_RETURN_NONE;
    at::Tensor ws;
    if (a[6] == Py_None) {
        const size_t need = lib.alternatives_workspace_bytes(&p, (int32_t)topk);
        ws = make(*x, {(int64_t)(need > 256 ? need : 256)}, at::kByte);
    } else if (!workspace_of(a[6], *x, p, ws)) {
        Py_RETURN_NONE;
    }
    const at::Tensor lp = y ? make(*x, {p.batch, p.length}, at::kFloat) : at::Tensor(), entropy = make(*x, {p.batch, p.length}, at::kFloat);
    const at::Tensor top = topk ? make(*x, {p.batch, p.length, topk}, at::kInt) : at::Tensor();
    const at::Tensor top_lp = topk ? make(*x, {p.batch, p.length, topk}, at::kFloat) : at::Tensor();
    const at::Tensor stats = want ? make(*x, {p.batch, p.length, 2}, at::kFloat) : at::Tensor();
    void* stream;
    if (!stream_of(*x, stream)) return nullptr;
    const ss_status rc = unlocked([&] {
        return lib.token_alternatives(data(x), data_as<int32_t>(y), data_as<uint8_t>(mask), &p, (int32_t)topk, ptr<float>(lp), ptr<float>(entropy),
                                      ptr<int32_t>(top), ptr<float>(top_lp), ptr<float>(stats), ws.data_ptr(), ws.nbytes(), stream);
    });
    if (rc != SS_OK) return PyLong_FromLong(rc);
    return result({{"logprobs", &lp}, {"entropy", &entropy}, {"top_tokens", &top}, {"top_logprobs", &top_lp}, {"stats", &stats}});
    END_HANDLE_TH_ERRORS
}

// token_alternatives_grad(logits, tokens, stats, entropy, grad_logprobs, grad_entropy, mask, temperature, grad_scale, grad_logits)
PyObject* token_alternatives_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 10) Py_RETURN_NONE;
    const at::Tensor* x = gpu_tensor(a[0]);
    ss_loss_params p;
    bool ok = true;
    if (!x || !describe(*x, p)) Py_RETURN_NONE;
    const at::Tensor *y = rows_of(a[1], at::kInt, *x, p, true, ok), *stats = ready(a[2], at::kFloat, *x), *entropy = rows_of(a[3], at::kFloat, *x, p, true, ok);
    const at::Tensor *g = rows_of(a[4], at::kFloat, *x, p, true, ok), *k = rows_of(a[5], at::kFloat, *x, p, true, ok), *mask = mask_of(a[6], *x, p, ok);
    if (!ok || !stats || stats->dim() != 3 || stats->size(0) != p.batch || stats->size(1) != p.length || stats->size(2) != 2) Py_RETURN_NONE;
    if ((!g && !k) || (g && !y) || (k && !entropy)) Py_RETURN_NONE;
    at::Tensor grad;
    if (!number(a[7], p.temperature) || !number(a[8], p.grad_scale) || !gradient_of(a[9], true, *x, nullptr, p, grad)) Py_RETURN_NONE;
    void* stream;
    if (!stream_of(*x, stream)) return nullptr;
    const ss_status rc = unlocked([&] {
        return lib.token_alternatives_grad(data(x), data_as<int32_t>(y), data_as<uint8_t>(mask), data_as<float>(stats), data_as<float>(entropy),
                                           data_as<float>(g), data_as<float>(k), &p, grad.data_ptr(), stream);
    });
    if (rc != SS_OK) return PyLong_FromLong(rc);
    written(a[9], grad);
    if (a[9] != Py_None) return Py_NewRef(a[9]);
    return THPVariable_Wrap(grad);
    END_HANDLE_TH_ERRORS
}

// use(workspace_bytes, token_logprobs, token_logprobs_grad, policy_loss, preference_loss, alternatives_workspace_bytes, token_alternatives,
//     token_alternatives_grad, current_raw_stream): the library's functions by their addresses, and what gives torch's current stream on a device
PyObject* use(PyObject*, PyObject* const* a, Py_ssize_t n) {
    constexpr int kFunctions = 8;
    if (n != kFunctions + 1) return PyErr_Format(PyExc_TypeError, "nine arguments");
    void* f[kFunctions];
    for (int i = 0; i < kFunctions; ++i) {
        f[i] = PyLong_AsVoidPtr(a[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    lib.workspace_bytes = reinterpret_cast<decltype(lib.workspace_bytes)>(f[0]);
    lib.token_logprobs = reinterpret_cast<decltype(lib.token_logprobs)>(f[1]);
    lib.token_logprobs_grad = reinterpret_cast<decltype(lib.token_logprobs_grad)>(f[2]);
    lib.policy_loss = reinterpret_cast<decltype(lib.policy_loss)>(f[3]);
    lib.preference_loss = reinterpret_cast<decltype(lib.preference_loss)>(f[4]);
    lib.alternatives_workspace_bytes = reinterpret_cast<decltype(lib.alternatives_workspace_bytes)>(f[5]);
    lib.token_alternatives = reinterpret_cast<decltype(lib.token_alternatives)>(f[6]);
    lib.token_alternatives_grad = reinterpret_cast<decltype(lib.token_alternatives_grad)>(f[7]);
    Py_INCREF(a[kFunctions]);
    Py_XSETREF(current_raw_stream, a[kFunctions]);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"use", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(use)), METH_FASTCALL, nullptr},
    {"token_logprobs", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(token_logprobs)), METH_FASTCALL, nullptr},
    {"token_logprobs_grad", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(token_logprobs_grad)), METH_FASTCALL, nullptr},
    {"policy_loss", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(policy_loss)), METH_FASTCALL, nullptr},
    {"preference_loss", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(preference_loss)), METH_FASTCALL, nullptr},
    {"token_alternatives", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(token_alternatives)), METH_FASTCALL, nullptr},
    {"token_alternatives_grad", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(token_alternatives_grad)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_loss_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__loss_calls(void) { return PyModule_Create(&module); }
