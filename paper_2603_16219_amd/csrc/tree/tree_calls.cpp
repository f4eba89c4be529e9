// The wrappers of calls with trees on arguments that need nothing done to them, in native code: the checks, the outputs and the call of the
// library.  Small calls wait for the host otherwise.
//
// Every function returns the wrapper's result, an integer (the library's status, not 0), or None for arguments that it leaves to the wrapper:
// whatever has to be converted, copied or refused, what is no plain GPU tensor, and tensors of another device than the current one.  No device
// code here.
#include "../calls_common.hpp"

#include <c10/core/impl/DeviceGuardImplInterface.h>

#include <cmath>

#include "specsteer_tree.h"

namespace {

// The library that the binding has loaded.
struct Library {
    decltype(&specsteer_tree_attention_workspace_bytes) attention_workspace_bytes;
    decltype(&specsteer_tree_attention) attention;
    decltype(&specsteer_tree_verify_workspace_bytes) verify_workspace_bytes;
    decltype(&specsteer_tree_verify) verify;
    decltype(&specsteer_tree_commit) commit;
} lib;

bool on_current_device(const at::Tensor& t) { return c10::impl::getDeviceGuardImpl(c10::DeviceType::CUDA)->getDevice() == t.device(); }

bool strides_of(const at::Tensor& t, int64_t (&s)[3]) {
    if (t.dim() != 4 || t.numel() == 0 || t.stride(3) != 1 || (reinterpret_cast<uintptr_t>(t.data_ptr()) & 15)) return false;
    for (int i = 0; i < 3; ++i) {
        if (t.size(i) > INT32_MAX) return false;
        s[i] = t.size(i) > 1 ? t.stride(i) : 0;
        if (t.size(i) > 1 && (s[i] <= 0 || (s[i] & 7))) return false;
    }
    return true;
}

// Integers of 32 bits of this shape; a null with `ok` unset if they are something else, with `ok` as it is for None where that may be.
const at::Tensor* ints_of(PyObject* o, const at::Tensor& like, int64_t n, int64_t m, bool may_miss, bool& ok) {
    if (o == Py_None) {
        ok = ok && may_miss;
        return nullptr;
    }
    const at::Tensor* t = ready(o, at::kInt, like);
    ok = ok && t && (m < 0 ? t->dim() == 1 && t->size(0) == n : t->dim() == 2 && t->size(0) == n && t->size(1) == m);
    return ok ? t : nullptr;
}
const int32_t* ints(const at::Tensor* t) { return t ? static_cast<const int32_t*>(t->data_ptr()) : nullptr; }

// The block's keys and values, the caches and the table, all on the current device.
struct Cache {
    const at::Tensor *k, *v, *kc, *vc, *table;
};
bool describe(PyObject* const* a, ss_tree_params& p, Cache& c) {
    c = Cache{gpu_tensor(a[0]), gpu_tensor(a[1]), gpu_tensor(a[2]), gpu_tensor(a[3]), gpu_tensor(a[4])};
    if (!c.k || !c.v || !c.kc || !c.vc || !c.table) return false;
    const at::Tensor &k = *c.k, &kc = *c.kc, &t = *c.table;
    if (k.scalar_type() != at::kBFloat16 && k.scalar_type() != at::kHalf) return false;
    if (!strides_of(k, p.k_stride) || !strides_of(kc, p.cache_stride) || !same_form(k, *c.v) || !same_form(kc, *c.vc)) return false;
    if ((reinterpret_cast<uintptr_t>(c.v->data_ptr()) | reinterpret_cast<uintptr_t>(c.vc->data_ptr())) & 15) return false;
    if (kc.scalar_type() != k.scalar_type() || kc.device() != k.device() || kc.size(2) != k.size(2) || kc.size(3) != k.size(3)) return false;
    if (t.scalar_type() != at::kInt || t.device() != k.device() || t.dim() != 2 || t.size(0) != k.size(0) || t.size(1) < 1 || t.size(1) > INT32_MAX ||
        !t.is_contiguous() || !on_current_device(k))
        return false;
    p.batch = (int32_t)k.size(0);
    p.nodes = (int32_t)(k.size(1) - 1);
    p.heads = p.kv_heads = (int32_t)k.size(2);
    p.head_dim = (int32_t)(k.size(3) <= INT32_MAX ? k.size(3) : 0);
    p.dtype = k.scalar_type() == at::kHalf ? SS_TREE_F16 : SS_BF16;
    p.pages = (int32_t)kc.size(0);
    p.page_size = (int32_t)kc.size(1);
    p.table_width = (int32_t)t.size(1);
    p.table_stride = 0;
    p.scale = 0.f;
    for (int i = 0; i < 3; ++i) p.q_stride[i] = p.out_stride[i] = 0;
    return true;
}

bool workspace_of(PyObject* o, const at::Tensor& like, size_t need, at::Tensor& out) {
    if (o == Py_None) {
        out = make(like, {(int64_t)(need > 256 ? need : 256)}, at::kByte);
        return true;
    }
    const at::Tensor* t = gpu_tensor(o);
    if (!t || !t->is_contiguous() || t->device() != like.device()) return false;
    out = *t;
    return true;
}

// Autograd learns that a tensor of the caller's was written.
void written(const at::Tensor& t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// attention(q, k, v, k_cache, v_cache, block_table, cache_len, parents, tree_len, scale, out, workspace)
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 12) Py_RETURN_NONE;
    ss_tree_params p;
    Cache c;
    const at::Tensor* q = gpu_tensor(a[0]);
    if (!q || !describe(a + 1, p, c) || !strides_of(*q, p.q_stride)) Py_RETURN_NONE;
    if (q->scalar_type() != c.k->scalar_type() || q->device() != c.k->device() || q->size(0) != p.batch || q->size(1) != p.nodes + 1 || q->size(3) != p.head_dim ||
        q->size(2) % p.kv_heads || (p.head_dim != 64 && p.head_dim != 128))
        Py_RETURN_NONE;
    bool ok = true;
    const at::Tensor* len = ints_of(a[6], *q, p.batch, -1, false, ok);
    const at::Tensor* parents = ints_of(a[7], *q, p.batch, p.nodes, true, ok);
    const at::Tensor* tree = ints_of(a[8], *q, p.batch, -1, true, ok);
    if (!ok) Py_RETURN_NONE;
    p.heads = (int32_t)q->size(2);
    if (a[9] == Py_None) p.scale = (float)(1.0 / std::sqrt((double)p.head_dim));
    else if (!number(a[9], p.scale)) Py_RETURN_NONE;
    at::Tensor out, ws;
    if (a[10] == Py_None) {
        out = make(*q, q->sizes(), q->scalar_type());
    } else {
        const at::Tensor* t = gpu_tensor(a[10]);
        if (!t || t->sizes() != q->sizes() || t->scalar_type() != q->scalar_type() || t->device() != q->device() || !strides_of(*t, p.out_stride)) Py_RETURN_NONE;
        for (const at::Tensor* in : {q, c.k, c.v, c.kc, c.vc})
            if (in->storage().data() == t->storage().data()) Py_RETURN_NONE;
        out = *t;
    }
    if (!workspace_of(a[11], *q, lib.attention_workspace_bytes(&p), ws)) Py_RETURN_NONE;
    void* stream;
    if (!stream_of(*q, stream)) return nullptr;
    const ss_status rc = unlocked([&] {
        return lib.attention(q->data_ptr(), c.k->data_ptr(), c.v->data_ptr(), c.kc->data_ptr(), c.vc->data_ptr(), ints(c.table), ints(len), ints(parents), ints(tree),
                             &p, out.data_ptr(), ws.data_ptr(), ws.nbytes(), stream);
    });
    if (rc != SS_OK) return PyLong_FromLong(rc);
    if (a[10] != Py_None) {
        written(out);
        return Py_NewRef(a[10]);
    }
    return THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}

// verify(G, S_ctx, S_noctx, tokens, uniforms, parents, lam, beta, temperature, tree_len, greedy, workspace)
PyObject* verify(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 12) Py_RETURN_NONE;
    const at::Tensor *g = gpu_tensor(a[0]), *sp = gpu_tensor(a[1]), *sm = gpu_tensor(a[2]);
    if (!g || !sp || !sm || g->dim() != 3 || g->numel() == 0 || !same_form(*g, *sp) || !same_form(*g, *sm) || !on_current_device(*g)) Py_RETURN_NONE;
    if (g->scalar_type() != at::kFloat && g->scalar_type() != at::kBFloat16) Py_RETURN_NONE;
    for (int i = 0; i < 3; ++i)
        if (g->size(i) > INT32_MAX) Py_RETURN_NONE;
    const int64_t B = g->size(0), R = g->size(1), V = g->size(2);
    if (g->stride(2) != 1 || (B > 1 && g->stride(0) == 0) || (R > 1 && g->stride(1) == 0)) Py_RETURN_NONE;
    bool ok = true, greedy;
    const at::Tensor* y = ints_of(a[3], *g, B, R - 1, false, ok);
    const at::Tensor* u = ready(a[4], at::kFloat, *g);
    const at::Tensor* parents = ints_of(a[5], *g, B, R - 1, true, ok);
    const at::Tensor* tree = ints_of(a[9], *g, B, -1, true, ok);
    ss_params p{(int32_t)B, (int32_t)(R - 1), (int32_t)V, g->scalar_type() == at::kFloat ? SS_F32 : SS_BF16, B > 1 ? g->stride(0) : 0, R > 1 ? g->stride(1) : 0, 0.f, 0.f, 0.f, 0u};
    if (!ok || !u || u->dim() != 2 || u->size(0) != B || u->size(1) != R || !number(a[6], p.lambda) || !number(a[7], p.beta) || !number(a[8], p.temperature) ||
        !truth(a[10], greedy))
        Py_RETURN_NONE;
    p.flags = greedy ? SS_FLAG_GREEDY : 0u;
    at::Tensor ws;
    if (!workspace_of(a[11], *g, lib.verify_workspace_bytes(&p), ws)) Py_RETURN_NONE;
    const at::Tensor len = make(*g, {B}, at::kInt), path = make(*g, {B, R - 1}, at::kInt), token = make(*g, {B}, at::kInt), lp = make(*g, {B}, at::kFloat);
    void* stream;
    if (!stream_of(*g, stream)) return nullptr;
    const ss_status rc = unlocked([&] {
        return lib.verify(g->data_ptr(), sp->data_ptr(), sm->data_ptr(), ints(y), ints(parents), ints(tree), static_cast<const float*>(u->data_ptr()), &p, ptr<int32_t>(len),
                          ptr<int32_t>(path), ptr<int32_t>(token), ptr<float>(lp), ws.data_ptr(), ws.nbytes(), stream);
    });
    if (rc != SS_OK) return PyLong_FromLong(rc);
    PyObject* out = PyDict_New();
    if (out && !(put(out, "accepted_len", len) && put(out, "path", path) && put(out, "next_token", token) && put(out, "next_token_logprob", lp))) Py_CLEAR(out);
    return out;
    END_HANDLE_TH_ERRORS
}

// commit(k, v, k_cache, v_cache, block_table, cache_len, accepted_len, path)
PyObject* commit(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 8) Py_RETURN_NONE;
    ss_tree_params p;
    Cache c;
    if (!describe(a, p, c) || (p.head_dim & 7) || p.head_dim < 8 || p.head_dim > 1024) Py_RETURN_NONE;
    for (const at::Tensor* in : {c.k, c.v})
        if (in->storage().data() == c.kc->storage().data() || in->storage().data() == c.vc->storage().data()) Py_RETURN_NONE;
    bool ok = true;
    const at::Tensor *len = ints_of(a[5], *c.k, p.batch, -1, false, ok), *accepted = ints_of(a[6], *c.k, p.batch, -1, false, ok);
    const at::Tensor* path = ints_of(a[7], *c.k, p.batch, p.nodes, true, ok);
    if (!ok) Py_RETURN_NONE;
    const at::Tensor out = make(*c.k, {p.batch}, at::kInt);
    void* stream;
    if (!stream_of(*c.k, stream)) return nullptr;
    const ss_status rc = unlocked([&] {
        return lib.commit(c.k->data_ptr(), c.v->data_ptr(), c.kc->data_ptr(), c.vc->data_ptr(), ints(c.table), ints(len), ints(accepted), ints(path), &p,
                          ptr<int32_t>(out), stream);
    });
    if (rc != SS_OK) return PyLong_FromLong(rc);
    written(*c.kc);
    written(*c.vc);
    return THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}

// use(attention_workspace_bytes, attention, verify_workspace_bytes, verify, commit, current_raw_stream): the library's functions by their addresses,
// and what gives torch's current stream on a device
PyObject* use(PyObject*, PyObject* const* a, Py_ssize_t n) {
    constexpr int kFunctions = 5;
    if (n != kFunctions + 1) return PyErr_Format(PyExc_TypeError, "six arguments");
    void* f[kFunctions];
    for (int i = 0; i < kFunctions; ++i) {
        f[i] = PyLong_AsVoidPtr(a[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    lib.attention_workspace_bytes = reinterpret_cast<decltype(lib.attention_workspace_bytes)>(f[0]);
    lib.attention = reinterpret_cast<decltype(lib.attention)>(f[1]);
    lib.verify_workspace_bytes = reinterpret_cast<decltype(lib.verify_workspace_bytes)>(f[2]);
    lib.verify = reinterpret_cast<decltype(lib.verify)>(f[3]);
    lib.commit = reinterpret_cast<decltype(lib.commit)>(f[4]);
    Py_INCREF(a[kFunctions]);
    Py_XSETREF(current_raw_stream, a[kFunctions]);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"use", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(use)), METH_FASTCALL, nullptr},
    {"attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(attention)), METH_FASTCALL, nullptr},
    {"verify", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(verify)), METH_FASTCALL, nullptr},
    {"commit", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(commit)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tree_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tree_calls(void) { return PyModule_Create(&module); }
