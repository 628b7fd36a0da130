// The host side of a small call: checks a call's tensors, fills the descriptor and calls the C ABI, without the per-tensor Python work.
//
//   call(function address, kinds, sm_scale, l2_eps, stream, workspace or None, tensors...) -> status, or None
//
// None means that something is not as a plain call has it (another type than torch.Tensor, not in device memory, not
// contiguous, another shape or type): nothing has been called, and the Python binding goes through its own checks, which
// raise what is to be raised.  One character of `kinds` per tensor says what it must be; None stands for NULL except for k:
//   q  [B][Lq][H][D], the inputs' type (the first tensor, which names the sizes and the type)      k  [B][Lkv][H][D], likewise
//   S  [B][H][D][D] fp32    W  [H][D][D], the inputs' type    r  [Lq][D/2] fp32    a  [B][H] fp32    t  [B][Lq][H] fp32
//   g  [B][Lq][H], [B][Lq] or [B][Lq][H][D], fp32 or bf16: sets the descriptor's gate mode and type
// Calls on the paged cache begin with P and take `causal` in the place of l2_eps; their descriptor is arl2_kv_desc, all of their tensors
// are on the current device, and a letter is
//   c  the pool, uint8 [n_pages][Hkv][page_size][bytes of a token]      b  [B][max_pages] int32
//   x  [B][Lq][H][D] bf16     y  [B][Lq][Hkv][D] bf16    r  [max_pages page_size][D/2] fp32    i, n  [B] int32 (n or None)
// Calls of the recurrence begin with C and take `raw_rows` in the place of sm_scale; their descriptor is arl2_scan_desc, all of their tensors are on
// the current device, and a letter is
//   q  [B][L][H][D] bf16 (the first names the sizes)     t  [B][L][H] fp32 or None     S  [B][H][D][D] fp32 or None     n  [B] int32 or None
// Calls of the rotation begin with O, the norm (n, h or r) and the pairing (0: neighbours, 1: halves), and take (axis_pairs, theta or None) in the place of
// sm_scale and norm_eps in that of l2_eps; their descriptor is arl2_rope_desc, all of their tensors are on the current device, and a letter is
//   q  [B][L][H][D] fp32 or bf16 (the first names the sizes and the type)      k  [B][L][Hk][D], likewise, or None (the first says whether there are keys)
//   x, z  like q and k, or None     w, u  the weights of queries and keys, of their type, or None     W, U  likewise, fp32     p  [L][axes] or [B][L][axes] int32
//   n  [B] int32 or None
// Measured: a call of the smallest size took 7 us to issue through ctypes, of them 3.5 in the library and the runtime.
#include <Python.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/arl2.h"

namespace {

constexpr int kMaxTensors = 13;

struct Checked {
    arl2_desc d{};
    const void *p[kMaxTensors] = {};
    bool sized = false;
};

int type_code(const at::Tensor &t)
{
    return t.scalar_type() == at::kFloat ? ARL2_F32 : t.scalar_type() == at::kBFloat16 ? ARL2_BF16 : -1;
}

bool is_shape(const at::Tensor &t, std::initializer_list<int64_t> want) { return t.sizes().equals(at::IntArrayRef(want)); }

// A plain tensor in device memory, contiguous; nullptr otherwise.
const at::Tensor *plain(PyObject *o)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.defined() && t.is_cuda() && t.is_contiguous() ? &t : nullptr;
}

bool check(Checked &c, char kind, PyObject *o, int i)
{
    arl2_desc &d = c.d;
    if (o == Py_None && i > 0) return kind != 'k';      // (keys name a size: the binding's checks refuse None)
    const at::Tensor *t = plain(o);
    if (t == nullptr) return false;
    const int type = type_code(*t);
    if (type < 0) return false;
    if (i == 0) {
        if (kind != 'q' || t->dim() != 4) return false;
        for (int64_t n : t->sizes())
            if (n > INT32_MAX) return false;
        d.B = (int32_t)t->size(0); d.Lq = d.Lkv = (int32_t)t->size(1); d.H = (int32_t)t->size(2); d.D = (int32_t)t->size(3);
        d.io_dtype = type;
    }
    const int64_t B = d.B, H = d.H, Lq = d.Lq, D = d.D;
    bool ok = false;
    switch (kind) {
    case 'q': ok = type == d.io_dtype && is_shape(*t, {B, Lq, H, D}); break;
    case 'k':
        if (!c.sized) {                       // the first of them names Lkv
            if (t->dim() != 4 || t->size(1) > INT32_MAX) return false;
            d.Lkv = (int32_t)t->size(1);
            c.sized = true;
        }
        ok = type == d.io_dtype && is_shape(*t, {B, d.Lkv, H, D});
        break;
    case 'W': ok = type == d.io_dtype && is_shape(*t, {H, D, D}); break;
    case 'S': ok = type == ARL2_F32 && is_shape(*t, {B, H, D, D}); break;
    case 'r': ok = type == ARL2_F32 && is_shape(*t, {Lq, D / 2}); break;
    case 'a': ok = type == ARL2_F32 && is_shape(*t, {B, H}); break;
    case 't': ok = type == ARL2_F32 && is_shape(*t, {B, Lq, H}); break;
    case 'g':
        d.g_dtype = type;
        d.g_mode = t->dim() == 4 ? ARL2_GATE_PER_ELEMENT : t->dim() == 2 ? ARL2_GATE_PER_TOKEN : ARL2_GATE_PER_HEAD;
        ok = t->dim() == 4 ? is_shape(*t, {B, Lq, H, D}) : t->dim() == 2 ? is_shape(*t, {B, Lq}) : is_shape(*t, {B, Lq, H});
        break;
    }
    if (ok) c.p[i] = t->data_ptr();
    return ok;
}

// The same for calls on the paged cache; the arrays that name the sizes may come after others.
bool check_kv(arl2_kv_desc &d, const char *kinds, PyObject *const *args, int n, const void **p)
{
    const at::Tensor *t[kMaxTensors] = {}, *rows = nullptr, *pool = nullptr, *table = nullptr;
    int device = -1;
    for (int i = 0; i < n; ++i) {
        if (args[i] == Py_None) {
            if (kinds[i] != 'n' && kinds[i] != 'r') return false;
            continue;
        }
        if ((t[i] = plain(args[i])) == nullptr) return false;
        if (device < 0) device = t[i]->get_device();
        if (t[i]->get_device() != device) return false;
        if ((kinds[i] == 'x' || kinds[i] == 'y') && rows == nullptr) rows = t[i];
        if (kinds[i] == 'c') pool = t[i];
        if (kinds[i] == 'b') table = t[i];
    }
    if (rows == nullptr || pool == nullptr || table == nullptr || rows->dim() != 4 || pool->dim() != 4 || table->dim() != 2) return false;
    if (device != (int)c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getDevice().index()) return false;
    for (const at::Tensor *x : {rows, pool, table})
        for (int64_t m : x->sizes())
            if (m > INT32_MAX) return false;
    const int64_t B = rows->size(0), L = rows->size(1), H = rows->size(2), D = rows->size(3), Hkv = pool->size(1), cap = table->size(1) * pool->size(2);
    d.B = (int32_t)B; d.Lq = (int32_t)L; d.H = (int32_t)H; d.D = (int32_t)D;
    d.n_pages = (int32_t)pool->size(0); d.Hkv = (int32_t)Hkv; d.page_size = (int32_t)pool->size(2); d.max_pages = (int32_t)table->size(1);
    for (int i = 0; i < n; ++i) {
        if (t[i] == nullptr) continue;
        const at::ScalarType type = t[i]->scalar_type();
        bool ok = false;
        switch (kinds[i]) {
        case 'c': ok = type == at::kByte && pool->size(3) == 2 * (D / 2 + D / 32); break;
        case 'b': ok = type == at::kInt && table->size(0) == B; break;
        case 'x': ok = type == at::kBFloat16 && is_shape(*t[i], {B, L, H, D}); break;
        case 'y': ok = type == at::kBFloat16 && is_shape(*t[i], {B, L, Hkv, D}); break;
        case 'r': ok = type == at::kFloat && is_shape(*t[i], {cap, D / 2}); break;
        case 'i': case 'n': ok = type == at::kInt && is_shape(*t[i], {B}); break;
        }
        if (!ok) return false;
        p[i] = t[i]->data_ptr();
    }
    return true;
}

// The same for calls of the recurrence.
bool check_scan(arl2_scan_desc &d, const char *kinds, PyObject *const *args, int n, const void **p)
{
    int64_t B = 0, L = 0, H = 0, D = 0;
    const int device = (int)c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getDevice().index();
    for (int i = 0; i < n; ++i) {
        if (args[i] == Py_None) {
            if (kinds[i] == 'q') return false;
            continue;
        }
        const at::Tensor *t = plain(args[i]);
        if (t == nullptr || t->get_device() != device) return false;
        if (i == 0) {
            if (t->dim() != 4) return false;
            for (int64_t m : t->sizes())
                if (m > INT32_MAX) return false;
            B = t->size(0); L = t->size(1); H = t->size(2); D = t->size(3);
            d.B = (int32_t)B; d.L = (int32_t)L; d.H = (int32_t)H; d.D = (int32_t)D;
        }
        const at::ScalarType type = t->scalar_type();
        bool ok = false;
        switch (kinds[i]) {
        case 'q': ok = type == at::kBFloat16 && is_shape(*t, {B, L, H, D}); break;
        case 't': ok = type == at::kFloat && is_shape(*t, {B, L, H}); break;
        case 'S': ok = type == at::kFloat && is_shape(*t, {B, H, D, D}); break;
        case 'n': ok = type == at::kInt && is_shape(*t, {B}); break;
        }
        if (!ok) return false;
        p[i] = t->data_ptr();
    }
    return true;
}

// The same for calls of the rotation.
bool check_rope(arl2_rope_desc &d, const char *kinds, PyObject *axes, PyObject *const *args, int n, const void **p)
{
    if (!PyTuple_CheckExact(axes) || PyTuple_GET_SIZE(axes) != 2) return false;
    PyObject *const pairs = PyTuple_GET_ITEM(axes, 0), *const theta = PyTuple_GET_ITEM(axes, 1);
    auto sequence = [](PyObject *o) { return PyTuple_CheckExact(o) || PyList_CheckExact(o); };
    if (!sequence(pairs) || (theta != Py_None && !sequence(theta))) return false;
    const Py_ssize_t n_axes = PySequence_Fast_GET_SIZE(pairs);
    if (n_axes < 1 || n_axes > 4 || (theta != Py_None && PySequence_Fast_GET_SIZE(theta) != n_axes)) return false;
    d.n_axes = (int32_t)n_axes;
    for (Py_ssize_t i = 0; i < n_axes; ++i) {
        PyObject *const m = PySequence_Fast_GET_ITEM(pairs, i);
        if (!PyLong_CheckExact(m)) return false;
        const long value = PyLong_AsLong(m);
        if (value < 0 || value > INT32_MAX) return false;
        d.axis_pairs[i] = (int32_t)value;
        if (theta == Py_None) continue;
        PyObject *const t = PySequence_Fast_GET_ITEM(theta, i);
        if (!PyFloat_CheckExact(t) && !PyLong_CheckExact(t)) return false;
        d.theta[i] = PyFloat_AsDouble(t);
    }
    if (PyErr_Occurred()) return false;
    d.norm = kinds[0] == 'h' ? ARL2_NORM_HEAD : kinds[0] == 'r' ? ARL2_NORM_ROW : ARL2_NORM_NONE;
    d.halves = kinds[1] == '1';
    kinds += 2;
    const at::Tensor *rows = nullptr, *keys = nullptr;
    bool no_keys = false;
    const int device = (int)c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getDevice().index();
    const at::Tensor *t[kMaxTensors] = {};
    for (int i = 0; i < n; ++i) {
        if (args[i] == Py_None) {
            if (kinds[i] == 'q' || kinds[i] == 'p') return false;
            if (kinds[i] == 'k' && keys == nullptr) no_keys = true;
            continue;
        }
        if ((t[i] = plain(args[i])) == nullptr || t[i]->get_device() != device) return false;
        if (kinds[i] == 'q' && rows == nullptr) rows = t[i];
        if (kinds[i] == 'k' && keys == nullptr) keys = t[i];
        if (kinds[i] == 'p' && t[i]->dim() != 2 && t[i]->dim() != 3) return false;
    }
    if (rows == nullptr || rows->dim() != 4 || (keys != nullptr && (no_keys || keys->dim() != 4))) return false;
    for (const at::Tensor *x : {rows, keys})
        for (int64_t m : x ? x->sizes() : at::IntArrayRef())
            if (m > INT32_MAX) return false;
    const int64_t B = rows->size(0), L = rows->size(1), H = rows->size(2), D = rows->size(3), Hk = keys ? keys->size(2) : 0;
    const at::ScalarType io = rows->scalar_type();
    if (type_code(*rows) < 0) return false;
    d.B = (int32_t)B; d.H = (int32_t)H; d.L = (int32_t)L; d.D = (int32_t)D; d.Hk = (int32_t)Hk; d.io_dtype = type_code(*rows);
    const bool head = d.norm == ARL2_NORM_HEAD;
    for (int i = 0; i < n; ++i) {
        if (t[i] == nullptr) continue;
        const at::ScalarType type = t[i]->scalar_type();
        bool ok = false;
        switch (kinds[i]) {
        case 'q': case 'x': ok = type == io && is_shape(*t[i], {B, L, H, D}); break;
        case 'k': case 'z': ok = type == io && is_shape(*t[i], {B, L, Hk, D}); break;
        case 'w': ok = type == io && is_shape(*t[i], {head ? D : H * D}); break;
        case 'u': ok = type == io && is_shape(*t[i], {head ? D : Hk * D}); break;
        case 'W': ok = type == at::kFloat && is_shape(*t[i], {head ? D : H * D}); break;
        case 'U': ok = type == at::kFloat && is_shape(*t[i], {head ? D : Hk * D}); break;
        case 'p':
            d.pos_per_stream = t[i]->dim() == 3;
            ok = type == at::kInt && (t[i]->dim() == 3 ? is_shape(*t[i], {B, L, n_axes}) : is_shape(*t[i], {L, n_axes}));
            break;
        case 'n': ok = type == at::kInt && is_shape(*t[i], {B}); break;
        }
        if (!ok) return false;
        p[i] = t[i]->data_ptr();
    }
    return true;
}

int invoke(void *f, const void *d, const void *const *p, int n)
{
    typedef const void *P;
    switch (n) {
    case 3: return ((int (*)(P, P, P, P))f)(d, p[0], p[1], p[2]);
    case 4: return ((int (*)(P, P, P, P, P))f)(d, p[0], p[1], p[2], p[3]);
    case 5: return ((int (*)(P, P, P, P, P, P))f)(d, p[0], p[1], p[2], p[3], p[4]);
    case 6: return ((int (*)(P, P, P, P, P, P, P))f)(d, p[0], p[1], p[2], p[3], p[4], p[5]);
    case 7: return ((int (*)(P, P, P, P, P, P, P, P))f)(d, p[0], p[1], p[2], p[3], p[4], p[5], p[6]);
    case 8: return ((int (*)(P, P, P, P, P, P, P, P, P))f)(d, p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7]);
    case 10:
        return ((int (*)(P, P, P, P, P, P, P, P, P, P, P))f)(d, p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], p[8], p[9]);
    case 12:
        return ((int (*)(P, P, P, P, P, P, P, P, P, P, P, P, P))f)(d, p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], p[8], p[9], p[10], p[11]);
    case 13:
        return ((int (*)(P, P, P, P, P, P, P, P, P, P, P, P, P, P))f)(d, p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], p[8], p[9], p[10], p[11], p[12]);
    }
    return -1;
}

PyObject *call(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    constexpr Py_ssize_t kFixed = 6;
    if (nargs <= kFixed || !PyBytes_CheckExact(args[1]) || nargs - kFixed > kMaxTensors) Py_RETURN_NONE;
    const int n = (int)(nargs - kFixed);
    const char *kinds = PyBytes_AS_STRING(args[1]);
    const bool kv = kinds[0] == 'P', scan = kinds[0] == 'C', rope = kinds[0] == 'O';
    if (PyBytes_GET_SIZE(args[1]) != n + (rope ? 3 : kv || scan)) Py_RETURN_NONE;
    void *f = PyLong_AsVoidPtr(args[0]);
    const double sm_scale = rope ? 0.0 : PyFloat_AsDouble(args[2]), l2_eps = PyFloat_AsDouble(args[3]);
    void *stream = PyLong_Check(args[4]) ? PyLong_AsVoidPtr(args[4]) : nullptr;
    if (PyErr_Occurred() || f == nullptr || !PyLong_Check(args[4])) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    if ((scan || rope) && l2_eps != 0.0 && (float)l2_eps == 0.f) Py_RETURN_NONE;      // (it would select the default)
    Checked c;
    arl2_kv_desc kd{};
    arl2_scan_desc sd{};
    arl2_rope_desc rd{};
    void *workspace = nullptr;
    size_t workspace_bytes = 0;
    try {
        if (kv) {
            if (!check_kv(kd, kinds + 1, args + kFixed, n, c.p)) Py_RETURN_NONE;
        } else if (scan) {
            if (!check_scan(sd, kinds + 1, args + kFixed, n, c.p)) Py_RETURN_NONE;
        } else if (rope) {
            if (!check_rope(rd, kinds + 1, args[2], args + kFixed, n, c.p)) {
                PyErr_Clear();
                Py_RETURN_NONE;
            }
        } else {
            for (int i = 0; i < n; ++i)
                if (!check(c, kinds[i], args[kFixed + i], i)) Py_RETURN_NONE;
        }
        if (args[5] != Py_None) {
            const at::Tensor *w = plain(args[5]);
            if (w == nullptr || ((kv || scan || rope) && w->get_device() != (int)c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getDevice().index())) Py_RETURN_NONE;
            workspace = w->data_ptr();
            workspace_bytes = w->nbytes();
        }
    } catch (...) {                           // a tensor without storage, or of a layout that has no such notion
        Py_RETURN_NONE;
    }
    if (kv) {
        kd.sm_scale = (float)sm_scale;
        kd.causal = l2_eps != 0.0;
        kd.workspace = workspace;
        kd.workspace_bytes = workspace_bytes;
        kd.stream = stream;
    }
    if (scan) {
        sd.raw_rows = sm_scale != 0.0;
        sd.l2_eps = (float)l2_eps;
        sd.workspace = workspace;
        sd.workspace_bytes = workspace_bytes;
        sd.stream = stream;
    }
    if (rope) {
        rd.norm_eps = (float)l2_eps;
        rd.workspace = workspace;
        rd.workspace_bytes = workspace_bytes;
        rd.stream = stream;
    }
    c.d.sm_scale = (float)sm_scale;
    c.d.l2_eps = (float)l2_eps;
    c.d.workspace = workspace;
    c.d.workspace_bytes = workspace_bytes;
    c.d.stream = stream;
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = invoke(f, kv ? (const void *)&kd : scan ? (const void *)&sd : rope ? (const void *)&rd : &c.d, c.p, n);
    Py_END_ALLOW_THREADS
    if (st < 0) Py_RETURN_NONE;
    return PyLong_FromLong(st);
}

PyMethodDef methods[] = {{"call", (PyCFunction)(void (*)(void))call, METH_FASTCALL, "Checks a call's tensors and calls the C ABI."},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_arl2_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__arl2_host(void)
{
    PyObject *m = PyModule_Create(&module);
    if (m != nullptr && PyModule_AddStringConstant(m, "built_for", ARL2_HOST_FOR) != 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
