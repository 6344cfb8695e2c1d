// Marshalling of the hot-path calls for Python, and of those around the frozen layer: the same checks as binding.py makes, on the tensors themselves.
//
// A call from Python took 10 us, of which the kernel of a small layer is 3: some thirty attribute reads and checks, a ctypes call with
// eleven conversions and the look-up of the current stream.  With them here it takes 3.3 to 4.4, most of it the launch (1 x 1024 x 1024,
// calls back to back 10.3 -> 4.7 us; the four calls of a 7B-shaped block at four rows 50 -> 39).  Whatever is not a plain call - a
// missing workspace, a tensor subclass, an active function or dispatch mode (torch.set_default_device installs one for good), a wrapped
// tensor, an argument that does not fit - gets None, and binding.py takes the call from there: it allocates, and it words the errors.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>

#include "../../include/fp6_linear.h"

namespace {

// the entry points of the loaded library, as binding.py found them
decltype(&fp6_linear) call_linear;
decltype(&fp6_linear_variant) call_variant;
decltype(&fp6_linear_fgq) call_fgq;
decltype(&fp5_linear) call_fp5;
decltype(&fp6_linear_v2) call_v2;
decltype(&fp6_linear_v2_bf16) call_v2_bf16;
decltype(&fp6_linear_group) call_group;
decltype(&fp6_linear_workspace_bytes) need_linear;
decltype(&fp6_linear_variant_workspace_bytes) need_variant;
decltype(&fp6_linear_fgq_workspace_bytes) need_fgq;
decltype(&fp5_linear_workspace_bytes) need_fp5;
decltype(&fp6_linear_v2_workspace_bytes) need_v2;          // of both plane-layout-2 calls
decltype(&fp6_linear_group_workspace_bytes) need_group;
PyObject* fail = nullptr;          // fail(status, name) raises

enum Kind { kLinear, kVariant, kFgq, kFp5, kV2, kV2Bf16, kKinds };
constexpr const char* kNames[kKinds] = {"fp6_linear", "fp6_linear_variant", "fp6_linear_fgq", "fp5_linear", "fp6_linear_v2",
                                        "fp6_linear_v2_bf16"};

bool modes_active()
{
    return at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set();
}

// A plain contiguous device tensor of this type, or nullptr.
const at::Tensor* plain(PyObject* o, c10::ScalarType type)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.scalar_type() != type || t.layout() != c10::kStrided || !t.is_contiguous()) return nullptr;
    const c10::DispatchKeySet keys = t.key_set();
    if (keys.has(c10::DispatchKey::Python) || keys.has(c10::DispatchKey::FuncTorchBatched) ||
        keys.has(c10::DispatchKey::FuncTorchGradWrapper) || keys.has(c10::DispatchKey::Functionalize))
        return nullptr;
    return &t;
}

bool whole(PyObject* o, int64_t* v)
{
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    *v = PyLong_AsLongLongAndOverflow(o, &overflow);
    return !overflow;
}

struct Layer {
    const void *x, *hi, *lo, *scales;
    void* y;
    int64_t M, N, K;
    const at::Tensor* X;
};

// X, planes, scales, N and K, each checked against the sizes that the others imply.
bool read_layer(PyObject* X, PyObject* hi, PyObject* lo, PyObject* scales, PyObject* n, PyObject* k, int64_t block, int64_t lo_div,
                c10::ScalarType type, Layer* l)
{
    if (!whole(n, &l->N) || !whole(k, &l->K)) return false;
    const int64_t N = l->N, K = l->K;
    if (N <= 0 || K <= 0 || N % FP6_TILE || K % FP6_TILE || N > (int64_t)1 << 30 || K > (int64_t)1 << 30) return false;
    if (block && (block < 0 || K % block)) return false;
    const at::Tensor *x = plain(X, type), *h = plain(hi, c10::kByte), *o = plain(lo, c10::kByte), *s = plain(scales, c10::kHalf);
    if (!x || !h || !o || !s || x->dim() != 2 || x->size(1) != K || x->size(0) < 1) return false;
    if (h->numel() != N * K / 2 || o->numel() != N * K / lo_div || s->numel() != N * (block ? K / block : 1)) return false;
    l->M = x->size(0);
    l->x = x->data_ptr();
    l->hi = h->data_ptr();
    l->lo = o->data_ptr();
    l->scales = s->data_ptr();
    l->X = x;
    return true;
}

bool read_out(PyObject* out, c10::ScalarType type, Layer* l)
{
    const at::Tensor* y = plain(out, type);
    if (!y || y->dim() != 2 || y->size(0) != l->M || y->size(1) != l->N) return false;
    l->y = y->data_ptr();
    return true;
}

// linear(kind, X, hi, lo, scales, N, K, block, out, workspace, variant, split_k) -> Y, or None
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t count)
{
    int64_t kind, block, variant, split_k;
    if (count != 12 || !fail || !whole(a[0], &kind) || kind < 0 || kind >= kKinds || !whole(a[7], &block) || !whole(a[10], &variant) ||
        !whole(a[11], &split_k) || variant != (int)variant || split_k != (int)split_k || modes_active())
        Py_RETURN_NONE;
    PyObject* result = nullptr;
    int status = FP6_OK;
    try {
        const c10::ScalarType type = kind == kV2Bf16 ? c10::kBFloat16 : c10::kHalf;
        Layer l;
        if (!read_layer(a[1], a[2], a[3], a[4], a[5], a[6], block, kind == kFp5 ? 8 : 4, type, &l)) Py_RETURN_NONE;
        if (kind == kFgq && block <= 0) Py_RETURN_NONE;
        const at::Tensor* ws = nullptr;
        if (a[9] == Py_None) {
            // a call that needs no workspace; one that does has it allocated by binding.py
            const int v = (int)variant, d = (int)split_k;
            const size_t need = kind == kLinear    ? need_linear(l.M, l.N, l.K)
                                : kind == kVariant ? need_variant(l.M, l.N, l.K, v, d)
                                : kind == kFgq     ? need_fgq(l.M, l.N, l.K, block, v, d)
                                : kind == kFp5     ? need_fp5(l.M, l.N, l.K, v, d)
                                                   : need_v2(l.M, l.N, l.K, v, d);
            if (need) Py_RETURN_NONE;
        } else {
            ws = plain(a[9], c10::kByte);
            if (!ws) Py_RETURN_NONE;
        }
        if (a[8] == Py_None) {
            const at::Tensor y = at::empty({l.M, l.N}, l.X->options());
            l.y = y.data_ptr();
            result = THPVariable_Wrap(y);
            if (!result) return nullptr;
        } else {
            if (!read_out(a[8], type, &l)) Py_RETURN_NONE;
            result = a[8];
            Py_INCREF(result);
        }
        void* w = ws ? ws->data_ptr() : nullptr;
        const size_t bytes = ws ? (size_t)ws->numel() : 0;
        void* stream = c10::hip::getCurrentHIPStream().stream();
        const uint16_t *x = (const uint16_t*)l.x, *s = (const uint16_t*)l.scales;
        uint16_t* y = (uint16_t*)l.y;
        Py_BEGIN_ALLOW_THREADS
        switch (kind) {
            case kLinear: status = call_linear(x, l.M, l.hi, l.lo, s, l.N, l.K, y, w, bytes, stream); break;
            case kVariant: status = call_variant(x, l.M, l.hi, l.lo, s, l.N, l.K, y, w, bytes, stream, (int)variant, (int)split_k); break;
            case kFgq: status = call_fgq(x, l.M, l.hi, l.lo, s, l.N, l.K, block, y, w, bytes, stream, (int)variant, (int)split_k); break;
            case kFp5: status = call_fp5(x, l.M, l.hi, l.lo, s, l.N, l.K, y, w, bytes, stream, (int)variant, (int)split_k); break;
            case kV2: status = call_v2(x, l.M, l.hi, l.lo, s, l.N, l.K, y, w, bytes, stream, (int)variant, (int)split_k); break;
            default: status = call_v2_bf16(x, l.M, l.hi, l.lo, s, l.N, l.K, y, w, bytes, stream, (int)variant, (int)split_k);
        }
        Py_END_ALLOW_THREADS
    } catch (...) {
        Py_XDECREF(result);          // (the allocation of Y threw, or the look-up of the stream behind it)
        Py_RETURN_NONE;
    }
    if (status == FP6_OK) return result;
    Py_DECREF(result);
    return PyObject_CallFunction(fail, "is", status, kNames[kind]);
}

// The tensors of a list's items, held while other threads may run and change the list: their memory would be given to others before the launch.
class Held {
    PyObject* p[4 * FP6_GROUP_MAX];
    int count = 0;

public:
    Held() = default;
    Held(const Held&) = delete;
    Held& operator=(const Held&) = delete;
    ~Held()
    {
        while (count) Py_DECREF(p[--count]);
    }
    void add(PyObject* o)
    {
        Py_INCREF(o);
        p[count++] = o;
    }
};

// group(layers, outs, workspace) -> list of Y, or None
PyObject* group(PyObject*, PyObject* const* a, Py_ssize_t count)
{
    if (count != 3 || !fail || modes_active()) Py_RETURN_NONE;
    auto sequence = [](PyObject* o) { return PyList_CheckExact(o) || PyTuple_CheckExact(o); };
    if (!sequence(a[0]) || !sequence(a[1])) Py_RETURN_NONE;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(a[0]);
    if (n < 1 || n > FP6_GROUP_MAX || PySequence_Fast_GET_SIZE(a[1]) < n) Py_RETURN_NONE;
    fp6_linear_problem problems[FP6_GROUP_MAX];
    PyObject* ys[FP6_GROUP_MAX];
    Held held;
    int status = FP6_OK;
    try {
        int64_t M = 0;
        for (Py_ssize_t i = 0; i < n; i++) {
            PyObject* p = PySequence_Fast_GET_ITEM(a[0], i);
            ys[i] = PySequence_Fast_GET_ITEM(a[1], i);
            Layer l;
            if (!sequence(p) || PySequence_Fast_GET_SIZE(p) != 6) Py_RETURN_NONE;
            PyObject** f = PySequence_Fast_ITEMS(p);
            if (!read_layer(f[0], f[1], f[2], f[3], f[4], f[5], 0, 4, c10::kHalf, &l) || (i && l.M != M) || !read_out(ys[i], c10::kHalf, &l))
                Py_RETURN_NONE;
            M = l.M;
            for (int k = 0; k < 4; k++) held.add(f[k]);
            problems[i] = fp6_linear_problem{(const uint16_t*)l.x, l.hi, l.lo, (const uint16_t*)l.scales, l.N, l.K, (uint16_t*)l.y};
        }
        const at::Tensor* ws = nullptr;
        if (a[2] == Py_None) {
            if (need_group(M, problems, (int)n)) Py_RETURN_NONE;
        } else {
            ws = plain(a[2], c10::kByte);
            if (!ws) Py_RETURN_NONE;
        }
        void* w = ws ? ws->data_ptr() : nullptr;
        const size_t bytes = ws ? (size_t)ws->numel() : 0;
        void* stream = c10::hip::getCurrentHIPStream().stream();
        for (Py_ssize_t i = 0; i < n; i++) Py_INCREF(ys[i]);
        Py_BEGIN_ALLOW_THREADS
        status = call_group(M, problems, (int)n, w, bytes, stream);
        Py_END_ALLOW_THREADS
    } catch (...) {
        Py_RETURN_NONE;
    }
    PyObject* list = status == FP6_OK ? PyList_New(n) : nullptr;
    for (Py_ssize_t i = 0; i < n; i++) {
        if (list) PyList_SET_ITEM(list, i, ys[i]);
        else Py_DECREF(ys[i]);
    }
    if (status != FP6_OK) return PyObject_CallFunction(fail, "is", status, "fp6_linear_group");
    return list;
}

// bind(address of each entry point in the order of the declarations above, fail)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t count)
{
    if (count != 14) return PyErr_Format(PyExc_TypeError, "bind takes thirteen addresses and a function");
    void* p[13];
    for (int i = 0; i < 13; i++) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    call_linear = (decltype(call_linear))p[0];
    call_variant = (decltype(call_variant))p[1];
    call_fgq = (decltype(call_fgq))p[2];
    call_fp5 = (decltype(call_fp5))p[3];
    call_v2 = (decltype(call_v2))p[4];
    call_v2_bf16 = (decltype(call_v2_bf16))p[5];
    call_group = (decltype(call_group))p[6];
    need_linear = (decltype(need_linear))p[7];
    need_variant = (decltype(need_variant))p[8];
    need_fgq = (decltype(need_fgq))p[9];
    need_fp5 = (decltype(need_fp5))p[10];
    need_v2 = (decltype(need_v2))p[11];
    need_group = (decltype(need_group))p[12];
    Py_INCREF(a[13]);
    PyObject* old = fail;
    fail = a[13];
    Py_XDECREF(old);
    Py_RETURN_NONE;
}

// ---- the operators around the frozen layer

decltype(&fp6_lora_group) call_lora_group;
decltype(&fp6_lora_backward) call_lora_backward;
decltype(&fp6_linear_grad) call_linear_grad;
decltype(&fp6_adamw) call_adamw;

// Checks of a call one after another; `ok` says whether all held.  Every tensor is a plain one on the current device.
struct Checked {
    bool ok = true;
    c10::DeviceIndex device = -1;

    const at::Tensor* tensor(PyObject* o, c10::ScalarType type)
    {
        const at::Tensor* t = ok ? plain(o, type) : nullptr;
        if (!t || (device >= 0 && t->device().index() != device)) {
            ok = false;
            return nullptr;
        }
        if (device < 0) {
            device = t->device().index();
            if (device != c10::hip::getCurrentHIPStream().device_index()) ok = false;
        }
        return t;
    }
    void* sized(PyObject* o, c10::ScalarType type, std::initializer_list<int64_t> sizes)
    {
        const at::Tensor* t = tensor(o, type);
        if (!t || t->dim() != (int64_t)sizes.size()) {
            ok = false;
            return nullptr;
        }
        int64_t d = 0;
        for (const int64_t n : sizes) ok = ok && t->size(d++) == n;
        return t->data_ptr();
    }
    void* flat(PyObject* o, c10::ScalarType type, int64_t count)
    {
        const at::Tensor* t = tensor(o, type);
        if (t && t->numel() != count) ok = false;
        return t ? t->data_ptr() : nullptr;
    }
    void* optional(PyObject* o, c10::ScalarType type, std::initializer_list<int64_t> sizes)
    {
        return o == Py_None ? nullptr : sized(o, type, sizes);
    }
};

struct Adapters {
    const void *x, *a, *b;
    int64_t M, N, K, rank, adapters;
    c10::ScalarType type;
};

// X [M,K], A [adapters, rank, K] and B [adapters, N, rank]
bool read_adapters(Checked& c, PyObject* X, PyObject* A, PyObject* B, Adapters* r)
{
    if (!THPVariable_CheckExact(X)) return false;
    const c10::ScalarType type = THPVariable_Unpack(X).scalar_type();
    if (type != c10::kHalf && type != c10::kBFloat16) return false;
    const at::Tensor *x = c.tensor(X, type), *a = c.tensor(A, type), *b = c.tensor(B, type);
    if (!c.ok || x->dim() != 2 || a->dim() != 3 || b->dim() != 3 || x->size(0) < 1 || x->size(1) != a->size(2) || b->size(0) != a->size(0) ||
        b->size(2) != a->size(1))
        return false;
    *r = Adapters{x->data_ptr(), a->data_ptr(), b->data_ptr(), x->size(0), b->size(1), x->size(1), a->size(1), a->size(0), type};
    return true;
}

bool read_workspace(Checked& c, PyObject* o, void** p, size_t* bytes)
{
    const at::Tensor* t = c.tensor(o, c10::kByte);
    if (!c.ok) return false;
    *p = t->data_ptr();
    *bytes = (size_t)t->numel();
    return true;
}

int type_of(c10::ScalarType t) { return t == c10::kBFloat16 ? FP6_BF16 : FP6_F16; }

// One projection of lora() and lora_group(): into `out`, or into Y where that is None.
bool read_projection(Checked& c, PyObject* X, PyObject* A, PyObject* B, PyObject* Y, PyObject* out, PyObject* hidden, Adapters* r,
                     fp6_lora_problem* p)
{
    if (!read_adapters(c, X, A, B, r)) return false;
    void* y = c.sized(Y, r->type, {r->M, r->N});
    void* o = out == Py_None ? y : c.sized(out, r->type, {r->M, r->N});
    void* h = c.optional(hidden, c10::kFloat, {r->M, r->rank});
    *p = fp6_lora_problem{(const uint16_t*)r->x, (const uint16_t*)r->a, (const uint16_t*)r->b, (const uint16_t*)y, (uint16_t*)o, (float*)h,
                          r->N, r->K, r->rank};
    return c.ok;
}

// lora(X, A, B, Y, index, scaling, hidden, out, workspace) -> out, or None
PyObject* lora(PyObject*, PyObject* const* a, Py_ssize_t count)
{
    if (count != 9 || !fail || modes_active()) Py_RETURN_NONE;
    PyObject* result = a[7] == Py_None ? a[3] : a[7];
    int status = FP6_OK;
    try {
        Checked c;
        Adapters r;
        fp6_lora_problem p;
        void* ws;
        size_t bytes;
        if (!read_projection(c, a[0], a[1], a[2], a[3], a[7], a[6], &r, &p)) Py_RETURN_NONE;
        const int32_t* index = (const int32_t*)c.optional(a[4], c10::kInt, {r.M});
        const float* scaling = (const float*)c.optional(a[5], c10::kFloat, {r.adapters});
        if (!read_workspace(c, a[8], &ws, &bytes)) Py_RETURN_NONE;
        void* stream = c10::hip::getCurrentHIPStream().stream();
        Py_INCREF(result);
        Py_BEGIN_ALLOW_THREADS
        status = call_lora_group(type_of(r.type), r.M, &p, 1, r.adapters, index, scaling, ws, bytes, stream);
        Py_END_ALLOW_THREADS
    } catch (...) {
        Py_RETURN_NONE;
    }
    if (status == FP6_OK) return result;
    Py_DECREF(result);
    return PyObject_CallFunction(fail, "is", status, "fp6_lora");
}

// lora_group(layers, index, scaling, outs or None, workspace) -> list of results, or None
PyObject* lora_group(PyObject*, PyObject* const* a, Py_ssize_t count)
{
    if (count != 5 || !fail || modes_active()) Py_RETURN_NONE;
    auto sequence = [](PyObject* o) { return PyList_CheckExact(o) || PyTuple_CheckExact(o); };
    if (!sequence(a[0]) || (a[3] != Py_None && !sequence(a[3]))) Py_RETURN_NONE;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(a[0]);
    if (n < 1 || n > FP6_GROUP_MAX || (a[3] != Py_None && PySequence_Fast_GET_SIZE(a[3]) != n)) Py_RETURN_NONE;
    fp6_lora_problem problems[FP6_GROUP_MAX];
    PyObject* results[FP6_GROUP_MAX];
    Held held;
    int status = FP6_OK;
    try {
        Checked c;
        Adapters first{}, r;
        void* ws;
        size_t bytes;
        for (Py_ssize_t i = 0; i < n; i++) {
            PyObject* l = PySequence_Fast_GET_ITEM(a[0], i);
            PyObject* out = a[3] == Py_None ? Py_None : PySequence_Fast_GET_ITEM(a[3], i);
            if (!sequence(l) || PySequence_Fast_GET_SIZE(l) != 4) Py_RETURN_NONE;
            PyObject** f = PySequence_Fast_ITEMS(l);
            if (!read_projection(c, f[0], f[1], f[2], f[3], out, Py_None, &r, &problems[i])) Py_RETURN_NONE;
            if (i == 0) first = r;
            if (r.M != first.M || r.adapters != first.adapters || r.type != first.type) Py_RETURN_NONE;
            results[i] = out == Py_None ? f[3] : out;
            for (int k = 0; k < 4; k++) held.add(f[k]);
        }
        const int32_t* index = (const int32_t*)c.optional(a[1], c10::kInt, {first.M});
        const float* scaling = (const float*)c.optional(a[2], c10::kFloat, {first.adapters});
        if (!read_workspace(c, a[4], &ws, &bytes)) Py_RETURN_NONE;
        void* stream = c10::hip::getCurrentHIPStream().stream();
        for (Py_ssize_t i = 0; i < n; i++) Py_INCREF(results[i]);
        Py_BEGIN_ALLOW_THREADS
        status = call_lora_group(type_of(first.type), first.M, problems, (int)n, first.adapters, index, scaling, ws, bytes, stream);
        Py_END_ALLOW_THREADS
    } catch (...) {
        Py_RETURN_NONE;
    }
    PyObject* list = status == FP6_OK ? PyList_New(n) : nullptr;
    for (Py_ssize_t i = 0; i < n; i++) {
        if (list) PyList_SET_ITEM(list, i, results[i]);
        else Py_DECREF(results[i]);
    }
    if (status != FP6_OK) return PyObject_CallFunction(fail, "is", status, "fp6_lora_group");
    return list;
}

// lora_backward(dY, X, hidden, A, B, dX or None, index, scaling, dA, dB, accumulate, out or None, workspace) -> (out, dA, dB), or None
PyObject* lora_backward(PyObject*, PyObject* const* a, Py_ssize_t count)
{
    if (count != 13 || !fail || modes_active() || (a[10] != Py_True && a[10] != Py_False) || (a[5] == Py_None && a[11] != Py_None))
        Py_RETURN_NONE;
    PyObject* result = a[11] == Py_None ? a[5] : a[11];
    PyObject* tuple = nullptr;
    int status = FP6_OK;
    try {
        Checked c;
        Adapters r;
        void* ws;
        size_t bytes;
        if (!read_adapters(c, a[1], a[3], a[4], &r)) Py_RETURN_NONE;
        const void* dy = c.sized(a[0], r.type, {r.M, r.N});
        const float* hidden = (const float*)c.sized(a[2], c10::kFloat, {r.M, r.rank});
        const void* dx = c.optional(a[5], r.type, {r.M, r.K});
        const int32_t* index = (const int32_t*)c.optional(a[6], c10::kInt, {r.M});
        const float* scaling = (const float*)c.optional(a[7], c10::kFloat, {r.adapters});
        float* da = (float*)c.sized(a[8], c10::kFloat, {r.adapters, r.rank, r.K});
        float* db = (float*)c.sized(a[9], c10::kFloat, {r.adapters, r.N, r.rank});
        void* out = c.optional(result, r.type, {r.M, r.K});
        if (!read_workspace(c, a[12], &ws, &bytes)) Py_RETURN_NONE;
        void* stream = c10::hip::getCurrentHIPStream().stream();
        tuple = PyTuple_Pack(3, result, a[8], a[9]);
        if (!tuple) return nullptr;
        const int accumulate = a[10] == Py_True;
        Py_BEGIN_ALLOW_THREADS
        status = call_lora_backward(type_of(r.type), (const uint16_t*)dy, (const uint16_t*)r.x, hidden, r.M, (const uint16_t*)r.a,
                                    (const uint16_t*)r.b, r.adapters, r.rank, index, scaling, (const uint16_t*)dx, (uint16_t*)out, da, db,
                                    accumulate, r.N, r.K, ws, bytes, stream);
        Py_END_ALLOW_THREADS
    } catch (...) {
        Py_XDECREF(tuple);
        Py_RETURN_NONE;
    }
    if (status == FP6_OK) return tuple;
    Py_DECREF(tuple);
    return PyObject_CallFunction(fail, "is", status, "fp6_lora_backward");
}

// linear_grad(dY, hi_t, lo_t, scales_t, ratio, N, K, format, out, workspace) -> out, or None
PyObject* linear_grad(PyObject*, PyObject* const* a, Py_ssize_t count)
{
    int64_t N, K, format;
    if (count != 10 || !fail || !whole(a[5], &N) || !whole(a[6], &K) || !whole(a[7], &format) || modes_active()) Py_RETURN_NONE;
    if (N <= 0 || K <= 0 || N % FP6_TILE || K % FP6_TILE || N > (int64_t)1 << 30 || K > (int64_t)1 << 30 || format < FP6_FORMAT_E3M1 ||
        format > FP6_FORMAT_E3M2_V2_BF16)
        Py_RETURN_NONE;
    int status = FP6_OK;
    try {
        Checked c;
        void* ws;
        size_t bytes;
        const c10::ScalarType type = format == FP6_FORMAT_E3M2_V2_BF16 ? c10::kBFloat16 : c10::kHalf;
        const at::Tensor* dy = c.tensor(a[0], type);
        if (!c.ok || dy->dim() != 2 || dy->size(1) != N || dy->size(0) < 1) Py_RETURN_NONE;
        const int64_t M = dy->size(0);
        const void *hi = c.flat(a[1], c10::kByte, N * K / 2), *lo = c.flat(a[2], c10::kByte, N * K / (format == FP6_FORMAT_E3M1 ? 8 : 4));
        const uint16_t* scales = (const uint16_t*)c.flat(a[3], c10::kHalf, K);
        const float* ratio = (const float*)c.flat(a[4], c10::kFloat, N);
        uint16_t* out = (uint16_t*)c.sized(a[8], type, {M, K});
        if (!read_workspace(c, a[9], &ws, &bytes)) Py_RETURN_NONE;
        const uint16_t* from = (const uint16_t*)dy->data_ptr();
        void* stream = c10::hip::getCurrentHIPStream().stream();
        Py_INCREF(a[8]);
        Py_BEGIN_ALLOW_THREADS
        status = call_linear_grad((int)format, from, M, hi, lo, scales, ratio, N, K, out, ws, bytes, stream);
        Py_END_ALLOW_THREADS
    } catch (...) {
        Py_RETURN_NONE;
    }
    if (status == FP6_OK) return a[8];
    Py_DECREF(a[8]);
    return PyObject_CallFunction(fail, "is", status, "fp6_linear_grad");
}

// adamw(table, items, state_bits, grad_type, copy_type, step, lr, beta1, beta2, eps, weight_decay, grad_scale, found_inf, seed) -> True, or None
PyObject* adamw(PyObject*, PyObject* const* a, Py_ssize_t count)
{
    int64_t items, bits, grad, copy, seed;
    if (count != 14 || !fail || modes_active() || !whole(a[1], &items) || !whole(a[2], &bits) || !whole(a[3], &grad) || !whole(a[4], &copy) ||
        !whole(a[13], &seed))
        Py_RETURN_NONE;
    for (int i = 7; i <= 10; i++)
        if (!PyFloat_CheckExact(a[i])) Py_RETURN_NONE;
    int status = FP6_OK;
    try {
        Checked c;
        const at::Tensor* table = c.tensor(a[0], c10::kByte);
        int32_t* step = (int32_t*)c.sized(a[5], c10::kInt, {1});
        fp6_adamw_options o{};
        if (PyFloat_CheckExact(a[6])) o.lr = PyFloat_AS_DOUBLE(a[6]);
        else o.lr_device = (const float*)c.sized(a[6], c10::kFloat, {1});
        o.beta1 = PyFloat_AS_DOUBLE(a[7]);
        o.beta2 = PyFloat_AS_DOUBLE(a[8]);
        o.eps = PyFloat_AS_DOUBLE(a[9]);
        o.weight_decay = PyFloat_AS_DOUBLE(a[10]);
        o.grad_scale = (const float*)c.optional(a[11], c10::kFloat, {1});
        o.found_inf = (const float*)c.optional(a[12], c10::kFloat, {1});
        o.seed = (uint32_t)seed;
        if (!c.ok) Py_RETURN_NONE;
        void* plan = table->data_ptr();
        void* stream = c10::hip::getCurrentHIPStream().stream();
        Py_BEGIN_ALLOW_THREADS
        status = call_adamw(plan, items, (int)bits, (int)grad, (int)copy, step, &o, stream);
        Py_END_ALLOW_THREADS
    } catch (...) {
        Py_RETURN_NONE;
    }
    if (status == FP6_OK) Py_RETURN_TRUE;
    return PyObject_CallFunction(fail, "is", status, "fp6_adamw");
}

// bind_adapters(address of each entry point in the order of the declarations above); `fail` is bind()'s
PyObject* bind_adapters(PyObject*, PyObject* const* a, Py_ssize_t count)
{
    if (count != 4) return PyErr_Format(PyExc_TypeError, "bind_adapters takes four addresses");
    void* p[4];
    for (int i = 0; i < 4; i++) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    call_lora_group = (decltype(call_lora_group))p[0];
    call_lora_backward = (decltype(call_lora_backward))p[1];
    call_linear_grad = (decltype(call_linear_grad))p[2];
    call_adamw = (decltype(call_adamw))p[3];
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"linear", (PyCFunction)(void (*)())linear, METH_FASTCALL, nullptr},
                         {"group", (PyCFunction)(void (*)())group, METH_FASTCALL, nullptr},
                         {"lora", (PyCFunction)(void (*)())lora, METH_FASTCALL, nullptr},
                         {"lora_group", (PyCFunction)(void (*)())lora_group, METH_FASTCALL, nullptr},
                         {"lora_backward", (PyCFunction)(void (*)())lora_backward, METH_FASTCALL, nullptr},
                         {"linear_grad", (PyCFunction)(void (*)())linear_grad, METH_FASTCALL, nullptr},
                         {"adamw", (PyCFunction)(void (*)())adamw, METH_FASTCALL, nullptr},
                         {"bind_adapters", (PyCFunction)(void (*)())bind_adapters, METH_FASTCALL, nullptr},
                         {"bind", (PyCFunction)(void (*)())bind, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&module); }
