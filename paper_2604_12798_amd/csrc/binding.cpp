// CPython module `_native`: the C ABI of libvfa.so (vfa.h) as Python functions with the same names and the same arguments in the
// same order, returning the status code.  Pointers are integers or None.  It checks no tensors (the package's __init__.py does).
// Converting the twenty arguments of a call that is refused at once takes 2.6 us through ctypes, one object at a time, and 0.2 us
// here (measured on the host; a step of two calls got 6.4 us shorter).  The conversions follow from the declared argument types, so
// a signature that changes in vfa.h changes here by itself.
//
// What the wrappers of __init__.py look up on every call, is_cuda, dtype, is_contiguous(), shape and data_ptr() of up to seven objects,
// is looked up here too (check_qkv, check_cache, bytes_of): the same attributes in the same order, so that whatever has them works as
// before, without an interpreter step for each.  Host time of a call, launches included, before / after in us: vfa_attn_fwd 7.1 / 5.3,
// an append and a decode step 12.4 / 10.2.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cstddef>
#include <cstdint>
#include <limits>
#include <tuple>
#include <type_traits>
#include <utility>

#include "vfa.h"

namespace {

// Whole numbers (and what has __index__): the low bits of the C type, as ctypes takes them; the entry point judges the range.
template <typename T, std::enable_if_t<std::is_integral_v<T>, int> = 0>
bool convert(PyObject* o, T& v) {
    v = (T)PyLong_AsUnsignedLongLongMask(o);
    return !(v == (T)-1 && PyErr_Occurred());
}
bool convert(PyObject* o, float& v) {
    v = (float)PyFloat_AsDouble(o);
    return !(v == -1.f && PyErr_Occurred());
}

// Attribute and method names, made once when the module is loaded.
struct Names {
    PyObject *data_ptr, *is_cuda, *dtype, *is_contiguous, *dim, *shape, *numel, *element_size, *get_device, *stride;
    bool make() {
        return (data_ptr = PyUnicode_InternFromString("data_ptr")) && (is_cuda = PyUnicode_InternFromString("is_cuda")) &&
               (dtype = PyUnicode_InternFromString("dtype")) && (is_contiguous = PyUnicode_InternFromString("is_contiguous")) &&
               (dim = PyUnicode_InternFromString("dim")) && (shape = PyUnicode_InternFromString("shape")) &&
               (numel = PyUnicode_InternFromString("numel")) && (element_size = PyUnicode_InternFromString("element_size")) &&
               (get_device = PyUnicode_InternFromString("get_device")) && (stride = PyUnicode_InternFromString("stride"));
    }
} names;

// A new reference that is given back at the end of the scope.
struct Ref {
    PyObject* o;
    explicit Ref(PyObject* x) : o(x) {}
    ~Ref() { Py_XDECREF(o); }
    Ref(const Ref&) = delete;
    Ref& operator=(const Ref&) = delete;
};
Ref attribute(PyObject* o, PyObject* name) { return Ref(PyObject_GetAttr(o, name)); }
Ref method(PyObject* o, PyObject* name) { return Ref(PyObject_CallMethodNoArgs(o, name)); }
// 1 = true, 0 = false, -1 = an error is set
int truth(const Ref& r) { return r.o ? PyObject_IsTrue(r.o) : -1; }

template <typename T>
bool convert(PyObject* o, T*& v) {
    v = nullptr;
    if (o == Py_None) return true;
    if (!PyLong_Check(o)) {
        PyErr_SetString(PyExc_TypeError, "a pointer is an integer or None");
        return false;
    }
    v = reinterpret_cast<T*>((uintptr_t)PyLong_AsUnsignedLongLongMask(o));
    return true;
}
// Whole numbers of the serving operators, whose lengths and positions users count in Python: one that its type does not hold makes the call a refused one
// (`held`), as the entry point would refuse it if it saw it.
template <typename T>
bool convert_held(PyObject* o, T& v, bool& held) {
    if constexpr (!std::is_integral_v<T>) {
        return convert(o, v);
    } else if constexpr (std::is_signed_v<T>) {
        int past = 0;
        const long long x = PyLong_AsLongLongAndOverflow(o, &past);
        if (x == -1 && !past && PyErr_Occurred()) return false;
        held = held && !past && x >= std::numeric_limits<T>::min() && x <= std::numeric_limits<T>::max();
        v = (T)x;
        return true;
    } else {
        static_assert(sizeof(T) == sizeof(unsigned long long));
        const Ref i(PyNumber_Index(o));
        if (!i.o) return false;
        v = (T)PyLong_AsUnsignedLongLong(i.o);
        if (v != (T)-1 || !PyErr_Occurred()) return true;
        if (!PyErr_ExceptionMatches(PyExc_OverflowError)) return false;
        PyErr_Clear();
        held = false;
        return true;
    }
}
template <bool TENSORS, bool HELD, typename T>
bool convert_any(PyObject* o, T& v, bool& held) {
    if constexpr (TENSORS && std::is_pointer_v<T>) {
        if (o == Py_None) return convert(o, v);
        const Ref p = method(o, names.data_ptr);
        return p.o && convert(p.o, v);
    } else if constexpr (HELD) {
        return convert_held(o, v, held);
    } else {
        return convert(o, v);
    }
}

// REFUSED: nothing, or what the function returns for arguments that it does not take
template <bool TENSORS, auto... REFUSED, typename R, typename... A, size_t... I>
PyObject* call(R (*f)(A...), PyObject* const* args, Py_ssize_t n, std::index_sequence<I...>) {
    if (n != (Py_ssize_t)sizeof...(A)) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", (Py_ssize_t)sizeof...(A), n);
        return nullptr;
    }
    std::tuple<A...> v{};
    bool held = true;
    const bool ok = (convert_any<TENSORS && I + 1 < sizeof...(A), sizeof...(REFUSED) != 0>(args[I], std::get<I>(v), held) && ...);
    if (!ok) return nullptr;
    if (!held) return PyLong_FromLongLong((0LL + ... + REFUSED));
    R r;
    Py_BEGIN_ALLOW_THREADS  // (as ctypes does: other threads run while the launches are enqueued)
    r = f(std::get<I>(v)...);
    Py_END_ALLOW_THREADS
    return std::is_unsigned_v<R> ? PyLong_FromUnsignedLongLong((unsigned long long)r) : PyLong_FromLongLong((long long)r);
}
template <bool TENSORS, auto F, auto... REFUSED>
struct Wrap;
template <bool TENSORS, typename R, typename... A, R (*F)(A...), auto... REFUSED>
struct Wrap<TENSORS, F, REFUSED...> {
    static PyObject* run(PyObject*, PyObject* const* args, Py_ssize_t n) { return call<TENSORS, REFUSED...>(F, args, n, std::index_sequence_for<A...>{}); }
};

// is_cuda, dtype, is_contiguous() and, unless dims < 0, dim() of a tensor are as they have to be: 1, 0, or -1 with an error set
int is_as_wanted(PyObject* t, PyObject* dtype, long dims) {
    int ok = truth(attribute(t, names.is_cuda));
    if (ok != 1) return ok;
    {
        const Ref d = attribute(t, names.dtype);
        ok = d.o ? PyObject_RichCompareBool(d.o, dtype, Py_EQ) : -1;
        if (ok != 1) return ok;
    }
    ok = truth(method(t, names.is_contiguous));
    if (ok != 1 || dims < 0) return ok;
    const Ref d = method(t, names.dim);
    if (!d.o) return -1;
    const long n = PyLong_AsLong(d.o);
    return n == -1 && PyErr_Occurred() ? -1 : n == dims;
}

// entries [0, n) of a shape
bool entries(const Ref& shape, Py_ssize_t n, bool all, long long* v) {
    if (!shape.o) return false;
    const Ref fast(PySequence_Fast(shape.o, "a shape is a sequence"));
    if (!fast.o) return false;
    const Py_ssize_t have = PySequence_Fast_GET_SIZE(fast.o);
    if (have < n || (all && have != n)) {
        PyErr_Format(PyExc_ValueError, "a shape of %zd entries was expected, not of %zd", n, have);
        return false;
    }
    for (Py_ssize_t i = 0; i < n; ++i) {
        v[i] = PyLong_AsLongLong(PySequence_Fast_GET_ITEM(fast.o, i));
        if (v[i] == -1 && PyErr_Occurred()) return false;
    }
    return true;
}

// check_qkv(Q, K, V, bfloat16) -> (B, Hq, Hkv, N, d)
PyObject* check_qkv(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 4) return PyErr_Format(PyExc_TypeError, "expected 4 arguments, got %zd", n);
    for (int i = 0; i < 3; ++i) {
        const int ok = is_as_wanted(args[i], args[3], 4);
        if (ok < 0) return nullptr;
        if (!ok) return PyErr_Format(PyExc_ValueError, "Q, K, V must be contiguous 4-d bf16 tensors on the GPU");
    }
    const Ref qs = attribute(args[0], names.shape), ks = attribute(args[1], names.shape), vs = attribute(args[2], names.shape);
    long long q[4], k[4];
    if (!entries(qs, 4, true, q) || !entries(ks, 4, true, k) || !vs.o) return nullptr;
    const int differ = PyObject_RichCompareBool(ks.o, vs.o, Py_NE);
    if (differ < 0) return nullptr;
    if (differ || k[0] != q[0] || k[2] != q[2] || k[3] != q[3])
        return PyErr_Format(PyExc_ValueError, "K, V must be [B, Hkv, N, d] matching Q [B, Hq, N, d]");
    return Py_BuildValue("(LLLLL)", q[0], q[1], k[1], q[2], q[3]);
}

// check_cache(q, K, V, bfloat16 or None) -> (B, Hq, d, Hkv, n_cap); None: the tensors' types are not looked at
PyObject* check_cache(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 4) return PyErr_Format(PyExc_TypeError, "expected 4 arguments, got %zd", n);
    long long q[3], k[3];
    if (!entries(attribute(args[0], names.shape), 3, true, q) || !entries(attribute(args[1], names.shape), 3, false, k)) return nullptr;
    for (int i = 0; i < 3 && args[3] != Py_None; ++i) {
        const int ok = is_as_wanted(args[i], args[3], -1);
        if (ok < 0) return nullptr;
        if (!ok) return PyErr_Format(PyExc_ValueError, "q, K, V must be contiguous bf16 tensors on the GPU");
    }
    return Py_BuildValue("(LLLLL)", q[0], q[1], q[2], k[1], k[2]);
}

// bytes_of(t): numel() * element_size()
PyObject* bytes_of(PyObject*, PyObject* t) {
    const Ref n = method(t, names.numel);
    if (!n.o) return nullptr;
    const Ref e = method(t, names.element_size);
    return e.o ? PyNumber_Multiply(n.o, e.o) : nullptr;
}

// The serving operators' tensors: 1, 0, or -1 with an error set, as above.  All of them lie on one GPU, whose index goes to `device` (-1 at first).
int on_device(PyObject* t, PyObject* dtype, long& device) {
    {
        const Ref d = attribute(t, names.dtype);
        const int ok = d.o ? PyObject_RichCompareBool(d.o, dtype, Py_EQ) : -1;
        if (ok != 1) return ok;
    }
    const Ref i = method(t, names.get_device);
    const long at = i.o ? PyLong_AsLong(i.o) : -1;
    if (at == -1 && PyErr_Occurred()) return -1;
    if (device < 0) device = at;
    return at >= 0 && at == device;  // (-1: a tensor of the host)
}
// ... of `n` dimensions, contiguous; the shape goes to v
int whole_tensor(PyObject* t, PyObject* dtype, long& device, Py_ssize_t n, long long* v) {
    int ok = on_device(t, dtype, device);
    if (ok == 1) ok = truth(method(t, names.is_contiguous));
    if (ok != 1) return ok;
    const Ref s = attribute(t, names.shape);
    if (!s.o) return -1;
    const Py_ssize_t have = PySequence_Size(s.o);
    if (have != n) return have < 0 ? -1 : 0;
    return entries(s, n, true, v) ? 1 : -1;
}
// ... of four dimensions, the last one contiguous; shape and strides
int rows_tensor(PyObject* t, PyObject* dtype, long& device, long long* v, long long* st) {
    const int ok = on_device(t, dtype, device);
    if (ok != 1) return ok;
    const Ref s = attribute(t, names.shape), r = method(t, names.stride);
    if (!s.o || !r.o) return -1;
    const Py_ssize_t have = PySequence_Size(s.o);
    if (have != 4) return have < 0 ? -1 : 0;
    if (!entries(s, 4, true, v) || !entries(r, 4, true, st)) return -1;
    for (int i = 0; i < 3; ++i)
        if (v[i] <= 1) st[i] = 0;  // (that of an axis of one entry means nothing, and torch lets it be anything)
    return st[3] == 1 || v[3] <= 1;
}
// Lengths or positions that are one number for all, or a contiguous int32 tensor of B entries on `device`: the tensor (or None) and the number (0).
// 1, 0 (refused), or -1 with an error set
struct Lengths {
    PyObject *at = nullptr, *number = nullptr;  // (new references)
    ~Lengths() { Py_XDECREF(at); Py_XDECREF(number); }
    Lengths() = default;
    Lengths(const Lengths&) = delete;
    Lengths& operator=(const Lengths&) = delete;
    int set(PyObject* x, PyObject* int32, long device, long long B) {
        if (!PyLong_Check(x) && PyObject_HasAttr(x, names.get_device)) {
            long long n[1];
            const int ok = whole_tensor(x, int32, device, 1, n);
            if (ok != 1 || n[0] != B) return ok == 1 ? 0 : ok;
            Py_INCREF(x);
            at = x;
            number = PyLong_FromLong(0);
        } else {
            Py_INCREF(Py_None);
            at = Py_None;
            number = PyNumber_Long(x);
        }
        return number ? 1 : -1;
    }
};
const char kLengths[] = "lengths and positions are numbers, or contiguous int32 tensors of an entry for each sequence on the same GPU";
PyObject* refused(int ok, const char* what) {
    if (ok == 0) PyErr_SetString(PyExc_ValueError, what);
    return nullptr;
}
// K8, V8, KS, VS of a cache; (B, Hkv, T, d / 64) go to v
int cache8(PyObject* const* c, PyObject* uint8, long& device, long long* v) {
    long long k[6], x[5], a[3], b[3];
    int ok = whole_tensor(c[0], uint8, device, 6, k);
    if (ok == 1) ok = whole_tensor(c[1], uint8, device, 5, x);
    if (ok == 1) ok = whole_tensor(c[2], uint8, device, 3, a);
    if (ok == 1) ok = whole_tensor(c[3], uint8, device, 3, b);
    if (ok != 1) return ok;
    for (int i = 0; i < 3; ++i)
        if (x[i] != k[i] || a[i] != k[i] || b[i] != k[i]) return 0;
    for (int i = 0; i < 4; ++i) v[i] = k[i];
    return k[4] == 64 && k[5] == 64 && x[3] == 64 * k[3] && x[4] == 64;
}
const char kCache8[] = "a cache is four contiguous uint8 tensors on one GPU: K8 [B, Hkv, T, d / 64, 64, 64], V8 [B, Hkv, T, d, 64], KS and VS [B, Hkv, T]";

// check_cache8(K8, V8, KS, VS, lengths, uint8, int32) -> (device, B, Hkv, n_cap, d, seq_lens, seq_len)
PyObject* check_cache8(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 7) return PyErr_Format(PyExc_TypeError, "expected 7 arguments, got %zd", n);
    long device = -1;
    long long c[4];
    int ok = cache8(args, args[5], device, c);
    if (ok != 1) return refused(ok, kCache8);
    Lengths l;
    ok = l.set(args[4], args[6], device, c[0]);
    if (ok != 1) return refused(ok, kLengths);
    return Py_BuildValue("(lLLLLOO)", device, c[0], c[1], 64 * c[2], 64 * c[3], l.at, l.number);
}
// check_kv8_append(K, V, K8, V8, KS, VS, old, new, bfloat16, uint8, int32) -> (device, B, Hkv, n_cap, n_in, d, strides of K, strides of V,
// old_lens, new_lens, n_old, n_new)
PyObject* check_kv8_append(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 11) return PyErr_Format(PyExc_TypeError, "expected 11 arguments, got %zd", n);
    long device = -1;
    long long c[4], k[4], v[4], ks[4], vs[4];
    int ok = cache8(args + 2, args[9], device, c);
    if (ok != 1) return refused(ok, kCache8);
    ok = rows_tensor(args[0], args[8], device, k, ks);
    if (ok == 1) ok = rows_tensor(args[1], args[8], device, v, vs);
    if (ok == 1) ok = k[0] == c[0] && k[1] == c[1] && k[3] == 64 * c[3] && v[0] == k[0] && v[1] == k[1] && v[2] == k[2] && v[3] == k[3];
    if (ok != 1) return refused(ok, "K, V must be bf16 tensors [B, Hkv, n_in, d] matching the cache and on its GPU, their last dimension contiguous");
    Lengths o, m;
    ok = o.set(args[6], args[10], device, c[0]);
    if (ok == 1) ok = m.set(args[7], args[10], device, c[0]);
    if (ok == 1) ok = (o.at == Py_None) == (m.at == Py_None);
    if (ok != 1) return refused(ok, "old_lens and new_lens are both numbers, or both contiguous int32 tensors of an entry for each sequence on the same GPU");
    return Py_BuildValue("(lLLLLLLLLLLLOOOO)", device, c[0], c[1], 64 * c[2], k[2], 64 * c[3], ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], o.at, m.at, o.number,
                         m.number);
}
// check_kv8_decode(q, K8, V8, KS, VS, lengths, bfloat16, uint8, int32) -> (device, B, Hq, Hkv, n_cap, n_q, d, seq_lens, n_keys)
PyObject* check_kv8_decode(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 9) return PyErr_Format(PyExc_TypeError, "expected 9 arguments, got %zd", n);
    long device = -1;
    long long c[4], q[4] = {0, 0, 1, 0};
    int ok = cache8(args + 1, args[7], device, c);
    if (ok != 1) return refused(ok, kCache8);
    const Ref dims = method(args[0], names.dim);
    const long nd = dims.o ? PyLong_AsLong(dims.o) : -1;
    if (nd == -1 && PyErr_Occurred()) return nullptr;
    ok = nd == 3 || nd == 4;
    if (ok == 1) ok = whole_tensor(args[0], args[6], device, nd, q);
    if (ok == 1 && nd == 3) { q[3] = q[2]; q[2] = 1; }
    if (ok == 1) ok = q[0] == c[0] && q[3] == 64 * c[3];
    if (ok != 1) return refused(ok, "q must be a contiguous bf16 tensor [B, Hq, n_q, d] or [B, Hq, d] matching the cache and on its GPU");
    Lengths l;
    ok = l.set(args[5], args[8], device, c[0]);
    if (ok != 1) return refused(ok, kLengths);
    return Py_BuildValue("(lLLLLLLOO)", device, c[0], q[1], c[1], 64 * c[2], q[2], q[3], l.at, l.number);
}
// check_norm_rope(q, k, v or None, q_weight or None, k_weight or None, cos_sin or None, position, bfloat16, float32, int32) -> (device, B, N, Hq, Hkv, d,
// strides of q, of k, of v, n_pos, rot, first_pos, first)
PyObject* check_norm_rope(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 10) return PyErr_Format(PyExc_TypeError, "expected 10 arguments, got %zd", n);
    long device = -1;
    long long q[4], k[4], v[4], qs[4], ks[4], vs[4] = {0, 0, 0, 0}, w[1], table[2] = {0, 0};
    int ok = rows_tensor(args[0], args[7], device, q, qs);
    if (ok == 1) ok = rows_tensor(args[1], args[7], device, k, ks);
    if (ok == 1) ok = k[0] == q[0] && k[1] == q[1] && k[3] == q[3];
    if (ok == 1 && args[2] != Py_None) {
        ok = rows_tensor(args[2], args[7], device, v, vs);
        if (ok == 1) ok = v[0] == k[0] && v[1] == k[1] && v[2] == k[2] && v[3] == k[3];
    }
    if (ok != 1) return refused(ok, "q [B, N, Hq, d], k and v [B, N, Hkv, d] must be bf16 tensors on one GPU, their last dimension contiguous");
    for (int i = 3; i < 5; ++i) {
        if (args[i] != Py_None) ok = whole_tensor(args[i], args[7], device, 1, w);
        if (ok == 1 && args[i] != Py_None) ok = w[0] == q[3];
        if (ok != 1) return refused(ok, "weights are contiguous bf16 tensors of d entries on the same GPU");
    }
    if (args[5] != Py_None) ok = whole_tensor(args[5], args[8], device, 2, table);
    if (ok != 1) return refused(ok, "cos_sin is a contiguous fp32 tensor [n_pos, rot] on the same GPU");
    Lengths first;
    ok = first.set(args[6], args[9], device, q[0]);
    if (ok != 1) return refused(ok, kLengths);
    return Py_BuildValue("(lLLLLLLLLLLLLLLLLOO)", device, q[0], q[1], q[2], k[2], q[3], qs[0], qs[1], qs[2], ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], table[0],
                         table[1], first.at, first.number);
}
// check_tensor(t, dtype, device, shape...): a contiguous tensor of that kind
PyObject* check_tensor(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n < 4 || n > 9) return PyErr_Format(PyExc_TypeError, "expected 4 to 9 arguments, got %zd", n);
    long device = PyLong_AsLong(args[2]);
    if (device == -1 && PyErr_Occurred()) return nullptr;
    long long want[6], have[6];
    for (Py_ssize_t i = 3; i < n; ++i) {
        want[i - 3] = PyLong_AsLongLong(args[i]);
        if (want[i - 3] == -1 && PyErr_Occurred()) return nullptr;
    }
    int ok = whole_tensor(args[0], args[1], device, n - 3, have);
    for (Py_ssize_t i = 0; ok == 1 && i < n - 3; ++i) ok = have[i] == want[i];
    if (ok < 0) return nullptr;
    return PyBool_FromLong(ok);
}

#define VFA_FUNCTION(f) (PyCFunction)(void (*)(void)) & f, METH_FASTCALL, nullptr
#define VFA_METHOD(name) {#name, VFA_FUNCTION((Wrap<false, &name>::run))}
#define VFA_METHODS(name) VFA_METHOD(name), {#name "_t", VFA_FUNCTION((Wrap<true, &name>::run))}
#define VFA_HELD_METHOD(name, refused) {#name, VFA_FUNCTION((Wrap<false, &name, refused>::run))}
#define VFA_HELD_METHODS(name) VFA_HELD_METHOD(name, VFA_ERR_INVALID_ARG), {#name "_t", VFA_FUNCTION((Wrap<true, &name, VFA_ERR_INVALID_ARG>::run))}
PyMethodDef methods[] = {
    VFA_METHOD(vfa_workspace_bytes), VFA_METHODS(vfa_kblock_summary), VFA_METHODS(vfa_kblock_summary_mode),
    VFA_METHODS(fa_baseline_fwd), VFA_METHODS(fa_lazy_rescale_fwd), VFA_METHODS(fa_lazy_rescale_softexp_fwd),
    VFA_METHODS(vfa_attn_fwd), VFA_METHODS(vsa_attn_fwd), VFA_METHODS(vfa_variant_fwd),
    VFA_METHODS(vfa_kblock_summary_append), VFA_METHODS(vfa_kblock_summary_append_varlen),
    VFA_METHOD(vfa_decode_workspace_bytes), VFA_METHODS(vfa_decode_fwd), VFA_METHODS(vfa_decode_noalloc_fwd), VFA_METHODS(vfa_decode_varlen_fwd),
    VFA_METHODS(vfa_fp8_quantize), VFA_METHOD(vfa_fp8_v_bytes), VFA_METHODS(vfa_fp8_pack_v), VFA_METHODS(vfa_fp8_attn_fwd), VFA_METHODS(vfa_fp8_attn_noexp_fwd),
    VFA_METHODS(vfa_mxfp4_quantize), VFA_METHOD(vfa_mxfp4_workspace_bytes), VFA_METHODS(vfa_mxfp4_attn_fwd), VFA_METHODS(vfa_mxfp4_attn_noexp_fwd),
    VFA_HELD_METHODS(vfa_qk_norm_rope_fwd), VFA_HELD_METHODS(vfa_kv8_append), VFA_HELD_METHODS(vfa_kv8_read), VFA_HELD_METHOD(vfa_kv8_decode_splits, 1),
    VFA_HELD_METHOD(vfa_kv8_decode_workspace_bytes, 0), VFA_HELD_METHODS(vfa_kv8_decode_fwd),
    {"check_qkv", VFA_FUNCTION(check_qkv)}, {"check_cache", VFA_FUNCTION(check_cache)},
    {"check_cache8", VFA_FUNCTION(check_cache8)}, {"check_kv8_append", VFA_FUNCTION(check_kv8_append)},
    {"check_kv8_decode", VFA_FUNCTION(check_kv8_decode)}, {"check_norm_rope", VFA_FUNCTION(check_norm_rope)}, {"check_tensor", VFA_FUNCTION(check_tensor)},
    {"bytes_of", &bytes_of, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", "The C ABI of libvfa.so.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return names.make() ? PyModule_Create(&module) : nullptr; }
