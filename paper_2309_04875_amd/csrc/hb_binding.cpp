// Argument marshalling of the Python binding in native code: a CPython module (paper_2309_04875_amd._binding) whose functions
// take torch tensors and call the C ABI of include/hb.h.
//
// What it is for: the calls on small tensors are bound by the host, and of the 6.6 us of one (2^16 elements) 2.5 were
// spent in Python on four tensors' checks and ctypes' conversions; here they take about 0.4.  A batch of 17 tensors of one small image
// was made in 25 us and is in 2.
//
// Every function is a short cut of the Python function of the same purpose in hb.py and returns NotImplemented, having done
// nothing, for whatever it does not know at sight: tensors of a subclass, of another type or device, not contiguous or of
// different sizes, numbers that are not plain ints, a stream of the caller's, outputs left out.  The Python function then
// goes on as if it had not been called, and raises what it always raised.
#include <Python.h>

#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <initializer_list>
#include <vector>

#include "../../include/hb.h"
#include "hb_gil.hpp"

namespace {

PyObject *g_check = nullptr;      // hb._check: raises the exception of a status

PyObject *not_known() { Py_RETURN_NOTIMPLEMENTED; }

const at::Tensor *tensor_of(PyObject *o, at::ScalarType type)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.defined() && t.scalar_type() == type && t.is_cuda() && t.is_contiguous() ? &t : nullptr;
}

// Tensors of one size, whose addresses go to `at`.
class Tensors {
  public:
    template <class Pointer>
    void take(PyObject *o, at::ScalarType type, Pointer *&at)
    {
        const at::Tensor *t = ok ? tensor_of(o, type) : nullptr;
        ok = t != nullptr && (n < 0 || n == t->numel());
        if (!ok) return;
        n = t->numel();
        at = static_cast<Pointer *>(t->data_ptr());
    }
    bool ok = true;
    int64_t n = -1;
};

// Plain ints, reduced as ctypes and the mask of a seed reduce them.
bool word_of(PyObject *o, uint64_t &v)
{
    if (!PyLong_CheckExact(o)) return false;
    v = PyLong_AsUnsignedLongLongMask(o);
    return true;
}
bool int_of(PyObject *o, int &v)
{
    uint64_t w = 0;
    const bool known = word_of(o, w);
    v = (int)(uint32_t)w;
    return known;
}

// An int that is one: others are the Python function's to refuse.
bool plain_int_of(PyObject *o, int &v)
{
    if (!PyLong_CheckExact(o)) return false;
    int over = 0;
    const long w = PyLong_AsLongAndOverflow(o, &over);
    v = (int)w;
    return over == 0 && w == v;
}

void *current_stream() { return c10::hip::getCurrentHIPStream(c10::hip::current_device()).stream(); }

// The result of a call, or the exception of its status.
PyObject *checked(int st, PyObject *result)
{
    if (st == HB_OK) return result;
    Py_XDECREF(result);
    PyObject *none = PyObject_CallFunction(g_check, "i", st);
    Py_XDECREF(none);
    return nullptr;                       // hb._check has raised
}

// Runs `body`, which returns what the function returns; C++ exceptions (tensors without memory of their own) are left to the
// Python function.  They come from before the C call, which throws none, and nothing after it does.
template <class Body>
PyObject *guarded(const Body &body)
{
    try {
        return body();
    } catch (const std::exception &) {
        PyErr_Clear();                    // where the exception came out of Python code (a dispatch mode of torch)
        return not_known();
    }
}

using SharesCall = int (*)(const int64_t *, const int64_t *, size_t, int, int, uint64_t, int64_t *, int64_t *, uint64_t *, void *);
using SharesCallEx = int (*)(const int64_t *, const int64_t *, size_t, int, int, uint64_t, int, int64_t *, int64_t *, uint64_t *, void *);

// shares(which, share0, share1, k, m, seed, dealer or None, out0, out1) -> (out0, out1, opened bits)
PyObject *shares(PyObject *, PyObject *const *a, Py_ssize_t count)
{
    static const SharesCall plain[] = {hb_drelu, hb_relu, hb_sign_shares};
    static const SharesCallEx ex[] = {hb_drelu_ex, hb_relu_ex};
    return guarded([&]() -> PyObject * {
        int which = -1, k = 0, m = 0, dealer = 0;
        uint64_t seed = 0, bits = 0;
        if (count != 9 || !int_of(a[0], which) || !int_of(a[3], k) || !int_of(a[4], m) || !word_of(a[5], seed)) return not_known();
        const bool has_dealer = a[6] != Py_None;
        if (which < 0 || which >= (has_dealer ? 2 : 3) || (has_dealer && !int_of(a[6], dealer))) return not_known();
        const int64_t *s0 = nullptr, *s1 = nullptr;
        int64_t *o0 = nullptr, *o1 = nullptr;
        Tensors t;
        t.take(a[1], at::kLong, s0);
        t.take(a[2], at::kLong, s1);
        t.take(a[7], at::kLong, o0);
        t.take(a[8], at::kLong, o1);
        if (!t.ok) return not_known();
        void *stream = current_stream();
        const int st = without_gil([&] {
            return has_dealer ? ex[which](s0, s1, (size_t)t.n, k, m, seed, dealer, o0, o1, &bits, stream)
                              : plain[which](s0, s1, (size_t)t.n, k, m, seed, o0, o1, &bits, stream);
        });
        return checked(st, st == HB_OK ? Py_BuildValue("OOK", a[7], a[8], (unsigned long long)bits) : nullptr);
    });
}

// parties(relu, shares, k, m, seed, outs) -> opened bits
PyObject *parties(PyObject *, PyObject *const *a, Py_ssize_t count)
{
    return guarded([&]() -> PyObject * {
        constexpr Py_ssize_t kMost = 8;
        int relu = 0, k = 0, m = 0;
        uint64_t seed = 0, bits = 0;
        if (count != 6 || !int_of(a[0], relu) || !int_of(a[2], k) || !int_of(a[3], m) || !word_of(a[4], seed)) return not_known();
        if (!PyList_CheckExact(a[1]) || !PyList_CheckExact(a[5])) return not_known();
        const Py_ssize_t p = PyList_GET_SIZE(a[1]);
        if (p < 1 || p > kMost || PyList_GET_SIZE(a[5]) != p) return not_known();
        const int64_t *in[kMost] = {};
        int64_t *out[kMost] = {};
        Tensors t;
        for (Py_ssize_t q = 0; q < p; ++q) t.take(PyList_GET_ITEM(a[1], q), at::kLong, in[q]);
        for (Py_ssize_t q = 0; q < p; ++q) t.take(PyList_GET_ITEM(a[5], q), at::kLong, out[q]);
        if (!t.ok) return not_known();
        void *stream = current_stream();
        const int st = without_gil([&] { return (relu ? hb_relu_mp : hb_drelu_mp)(in, (int)p, (size_t)t.n, k, m, seed, out, &bits, stream); });
        return checked(st, st == HB_OK ? PyLong_FromUnsignedLongLong(bits) : nullptr);
    });
}

// batch(relu, list of (share0, share1, out0, out1, k, m, seed), dealer or None) -> opened bits
PyObject *batch(PyObject *, PyObject *const *a, Py_ssize_t count)
{
    return guarded([&]() -> PyObject * {
        int relu = 0, dealer = 0;
        if (count != 3 || !int_of(a[0], relu) || (!PyList_CheckExact(a[1]) && !PyTuple_CheckExact(a[1]))) return not_known();
        const bool has_dealer = a[2] != Py_None;
        if (has_dealer && !int_of(a[2], dealer)) return not_known();
        const Py_ssize_t items = PySequence_Fast_GET_SIZE(a[1]);
        std::vector<hb_tensor> set((size_t)items);
        for (Py_ssize_t i = 0; i < items; ++i) {
            PyObject *item = PySequence_Fast_GET_ITEM(a[1], i);
            if (!PyTuple_CheckExact(item) || PyTuple_GET_SIZE(item) != 7) return not_known();
            hb_tensor &d = set[(size_t)i];
            Tensors t;
            t.take(PyTuple_GET_ITEM(item, 0), at::kLong, d.share0);
            t.take(PyTuple_GET_ITEM(item, 1), at::kLong, d.share1);
            t.take(PyTuple_GET_ITEM(item, 2), at::kLong, d.out0);
            t.take(PyTuple_GET_ITEM(item, 3), at::kLong, d.out1);
            if (!t.ok || !int_of(PyTuple_GET_ITEM(item, 4), d.k) || !int_of(PyTuple_GET_ITEM(item, 5), d.m) ||
                !word_of(PyTuple_GET_ITEM(item, 6), d.seed))
                return not_known();
            d.n = (size_t)t.n;
        }
        uint64_t bits = 0;
        void *stream = current_stream();
        const int st = without_gil([&] {
            if (has_dealer) return (relu ? hb_relu_batch_ex : hb_drelu_batch_ex)(set.data(), set.size(), dealer, &bits, stream);
            return (relu ? hb_relu_batch : hb_drelu_batch)(set.data(), set.size(), &bits, stream);
        });
        return checked(st, st == HB_OK ? PyLong_FromUnsignedLongLong(bits) : nullptr);
    });
}

// plan_run(address of the plan) -> opened bits
PyObject *plan_run(PyObject *, PyObject *plan)
{
    return guarded([&]() -> PyObject * {
        uint64_t address = 0, bits = 0;
        if (!word_of(plan, address) || address == 0) return not_known();
        void *stream = current_stream();
        const int st = without_gil([&] { return hb_plan_run(reinterpret_cast<const hb_plan *>(address), &bits, stream); });
        return checked(st, st == HB_OK ? PyLong_FromUnsignedLongLong(bits) : nullptr);
    });
}

PyObject *given(PyObject *o)
{
    Py_INCREF(o);
    return o;
}

// sim_relu(x, k, m, seed, share_seed, out) -> out
PyObject *sim_relu(PyObject *, PyObject *const *a, Py_ssize_t count)
{
    return guarded([&]() -> PyObject * {
        int k = 0, m = 0;
        uint64_t seed = 0, share_seed = 0;
        if (count != 6 || !int_of(a[1], k) || !int_of(a[2], m) || !word_of(a[3], seed) || !word_of(a[4], share_seed)) return not_known();
        const float *x = nullptr;
        float *y = nullptr;
        Tensors t;
        t.take(a[0], at::kFloat, x);
        t.take(a[5], at::kFloat, y);
        if (!t.ok) return not_known();
        void *stream = current_stream();
        const int st = without_gil([&] { return hb_sim_relu_f32(x, (size_t)t.n, k, m, seed, share_seed, y, stream); });
        return checked(st, st == HB_OK ? given(a[5]) : nullptr);
    });
}

// share(x, share_seed, share0, share1) -> (share0, share1)
PyObject *share(PyObject *, PyObject *const *a, Py_ssize_t count)
{
    return guarded([&]() -> PyObject * {
        uint64_t seed = 0;
        if (count != 4 || !word_of(a[1], seed)) return not_known();
        const float *x = nullptr;
        int64_t *s0 = nullptr, *s1 = nullptr;
        Tensors t;
        t.take(a[0], at::kFloat, x);
        t.take(a[2], at::kLong, s0);
        t.take(a[3], at::kLong, s1);
        if (!t.ok) return not_known();
        void *stream = current_stream();
        const int st = without_gil([&] { return hb_share_f32(x, (size_t)t.n, seed, s0, s1, stream); });
        return checked(st, st == HB_OK ? PyTuple_Pack(2, a[2], a[3]) : nullptr);
    });
}

// reveal(share0, share1, out) -> out
PyObject *reveal(PyObject *, PyObject *const *a, Py_ssize_t count)
{
    return guarded([&]() -> PyObject * {
        if (count != 3) return not_known();
        const int64_t *s0 = nullptr, *s1 = nullptr;
        float *y = nullptr;
        Tensors t;
        t.take(a[0], at::kLong, s0);
        t.take(a[1], at::kLong, s1);
        t.take(a[2], at::kFloat, y);
        if (!t.ok) return not_known();
        void *stream = current_stream();
        const int st = without_gil([&] { return hb_reveal_f32(s0, s1, (size_t)t.n, y, stream); });
        return checked(st, st == HB_OK ? given(a[2]) : nullptr);
    });
}

// eco_scan(share0, share1, counts) -> counts
PyObject *eco_scan(PyObject *, PyObject *const *a, Py_ssize_t count)
{
    return guarded([&]() -> PyObject * {
        if (count != 3) return not_known();
        const int64_t *s0 = nullptr, *s1 = nullptr;
        int64_t *counts = nullptr;
        Tensors t, c;
        t.take(a[0], at::kLong, s0);
        t.take(a[1], at::kLong, s1);
        c.take(a[2], at::kLong, counts);
        if (!t.ok || !c.ok || c.n != 64) return not_known();
        void *stream = current_stream();
        const int st = without_gil([&] { return hb_eco_scan(s0, s1, (size_t)t.n, reinterpret_cast<uint64_t *>(counts), stream); });
        return checked(st, st == HB_OK ? given(a[2]) : nullptr);
    });
}

// party(share0, share1, k, m, seed, dealer or None, out0, out1, workspace) -> (out0, out1, wire 0, wire 1, wire bytes)
PyObject *party(PyObject *, PyObject *const *a, Py_ssize_t count)
{
    return guarded([&]() -> PyObject * {
        int k = 0, m = 0, dealer = 0;
        uint64_t seed = 0, bytes = 0;
        if (count != 9 || !int_of(a[2], k) || !int_of(a[3], m) || !word_of(a[4], seed)) return not_known();
        const bool has_dealer = a[5] != Py_None;
        if (has_dealer && !int_of(a[5], dealer)) return not_known();
        const int64_t *s0 = nullptr, *s1 = nullptr;
        int64_t *o0 = nullptr, *o1 = nullptr;
        Tensors t;
        t.take(a[0], at::kLong, s0);
        t.take(a[1], at::kLong, s1);
        t.take(a[6], at::kLong, o0);
        t.take(a[7], at::kLong, o1);
        const at::Tensor *workspace = tensor_of(a[8], at::kByte);
        if (!t.ok || workspace == nullptr || workspace->dim() != 1) return not_known();
        const size_t n = (size_t)t.n, workspace_bytes = (size_t)workspace->numel();
        // The views of the wires are made before the launch: what throws here has not been enqueued and may be left to the Python
        // function, which would enqueue it a second time otherwise.
        const int64_t words = (int64_t)(has_dealer ? hb_party_wire_words_ex(n, k, m, dealer) : hb_party_wire_words(n, k, m));
        THPObjectPtr wires[2];
        for (int p = 0; p < 2; ++p) {
            const int64_t at = (int64_t)(has_dealer ? hb_party_wire_offset_ex(n, k, m, dealer, p) : hb_party_wire_offset(n, k, m, p));
            wires[p] = THPVariable_Wrap(workspace->slice(0, at, at + 8 * words).view(at::kLong));
        }
        void *to = workspace->data_ptr(), *stream = current_stream();
        const int st = without_gil([&] {
            return has_dealer ? hb_relu_party_ex(s0, s1, n, k, m, seed, dealer, o0, o1, to, workspace_bytes, &bytes, stream)
                              : hb_relu_party(s0, s1, n, k, m, seed, o0, o1, to, workspace_bytes, &bytes, stream);
        });
        if (st != HB_OK) return checked(st, nullptr);
        return Py_BuildValue("OOOOK", a[6], a[7], wires[0].get(), wires[1].get(), (unsigned long long)bytes);
    });
}

// A tensor of a given type and shape (-1: any size there).
const at::Tensor *shaped(PyObject *o, at::ScalarType type, std::initializer_list<int64_t> shape)
{
    const at::Tensor *t = tensor_of(o, type);
    if (t == nullptr || (size_t)t->dim() != shape.size()) return nullptr;
    int64_t d = 0;
    for (const int64_t want : shape) {
        const int64_t have = t->size(d++);
        if (want >= 0 && have != want) return nullptr;
    }
    return t;
}
template <class Pointer>
bool take_shaped(PyObject *o, at::ScalarType type, std::initializer_list<int64_t> shape, Pointer *&at)
{
    const at::Tensor *t = shaped(o, type, shape);
    if (t == nullptr) return false;
    at = static_cast<Pointer *>(t->data_ptr());
    return true;
}

// linear(x0, x1, weight, scales, group, frac, seed, out0, out1) -> (out0, out1, opened bits)
PyObject *linear(PyObject *, PyObject *const *a, Py_ssize_t count)
{
    return guarded([&]() -> PyObject * {
        int group = 0, frac = 0;
        uint64_t seed = 0, bits = 0;
        if (count != 9 || !plain_int_of(a[4], group) || !plain_int_of(a[5], frac) || !word_of(a[6], seed) || group < 1) return not_known();
        const at::Tensor *x = tensor_of(a[0], at::kLong), *weight = shaped(a[2], at::kByte, {-1, -1});
        if (x == nullptr || weight == nullptr || x->dim() < 1) return not_known();
        const int64_t in = x->size(-1), out = weight->size(0);
        if (in < 1 || weight->size(1) != (in + 1) / 2) return not_known();
        const at::Tensor *y[2] = {tensor_of(a[7], at::kLong), tensor_of(a[8], at::kLong)}, *x1 = tensor_of(a[1], at::kLong);
        if (x1 == nullptr || x1->sizes() != x->sizes()) return not_known();
        for (const at::Tensor *t : y) {
            if (t == nullptr || t->dim() != x->dim() || t->size(-1) != out) return not_known();
            for (int64_t d = 0; d + 1 < x->dim(); ++d) {
                if (t->size(d) != x->size(d)) return not_known();
            }
        }
        const int32_t *scales = nullptr;
        if (!take_shaped(a[3], at::kInt, {out, (in + group - 1) / group}, scales)) return not_known();
        const int64_t *s0 = static_cast<const int64_t *>(x->data_ptr()), *s1 = static_cast<const int64_t *>(x1->data_ptr());
        int64_t *o0 = static_cast<int64_t *>(y[0]->data_ptr()), *o1 = static_cast<int64_t *>(y[1]->data_ptr());
        const uint8_t *w = static_cast<const uint8_t *>(weight->data_ptr());
        const size_t rows = (size_t)(x->numel() / in);
        void *stream = current_stream();
        const int st = without_gil([&] { return hb_linear_q4(s0, s1, rows, (size_t)in, (size_t)out, w, scales, group, frac, seed, o0, o1, &bits, stream); });
        return checked(st, st == HB_OK ? Py_BuildValue("OOK", a[7], a[8], (unsigned long long)bits) : nullptr);
    });
}

// The struct of a cache, from its three tensors as they are now.
bool take_cache(PyObject *const *a, hb_cache &c)
{
    const at::Tensor *keys = shaped(a[0], at::kLong, {-1, -1, -1, -1}), *values = tensor_of(a[1], at::kLong);
    if (keys == nullptr || values == nullptr || values->sizes() != keys->sizes() || !take_shaped(a[2], at::kLong, {keys->size(0)}, c.page_seeds)) return false;
    for (int64_t d = 1; d < 4; ++d) {
        if (keys->size(d) > INT32_MAX) return false;
    }
    c.keys = static_cast<int64_t *>(keys->data_ptr());
    c.values = static_cast<int64_t *>(values->data_ptr());
    c.pages = (size_t)keys->size(0);
    c.heads = (int)keys->size(1);
    c.page = (int)keys->size(2);
    c.dim = (int)keys->size(3);
    return true;
}

// cache(keys, values, page_seeds) -> the bytes of their struct hb_cache
PyObject *cache(PyObject *, PyObject *const *a, Py_ssize_t count)
{
    return guarded([&]() -> PyObject * {
        hb_cache c = {};
        if (count != 3 || !take_cache(a, c)) return not_known();
        return PyBytes_FromStringAndSize(reinterpret_cast<const char *>(&c), sizeof(c));
    });
}

// append(keys, values, page_seeds, k0, k1, v0, v1, slots, positions, cos, sin, frac, seed, q0, q1, q_mul, q_out0, q_out1) -> (q_out0, q_out1, opened bits);
// positions, cos and sin, or the queries and their outputs, may all be None
PyObject *append(PyObject *, PyObject *const *a, Py_ssize_t count)
{
    return guarded([&]() -> PyObject * {
        hb_cache c = {};
        int frac = 0, q_mul = 0;
        uint64_t seed = 0, bits = 0;
        if (count != 18 || !take_cache(a, c) || !plain_int_of(a[11], frac) || !word_of(a[12], seed) || !plain_int_of(a[15], q_mul)) return not_known();
        const at::Tensor *slots = shaped(a[7], at::kLong, {-1});
        if (slots == nullptr) return not_known();
        const int64_t tokens = slots->size(0);
        const int64_t *kv[4] = {}, *q[2] = {}, *to = static_cast<const int64_t *>(slots->data_ptr());
        for (int i = 0; i < 4; ++i) {
            if (!take_shaped(a[3 + i], at::kLong, {tokens, c.heads, c.dim}, kv[i])) return not_known();
        }
        const int32_t *positions = nullptr, *cos = nullptr, *sin = nullptr;
        int64_t rows = 0, half = 0, heads = 0;
        if (a[8] != Py_None || a[9] != Py_None || a[10] != Py_None) {
            const at::Tensor *table = shaped(a[9], at::kInt, {-1, -1});
            if (table == nullptr) return not_known();
            rows = table->size(0);
            half = table->size(1);
            cos = static_cast<const int32_t *>(table->data_ptr());
            if (half > c.dim || !take_shaped(a[10], at::kInt, {rows, half}, sin) || !take_shaped(a[8], at::kInt, {tokens}, positions)) return not_known();
        }
        int64_t *o[2] = {};
        if (a[13] != Py_None || a[14] != Py_None) {
            const at::Tensor *query = shaped(a[13], at::kLong, {tokens, -1, c.dim});
            if (query == nullptr || query->size(1) > INT32_MAX) return not_known();
            heads = query->size(1);
            q[0] = static_cast<const int64_t *>(query->data_ptr());
            if (!take_shaped(a[14], at::kLong, {tokens, heads, c.dim}, q[1])) return not_known();
            for (int i = 0; i < 2; ++i) {
                if (!take_shaped(a[16 + i], at::kLong, {tokens, heads, c.dim}, o[i])) return not_known();
            }
        }
        void *stream = current_stream();
        const int st = without_gil([&] {
            return hb_cache_append(&c, kv[0], kv[1], kv[2], kv[3], (size_t)tokens, to, positions, cos, sin, (size_t)rows, (int)(2 * half), frac, q[0], q[1],
                                   (int)heads, q_mul, seed, o[0], o[1], &bits, stream);
        });
        return checked(st, st == HB_OK ? Py_BuildValue("OOK", a[16], a[17], (unsigned long long)bits) : nullptr);
    });
}

// attention(keys, values, page_seeds, q0, q1, page_table, lens, max_len, k, m, seed, out0, out1, workspace) -> (out0, out1, opened bits)
PyObject *attention(PyObject *, PyObject *const *a, Py_ssize_t count)
{
    return guarded([&]() -> PyObject * {
        hb_cache c = {};
        int max_len = 0, k = 0, m = 0;
        uint64_t seed = 0, bits = 0;
        if (count != 14 || !take_cache(a, c) || !plain_int_of(a[7], max_len) || !plain_int_of(a[8], k) || !plain_int_of(a[9], m) || !word_of(a[10], seed) || max_len < 0)
            return not_known();
        const at::Tensor *query = shaped(a[3], at::kLong, {-1, -1, c.dim}), *workspace = shaped(a[13], at::kByte, {-1});
        if (query == nullptr || workspace == nullptr || query->size(1) > INT32_MAX) return not_known();
        const int64_t batch = query->size(0), heads = query->size(1);
        const at::Tensor *table = shaped(a[5], at::kInt, {batch, -1});
        const int64_t *q0 = static_cast<const int64_t *>(query->data_ptr()), *q1 = nullptr;
        int64_t *o[2] = {};
        const int32_t *lens = nullptr;
        if (table == nullptr || !take_shaped(a[4], at::kLong, {batch, heads, c.dim}, q1) || !take_shaped(a[6], at::kInt, {batch}, lens)) return not_known();
        for (int i = 0; i < 2; ++i) {
            if (!take_shaped(a[11 + i], at::kLong, {batch, heads, c.dim}, o[i])) return not_known();
        }
        const int32_t *pages = static_cast<const int32_t *>(table->data_ptr());
        const size_t width = (size_t)table->size(1), room = (size_t)workspace->numel();
        void *to = workspace->data_ptr(), *stream = current_stream();
        const int st = without_gil([&] {
            return hb_attention(&c, q0, q1, (size_t)batch, (int)heads, pages, width, lens, (size_t)max_len, k, m, seed, o[0], o[1], to, room, &bits, stream);
        });
        return checked(st, st == HB_OK ? Py_BuildValue("OOK", a[11], a[12], (unsigned long long)bits) : nullptr);
    });
}

PyObject *initialise(PyObject *, PyObject *check)
{
    Py_INCREF(check);
    Py_XDECREF(g_check);
    g_check = check;
    Py_RETURN_NONE;
}

#define HB_FAST(name, doc) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, doc}
PyMethodDef g_methods[] = {
    HB_FAST(shares, "DReLU, ReLU or sign shares of a pair of share tensors"),
    HB_FAST(parties, "DReLU or ReLU among several parties"),
    HB_FAST(batch, "DReLU or ReLU of a set of tensors"),
    HB_FAST(sim_relu, "simulator ReLU of floats"),
    HB_FAST(share, "encode and share floats"),
    HB_FAST(reveal, "open and decode shares"),
    HB_FAST(eco_scan, "zero-error scan"),
    HB_FAST(party, "party-faithful ReLU"),
    HB_FAST(linear, "linear layer with 4-bit weights"),
    HB_FAST(cache, "struct of a paged cache"),
    HB_FAST(append, "keys and values into a paged cache"),
    HB_FAST(attention, "attention over a paged cache"),
    {"plan_run", plan_run, METH_O, "enqueue a plan"},
    {"initialise", initialise, METH_O, "the function that raises the exception of a status"},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_binding", "argument marshalling of hb.py", -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding()
{
    PyObject *module = PyModule_Create(&g_module);
    if (module != nullptr && PyModule_AddStringConstant(module, "torch_version", HB_TORCH_VERSION) != 0) Py_CLEAR(module);
    return module;
}
