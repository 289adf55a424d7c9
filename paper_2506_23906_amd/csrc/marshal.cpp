// The argument marshalling of binding.py for the calls that a program makes over and over, as a CPython extension: tensors to
// pointers, the current stream, the call of the C entry point.  A call on a short vector takes the GPU three microseconds; with
// properties asked for one by one in Python and ctypes converting ten arguments, the host took 4.7 to issue it (segmented scan of
// 3000 values; see binding.py for what it takes now).
// Every function returns the status of the entry point, or None for a call it leaves to binding.py: arguments left out, types it does
// not know, subclasses of Tensor, tensors that are not contiguous GPU memory (binding.py raises what it raises for those).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>

#include "mmvseg.h"

namespace {

struct {
    decltype(&mmv_segscan) segscan;
    decltype(&mmv_segsum) segsum;
    decltype(&mmv_scan) scan;
    decltype(&mmv_compress) compress;
    decltype(&mmv_spmv_coo) spmv_coo, spmv_coo_run;
    decltype(&mmv_spmv_csr) spmv_csr, spmv_csr_run;
} g_entry;

struct LeftToPython {};   // thrown and caught in here

struct Array {
    void *ptr;
    uint64_t numel;
    at::ScalarType type;
};
Array array(PyObject *o) {
    if (!THPVariable_CheckExact(o)) throw LeftToPython();
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || !t.is_contiguous()) throw LeftToPython();
    return {t.data_ptr(), (uint64_t)t.numel(), t.scalar_type()};
}
uint64_t number(PyObject *o) {
    if (!PyLong_CheckExact(o)) throw LeftToPython();
    return PyLong_AsUnsignedLongLongMask(o);
}
mmv_dtype value_type(const Array &a) {
    switch (a.type) {
        case at::kFloat: return MMV_F32_F32;
        case at::kHalf: return MMV_F16_F32;
        case at::kBFloat16: return MMV_BF16_F32;
        case at::kChar: return MMV_I8_I32;
        case at::kByte: return MMV_U8_XOR;
        default: throw LeftToPython();
    }
}
mmv_flag_fmt flag_format(const Array &a) {
    if (a.type == at::kByte) return MMV_FLAGS_U8;
    if (a.type == at::kInt) return MMV_FLAGS_PACKED32;
    throw LeftToPython();
}
mmv_variant variant(PyObject *o) {
    if (PyUnicode_CheckExact(o)) {
        if (PyUnicode_CompareWithASCIIString(o, "mfma") == 0) return MMV_VARIANT_MFMA;
        if (PyUnicode_CompareWithASCIIString(o, "shuffle") == 0) return MMV_VARIANT_SHUFFLE;
    }
    throw LeftToPython();
}
void *stream(PyObject *o) {   // (None: the current one of the current device)
    if (o != Py_None) throw LeftToPython();
    return (void *)c10::hip::getCurrentHIPStream().stream();
}

template <typename Body> PyObject *guarded(Py_ssize_t got, Py_ssize_t want, Body body) {
    if (got != want) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        return PyLong_FromLong((long)body());
    } catch (...) {   // (also what torch throws for tensors without memory of their own)
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}
struct WithoutGil {
    PyThreadState *state = PyEval_SaveThread();
    ~WithoutGil() { PyEval_RestoreThread(state); }
};

// segscan(x, flags, n, z, variant, ws, stream)
PyObject *segscan(PyObject *, PyObject *const *a, Py_ssize_t count) {
    return guarded(count, 7, [&] {
        const Array x = array(a[0]), f = array(a[1]), z = array(a[3]), ws = array(a[5]);
        const uint64_t n = a[2] == Py_None ? x.numel : number(a[2]);
        const mmv_dtype dt = value_type(x);
        const mmv_flag_fmt ff = flag_format(f);
        const mmv_variant v = variant(a[4]);
        void *const s = stream(a[6]);
        WithoutGil free;
        return g_entry.segscan(x.ptr, f.ptr, n, z.ptr, dt, ff, v, ws.ptr, ws.numel, s);
    });
}
// segsum(x, flags, n, out, nseg, variant, ws, stream)
PyObject *segsum(PyObject *, PyObject *const *a, Py_ssize_t count) {
    return guarded(count, 8, [&] {
        const Array x = array(a[0]), f = array(a[1]), out = array(a[3]), nseg = array(a[4]), ws = array(a[6]);
        const uint64_t n = a[2] == Py_None ? x.numel : number(a[2]);
        const mmv_dtype dt = value_type(x);
        const mmv_flag_fmt ff = flag_format(f);
        const mmv_variant v = variant(a[5]);
        void *const s = stream(a[7]);
        WithoutGil free;
        return g_entry.segsum(x.ptr, f.ptr, n, out.ptr, out.numel, (uint64_t *)nseg.ptr, dt, ff, v, ws.ptr, ws.numel, s);
    });
}
// scan(x, n, z, variant, ws, stream)
PyObject *scan(PyObject *, PyObject *const *a, Py_ssize_t count) {
    return guarded(count, 6, [&] {
        const Array x = array(a[0]), z = array(a[2]), ws = array(a[4]);
        const uint64_t n = a[1] == Py_None ? x.numel : number(a[1]);
        const mmv_dtype dt = value_type(x);
        const mmv_variant v = variant(a[3]);
        void *const s = stream(a[5]);
        WithoutGil free;
        return g_entry.scan(x.ptr, n, z.ptr, dt, v, ws.ptr, ws.numel, s);
    });
}
// compress(x, mask, n, out, count, ws, stream)
PyObject *compress(PyObject *, PyObject *const *a, Py_ssize_t args) {
    return guarded(args, 7, [&] {
        Array x = {};
        if (a[0] != Py_None) {
            x = array(a[0]);
            if (c10::elementSize(x.type) != 4) throw LeftToPython();
        }
        const Array mask = array(a[1]), out = array(a[3]), count = array(a[4]), ws = array(a[5]);
        const uint64_t n = number(a[2]);
        const mmv_flag_fmt ff = flag_format(mask);
        void *const s = stream(a[6]);
        WithoutGil free;
        return g_entry.compress(x.ptr, mask.ptr, n, out.ptr, out.numel, (uint64_t *)count.ptr, ff, ws.ptr, ws.numel, s);
    });
}
// ...(n_rows, n_cols, nnz, row or rowptr, col, val, x, y, variant, ws, stream)
template <typename Entry> PyObject *spmv(Entry entry, PyObject *const *a, Py_ssize_t args) {
    return guarded(args, 11, [&] {
        const uint64_t n_rows = number(a[0]), n_cols = number(a[1]);
        const Array row = array(a[3]), col = array(a[4]), val = array(a[5]), x = array(a[6]), y = array(a[7]), ws = array(a[9]);
        const uint64_t nnz = a[2] == Py_None ? val.numel : number(a[2]);
        const mmv_variant v = variant(a[8]);
        void *const s = stream(a[10]);
        WithoutGil free;
        return entry(n_rows, n_cols, nnz, (const int32_t *)row.ptr, (const int32_t *)col.ptr, (const float *)val.ptr, (const float *)x.ptr,
                     (float *)y.ptr, v, ws.ptr, ws.numel, s);
    });
}
PyObject *spmv_coo(PyObject *, PyObject *const *a, Py_ssize_t n) { return spmv(g_entry.spmv_coo, a, n); }
PyObject *spmv_csr(PyObject *, PyObject *const *a, Py_ssize_t n) { return spmv(g_entry.spmv_csr, a, n); }
PyObject *spmv_coo_run(PyObject *, PyObject *const *a, Py_ssize_t n) { return spmv(g_entry.spmv_coo_run, a, n); }
PyObject *spmv_csr_run(PyObject *, PyObject *const *a, Py_ssize_t n) { return spmv(g_entry.spmv_csr_run, a, n); }

// ---- the calls of a serving step (the checks are those of binding.py, which raises what it finds wrong) --------------

struct {
    decltype(&mmv_page_tables) page_tables;
    decltype(&mmv_cache_append) cache_append;
    decltype(&mmv_paged_attention) paged_attention;
    decltype(&mmv_decay_attention) decay_attention;
    decltype(&mmv_decay_step) decay_step;
    decltype(&mmv_block_append) block_append;
    decltype(&mmv_block_read) block_read;
    decltype(&mmv_block_attention) block_attention;
    decltype(&mmv_delta_attention) delta_attention;
    decltype(&mmv_delta_step) delta_step;
} g_serving;

const at::Tensor &tensor(PyObject *o, at::ScalarType type) {
    if (!THPVariable_CheckExact(o)) throw LeftToPython();
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.scalar_type() != type) throw LeftToPython();
    return t;
}
template <typename T> T *array_of(PyObject *o, at::ScalarType type, int64_t numel) {   // contiguous, at least so many
    const at::Tensor &t = tensor(o, type);
    if (!t.is_contiguous() || t.numel() < numel) throw LeftToPython();
    return (T *)t.data_ptr();
}
template <typename T> T *shaped(PyObject *o, at::ScalarType type, std::initializer_list<int64_t> shape) {   // contiguous, of this shape
    const at::Tensor &t = tensor(o, type);
    if (!t.is_contiguous() || !t.sizes().equals(shape)) throw LeftToPython();
    return (T *)t.data_ptr();
}
at::ScalarType value_of(PyObject *o, int64_t dims) {
    if (!THPVariable_CheckExact(o)) throw LeftToPython();
    const at::Tensor &t = THPVariable_Unpack(o);
    if (t.dim() != dims || (t.scalar_type() != at::kHalf && t.scalar_type() != at::kBFloat16)) throw LeftToPython();
    return t.scalar_type();
}
mmv_type type_of(at::ScalarType t) { return t == at::kHalf ? MMV_TYPE_F16 : MMV_TYPE_BF16; }
struct Tokens {
    const void *ptr;
    uint64_t stride;
};
Tokens tokens(PyObject *o, at::ScalarType type, int64_t n, int64_t heads, int64_t dim) {   // the heads of a token one after the other
    const at::Tensor &t = tensor(o, type);
    if (!t.sizes().equals({n, heads, dim})) throw LeftToPython();
    if (t.numel() && ((dim > 1 && t.stride(2) != 1) || (heads > 1 && t.stride(1) != dim))) throw LeftToPython();
    return {t.data_ptr(), (uint64_t)(n > 1 ? t.stride(0) : heads * dim)};
}
struct Rows {
    int32_t *ptr;
    uint64_t width, stride;
};
Rows rows(PyObject *o, int64_t n) {
    const at::Tensor &t = tensor(o, at::kInt);
    if (t.dim() != 2 || t.size(0) < n || (t.size(1) > 1 && t.stride(1) != 1)) throw LeftToPython();
    return {(int32_t *)t.data_ptr(), (uint64_t)t.size(1), (uint64_t)(t.size(0) > 1 ? t.stride(0) : t.size(1))};
}
float real(PyObject *o) {
    if (!PyFloat_CheckExact(o)) throw LeftToPython();
    return (float)PyFloat_AS_DOUBLE(o);
}
uint32_t number32(PyObject *o) {
    if (!PyLong_CheckExact(o)) throw LeftToPython();
    const long v = PyLong_AsLong(o);
    if (v < 0 || v > 0x7fffffffL) throw LeftToPython();
    return (uint32_t)v;
}
template <typename Cache = mmv_paged_cache> const Cache *cache_of(PyObject *address) {   // (the address of binding.py's own structure)
    if (!PyLong_CheckExact(address)) throw LeftToPython();
    return (const Cache *)PyLong_AsVoidPtr(address);
}
struct Scratch {
    void *ptr;
    size_t bytes;
};
Scratch scratch(PyObject *o) {
    const Array a = array(o);
    return {a.ptr, (size_t)(a.numel * c10::elementSize(a.type))};
}

// page_tables(cached, new, free, table, page, max_tokens, out, ws, stream)
PyObject *page_tables(PyObject *, PyObject *const *a, Py_ssize_t count) {
    return guarded(count, 9, [&] {
        if (!PyTuple_Check(a[6]) || PyTuple_GET_SIZE(a[6]) != 5) throw LeftToPython();
        const int64_t n = tensor(a[1], at::kInt).numel(), most = number32(a[5]);
        const auto *cached = array_of<const int32_t>(a[0], at::kInt, n), *fresh = array_of<const int32_t>(a[1], at::kInt, n), *free_pages = array_of<const int32_t>(a[2], at::kInt, 0);
        const uint64_t free_count = THPVariable_Unpack(a[2]).numel();
        const Rows table = rows(a[3], n);
        const uint32_t page = number32(a[4]);
        PyObject *const *out = &PyTuple_GET_ITEM(a[6], 0);
        auto *offsets = array_of<int32_t>(out[0], at::kInt, n + 1), *context = array_of<int32_t>(out[1], at::kInt, n), *positions = array_of<int32_t>(out[3], at::kInt, most);
        auto *slots = array_of<int64_t>(out[2], at::kLong, most), *used = array_of<int64_t>(out[4], at::kLong, 2);
        const Scratch ws = scratch(a[7]);
        void *const s = stream(a[8]);
        WithoutGil free;
        return g_serving.page_tables(n, cached, fresh, free_pages, free_count, table.ptr, table.width, table.stride, page, most, offsets, context, slots, positions, used, ws.ptr, ws.bytes, s);
    });
}
// cache_append, block_append(k, v, slots, address of the cache, stream)
template <typename Cache, typename Entry> PyObject *append(Entry entry, PyObject *const *a, Py_ssize_t count) {
    return guarded(count, 5, [&] {
        const at::ScalarType type = value_of(a[0], 3);
        const Cache *cache = cache_of<Cache>(a[3]);
        const int64_t n = THPVariable_Unpack(a[0]).size(0);
        const Tokens k = tokens(a[0], type, n, cache->heads, cache->dim), v = tokens(a[1], type, n, cache->heads, cache->dim);
        const auto *slots = array_of<const int64_t>(a[2], at::kLong, n);
        void *const s = stream(a[4]);
        WithoutGil free;
        return entry(n, k.ptr, k.stride, v.ptr, v.stride, type_of(type), slots, cache, s);
    });
}
// paged_attention, block_attention(q, address of the cache, table, context, scale, window, out, lse, ws, stream)
template <typename Cache, typename Entry> PyObject *attention(Entry entry, PyObject *const *a, Py_ssize_t count) {
    return guarded(count, 10, [&] {
        const at::ScalarType type = value_of(a[0], 3);
        const Cache *cache = cache_of<Cache>(a[1]);
        const at::Tensor &t = THPVariable_Unpack(a[0]);
        const int64_t n = t.size(0), heads = t.size(1), dim = cache->dim;
        const Tokens q = tokens(a[0], type, n, heads, dim);
        const Rows table = rows(a[2], n);
        const auto *context = array_of<const int32_t>(a[3], at::kInt, n);
        const float scale = real(a[4]);
        const uint32_t window = number32(a[5]);
        void *const out = shaped<void>(a[6], type, {n, heads, dim});
        float *const lse = a[7] == Py_None ? nullptr : shaped<float>(a[7], at::kFloat, {n, heads});
        const Scratch ws = scratch(a[8]);
        void *const s = stream(a[9]);
        WithoutGil free;
        return entry(n, heads, q.ptr, q.stride, type_of(type), cache, table.ptr, table.width, table.stride, context, scale, window, out, lse, ws.ptr, ws.bytes, s);
    });
}
PyObject *cache_append(PyObject *, PyObject *const *a, Py_ssize_t n) { return append<mmv_paged_cache>(g_serving.cache_append, a, n); }
PyObject *block_append(PyObject *, PyObject *const *a, Py_ssize_t n) { return append<mmv_block_cache>(g_serving.block_append, a, n); }
PyObject *paged_attention(PyObject *, PyObject *const *a, Py_ssize_t n) { return attention<mmv_paged_cache>(g_serving.paged_attention, a, n); }
PyObject *block_attention(PyObject *, PyObject *const *a, Py_ssize_t n) { return attention<mmv_block_cache>(g_serving.block_attention, a, n); }
// block_read(address of the cache, table, offsets, first, out, stream)
PyObject *block_read(PyObject *, PyObject *const *a, Py_ssize_t count) {
    return guarded(count, 6, [&] {
        const mmv_block_cache *cache = cache_of<mmv_block_cache>(a[0]);
        if (!PyTuple_CheckExact(a[4]) || PyTuple_GET_SIZE(a[4]) != 2) throw LeftToPython();
        PyObject *const ok = PyTuple_GET_ITEM(a[4], 0), *const ov = PyTuple_GET_ITEM(a[4], 1);
        const at::ScalarType type = value_of(ok, 3);
        const int64_t n = tensor(a[2], at::kInt).numel() - 1, count_out = THPVariable_Unpack(ok).size(0);
        if (n < 0) throw LeftToPython();
        const auto *offsets = array_of<const int32_t>(a[2], at::kInt, n + 1), *first = a[3] == Py_None ? nullptr : array_of<const int32_t>(a[3], at::kInt, n);
        const Rows table = rows(a[1], n);
        const Tokens k = tokens(ok, type, count_out, cache->heads, cache->dim), v = tokens(ov, type, count_out, cache->heads, cache->dim);
        void *const s = stream(a[5]);
        WithoutGil free;
        return g_serving.block_read(n, count_out, offsets, first, table.ptr, table.width, table.stride, cache, type_of(type), (void *)k.ptr, k.stride, (void *)v.ptr, v.stride, s);
    });
}
// What the recurrences take: q, k, v, log_decay (the delta rule beta too), scale, state_in, state_out, state_index, out
struct Recurrence {
    at::ScalarType type;
    int64_t n, heads, kv, dk, dv;
    Tokens q, k, v;
    const float *log_decay, *beta, *in;
    float *out_states, scale;
    uint64_t states;
    const int32_t *index;
    void *out;
    void set_states(PyObject *from, PyObject *to, PyObject *which, PyObject *result, int64_t requests) {   // (fewer than 0: one for each token)
        int64_t count = -1;
        const auto state = [&](PyObject *o) -> float * {
            if (o == Py_None) return nullptr;
            const at::Tensor &t = tensor(o, at::kFloat);
            if (!t.is_contiguous() || t.dim() != 4 || t.size(1) != heads || t.size(2) != dk || t.size(3) != dv || (count >= 0 && t.size(0) != count)) throw LeftToPython();
            count = t.size(0);
            return (float *)t.data_ptr();
        };
        in = state(from), out_states = state(to);
        states = count < 0 ? 0 : count;
        index = which == Py_None ? nullptr : array_of<const int32_t>(which, at::kInt, requests < 0 ? n : requests);
        out = shaped<void>(result, type, {n, heads, dv});
    }
};
Recurrence recurrence(PyObject *q, PyObject *k, PyObject *v, PyObject *log_decay, PyObject *scale, PyObject *in, PyObject *out_states, PyObject *index, PyObject *out, int64_t requests) {
    Recurrence R = {};
    R.type = value_of(q, 3);
    value_of(v, 3);
    const at::Tensor &tq = THPVariable_Unpack(q), &tv = THPVariable_Unpack(v);
    R.n = tq.size(0), R.heads = tq.size(1), R.dk = tq.size(2), R.kv = tv.size(1), R.dv = tv.size(2);
    R.q = tokens(q, R.type, R.n, R.heads, R.dk), R.k = tokens(k, R.type, R.n, R.kv, R.dk), R.v = tokens(v, R.type, R.n, R.kv, R.dv);
    R.log_decay = array_of<const float>(log_decay, at::kFloat, R.heads);
    R.scale = real(scale);
    R.set_states(in, out_states, index, out, requests);
    return R;
}
// decay_attention(q, k, v, offsets, log_decay, scale, state_in, state_out, state_index, out, ws, stream)
PyObject *decay_attention(PyObject *, PyObject *const *a, Py_ssize_t count) {
    return guarded(count, 12, [&] {
        const int64_t n = tensor(a[3], at::kInt).numel() - 1;
        if (n < 0) throw LeftToPython();
        const auto *offsets = array_of<const int32_t>(a[3], at::kInt, n + 1);
        const Recurrence R = recurrence(a[0], a[1], a[2], a[4], a[5], a[6], a[7], a[8], a[9], n);
        const Scratch ws = scratch(a[10]);
        void *const s = stream(a[11]);
        WithoutGil free;
        return g_serving.decay_attention(n, R.n, R.heads, R.kv, R.dk, R.dv, R.q.ptr, R.q.stride, R.k.ptr, R.k.stride, R.v.ptr, R.v.stride, type_of(R.type), offsets, R.log_decay, R.scale,
                                         R.in, R.out_states, R.states, R.index, R.out, ws.ptr, ws.bytes, s);
    });
}
// decay_step(q, k, v, log_decay, state_in, state_out, scale, state_index, out, stream)
PyObject *decay_step(PyObject *, PyObject *const *a, Py_ssize_t count) {
    return guarded(count, 10, [&] {
        const Recurrence R = recurrence(a[0], a[1], a[2], a[3], a[6], a[4], a[5], a[7], a[8], -1);
        void *const s = stream(a[9]);
        WithoutGil free;
        return g_serving.decay_step(R.n, R.heads, R.kv, R.dk, R.dv, R.q.ptr, R.q.stride, R.k.ptr, R.k.stride, R.v.ptr, R.v.stride, type_of(R.type), R.log_decay, R.scale, R.in, R.out_states,
                                    R.states, R.index, R.out, s);
    });
}
Recurrence delta_rule(PyObject *q, PyObject *k, PyObject *v, PyObject *log_decay, PyObject *beta, PyObject *scale, PyObject *in, PyObject *out_states, PyObject *index, PyObject *out,
                      int64_t requests) {
    Recurrence R = {};
    R.type = value_of(q, 3);
    value_of(v, 3);
    const at::Tensor &tq = THPVariable_Unpack(q), &tv = THPVariable_Unpack(v);
    R.n = tq.size(0), R.kv = tq.size(1), R.dk = tq.size(2), R.heads = tv.size(1), R.dv = tv.size(2);
    R.q = tokens(q, R.type, R.n, R.kv, R.dk), R.k = tokens(k, R.type, R.n, R.kv, R.dk), R.v = tokens(v, R.type, R.n, R.heads, R.dv);
    R.log_decay = shaped<const float>(log_decay, at::kFloat, {R.n, R.heads}), R.beta = shaped<const float>(beta, at::kFloat, {R.n, R.heads});
    R.scale = real(scale);
    R.set_states(in, out_states, index, out, requests);
    return R;
}
// delta_attention(q, k, v, offsets, log_decay, beta, scale, state_in, state_out, state_index, out, ws, stream)
PyObject *delta_attention(PyObject *, PyObject *const *a, Py_ssize_t count) {
    return guarded(count, 13, [&] {
        const int64_t n = tensor(a[3], at::kInt).numel() - 1;
        if (n < 0) throw LeftToPython();
        const auto *offsets = array_of<const int32_t>(a[3], at::kInt, n + 1);
        const Recurrence R = delta_rule(a[0], a[1], a[2], a[4], a[5], a[6], a[7], a[8], a[9], a[10], n);
        const Scratch ws = scratch(a[11]);
        void *const s = stream(a[12]);
        WithoutGil free;
        return g_serving.delta_attention(n, R.n, R.heads, R.kv, R.dk, R.dv, R.q.ptr, R.q.stride, R.k.ptr, R.k.stride, R.v.ptr, R.v.stride, type_of(R.type), offsets, R.log_decay, R.beta,
                                         R.scale, R.in, R.out_states, R.states, R.index, R.out, ws.ptr, ws.bytes, s);
    });
}
// delta_step(q, k, v, log_decay, beta, state_in, state_out, scale, state_index, out, stream)
PyObject *delta_step(PyObject *, PyObject *const *a, Py_ssize_t count) {
    return guarded(count, 11, [&] {
        const Recurrence R = delta_rule(a[0], a[1], a[2], a[3], a[4], a[7], a[5], a[6], a[8], a[9], -1);
        void *const s = stream(a[10]);
        WithoutGil free;
        return g_serving.delta_step(R.n, R.heads, R.kv, R.dk, R.dv, R.q.ptr, R.q.stride, R.k.ptr, R.k.stride, R.v.ptr, R.v.stride, type_of(R.type), R.log_decay, R.beta, R.scale, R.in,
                                    R.out_states, R.states, R.index, R.out, s);
    });
}
// bind_serving(addresses of mmv_page_tables, mmv_cache_append, mmv_paged_attention, mmv_decay_attention, mmv_decay_step, mmv_block_append, mmv_block_read,
// mmv_block_attention, mmv_delta_attention, mmv_delta_step)
PyObject *bind_serving(PyObject *, PyObject *const *a, Py_ssize_t count) {
    void *p[10];
    if (count != 10) {
        PyErr_SetString(PyExc_TypeError, "bind_serving takes ten addresses");
        return nullptr;
    }
    for (int i = 0; i < 10; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (!p[i] && PyErr_Occurred()) return nullptr;
    }
    g_serving = {(decltype(&mmv_page_tables))p[0], (decltype(&mmv_cache_append))p[1], (decltype(&mmv_paged_attention))p[2], (decltype(&mmv_decay_attention))p[3],
                 (decltype(&mmv_decay_step))p[4], (decltype(&mmv_block_append))p[5], (decltype(&mmv_block_read))p[6], (decltype(&mmv_block_attention))p[7],
                 (decltype(&mmv_delta_attention))p[8], (decltype(&mmv_delta_step))p[9]};
    Py_RETURN_NONE;
}

// bind(addresses of mmv_segscan, mmv_segsum, mmv_scan, mmv_compress, mmv_spmv_coo, mmv_spmv_csr, mmv_spmv_coo_run, mmv_spmv_csr_run)
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t count) {
    void *p[8];
    if (count != 8) {
        PyErr_SetString(PyExc_TypeError, "bind takes eight addresses");
        return nullptr;
    }
    for (int i = 0; i < 8; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (!p[i] && PyErr_Occurred()) return nullptr;
    }
    g_entry = {(decltype(&mmv_segscan))p[0], (decltype(&mmv_segsum))p[1], (decltype(&mmv_scan))p[2], (decltype(&mmv_compress))p[3],
               (decltype(&mmv_spmv_coo))p[4], (decltype(&mmv_spmv_coo))p[6], (decltype(&mmv_spmv_csr))p[5], (decltype(&mmv_spmv_csr))p[7]};
    Py_RETURN_NONE;
}

#define MMV_METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {MMV_METHOD(bind),     MMV_METHOD(segscan),      MMV_METHOD(segsum),       MMV_METHOD(scan),
                           MMV_METHOD(compress), MMV_METHOD(spmv_coo),     MMV_METHOD(spmv_csr),     MMV_METHOD(spmv_coo_run),
                           MMV_METHOD(spmv_csr_run), MMV_METHOD(page_tables),  MMV_METHOD(cache_append), MMV_METHOD(paged_attention),
                           MMV_METHOD(decay_attention), MMV_METHOD(decay_step), MMV_METHOD(block_append), MMV_METHOD(block_read), MMV_METHOD(block_attention),
                           MMV_METHOD(delta_attention), MMV_METHOD(delta_step), MMV_METHOD(bind_serving), {nullptr, nullptr, 0, nullptr}};
#undef MMV_METHOD
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_marshal", "Argument marshalling of the calls of libmmvseg.so.", -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) {
    PyObject *m = PyModule_Create(&g_module);
    if (m && PyModule_AddStringConstant(m, "torch_version", MMV_TORCH_VERSION) < 0) Py_CLEAR(m);   // (binding.py uses it with this one only)
    return m;
}
