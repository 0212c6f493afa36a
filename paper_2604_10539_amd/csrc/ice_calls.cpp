// The Python side of the 4-bit cache's calls: checks torch tensors, allocates outputs and scratch with torch's allocator, and
// passes addresses on to the C ABI.  No arithmetic.  A decode step calls these once or twice per layer, so what a call costs the
// host counts as much as what it costs the GPU (us per call on the host, by ctypes and Python and so: attend 16.6 and 8.9, attend_tokens
// 12.6 and 5.5, plan 8.5 and 4.0).
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdarg>
#include <cstdio>

#include "icecache.h"

namespace {

using at::Tensor;

// set by bind(): the library's entry points and the exception class
struct {
    decltype(&ice_last_error) last_error;
    decltype(&ice_plan_blocks) plan_blocks;
    decltype(&ice_cache_write) write;
    decltype(&ice_cache_read) read;
    decltype(&ice_cache_attend_bytes) attend_bytes;
    decltype(&ice_cache_attend) attend;
    decltype(&ice_cache_attend_tokens_bytes) tokens_bytes;
    decltype(&ice_cache_attend_tokens) tokens;
    decltype(&ice_plan_sources) plan_sources;
    decltype(&ice_cache_append) append;
    decltype(&ice_cache_attend_cross_bytes) cross_bytes;
    decltype(&ice_cache_attend_cross) cross;
    decltype(&ice_cache_attend_shared_bytes) shared_bytes;
    decltype(&ice_cache_attend_shared) shared;
} lib = {};
PyObject *ice_error = nullptr;

struct Refused {};  // a Python exception is set

[[noreturn]] void refuse(int status, const char *text) {
    if (PyObject *e = PyObject_CallFunction(ice_error, "is", status, text)) {
        PyErr_SetObject(ice_error, e);
        Py_DECREF(e);
    }
    throw Refused();
}
[[noreturn]] void refuse_shape(const char *format, ...) {
    char text[256];
    va_list ap;
    va_start(ap, format);
    vsnprintf(text, sizeof(text), format, ap);
    va_end(ap);
    refuse(ICE_ERR_SHAPE, text);
}
void check(ice_status_t st) {
    if (st != ICE_OK) refuse(st, lib.last_error());
}

const Tensor &tensor(PyObject *o, const char *name) {
    if (!THPVariable_Check(o)) refuse_shape("%s: a tensor", name);
    return THPVariable_Unpack(o);
}
long long number(PyObject *o, const char *name, long long low, long long high) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused();
    if (v < low || v > high) refuse_shape("%s %lld is outside [%lld, %lld]", name, v, low, high);
    return v;
}
int int32_of(PyObject *o, const char *name) { return (int)number(o, name, INT32_MIN, INT32_MAX); }

// The cache that a call is about: its description, its GPU and the stream.
struct Cache {
    const ice_cache_t *c;
    int device;
    void *stream;
    Cache(PyObject *const *args) {
        c = reinterpret_cast<const ice_cache_t *>(PyLong_AsVoidPtr(args[0]));
        device = (int)PyLong_AsLong(args[1]);
        stream = PyLong_AsVoidPtr(args[2]);
        if (PyErr_Occurred()) throw Refused();
    }
    bool here(const Tensor &t) const { return t.is_cuda() && t.get_device() == device; }
    at::TensorOptions options(at::ScalarType type) const { return at::TensorOptions().dtype(type).device(at::kCUDA, (c10::DeviceIndex)device); }
    // contiguous int32 of this shape (its last sizes may be left to the caller: -1)
    const int32_t *ints(const Tensor &t, const char *name, std::initializer_list<int64_t> shape) const {
        bool ok = t.scalar_type() == at::kInt && (size_t)t.dim() == shape.size() && here(t) && t.is_contiguous();
        int64_t d = 0;
        for (int64_t n : shape) {
            ok = ok && (n < 0 || t.size(d) == n);
            ++d;
        }
        if (!ok) refuse_shape("%s: contiguous int32 on the cache's device, of the sizes of the others", name);
        return t.const_data_ptr<int32_t>();
    }
    // rows [tokens, heads, 128] of bf16, heads and values side by side
    const void *rows(const Tensor &t, const char *name, int64_t *stride) const {
        if (!(t.dim() == 3 && t.size(2) == 128 && t.stride(2) == 1 && (t.stride(1) == 128 || t.size(1) == 1) && here(t) &&
              (t.scalar_type() == at::kBFloat16 || t.scalar_type() == at::kShort)))
            refuse_shape("%s: bf16 [tokens, heads, 128] on the cache's device, heads and values side by side", name);
        *stride = t.size(0) > 1 ? t.stride(0) : t.size(1) * 128;  // (of a single row it may be anything)
        return t.const_data_ptr();
    }
    struct Table {
        int n, width;
        const int32_t *seq_len, *table;
    };
    Table table(PyObject *seq_len, PyObject *block_table) const {
        const Tensor &s = tensor(seq_len, "seq_len"), &t = tensor(block_table, "block_table");
        const int32_t *sp = ints(s, "seq_len", {-1});
        if (s.size(0) > INT32_MAX) refuse_shape("seq_len: too many requests");
        const int32_t *tp = ints(t, "block_table", {s.size(0), -1});
        if (t.size(1) > INT32_MAX) refuse_shape("block_table: rows too long");
        return {(int)s.size(0), (int)t.size(1), sp, tp};
    }
};

// out and lse of an attention call, as given or new
struct Outputs {
    Tensor out, lse;
    int kind;
    Outputs(const Cache &c, const Tensor &q, PyObject *given, bool bf16, PyObject *given_lse, bool with_lse) {
        if (given == Py_None) {
            out = at::empty(q.sizes(), c.options(bf16 ? at::kBFloat16 : at::kFloat));
        } else {
            out = tensor(given, "out");
            if (!(out.sizes() == q.sizes() && out.is_contiguous() && c.here(out) && (out.scalar_type() == at::kFloat || out.scalar_type() == at::kBFloat16)))
                refuse_shape("out: contiguous float32 or bfloat16 of q's shape on the cache's device");
        }
        kind = out.scalar_type() == at::kFloat ? ICE_OUT_F32 : ICE_OUT_BF16;
        if (given_lse != Py_None) {
            lse = tensor(given_lse, "lse");
            if (!(lse.dim() == 2 && lse.size(0) == q.size(0) && lse.size(1) == q.size(1) && lse.scalar_type() == at::kFloat && lse.is_contiguous() && c.here(lse)))
                refuse_shape("lse: contiguous float32 [tokens, heads] on the cache's device");
        } else if (with_lse) {
            lse = at::empty({q.size(0), q.size(1)}, c.options(at::kFloat));
        }
    }
    float *lse_ptr() const { return lse.defined() ? lse.data_ptr<float>() : nullptr; }
    PyObject *result(PyObject *given, PyObject *given_lse) const {
        auto object = [](const Tensor &t, PyObject *old) {
            if (old == Py_None) return THPVariable_Wrap(t);
            Py_INCREF(old);
            return old;
        };
        PyObject *o = object(out, given);
        if (!lse.defined() || !o) return o;
        PyObject *l = object(lse, given_lse);
        if (!l) {
            Py_DECREF(o);
            return nullptr;
        }
        PyObject *both = PyTuple_New(2);
        if (!both) {
            Py_DECREF(o);
            Py_DECREF(l);
            return nullptr;
        }
        PyTuple_SET_ITEM(both, 0, o);
        PyTuple_SET_ITEM(both, 1, l);
        return both;
    }
};

// Scratch of one call: from torch's allocator each time (under capture from the graph's own pool), so that calls on other streams and
// other graphs never share it.
struct Scratch {
    Tensor t;
    size_t bytes;
    Scratch(const Cache &c, size_t n) : bytes(n) {
        if (n) t = at::empty({(int64_t)n}, c.options(at::kByte));
    }
    void *ptr() const { return bytes ? t.data_ptr() : nullptr; }
};

int group_of(const Cache &c, const Tensor &q) {
    const int64_t heads = c.c->n_kv_heads;
    if (q.size(1) % heads) refuse_shape("q: a multiple of %d heads", (int)heads);
    if (q.size(1) / heads > INT32_MAX || q.size(0) > INT32_MAX) refuse_shape("q: too many rows");
    return (int)(q.size(1) / heads);
}

template <typename F>
PyObject *guarded(Py_ssize_t have, Py_ssize_t want, F f) {
    HANDLE_TH_ERRORS
    if (have != want) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        return f();
    } catch (const Refused &) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// (desc, device, stream, q, query_start, seq_len, table, max_query or None, max_len or None, window, out or None, bf16, lse or None, with_lse)
PyObject *call_attend(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 14, [&]() -> PyObject * {
        const Cache c(a);
        const Tensor &q = tensor(a[3], "q");
        int64_t stride = 0;
        const void *qp = c.rows(q, "q", &stride);
        const int group = group_of(c, q);
        const Cache::Table t = c.table(a[5], a[6]);
        const int32_t *start = c.ints(tensor(a[4], "query_start"), "query_start", {(int64_t)t.n + 1});
        const int tokens = (int)q.size(0), window = int32_of(a[9], "window");
        int max_query = a[7] == Py_None ? tokens : int32_of(a[7], "max_query");
        if (max_query > tokens) max_query = tokens;
        const int64_t cap = (int64_t)t.width * c.c->block_size;
        const int max_len = a[8] == Py_None ? (int)std::min<int64_t>(cap, 1 << 30) : int32_of(a[8], "max_len");
        const Outputs o(c, q, a[10], a[11] == Py_True, a[12], a[13] == Py_True);
        if (tokens) {
            const Scratch w(c, lib.attend_bytes(c.c, group, t.n, max_query, max_len));
            check(lib.attend(c.c, qp, stride, group, t.n, start, tokens, max_query, t.seq_len, max_len, t.table, t.width, window, o.out.data_ptr(), o.kind,
                             o.lse_ptr(), w.ptr(), w.bytes, c.stream));
        }
        return o.result(a[10], a[12]);
    });
}

// (desc, device, stream, q, seq_len, table, token_pos, n_tok, out or None, bf16, lse or None, with_lse)
PyObject *call_attend_tokens(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 12, [&]() -> PyObject * {
        const Cache c(a);
        const Tensor &q = tensor(a[3], "q"), &pos = tensor(a[6], "token_pos");
        int64_t stride = 0;
        const void *qp = c.rows(q, "q", &stride);
        const int group = group_of(c, q);
        const Cache::Table t = c.table(a[4], a[5]);
        if (q.size(0) != t.n) refuse_shape("q: one row per request");
        const int32_t *pp = c.ints(pos, "token_pos", {t.n, c.c->n_kv_heads, -1});
        if (pos.size(2) > INT32_MAX) refuse_shape("token_pos: lists too long");
        const int32_t *np = c.ints(tensor(a[7], "n_tok"), "n_tok", {t.n, c.c->n_kv_heads});
        const int most = (int)pos.size(2);
        const Outputs o(c, q, a[8], a[9] == Py_True, a[10], a[11] == Py_True);
        const Scratch w(c, lib.tokens_bytes(c.c, group, t.n, most));
        check(lib.tokens(c.c, qp, stride, group, t.n, t.seq_len, t.table, t.width, pp, np, most, o.out.data_ptr(), o.kind, o.lse_ptr(), w.ptr(), w.bytes, c.stream));
        return o.result(a[8], a[10]);
    });
}

// (desc, device, stream, k, v, slots)
PyObject *call_write(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 6, [&]() -> PyObject * {
        const Cache c(a);
        const Tensor &k = tensor(a[3], "k"), &v = tensor(a[4], "v");
        int64_t ks = 0, vs = 0;
        const void *kp = c.rows(k, "k", &ks), *vp = c.rows(v, "v", &vs);
        if (k.sizes() != v.sizes() || k.size(1) != c.c->n_kv_heads || k.size(0) > INT32_MAX) refuse_shape("k and v: [tokens, %d, 128]", c.c->n_kv_heads);
        const int32_t *slots = c.ints(tensor(a[5], "slots"), "slots", {k.size(0)});
        check(lib.write(c.c, kp, vp, ks, vs, slots, (int)k.size(0), c.stream));
        Py_RETURN_NONE;
    });
}

// (desc, device, stream, table, seq_len, n_rows, first or None, K or None, V or None)
PyObject *call_read(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 9, [&]() -> PyObject * {
        const Cache c(a);
        const Cache::Table t = c.table(a[4], a[3]);
        const int n_rows = (int)number(a[5], "n_rows", 0, INT32_MAX);
        const int32_t *first = a[6] == Py_None ? nullptr : c.ints(tensor(a[6], "first"), "first", {t.n});
        const std::array<int64_t, 4> shape = {t.n, c.c->n_kv_heads, n_rows, 128};
        Tensor out[2];
        for (int i = 0; i < 2; ++i) {
            if (a[7 + i] == Py_None) {
                out[i] = at::empty(shape, c.options(at::kBFloat16));
                continue;
            }
            out[i] = tensor(a[7 + i], "out");
            if (!(out[i].sizes() == at::IntArrayRef(shape) && out[i].is_contiguous() && c.here(out[i]) &&
                  (out[i].scalar_type() == at::kBFloat16 || out[i].scalar_type() == at::kShort)))
                refuse_shape("out: two contiguous bf16 tensors [requests, n_kv_heads, n_rows, 128]");
        }
        check(lib.read(c.c, t.n, t.seq_len, t.table, t.width, first, n_rows, out[0].data_ptr(), out[1].data_ptr(), c.stream));
        PyObject *k = THPVariable_Wrap(out[0]), *v = THPVariable_Wrap(out[1]);
        PyObject *both = k && v ? PyTuple_Pack(2, k, v) : nullptr;
        Py_XDECREF(k);
        Py_XDECREF(v);
        return both;
    });
}

// (stream, block_size, new_len, cached_len, seq_len, table, free_ids, n_free, n_free_left, query_start, slots, info)
PyObject *call_plan(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 12, [&]() -> PyObject * {
        void *stream = PyLong_AsVoidPtr(a[0]);
        if (PyErr_Occurred()) throw Refused();
        const int block_size = int32_of(a[1], "block_size");
        const Tensor &table = tensor(a[5], "block_table");
        const int64_t requests = tensor(a[2], "new_len").numel(), n_blocks = tensor(a[6], "free_ids").numel(), n_slots = tensor(a[10], "slots").numel();
        if (table.dim() != 2 || table.size(0) != requests) refuse_shape("block_table: [requests, max_blocks]");
        if (n_blocks > INT32_MAX || n_slots > INT32_MAX || requests > INT32_MAX || table.size(1) > INT32_MAX) refuse_shape("an array is too long");
        static const char *const names[10] = {"new_len", "cached_len", "seq_len", "block_table", "free_ids", "n_free", "n_free_left", "query_start", "slots", "info"};
        const int64_t sizes[10] = {requests, requests, requests, table.numel(), n_blocks, 1, 1, requests + 1, n_slots, 4};
        int32_t *p[10];
        for (int i = 0; i < 10; ++i) {
            const Tensor &t = tensor(a[2 + i], names[i]);
            if (!(t.scalar_type() == at::kInt && t.numel() == sizes[i] && t.is_contiguous() && t.device() == table.device()))
                refuse_shape("%s: contiguous int32 of %lld entries on the block table's device", names[i], (long long)sizes[i]);
            p[i] = t.data_ptr<int32_t>();
        }
        if (!table.is_cuda()) refuse(ICE_ERR_INVALID_ARG, "the arrays must be on a GPU");
        check(lib.plan_blocks((int)requests, block_size, (int)table.size(1), (int)n_blocks, p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], p[8], (int)n_slots, p[9],
                              stream));
        Py_RETURN_NONE;
    });
}

// (stream, source, query_start, seq_len or None, plan, n_rows, n_tokens)
PyObject *call_plan_sources(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 7, [&]() -> PyObject * {
        void *stream = PyLong_AsVoidPtr(a[0]);
        if (PyErr_Occurred()) throw Refused();
        const int n_rows = int32_of(a[5], "n_rows"), n_tokens = int32_of(a[6], "n_tokens");
        const Tensor &source = tensor(a[1], "source");
        const int64_t requests = source.numel();
        if (requests > INT32_MAX) refuse_shape("source: too many requests");
        static const char *const names[4] = {"source", "query_start", "seq_len", "plan"};
        const int64_t sizes[4] = {requests, requests + 1, requests, 2 * (int64_t)n_rows + 2 + 2 * (int64_t)n_tokens};
        int32_t *p[4];
        for (int i = 0; i < 4; ++i) {
            p[i] = nullptr;
            if (i == 2 && a[3] == Py_None) continue;
            const Tensor &t = tensor(a[1 + i], names[i]);
            if (!(t.scalar_type() == at::kInt && t.numel() == sizes[i] && t.is_contiguous() && t.device() == source.device()))
                refuse_shape("%s: contiguous int32 of %lld entries on source's device", names[i], (long long)sizes[i]);
            p[i] = t.data_ptr<int32_t>();
        }
        if (!source.is_cuda()) refuse(ICE_ERR_INVALID_ARG, "the arrays must be on a GPU");
        check(lib.plan_sources((int)requests, n_rows, n_tokens, p[0], p[1], p[2], p[3], stream));
        Py_RETURN_NONE;
    });
}

// (desc, device, stream, k, v, query_start, seq_len, table, q or None, out or None, rope or None, neighbours, source or None)
PyObject *call_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 13, [&]() -> PyObject * {
        const Cache c(a);
        const Tensor &k = tensor(a[3], "k"), &v = tensor(a[4], "v");
        int64_t ks = 0, vs = 0, qs = 0, os = 0;
        const void *kp = c.rows(k, "k", &ks), *vp = c.rows(v, "v", &vs), *qp = nullptr;
        if (k.sizes() != v.sizes() || k.size(1) != c.c->n_kv_heads || k.size(0) > INT32_MAX) refuse_shape("k and v: [tokens, %d, 128]", c.c->n_kv_heads);
        const int tokens = (int)k.size(0);
        const Cache::Table t = c.table(a[6], a[7]);
        const int32_t *start = c.ints(tensor(a[5], "query_start"), "query_start", {(int64_t)t.n + 1});
        const int32_t *source = a[12] == Py_None ? nullptr : c.ints(tensor(a[12], "source"), "source", {t.n});
        const float *rope = nullptr;
        int positions = 0, rotated = 0, heads = 0;
        if (a[10] != Py_None) {
            const Tensor &r = tensor(a[10], "rope");
            if (!(r.scalar_type() == at::kFloat && r.dim() == 2 && r.is_contiguous() && c.here(r) && r.size(0) <= INT32_MAX && r.size(1) <= 128))
                refuse_shape("rope: contiguous float32 [positions, up to 128] on the cache's device");
            if (r.numel() == 0) refuse_shape("rope: an empty table");  // (it may have no address, which is how none is handed over)
            rope = r.const_data_ptr<float>();
            positions = (int)r.size(0);
            rotated = (int)r.size(1);
        }
        Tensor out;
        void *op = nullptr;
        if (a[8] == Py_None) {
            if (a[9] != Py_None) refuse_shape("out: only with q");
        } else {
            const Tensor &q = tensor(a[8], "q");
            qp = c.rows(q, "q", &qs);
            if (q.size(0) != tokens || q.size(1) < 1 || q.size(1) > 65536) refuse_shape("q: [%d, heads, 128]", tokens);
            heads = (int)q.size(1);
            if (a[9] == Py_None) out = at::empty(q.sizes(), c.options(q.scalar_type()));
            else out = tensor(a[9], "out");
            op = const_cast<void *>(c.rows(out, "out", &os));
            if (out.sizes() != q.sizes()) refuse_shape("out: q's shape");
        }
        check(lib.append(c.c, qp, qs, heads, op, os, kp, vp, ks, vs, tokens, t.n, start, t.seq_len, source, t.table, t.width, rope, positions, rotated,
                         a[11] == Py_True, c.stream));
        if (a[8] == Py_None) Py_RETURN_NONE;
        if (a[9] == Py_None) return THPVariable_Wrap(out);
        Py_INCREF(a[9]);
        return a[9];
    });
}

// The sorted list of a step's queries, for a table of `rows` rows and the rows of q.
const int32_t *list_of(const Cache &c, PyObject *plan, int64_t rows, int64_t tokens) {
    return c.ints(tensor(plan, "plan"), "plan", {2 * rows + 2 + 2 * tokens});
}
// What the host knows of the most queries, or None: `most` then; never more than that.
int most_of(PyObject *o, const char *name, int most) {
    const int v = o == Py_None ? most : int32_of(o, name);
    return v > most ? most : v;
}
int longest_of(PyObject *o, const char *name, int64_t cap) { return o == Py_None ? (int)std::min<int64_t>(cap, 1 << 30) : int32_of(o, name); }

// (desc, device, stream, q, plan, seq_len, table, max_shared or None, max_len or None, out or None, bf16, lse or None, with_lse)
PyObject *call_attend_cross(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 13, [&]() -> PyObject * {
        const Cache c(a);
        const Tensor &q = tensor(a[3], "q");
        int64_t stride = 0;
        const void *qp = c.rows(q, "q", &stride);
        const int group = group_of(c, q), tokens = (int)q.size(0);
        const Cache::Table t = c.table(a[5], a[6]);
        const int32_t *plan = list_of(c, a[4], t.n, tokens);
        const int most = most_of(a[7], "max_shared", tokens), longest = longest_of(a[8], "max_len", (int64_t)t.width * c.c->block_size);
        const Outputs o(c, q, a[9], a[10] == Py_True, a[11], a[12] == Py_True);
        if (tokens) {
            const Scratch w(c, lib.cross_bytes(c.c, group, t.n, most, longest));
            check(lib.cross(c.c, qp, stride, group, t.n, plan, tokens, most, t.seq_len, longest, t.table, t.width, o.out.data_ptr(), o.kind, o.lse_ptr(), w.ptr(),
                            w.bytes, c.stream));
        }
        return o.result(a[9], a[11]);
    });
}

// (desc, device, stream, q, query_start, source, plan, seq_len, table, max_query, max_shared, max_len, max_source (or None each), window, out or None, bf16,
// lse or None, with_lse)
PyObject *call_attend_shared(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 18, [&]() -> PyObject * {
        const Cache c(a);
        const Tensor &q = tensor(a[3], "q");
        int64_t stride = 0;
        const void *qp = c.rows(q, "q", &stride);
        const int group = group_of(c, q), tokens = (int)q.size(0), window = int32_of(a[13], "window");
        const Cache::Table t = c.table(a[7], a[8]);
        const int32_t *start = c.ints(tensor(a[4], "query_start"), "query_start", {(int64_t)t.n + 1}), *source = c.ints(tensor(a[5], "source"), "source", {t.n});
        const int32_t *plan = list_of(c, a[6], t.n, tokens);
        const int64_t cap = (int64_t)t.width * c.c->block_size;
        const int most = most_of(a[9], "max_query", tokens), shared = most_of(a[10], "max_shared", tokens);
        const int longest = longest_of(a[11], "max_len", cap), longest_source = longest_of(a[12], "max_source", cap);
        const Outputs o(c, q, a[14], a[15] == Py_True, a[16], a[17] == Py_True);
        if (tokens) {
            const Scratch w(c, lib.shared_bytes(c.c, group, t.n, tokens, most, shared, longest, longest_source));
            check(lib.shared(c.c, qp, stride, group, t.n, start, source, plan, tokens, most, shared, t.seq_len, longest, longest_source, t.table, t.width, window,
                             o.out.data_ptr(), o.kind, o.lse_ptr(), w.ptr(), w.bytes, c.stream));
        }
        return o.result(a[14], a[16]);
    });
}

// (IceError, addresses of the entry points in the order of `lib`)
PyObject *call_bind(PyObject *, PyObject *const *a, Py_ssize_t n) {
    constexpr int kEntries = 14;
    return guarded(n, 1 + kEntries, [&]() -> PyObject * {
        void *p[kEntries];
        for (int i = 0; i < kEntries; ++i) p[i] = PyLong_AsVoidPtr(a[1 + i]);
        if (PyErr_Occurred()) throw Refused();
        Py_INCREF(a[0]);
        Py_XDECREF(ice_error);
        ice_error = a[0];
        lib.last_error = reinterpret_cast<decltype(lib.last_error)>(p[0]);
        lib.plan_blocks = reinterpret_cast<decltype(lib.plan_blocks)>(p[1]);
        lib.write = reinterpret_cast<decltype(lib.write)>(p[2]);
        lib.read = reinterpret_cast<decltype(lib.read)>(p[3]);
        lib.attend_bytes = reinterpret_cast<decltype(lib.attend_bytes)>(p[4]);
        lib.attend = reinterpret_cast<decltype(lib.attend)>(p[5]);
        lib.tokens_bytes = reinterpret_cast<decltype(lib.tokens_bytes)>(p[6]);
        lib.tokens = reinterpret_cast<decltype(lib.tokens)>(p[7]);
        lib.plan_sources = reinterpret_cast<decltype(lib.plan_sources)>(p[8]);
        lib.append = reinterpret_cast<decltype(lib.append)>(p[9]);
        lib.cross_bytes = reinterpret_cast<decltype(lib.cross_bytes)>(p[10]);
        lib.cross = reinterpret_cast<decltype(lib.cross)>(p[11]);
        lib.shared_bytes = reinterpret_cast<decltype(lib.shared_bytes)>(p[12]);
        lib.shared = reinterpret_cast<decltype(lib.shared)>(p[13]);
        Py_RETURN_NONE;
    });
}

#define ICE_METHOD(name) {#name, (PyCFunction)(void (*)(void))call_##name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ICE_METHOD(attend), ICE_METHOD(attend_tokens), ICE_METHOD(write), ICE_METHOD(read),
                         ICE_METHOD(plan),   ICE_METHOD(plan_sources),  ICE_METHOD(append), ICE_METHOD(attend_cross),
                         ICE_METHOD(attend_shared), ICE_METHOD(bind),   {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
