// Python binding of the per-step calls of include/moe_kv.h (module _kv_native, wrapped by kv_cache.py).
//
// Argument marshalling only, like the ctypes binding of the other entry points.  A decoding step makes these calls once
// per layer on kernels of a few microseconds; ctypes and the checks in Python cost 17 to 35 us a call on the host, this
// file 3 to 6, so that a step of small calls is not bound by the host.
#include <Python.h>

#include <ATen/cuda/CUDAContext.h>
#include <ATen/cuda/EmptyTensor.h>
#include <ATen/core/TensorBase.h>
#include <ATen/TensorUtils.h>
#include <ATen/EmptyTensor.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAGuard.h>
#include <torch/csrc/autograd/python_variable.h>

#include "moe_kv.h"

namespace {

struct Fail { const char *what; };          // becomes an AssertionError, as the checks of the other binding

#define WANT(cond, what) do { if (!(cond)) throw Fail{what}; } while (0)

struct Args {
    PyObject *const *v;
    Py_ssize_t n, at = 0;
    int device = -1;
    PyObject *next() { WANT(at < n, "too few arguments"); return v[at++]; }
    long long i64() {
        const long long x = PyLong_AsLongLong(next());
        if (x == -1 && PyErr_Occurred()) throw Fail{nullptr};
        return x;
    }
    int32_t i32() {
        const long long x = i64();
        WANT(x >= INT32_MIN && x <= INT32_MAX, "an integer argument does not fit 32 bits");
        return (int32_t)x;
    }
    float f32() {
        const double x = PyFloat_AsDouble(next());
        if (x == -1.0 && PyErr_Occurred()) throw Fail{nullptr};
        return (float)x;
    }
    // nullptr for None
    const at::Tensor *tensor_or_none() {
        PyObject *o = next();
        if (o == Py_None) return nullptr;
        WANT(THPVariable_Check(o), "a tensor is wanted");
        const at::Tensor &t = THPVariable_Unpack(o);
        WANT(t.is_cuda(), "a CUDA tensor is wanted");
        WANT(device < 0 || t.get_device() == device, "a tensor is not on the plan's device");
        return &t;
    }
    const at::Tensor &tensor() {
        const at::Tensor *t = tensor_or_none();
        WANT(t != nullptr, "a tensor is wanted, not None");
        return *t;
    }
    const at::Tensor &dense(at::ScalarType type, const char *what) {
        const at::Tensor &t = tensor();
        WANT(t.scalar_type() == type && t.is_contiguous(), what);
        return t;
    }
};

struct Plan {
    moe_kv_plan_t *handle;
    int32_t heads, kv_heads, dim;
    int64_t page_bytes;
    at::ScalarType type;
    int device;
};

// handle, n_heads, n_kv_heads, head_dim, page bytes, dtype code, device
Plan plan_of(Args &a) {
    Plan p{};
    PyObject *t = a.next();
    WANT(PyTuple_CheckExact(t) && PyTuple_GET_SIZE(t) == 7, "a plan is wanted");
    auto get = [&](int i) { return PyLong_AsLongLong(PyTuple_GET_ITEM(t, i)); };
    p.handle = (moe_kv_plan_t *)get(0);
    p.heads = (int32_t)get(1); p.kv_heads = (int32_t)get(2); p.dim = (int32_t)get(3); p.page_bytes = get(4);
    p.type = get(5) == MOE_BF16 ? at::kBFloat16 : at::kFloat;
    p.device = (int)get(6);
    WANT(!PyErr_Occurred() && p.handle != nullptr, "a closed plan");
    a.device = p.device;
    return p;
}

moe_kv_rows_t rows_of(const at::Tensor &x, const Plan &p, int64_t heads, const char *what) {
    WANT(x.dim() == 3 && x.scalar_type() == p.type && x.size(2) == p.dim && (heads < 0 || x.size(1) == heads) && x.stride(2) == 1, what);
    return moe_kv_rows_t{x.data_ptr(), x.stride(0), x.stride(1)};
}

at::Tensor fresh(at::IntArrayRef size, at::ScalarType type, int device) {
    return at::detail::empty_cuda(size, type, c10::Device(c10::kCUDA, (c10::DeviceIndex)device), std::nullopt);
}

// A part of a fresh buffer as a tensor of its own: several outputs cost one allocation
at::Tensor part_of(const at::Tensor &base, int64_t offset, at::IntArrayRef size) {
    at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(base.storage()), base.key_set(), base.dtype());
    t.unsafeGetTensorImpl()->set_storage_offset(offset);
    t.unsafeGetTensorImpl()->set_sizes_contiguous(size);
    return t;
}

void *stream_of(const Plan &p) { return (void *)at::cuda::getCurrentCUDAStream((c10::DeviceIndex)p.device).stream(); }

int32_t pages_of(const at::Tensor &cache, const Plan &p) {
    WANT(cache.scalar_type() == at::kByte && cache.is_contiguous() && cache.dim() > 0, "cache: dense uint8 wanted");
    const int64_t n = cache.size(0);
    WANT(n <= INT32_MAX && (int64_t)cache.numel() == n * p.page_bytes, "cache of another shape");
    return (int32_t)n;
}

struct Turns { const int32_t *position = nullptr; const float *table = nullptr; int32_t n = 0, rot = 0; };
Turns turns_of(Args &a, int64_t tokens) {       // positions, turns; both None: nothing turns
    const at::Tensor *pos = a.tensor_or_none(), *tab = a.tensor_or_none();
    Turns t;
    if (!tab) return t;
    WANT(pos && pos->scalar_type() == at::kInt && pos->is_contiguous() && pos->dim() == 1 && pos->size(0) == tokens, "positions: int32, one for each token");
    WANT(tab->scalar_type() == at::kFloat && tab->is_contiguous() && tab->dim() == 3 && tab->size(2) == 2 && tab->size(0) <= INT32_MAX, "turns: [positions, pairs, 2] fp32");
    t.position = pos->data_ptr<int32_t>();
    t.table = tab->data_ptr<float>();
    t.n = (int32_t)tab->size(0);
    t.rot = (int32_t)(2 * tab->size(1));
    return t;
}

// (status, outputs...)
PyObject *answer(int status, std::initializer_list<at::Tensor> out) {
    PyObject *t = PyTuple_New(1 + (Py_ssize_t)out.size());
    if (!t) return nullptr;
    PyTuple_SET_ITEM(t, 0, PyLong_FromLong(status));
    Py_ssize_t i = 1;
    for (const at::Tensor &x : out) PyTuple_SET_ITEM(t, i++, THPVariable_Wrap(x));
    return t;
}

template <typename F>
PyObject *guarded(PyObject *const *args, Py_ssize_t n, F f) {
    try {
        Args a{args, n};
        return f(a);
    } catch (const Fail &e) {
        if (e.what) PyErr_SetString(PyExc_AssertionError, e.what);
        return nullptr;
    } catch (const c10::OutOfMemoryError &e) {
        PyErr_SetString(PyExc_MemoryError, e.what_without_backtrace());
        return nullptr;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

PyObject *tables(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return guarded(args, n, [](Args &a) {
        const Plan p = plan_of(a);
        const c10::cuda::CUDAGuard guard((c10::DeviceIndex)p.device);
        const at::Tensor &ctx = a.dense(at::kInt, "ctx_len: dense int32 wanted"), &fresh_len = a.dense(at::kInt, "new_len: dense int32 wanted");
        const at::Tensor &free_pages = a.dense(at::kInt, "free_pages: dense int32 wanted"), &table = a.dense(at::kInt, "block_table: dense int32 wanted");
        const int64_t tokens = a.i64(), req = ctx.numel();
        WANT(ctx.dim() == 1 && fresh_len.numel() == req && table.dim() == 2 && table.size(0) == req, "lengths and block_table of different numbers of requests");
        WANT(tokens >= 0 && tokens <= INT32_MAX && free_pages.numel() <= INT32_MAX && table.size(1) <= INT32_MAX, "a size does not fit 32 bits");
        const at::Tensor words = fresh({tokens + 2 * req + 2}, at::kInt, p.device);
        at::Tensor pos = part_of(words, 0, {tokens}), kv_len = part_of(words, tokens, {req}), cu = part_of(words, tokens + req, {req + 1});
        at::Tensor taken = part_of(words, tokens + 2 * req + 1, {1}), slot = fresh({tokens}, at::kLong, p.device);
        const int rc = moe_kv_tables(p.handle, ctx.data_ptr<int32_t>(), fresh_len.data_ptr<int32_t>(), (int32_t)req, free_pages.data_ptr<int32_t>(),
                                     (int32_t)free_pages.numel(), table.data_ptr<int32_t>(), (int32_t)table.size(1), (int32_t)tokens,
                                     kv_len.data_ptr<int32_t>(), cu.data_ptr<int32_t>(), pos.data_ptr<int32_t>(), slot.data_ptr<int64_t>(),
                                     taken.data_ptr<int32_t>(), stream_of(p));
        return answer(rc, {kv_len, cu, pos, slot, taken});
    });
}

PyObject *rope(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return guarded(args, n, [](Args &a) {
        const Plan p = plan_of(a);
        const c10::cuda::CUDAGuard guard((c10::DeviceIndex)p.device);
        const at::Tensor &x = a.tensor();
        const moe_kv_rows_t rows = rows_of(x, p, -1, "x: [tokens, heads, head_dim] of the plan's type wanted");
        WANT(x.size(0) <= INT32_MAX && x.size(1) <= INT32_MAX, "x is too large");
        const Turns t = turns_of(a, x.size(0));
        const int32_t layout = a.i32(), inverse = a.i32();
        const at::Tensor *given = a.tensor_or_none();
        at::Tensor out = given ? *given : fresh(x.sizes(), p.type, p.device);
        WANT(out.sizes() == x.sizes() && out.scalar_type() == p.type && out.stride(2) == 1, "out: as x wanted");
        const int rc = moe_rope(p.handle, &rows, (int32_t)x.size(0), (int32_t)x.size(1), t.position, t.table, t.n, t.rot, layout, inverse,
                                out.data_ptr(), out.stride(0), out.stride(1), stream_of(p));
        return answer(rc, {out});
    });
}

PyObject *append(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return guarded(args, n, [](Args &a) {
        const Plan p = plan_of(a);
        const c10::cuda::CUDAGuard guard((c10::DeviceIndex)p.device);
        const at::Tensor *q = a.tensor_or_none();
        const at::Tensor &k = a.tensor(), &v = a.tensor();
        const at::Tensor &slots = a.dense(at::kLong, "slots: dense int64 wanted"), &cache = a.tensor();
        const moe_kv_rows_t kr = rows_of(k, p, p.kv_heads, "k: [tokens, n_kv_heads, head_dim] of the plan's type wanted");
        const moe_kv_rows_t vr = rows_of(v, p, p.kv_heads, "v: [tokens, n_kv_heads, head_dim] of the plan's type wanted");
        const int64_t tokens = k.size(0);
        WANT(tokens <= INT32_MAX && v.size(0) == tokens && slots.numel() == tokens, "k, v and slots of different numbers of tokens");
        const Turns t = turns_of(a, tokens);
        const int32_t layout = a.i32();
        const float ks = a.f32(), vs = a.f32();
        const at::Tensor *given = a.tensor_or_none();
        moe_kv_rows_t qr{};
        at::Tensor out;
        if (q) {
            qr = rows_of(*q, p, p.heads, "q: [tokens, n_heads, head_dim] of the plan's type wanted");
            WANT(q->size(0) == tokens, "q and k of different numbers of tokens");
            out = given ? *given : fresh(q->sizes(), p.type, p.device);
            WANT(out.sizes() == q->sizes() && out.scalar_type() == p.type && out.is_contiguous(), "q_out: dense, as q wanted");
        }
        const int rc = moe_kv_append(p.handle, q ? &qr : nullptr, &kr, &vr, (int32_t)tokens, t.position, t.table, t.n, t.rot, layout,
                                     slots.data_ptr<int64_t>(), ks, vs, q ? out.data_ptr() : nullptr, cache.data_ptr(), pages_of(cache, p), stream_of(p));
        if (!q) return answer(rc, {});
        return answer(rc, {out});
    });
}

PyObject *read(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return guarded(args, n, [](Args &a) {
        const Plan p = plan_of(a);
        const c10::cuda::CUDAGuard guard((c10::DeviceIndex)p.device);
        const at::Tensor &cache = a.tensor(), &slots = a.dense(at::kLong, "slots: dense int64 wanted");
        const float ks = a.f32(), vs = a.f32();
        WANT(slots.numel() <= INT32_MAX, "too many slots");
        const at::Tensor both = fresh({2, slots.numel(), p.kv_heads, p.dim}, p.type, p.device);
        at::Tensor k = part_of(both, 0, {slots.numel(), p.kv_heads, p.dim}), v = part_of(both, both.numel() / 2, {slots.numel(), p.kv_heads, p.dim});
        const int rc = moe_kv_read(p.handle, cache.data_ptr(), pages_of(cache, p), slots.data_ptr<int64_t>(), (int32_t)slots.numel(), ks, vs,
                                   k.data_ptr(), v.data_ptr(), stream_of(p));
        return answer(rc, {k, v});
    });
}

PyObject *attention(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return guarded(args, n, [](Args &a) {
        const Plan p = plan_of(a);
        const c10::cuda::CUDAGuard guard((c10::DeviceIndex)p.device);
        const at::Tensor &q = a.tensor();
        const moe_kv_rows_t rows = rows_of(q, p, p.heads, "q: [tokens, n_heads, head_dim] of the plan's type wanted");
        const at::Tensor &cu = a.dense(at::kInt, "cu_new: dense int32 wanted"), &len = a.dense(at::kInt, "kv_len: dense int32 wanted");
        const at::Tensor &table = a.dense(at::kInt, "block_table: dense int32 wanted"), &cache = a.tensor();
        const int64_t req = len.numel();
        WANT(req <= INT32_MAX && q.size(0) <= INT32_MAX && cu.numel() == req + 1 && table.dim() == 2 && table.size(0) == req && table.size(1) <= INT32_MAX,
             "cu_new, kv_len and block_table of different numbers of requests");
        const int32_t max_new = a.i32(), window = a.i32(), sinks = a.i32();
        const float scale = a.f32(), ks = a.f32(), vs = a.f32();
        const at::Tensor *given = a.tensor_or_none();
        at::Tensor out = given ? *given : fresh(q.sizes(), p.type, p.device);
        WANT(out.sizes() == q.sizes() && out.scalar_type() == p.type && out.is_contiguous(), "out: dense, as q wanted");
        const int rc = moe_kv_attention(p.handle, &rows, (int32_t)q.size(0), cu.data_ptr<int32_t>(), len.data_ptr<int32_t>(), (int32_t)req, max_new,
                                        table.data_ptr<int32_t>(), (int32_t)table.size(1), cache.data_ptr(), pages_of(cache, p), scale, ks, vs, window, sinks,
                                        out.data_ptr(), stream_of(p));
        return answer(rc, {out});
    });
}

#define ENTRY(name, doc) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, doc}
PyMethodDef methods[] = {
    ENTRY(tables, "moe_kv_tables"), ENTRY(rope, "moe_rope"), ENTRY(append, "moe_kv_append"), ENTRY(read, "moe_kv_read"),
    ENTRY(attention, "moe_kv_attention"), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kv_native", "Per-step calls of include/moe_kv.h", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kv_native() { return PyModule_Create(&module); }
