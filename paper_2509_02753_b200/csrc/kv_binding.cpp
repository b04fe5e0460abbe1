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

// cu_new, kv_len, block_table: the requests of a call
struct Requests { const int32_t *cu, *len, *table; int32_t n, width; };
Requests requests_of(Args &a) {
    const at::Tensor &cu = a.dense(at::kInt, "cu_new: dense int32 wanted"), &len = a.dense(at::kInt, "kv_len: dense int32 wanted");
    const at::Tensor &table = a.dense(at::kInt, "block_table: dense int32 wanted");
    const int64_t n = len.numel();
    WANT(n <= INT32_MAX && cu.numel() == n + 1 && table.dim() == 2 && table.size(0) == n && table.size(1) <= INT32_MAX,
         "cu_new, kv_len and block_table of different numbers of requests");
    return Requests{cu.data_ptr<int32_t>(), len.data_ptr<int32_t>(), table.data_ptr<int32_t>(), (int32_t)n, (int32_t)table.size(1)};
}

// q and the output of an attention call
moe_kv_rows_t queries_of(const at::Tensor &q, const Plan &p) {
    WANT(q.dim() > 0 && q.size(0) <= INT32_MAX, "q is too large");
    return rows_of(q, p, p.heads, "q: [tokens, n_heads, head_dim] of the plan's type wanted");
}
at::Tensor output_of(const at::Tensor *given, const at::Tensor &q, const Plan &p) {
    at::Tensor out = given ? *given : fresh(q.sizes(), p.type, p.device);
    WANT(out.sizes() == q.sizes() && out.scalar_type() == p.type && out.is_contiguous(), "out: dense, as q wanted");
    return out;
}

int32_t summaries_of(const at::Tensor &s, const Plan &p) {
    WANT(s.scalar_type() == at::kByte && s.is_contiguous() && s.dim() > 0, "summaries: dense uint8 wanted");
    const int64_t n = s.size(0), width = p.dim <= 64 ? 64 : p.dim <= 128 ? 128 : 256;
    WANT(n <= INT32_MAX && (int64_t)s.numel() == n * p.kv_heads * (2 * width + 16), "summaries of another shape");
    return (int32_t)n;
}

PyObject *shared_prefix(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return guarded(args, n, [](Args &a) {
        const Plan p = plan_of(a);
        const c10::cuda::CUDAGuard guard((c10::DeviceIndex)p.device);
        const at::Tensor &groups = a.dense(at::kInt, "cu_group: dense int32 wanted");
        const Requests r = requests_of(a);
        const int64_t g = groups.numel() - 1;
        WANT(groups.dim() == 1 && g >= 0 && g <= INT32_MAX, "cu_group: the groups' first requests and the end wanted");
        const at::Tensor words = fresh({g + r.n}, at::kInt, p.device);
        at::Tensor shared = part_of(words, 0, {g}), start = part_of(words, g, {r.n});
        const int rc = moe_kv_shared_prefix(p.handle, groups.data_ptr<int32_t>(), (int32_t)g, r.cu, r.len, r.n, r.table, r.width, shared.data_ptr<int32_t>(),
                                            start.data_ptr<int32_t>(), stream_of(p));
        return answer(rc, {shared, start});
    });
}

PyObject *attention_shared(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return guarded(args, n, [](Args &a) {
        const Plan p = plan_of(a);
        const c10::cuda::CUDAGuard guard((c10::DeviceIndex)p.device);
        const at::Tensor &q = a.tensor();
        const moe_kv_rows_t rows = queries_of(q, p);
        const Requests r = requests_of(a);
        const at::Tensor &cache = a.tensor(), &groups = a.dense(at::kInt, "cu_group: dense int32 wanted");
        const at::Tensor &shared = a.dense(at::kInt, "shared_len: dense int32 wanted"), &start = a.dense(at::kInt, "start: dense int32 wanted");
        const int64_t g = groups.numel() - 1;
        WANT(g >= 0 && g <= INT32_MAX && shared.numel() == g && start.numel() == r.n, "cu_group, shared_len and start of different numbers");
        const int32_t max_new = a.i32(), max_group = a.i32();
        const float scale = a.f32(), ks = a.f32(), vs = a.f32();
        const at::Tensor out = output_of(a.tensor_or_none(), q, p);
        const int64_t bytes = (int64_t)moe_kv_shared_scratch_bytes(p.handle, (int32_t)q.size(0), r.n, max_new, (int32_t)g, max_group, r.width);
        const at::Tensor scratch = bytes > 0 ? fresh({bytes}, at::kByte, p.device) : at::Tensor();
        const int rc = moe_kv_attention_shared(p.handle, &rows, (int32_t)q.size(0), r.cu, r.len, r.n, max_new, r.table, r.width, cache.data_ptr(), pages_of(cache, p),
                                               groups.data_ptr<int32_t>(), (int32_t)g, max_group, shared.data_ptr<int32_t>(), start.data_ptr<int32_t>(), scale, ks, vs,
                                               bytes > 0 ? scratch.data_ptr() : nullptr, (uint64_t)bytes, out.data_ptr(), stream_of(p));
        return answer(rc, {out});
    });
}

PyObject *summarise(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return guarded(args, n, [](Args &a) {
        const Plan p = plan_of(a);
        const c10::cuda::CUDAGuard guard((c10::DeviceIndex)p.device);
        const Requests r = requests_of(a);
        const at::Tensor &cache = a.tensor(), &summaries = a.tensor();
        const int32_t tokens = a.i32(), pages = pages_of(cache, p);
        WANT(summaries_of(summaries, p) == pages, "summaries and cache of different numbers of pages");
        const int rc = moe_kv_summarise(p.handle, r.cu, r.len, r.n, tokens, r.table, r.width, cache.data_ptr(), pages, summaries.data_ptr(), stream_of(p));
        return answer(rc, {});
    });
}

PyObject *read_summaries(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return guarded(args, n, [](Args &a) {
        const Plan p = plan_of(a);
        const c10::cuda::CUDAGuard guard((c10::DeviceIndex)p.device);
        const at::Tensor &summaries = a.tensor(), &pages = a.dense(at::kInt, "pages: dense int32 wanted");
        const float ks = a.f32();
        const int64_t m = pages.numel();
        WANT(m <= INT32_MAX, "too many pages");
        const at::Tensor both = fresh({2, m, p.kv_heads, p.dim}, at::kFloat, p.device);
        at::Tensor high = part_of(both, 0, {m, p.kv_heads, p.dim}), low = part_of(both, both.numel() / 2, {m, p.kv_heads, p.dim});
        const int rc = moe_kv_read_summaries(p.handle, summaries.data_ptr(), summaries_of(summaries, p), pages.data_ptr<int32_t>(), (int32_t)m, ks,
                                             high.data_ptr<float>(), low.data_ptr<float>(), stream_of(p));
        return answer(rc, {high, low});
    });
}

PyObject *select(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return guarded(args, n, [](Args &a) {
        const Plan p = plan_of(a);
        const c10::cuda::CUDAGuard guard((c10::DeviceIndex)p.device);
        const at::Tensor &q = a.tensor();
        const moe_kv_rows_t rows = queries_of(q, p);
        const Requests r = requests_of(a);
        const at::Tensor &summaries = a.tensor();
        const int32_t n_select = a.i32(), first = a.i32(), last = a.i32(), max_new = a.i32();
        const at::Tensor *given = a.tensor_or_none();
        WANT(n_select >= 1, "n_select: at least one page wanted");
        const at::Tensor out = given ? *given : fresh({q.size(0), p.kv_heads, n_select}, at::kInt, p.device);
        WANT(out.scalar_type() == at::kInt && out.is_contiguous() && out.dim() == 3 && out.size(0) == q.size(0) && out.size(1) == p.kv_heads && out.size(2) == n_select,
             "out: dense int32 [tokens, n_kv_heads, n_select] wanted");
        const int rc = moe_kv_select(p.handle, &rows, (int32_t)q.size(0), r.cu, r.len, r.n, max_new, r.table, r.width, summaries.data_ptr(), summaries_of(summaries, p),
                                     n_select, first, last, out.data_ptr<int32_t>(), stream_of(p));
        return answer(rc, {out});
    });
}

PyObject *attention_selected(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return guarded(args, n, [](Args &a) {
        const Plan p = plan_of(a);
        const c10::cuda::CUDAGuard guard((c10::DeviceIndex)p.device);
        const at::Tensor &q = a.tensor();
        const moe_kv_rows_t rows = queries_of(q, p);
        const Requests r = requests_of(a);
        const at::Tensor &cache = a.tensor(), &selected = a.dense(at::kInt, "selected: dense int32 wanted");
        WANT(selected.dim() == 3 && selected.size(0) == q.size(0) && selected.size(1) == p.kv_heads && selected.size(2) <= INT32_MAX,
             "selected: [tokens, n_kv_heads, pages] wanted");
        const float scale = a.f32(), ks = a.f32(), vs = a.f32();
        const at::Tensor out = output_of(a.tensor_or_none(), q, p);
        const int rc = moe_kv_attention_selected(p.handle, &rows, (int32_t)q.size(0), r.cu, r.len, r.n, r.table, r.width, cache.data_ptr(), pages_of(cache, p),
                                                 selected.data_ptr<int32_t>(), (int32_t)selected.size(2), scale, ks, vs, out.data_ptr(), stream_of(p));
        return answer(rc, {out});
    });
}

#define ENTRY(name, doc) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, doc}
PyMethodDef methods[] = {
    ENTRY(tables, "moe_kv_tables"), ENTRY(rope, "moe_rope"), ENTRY(append, "moe_kv_append"), ENTRY(read, "moe_kv_read"),
    ENTRY(attention, "moe_kv_attention"), ENTRY(shared_prefix, "moe_kv_shared_prefix"), ENTRY(attention_shared, "moe_kv_attention_shared"),
    ENTRY(summarise, "moe_kv_summarise"), ENTRY(read_summaries, "moe_kv_read_summaries"), ENTRY(select, "moe_kv_select"),
    ENTRY(attention_selected, "moe_kv_attention_selected"), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kv_native", "Per-step calls of include/moe_kv.h", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kv_native() { return PyModule_Create(&module); }
