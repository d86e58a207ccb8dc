// Python calls of the paged-cache operators: checks of the tensors, marshalling into the C ABI, outputs and workspaces.  These run once per layer and
// token of a serving loop, where the interpreter's share of a call was two to four times the kernel's time; the calls that are made once per
// step or less go through ctypes (__init__.py).
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <stdarg.h>
#include <string>

#include "../../include/spd.h"

namespace {

// what ends a call: a Python exception that is set already
struct Raised {};

PyObject *g_check = nullptr; // _check(where, status) of the package: raises SpdError

[[noreturn]] void value_error(const char *format, ...)
{
    va_list ap;
    va_start(ap, format);
    PyErr_FormatV(PyExc_ValueError, format, ap);
    va_end(ap);
    throw Raised{};
}

void check(const char *where, int rc)
{
    if (rc == SPD_OK) return;
    PyObject *r = PyObject_CallFunction(g_check, "si", where, rc);
    Py_XDECREF(r);
    if (!PyErr_Occurred()) PyErr_Format(PyExc_RuntimeError, "%s: status %d", where, rc);
    throw Raised{};
}

const at::Tensor &tensor(PyObject *o, const char *name)
{
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s: a tensor", name);
        throw Raised{};
    }
    return THPVariable_Unpack(o);
}
const at::Tensor *maybe_tensor(PyObject *o, const char *name) { return o == Py_None ? nullptr : &tensor(o, name); }
int32_t int32_arg(PyObject *o)
{
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    return v > 0x7fffffffL ? 0x7fffffff : v < -0x80000000L ? -0x7fffffff - 1 : (int32_t)v;
}

int index_of(const at::Tensor &t) { return t.is_cuda() ? (int)t.get_device() : -1; }
bool sizes_are(const at::Tensor &t, std::initializer_list<int64_t> s) { return t.sizes().equals(at::IntArrayRef(s)); }

// the pages' tensors as the C ABI wants them; device in `dev`
spd_kv_cache kv_cache(PyObject *k_obj, PyObject *v_obj, PyObject *ks_obj, PyObject *vs_obj, int &dev)
{
    const at::Tensor &k = tensor(k_obj, "k_pages"), &v = tensor(v_obj, "v_pages");
    int fmt = -1;
    switch (k.scalar_type()) {
    case at::kFloat: fmt = SPD_KV_F32; break;
    case at::kBFloat16: fmt = SPD_KV_BF16; break;
    case at::kFloat8_e4m3fn: fmt = SPD_KV_E4M3; break;
    case at::kChar: fmt = SPD_KV_INT8; break;
    case at::kByte: fmt = SPD_KV_INT4; break;
    default: break;
    }
    dev = index_of(k);
    if (fmt < 0 || k.dim() != 4 || dev < 0 || !k.is_contiguous())
        value_error("k_pages: contiguous CUDA tensor [n_pages, n_kv_heads, page, head_dim] of float32, bfloat16, float8_e4m3fn or int8, "
                    "or uint8 with head_dim / 2 bytes per row (4 bits)");
    if (v.scalar_type() != k.scalar_type() || !v.sizes().equals(k.sizes()) || index_of(v) != dev || !v.is_contiguous()) value_error("v_pages: like k_pages");
    const int64_t pages = k.size(0), heads = k.size(1), page = k.size(2), d = fmt == SPD_KV_INT4 ? 2 * k.size(3) : k.size(3);
    const at::Tensor *s[2] = {maybe_tensor(ks_obj, "k_scales"), maybe_tensor(vs_obj, "v_scales")};
    for (int i = 0; i < 2; ++i) {
        const char *name = i ? "v_scales" : "k_scales";
        if (fmt == SPD_KV_INT4) {
            if (!s[i] || index_of(*s[i]) != dev || s[i]->scalar_type() != at::kBFloat16 || !sizes_are(*s[i], {pages, heads, page, 2, 2}) || !s[i]->is_contiguous())
                value_error("%s: contiguous bfloat16 [n_pages, n_kv_heads, page, 2, 2] on the pages' device (4-bit caches)", name);
        } else if (fmt >= SPD_KV_E4M3) {
            if (!s[i] || index_of(*s[i]) != dev || s[i]->scalar_type() != at::kFloat || !sizes_are(*s[i], {pages, heads, page}) || !s[i]->is_contiguous())
                value_error("%s: contiguous float32 [n_pages, n_kv_heads, page] on the pages' device (8-bit caches)", name);
        } else if (s[i])
            value_error("k_scales / v_scales: for 8-bit and 4-bit caches only");
    }
    if (pages > 0x7fffffff || heads > 0x7fffffff || page > 0x7fffffff || d > 0x7fffffff) value_error("k_pages: sizes beyond 32 bits");
    return spd_kv_cache{k.data_ptr(), v.data_ptr(), s[0] ? (float *)s[0]->data_ptr() : nullptr, s[1] ? (float *)s[1]->data_ptr() : nullptr,
                        (int32_t)pages, (int32_t)heads, (int32_t)page, (int32_t)d, fmt};
}

int32_t *int32s(PyObject *o, const char *name, int dev, std::initializer_list<int64_t> shape)
{
    const at::Tensor &t = tensor(o, name);
    if (t.scalar_type() != at::kInt || index_of(t) != dev || !sizes_are(t, shape) || !t.is_contiguous()) {
        std::string s;
        for (int64_t n : shape) s += (s.empty() ? "" : ", ") + std::to_string(n);
        value_error("%s: contiguous int32 tensor [%s] on the pages' device", name, s.c_str());
    }
    return (int32_t *)t.data_ptr();
}

spd_ragged ragged(PyObject *cu, PyObject *lens, PyObject *table_obj, int dev, int64_t n_tokens)
{
    const at::Tensor &table = tensor(table_obj, "block_table");
    if (table.dim() != 2) value_error("block_table: [B, max_pages]");
    const int64_t B = table.size(0), width = table.size(1);
    if (B > 0x7ffffffe || width > 0x7fffffff || n_tokens > 0x7fffffff) value_error("block_table: sizes beyond 32 bits");
    return spd_ragged{int32s(cu, "cu_new", dev, {B + 1}), int32s(lens, "seq_lens", dev, {B}), int32s(table_obj, "block_table", dev, {B, width}),
                      (int32_t)B, (int32_t)width, (int32_t)n_tokens};
}

// A [n_tokens, heads, head_dim] tensor whose heads lie side by side; the elements between its rows
int64_t rows(const char *name, const at::Tensor &t, int dev, int64_t heads, int64_t d)
{
    if (t.dim() != 3 || index_of(t) != dev || (t.scalar_type() != at::kFloat && t.scalar_type() != at::kBFloat16) || t.size(1) != heads || t.size(2) != d ||
        t.stride(2) != 1 || (t.stride(1) != d && heads > 1))
        value_error("%s: float32 or bfloat16 [n_tokens, %lld, %lld] on the pages' device, heads side by side in a row", name, (long long)heads, (long long)d);
    return t.size(0) > 1 ? t.stride(0) : heads * d;
}
int32_t dtype_of(const at::Tensor &t) { return t.scalar_type() == at::kBFloat16; }

int32_t *flag(PyObject *o, int dev)
{
    const at::Tensor &t = tensor(o, "err");
    if (index_of(t) != dev || t.scalar_type() != at::kInt || t.numel() < 1) value_error("err: int32 tensor on the pages' device");
    return (int32_t *)t.data_ptr();
}

// f() without the interpreter's lock: other threads run while the driver makes a call wait (a full queue, an allocation)
template <typename F> auto unlocked(F f)
{
    struct Lock {
        PyThreadState *state = PyEval_SaveThread();
        ~Lock() { PyEval_RestoreThread(state); }
    } lock;
    return f();
}

struct OnDevice { // makes `dev` current; its current stream
    c10::cuda::OptionalCUDAGuard guard;
    void *stream;
    explicit OnDevice(int dev)
    {
        if (c10::cuda::current_device() != dev) guard.set_index((c10::DeviceIndex)dev);
        stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream();
    }
};

template <typename F> PyObject *guarded(Py_ssize_t n, Py_ssize_t want, F f)
{
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "%zd arguments, %zd expected", n, want);
        return nullptr;
    }
    try {
        return f();
    } catch (const Raised &) {
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "an exception without a description");
    }
    return nullptr;
}

// k, v, k_pages, v_pages, cu_new, seq_lens, block_table, err, k_scales, v_scales
PyObject *kv_write(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 10, [&]() -> PyObject * {
        int dev;
        const spd_kv_cache c = kv_cache(a[2], a[3], a[8], a[9], dev);
        const at::Tensor &k = tensor(a[0], "k"), &v = tensor(a[1], "v");
        if (k.scalar_type() != v.scalar_type() || !k.sizes().equals(v.sizes())) value_error("k and v: same dtype and shape");
        const int64_t ks = rows("k", k, dev, c.n_kv_heads, c.head_dim), vs = rows("v", v, dev, c.n_kv_heads, c.head_dim);
        const spd_ragged r = ragged(a[4], a[5], a[6], dev, k.size(0));
        int32_t *err = flag(a[7], dev);
        const OnDevice on(dev);
        void *kd = k.data_ptr(), *vd = v.data_ptr();
        check("spd_kv_write", unlocked([&] { return spd_kv_write(&c, &r, kd, vd, ks, vs, dtype_of(k), err, on.stream); }));
        Py_RETURN_NONE;
    });
}

// k, v, k_pages, v_pages, slots, err, k_scales, v_scales
PyObject *kv_write_slots(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 8, [&]() -> PyObject * {
        int dev;
        const spd_kv_cache c = kv_cache(a[2], a[3], a[6], a[7], dev);
        const at::Tensor &k = tensor(a[0], "k"), &v = tensor(a[1], "v");
        if (k.scalar_type() != v.scalar_type() || !k.sizes().equals(v.sizes())) value_error("k and v: same dtype and shape");
        const int64_t ks = rows("k", k, dev, c.n_kv_heads, c.head_dim), vs = rows("v", v, dev, c.n_kv_heads, c.head_dim), tokens = k.size(0);
        const int32_t *slots = int32s(a[4], "slots", dev, {tokens});
        if (tokens > 0x7fffffff) value_error("k: sizes beyond 32 bits");
        int32_t *err = flag(a[5], dev);
        const OnDevice on(dev);
        void *kd = k.data_ptr(), *vd = v.data_ptr();
        check("spd_kv_write_slots", unlocked([&] { return spd_kv_write_slots(&c, slots, (int32_t)tokens, kd, vd, ks, vs, dtype_of(k), err, on.stream); }));
        Py_RETURN_NONE;
    });
}

// k_pages, v_pages, cu, starts, block_table, err, n_tokens, bf16 (or -1: out given), k_scales, v_scales, k_out, v_out -> (k, v)
PyObject *kv_read(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 12, [&]() -> PyObject * {
        int dev;
        const spd_kv_cache c = kv_cache(a[0], a[1], a[8], a[9], dev);
        at::Tensor k, v;
        const int bf16 = int32_arg(a[7]);
        if (bf16 >= 0) {
            const int64_t tokens = PyLong_AsLongLong(a[6]);
            if (PyErr_Occurred()) throw Raised{};
            const auto options = tensor(a[0], "k_pages").options().dtype(bf16 ? at::kBFloat16 : at::kFloat);
            unlocked([&] {
                k = at::empty({tokens, c.n_kv_heads, c.head_dim}, options);
                v = at::empty({tokens, c.n_kv_heads, c.head_dim}, options);
            });
        } else {
            k = tensor(a[10], "out");
            v = tensor(a[11], "out");
            if (k.scalar_type() != v.scalar_type() || !k.sizes().equals(v.sizes())) value_error("out: two tensors of one dtype and shape");
        }
        const int64_t ks = rows("k", k, dev, c.n_kv_heads, c.head_dim), vs = rows("v", v, dev, c.n_kv_heads, c.head_dim);
        const spd_ragged r = ragged(a[2], a[3], a[4], dev, k.size(0));
        int32_t *err = flag(a[5], dev);
        {
            const OnDevice on(dev);
            void *kd = k.data_ptr(), *vd = v.data_ptr();
            check("spd_kv_read", unlocked([&] { return spd_kv_read(&c, &r, kd, vd, ks, vs, dtype_of(k), err, on.stream); }));
        }
        PyObject *pair = PyTuple_New(2);
        if (!pair) throw Raised{};
        PyTuple_SET_ITEM(pair, 0, THPVariable_Wrap(k));
        PyTuple_SET_ITEM(pair, 1, THPVariable_Wrap(v));
        return pair;
    });
}

// q, k_pages, v_pages, cu_new, seq_lens, block_table, max_new, max_context, err, window, sinks, scale, k_scales, v_scales, out, workspace -> out
PyObject *paged_attention(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 16, [&]() -> PyObject * {
        int dev;
        const spd_kv_cache c = kv_cache(a[1], a[2], a[12], a[13], dev);
        const at::Tensor &q = tensor(a[0], "q");
        if (q.dim() != 3) value_error("q: [n_tokens, n_q_heads, head_dim]");
        const int64_t tokens = q.size(0), nq = q.size(1), d = q.size(2), qs = rows("q", q, dev, nq, c.head_dim);
        if (nq > 0x7fffffff) value_error("q: sizes beyond 32 bits");
        at::Tensor out;
        int64_t os = nq * d;
        if (a[14] == Py_None) unlocked([&] { out = at::empty({tokens, nq, d}, q.options()); });
        else {
            out = tensor(a[14], "out");
            if (out.scalar_type() != q.scalar_type() || !out.sizes().equals(q.sizes())) value_error("out: shape and dtype of q");
            os = rows("out", out, dev, nq, d);
        }
        const spd_ragged r = ragged(a[3], a[4], a[5], dev, tokens);
        const int32_t max_new = int32_arg(a[6]), max_context = int32_arg(a[7]), window = int32_arg(a[9]), sinks = int32_arg(a[10]);
        double scale = 1.0 / std::sqrt((double)d);
        if (a[11] != Py_None) {
            scale = PyFloat_AsDouble(a[11]);
            if (PyErr_Occurred()) throw Raised{};
        }
        int32_t *err = flag(a[8], dev);
        at::Tensor ws;
        void *ws_ptr = nullptr;
        size_t ws_bytes = 0;
        if (a[15] != Py_None) {
            ws = tensor(a[15], "workspace");
            if (index_of(ws) != dev || ws.scalar_type() != at::kByte || !ws.is_contiguous()) value_error("workspace: contiguous uint8 tensor on the pages' device");
            ws_ptr = ws.data_ptr();
            ws_bytes = (size_t)ws.numel();
        }
        {
            const OnDevice on(dev);
            void *qd = q.data_ptr(), *od = out.data_ptr();
            const bool own_ws = a[15] == Py_None;
            check("spd_paged_attention", unlocked([&] {
                // what the arguments ask for; what they are refused for the call itself says
                if (own_ws && spd_paged_attention_workspace_bytes(&c, r.B, r.n_tokens, dtype_of(q), (int32_t)nq, max_new, max_context, window, sinks, &ws_bytes) == SPD_OK &&
                    ws_bytes && r.B && r.n_tokens) {
                    ws = at::empty({(int64_t)ws_bytes}, q.options().dtype(at::kByte));
                    ws_ptr = ws.data_ptr();
                }
                return spd_paged_attention(&c, &r, qd, qs, od, os, dtype_of(q), (int32_t)nq, max_new, max_context, (float)scale, window, sinks, ws_ptr, ws_ptr ? ws_bytes : 0, err,
                                           on.stream);
            }));
        }
        if (a[14] != Py_None) {
            Py_INCREF(a[14]);
            return a[14];
        }
        return THPVariable_Wrap(out);
    });
}

// seq_lens, new_lens, block_table, free_pages, n_free, page, n_pages, n_tokens, err, out (None or five tensors) -> five tensors
PyObject *plan_batch(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 10, [&]() -> PyObject * {
        const at::Tensor &table = tensor(a[2], "block_table");
        const int dev = index_of(table);
        if (table.dim() != 2 || dev < 0) value_error("block_table: CUDA tensor [B, max_pages]");
        const int64_t B = table.size(0), width = table.size(1);
        if (B > 0x7ffffffe || width > 0x7fffffff) value_error("block_table: sizes beyond 32 bits");
        const int32_t page = int32_arg(a[5]), n_pages = int32_arg(a[6]), n_tokens = int32_arg(a[7]);
        if (n_tokens < 0 || n_tokens > 1 << 30) check("spd_plan_batch", SPD_EINVAL); // before there are outputs of such a size
        const int64_t sizes[5] = {B + 1, n_tokens, n_tokens, B, 1};
        static const char *const names[5] = {"out.cu_new", "out.positions", "out.slots", "out.next_lens", "out.n_free"};
        PyObject *result = nullptr;
        int32_t *p[5];
        if (a[9] == Py_None) {
            result = PyTuple_New(5);
            if (!result) throw Raised{};
            at::AutoDispatchBelowADInplaceOrView views;
            const at::Tensor all = unlocked([&] { return at::empty({2 * B + 2 + 2 * (int64_t)n_tokens}, table.options().dtype(at::kInt)); });
            int64_t at_ = 0;
            for (int i = 0; i < 5; ++i) {
                const at::Tensor t = all.narrow(0, at_, sizes[i]);
                p[i] = (int32_t *)all.data_ptr() + at_;
                at_ += sizes[i];
                PyTuple_SET_ITEM(result, i, THPVariable_Wrap(t));
            }
        } else {
            if (!PyTuple_Check(a[9]) || PyTuple_GET_SIZE(a[9]) != 5) value_error("out: a BatchPlan");
            for (int i = 0; i < 5; ++i) p[i] = int32s(PyTuple_GET_ITEM(a[9], i), names[i], dev, {sizes[i]});
            result = a[9];
            Py_INCREF(result);
        }
        try {
            const spd_page_pool pool{int32s(a[3], "free_pages", dev, {n_pages}), int32s(a[4], "n_free", dev, {1}), p[4], n_pages, page};
            const int32_t *lens = int32s(a[0], "seq_lens", dev, {B}), *news = int32s(a[1], "new_lens", dev, {B});
            int32_t *entries = int32s(a[2], "block_table", dev, {B, width}), *err = flag(a[8], dev);
            const OnDevice on(dev);
            check("spd_plan_batch", unlocked([&] { return spd_plan_batch(&pool, lens, news, (int32_t)B, entries, (int32_t)width, n_tokens, p[0], p[1], p[2], p[3], err, on.stream); }));
        } catch (...) {
            Py_DECREF(result);
            throw;
        }
        return result;
    });
}

PyObject *set_check(PyObject *, PyObject *f)
{
    Py_INCREF(f);
    Py_XSETREF(g_check, f);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"kv_write", (PyCFunction)(void (*)(void))kv_write, METH_FASTCALL, nullptr},
    {"kv_write_slots", (PyCFunction)(void (*)(void))kv_write_slots, METH_FASTCALL, nullptr},
    {"kv_read", (PyCFunction)(void (*)(void))kv_read, METH_FASTCALL, nullptr},
    {"paged_attention", (PyCFunction)(void (*)(void))paged_attention, METH_FASTCALL, nullptr},
    {"plan_batch", (PyCFunction)(void (*)(void))plan_batch, METH_FASTCALL, nullptr},
    {"set_check", set_check, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", "Calls of the paged-cache operators.", -1, methods, nullptr, nullptr, nullptr, nullptr};

} // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
