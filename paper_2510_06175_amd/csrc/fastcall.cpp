// Python module _fastcall: the argument checks of binding.py and the library call, in one native call.
//
// The checks of a step's 11 tensors (device, type, shape, contiguity, each an attribute read by the interpreter) and
// the conversion of 20 arguments by ctypes are host time in front of a launch that may itself take less:
// appends of one token to 32 sequences, called back to back, 7.9 us each by ctypes, 5.8 here (the kernel then bounds them);
// steps of 1000 tokens 10.12 -> 9.99 us, longer ones unchanged.
//
// Every function returns the library's status, or None where an argument is not what it expects: binding.py then
// goes through its own checks, which say what is wrong (or accept what only they can judge, such as subclasses
// of torch.Tensor).  Nothing is kept between calls but the library's functions and the one that finds the stream.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <exception>
#include <initializer_list>

#include "../../include/vecinfer.h"

namespace {

decltype(&vecinfer_encode_keys) encode_keys;
decltype(&vecinfer_encode_values) encode_values;
decltype(&vecinfer_append_kv) append_kv;
decltype(&vecinfer_decode_attention) decode_attention;
decltype(&vecinfer_decode_attention_residual) decode_residual;
decltype(&vecinfer_decode_step) decode_step;
decltype(&vecinfer_rotary) rotary_call;
decltype(&vecinfer_paged_append) paged_append_call;
decltype(&vecinfer_paged_attention) paged_attention_call;
decltype(&vecinfer_paged_evict) paged_evict_call;
PyObject *find_stream;                   // binding._stream
PyObject *find_stream_on;                // binding._stream_on
PyObject *get_device, *get_stream;       // torch's own functions for the current device and its stream's handle, or None

struct Refused {};                       // an argument that the interpreter's checks have to look at
struct Raised {};                        // Python's error is set

const at::Tensor &tensor(PyObject *o)
{
    if (!THPVariable_CheckExact(o)) throw Refused();
    return THPVariable_Unpack(o);
}

// A contiguous tensor on the GPU of this type and shape.
void *pointer(const at::Tensor &t, at::ScalarType type, std::initializer_list<int64_t> shape)
{
    if (!t.is_cuda() || t.scalar_type() != type || !t.sizes().equals(c10::IntArrayRef(shape)) || !t.is_contiguous()) throw Refused();
    return t.data_ptr();
}

void *pointer(PyObject *o, at::ScalarType type, std::initializer_list<int64_t> shape) { return pointer(tensor(o), type, shape); }

int64_t extent(const at::Tensor &t, int64_t dims, int64_t i)
{
    if (t.dim() != dims) throw Refused();
    return t.size(i);
}

int64_t integer(PyObject *o)
{
    if (!PyLong_CheckExact(o)) throw Refused();
    int overflow = 0;
    const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
    if (overflow) throw Refused();
    return v;
}

int32_t integer32(PyObject *o)
{
    const int64_t v = integer(o);
    if (v != (int32_t)v) throw Refused();
    return (int32_t)v;
}

void *address(PyObject *o)
{
    void *p = PyLong_Check(o) ? PyLong_AsVoidPtr(o) : nullptr;
    if (PyErr_Occurred()) {
        PyErr_Clear();
        throw Refused();
    }
    return p;
}

// The stream's handle, asked for after the checks as the interpreter's path does, and what that raises is raised: it may
// be an interrupt, which a second attempt would not see.
void *stream_of(PyObject *o)
{
    PyObject *const r = PyObject_CallFunctionObjArgs(find_stream, o, nullptr);
    if (!r) throw Raised();
    struct Release {
        PyObject *r;
        ~Release() { Py_DECREF(r); }
    } release{r};
    return address(r);
}

// What a call needs of its configuration.
struct Cfg {
    const vecinfer_cfg *c;
    int64_t D, Hq, Hkv;
    explicit Cfg(PyObject *o) : c(static_cast<const vecinfer_cfg *>(address(o)))
    {
        if (!c) throw Refused();
        D = c->head_dim;
        Hq = c->num_q_heads;
        Hkv = c->num_kv_heads;
        if (c->k_sub_dim < 1 || c->v_sub_dim < 1 || c->k_bits < 1 || c->v_bits < 1 || c->k_bits > 30 || c->v_bits > 30) throw Refused();
    }
    int64_t row(bool keys) const { return D / (keys ? c->k_sub_dim : c->v_sub_dim) * (keys ? c->k_bits : c->v_bits) / 8; }
    void *codebook(PyObject *o, bool keys) const
    {
        const int64_t d = keys ? c->k_sub_dim : c->v_sub_dim, bits = keys ? c->k_bits : c->v_bits;
        return bits == 8 ? pointer(o, at::kHalf, {Hkv, D / d, 256, d}) : pointer(o, at::kHalf, {Hkv, (int64_t)1 << bits, d});
    }
    const float *lambda(PyObject *o) const { return static_cast<const float *>(pointer(o, at::kFloat, {Hkv, D})); }
    uint8_t *codes(PyObject *o, bool keys, int64_t B, int64_t n_cap) const
    {
        return static_cast<uint8_t *>(pointer(o, at::kByte, {B, Hkv, n_cap, row(keys)}));
    }
};

// f: a call of the library, which throws nothing.  (Where the interpreter is shutting down, PyEval_RestoreThread ends
// a daemon thread by unwinding it: no destructor and no catch-all may stand in its way, or the process aborts.)
template <typename F>
int without_gil(F &&f)
{
    PyThreadState *const state = PyEval_SaveThread();
    const int rc = f();
    PyEval_RestoreThread(state);
    return rc;
}

// f() -> status; None for anything that is not as expected (also torch's own exceptions: wrapped tensors
// have no data pointer).
template <typename F>
PyObject *guarded(F &&f)
{
    try {
        return PyLong_FromLong(f());
    } catch (const Raised &) {
        return nullptr;
    } catch (const Refused &) {
    } catch (const std::exception &) {
    }
    Py_RETURN_NONE;
}

// encode(cfg, x, lambda or None (values), codebook, codes, pos0, stream)
PyObject *encode(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&] {
        if (n != 7) throw Refused();
        const Cfg cfg(a[0]);
        const bool keys = a[2] != Py_None;
        const at::Tensor &x = tensor(a[1]);
        const int64_t B = extent(x, 4, 0), T = extent(x, 4, 2), n_cap = extent(tensor(a[4]), 4, 2), pos0 = integer(a[5]);
        const void *const px = pointer(x, at::kHalf, {B, cfg.Hkv, T, cfg.D});
        const float *const lam = keys ? cfg.lambda(a[2]) : nullptr;
        const void *const cb = cfg.codebook(a[3], keys);
        uint8_t *const idx = cfg.codes(a[4], keys, B, n_cap);
        if (B != (int32_t)B) throw Refused();
        void *const stream = stream_of(a[6]);
        return without_gil([&] {
            return keys ? encode_keys(cfg.c, px, lam, cb, idx, (int32_t)B, T, pos0, n_cap, stream)
                        : encode_values(cfg.c, px, cb, idx, (int32_t)B, T, pos0, n_cap, stream);
        });
    });
}

// append(cfg, k, v, lambda, cb_k, cb_v, k_idx, v_idx, pos0, stream)
PyObject *append(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&] {
        if (n != 10) throw Refused();
        const Cfg cfg(a[0]);
        const at::Tensor &k = tensor(a[1]);
        const int64_t B = extent(k, 4, 0), T = extent(k, 4, 2), n_cap = extent(tensor(a[6]), 4, 2), pos0 = integer(a[8]);
        const void *const pk = pointer(k, at::kHalf, {B, cfg.Hkv, T, cfg.D}), *const pv = pointer(a[2], at::kHalf, {B, cfg.Hkv, T, cfg.D});
        const float *const lam = cfg.lambda(a[3]);
        const void *const cb_k = cfg.codebook(a[4], true), *const cb_v = cfg.codebook(a[5], false);
        uint8_t *const k_idx = cfg.codes(a[6], true, B, n_cap), *const v_idx = cfg.codes(a[7], false, B, n_cap);
        if (B != (int32_t)B) throw Refused();
        void *const stream = stream_of(a[9]);
        return without_gil([&] { return append_kv(cfg.c, pk, pv, lam, cb_k, cb_v, k_idx, v_idx, (int32_t)B, T, pos0, n_cap, stream); });
    });
}

// decode(cfg, q, lambda, cb_k, cb_v, k_idx, v_idx, workspace, out, lse or None, seq_lens or None, N or None, num_splits,
//        variant, stream [, k_new, v_new] [, k_res, v_res, res_lens or None, R or None])
PyObject *decode(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&] {
        if (n != 15 && n != 17 && n != 19) throw Refused();
        const Cfg cfg(a[0]);
        const at::Tensor &q = tensor(a[1]), &ws = tensor(a[7]);
        const int64_t B = extent(q, 3, 0), n_cap = extent(tensor(a[5]), 4, 2), N = a[11] == Py_None ? n_cap : integer(a[11]);
        const void *const pq = pointer(q, at::kHalf, {B, cfg.Hq, cfg.D});
        const float *const lam = cfg.lambda(a[2]);
        const void *const cb_k = cfg.codebook(a[3], true), *const cb_v = cfg.codebook(a[4], false);
        uint8_t *const k_idx = cfg.codes(a[5], true, B, n_cap), *const v_idx = cfg.codes(a[6], false, B, n_cap);
        void *const out = pointer(a[8], at::kHalf, {B, cfg.Hq, cfg.D});
        float *const lse = a[9] == Py_None ? nullptr : static_cast<float *>(pointer(a[9], at::kFloat, {B, cfg.Hq}));
        const int32_t *const lens = a[10] == Py_None ? nullptr : static_cast<const int32_t *>(pointer(a[10], at::kInt, {B}));
        const int32_t splits = integer32(a[12]), variant = integer32(a[13]);
        void *const wp = ws.data_ptr();
        const size_t wb = (size_t)ws.numel() * ws.element_size();
        if (B != (int32_t)B) throw Refused();
        const int32_t b = (int32_t)B;
        if (n == 15) {
            void *const stream = stream_of(a[14]);
            return without_gil([&] {
                return decode_attention(cfg.c, pq, lam, cb_k, cb_v, k_idx, v_idx, lens, b, N, n_cap, splits, variant, wp, wb, out, lse, stream);
            });
        }
        if (n == 17) {
            const void *const k = pointer(a[15], at::kHalf, {B, cfg.Hkv, 1, cfg.D}), *const v = pointer(a[16], at::kHalf, {B, cfg.Hkv, 1, cfg.D});
            void *const stream = stream_of(a[14]);
            return without_gil([&] {
                return decode_step(cfg.c, pq, k, v, lam, cb_k, cb_v, k_idx, v_idx, lens, b, N, n_cap, splits, variant, wp, wb, out, lse, stream);
            });
        }
        const int64_t r_cap = extent(tensor(a[15]), 4, 2);
        const void *const k = pointer(a[15], at::kHalf, {B, cfg.Hkv, r_cap, cfg.D}), *const v = pointer(a[16], at::kHalf, {B, cfg.Hkv, r_cap, cfg.D});
        const int32_t *const res = a[17] == Py_None ? nullptr : static_cast<const int32_t *>(pointer(a[17], at::kInt, {B}));
        if (a[18] == Py_None && r_cap != (int32_t)r_cap) throw Refused();
        const int32_t R = a[18] == Py_None ? (int32_t)r_cap : integer32(a[18]);
        void *const stream = stream_of(a[14]);
        return without_gil([&] {
            return decode_residual(cfg.c, pq, lam, cb_k, cb_v, k_idx, v_idx, lens, b, N, n_cap, k, v, res, R, r_cap, splits, variant, wp, wb, out,
                                   lse, stream);
        });
    });
}

// bind(addresses of the library's functions, in the order of the variables above, then the function for streams)
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 7) {
        PyErr_SetString(PyExc_TypeError, "bind: six addresses and a function");
        return nullptr;
    }
    void *p[6];
    for (int i = 0; i < 6; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    Py_INCREF(a[6]);
    Py_XDECREF(find_stream);
    find_stream = a[6];
    encode_keys = reinterpret_cast<decltype(encode_keys)>(p[0]);
    encode_values = reinterpret_cast<decltype(encode_values)>(p[1]);
    append_kv = reinterpret_cast<decltype(append_kv)>(p[2]);
    decode_attention = reinterpret_cast<decltype(decode_attention)>(p[3]);
    decode_residual = reinterpret_cast<decltype(decode_residual)>(p[4]);
    decode_step = reinterpret_cast<decltype(decode_step)>(p[5]);
    Py_RETURN_NONE;
}

// ---- the paged cache and rotary positions

// What a call needs of its pages, and of the device that they are on.
struct Pool {
    const vecinfer_pages *p;
    at::ScalarType type;
    int64_t D, Hkv, device;
    Pool(PyObject *o, PyObject *dev) : p(static_cast<const vecinfer_pages *>(address(o))), device(integer(dev))
    {
        if (!p) throw Refused();
        type = p->dtype == VECINFER_BF16 ? at::kBFloat16 : at::kHalf;
        D = p->head_dim;
        Hkv = p->num_kv_heads;
    }
};

void on(const at::Tensor &t, int64_t device)
{
    if (!t.is_cuda() || t.get_device() != device) throw Refused();
}

// A contiguous tensor on that device, or None.
template <typename T>
T *flat(PyObject *o, int64_t device, at::ScalarType type, std::initializer_list<int64_t> shape)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o);
    on(t, device);
    return static_cast<T *>(pointer(t, type, shape));
}

// A tensor of any strides with adjacent channels, and the strides of its other axes (an axis of one index has none).
template <int N>
void *rows(const at::Tensor &t, int64_t device, at::ScalarType type, std::initializer_list<int64_t> shape, int64_t (&steps)[N], bool written = false)
{
    on(t, device);
    if (t.scalar_type() != type || !t.sizes().equals(c10::IntArrayRef(shape)) || t.dim() != N + 1) throw Refused();
    if (t.size(N) > 1 && t.stride(N) != 1) throw Refused();
    for (int i = 0; i < N; ++i) {
        steps[i] = t.size(i) > 1 ? t.stride(i) : 0;
        if (written && t.size(i) > 1 && steps[i] == 0) throw Refused();
    }
    return t.data_ptr();
}

// The stream for work on that device; raises where it is not the current one.  The usual case, the current stream of the
// current device, is asked of torch's own functions (0.2 us less than by binding._stream_on, of 4 for a small call).
void *stream_on(PyObject *o, int64_t device)
{
    if (o == Py_None && get_device != Py_None && get_stream != Py_None) {
        PyObject *const d = PyObject_CallNoArgs(get_device);
        if (!d) throw Raised();
        const bool current = PyLong_CheckExact(d) && PyLong_AsLongLong(d) == device;
        PyObject *const s = current ? PyObject_CallOneArg(get_stream, d) : nullptr;
        Py_DECREF(d);
        if (current) {
            if (!s) throw Raised();
            void *const p = PyLong_Check(s) ? PyLong_AsVoidPtr(s) : nullptr;
            Py_DECREF(s);
            if (PyErr_Occurred()) throw Raised();
            return p;
        }
    }
    PyObject *const dev = PyLong_FromLongLong(device);
    if (!dev) throw Raised();
    PyObject *const r = PyObject_CallFunctionObjArgs(find_stream_on, o, dev, nullptr);
    Py_DECREF(dev);
    if (!r) throw Raised();
    struct Release {
        PyObject *r;
        ~Release() { Py_DECREF(r); }
    } release{r};
    return address(r);
}

int32_t narrow(int64_t v)
{
    if (v != (int32_t)v) throw Refused();
    return (int32_t)v;
}

// rotary(cfg, table, x, out, positions or None, pos0, inverse, stream)
PyObject *rotary(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&] {
        if (n != 8) throw Refused();
        const vecinfer_rotary_cfg *const cfg = static_cast<const vecinfer_rotary_cfg *>(address(a[0]));
        const at::Tensor &x = tensor(a[2]), &out = tensor(a[3]);
        const int64_t B = extent(x, 4, 0), H = x.size(1), T = x.size(2), D = cfg->head_dim, dev = x.is_cuda() ? x.get_device() : -1;
        const at::ScalarType type = x.scalar_type();
        if (type != at::kHalf && type != at::kBFloat16) throw Refused();
        int64_t xs[3], os[3];
        const void *const px = rows(x, dev, type, {B, H, T, D}, xs);
        void *const po = rows(out, dev, type, {B, H, T, D}, os, true);
        const uint64_t *const table = reinterpret_cast<const uint64_t *>(flat<int64_t>(a[1], dev, at::kLong, {(int64_t)(cfg->rot_dim / 2)}));
        const int32_t *const pos = flat<int32_t>(a[4], dev, at::kInt, {B, T});
        const int64_t pos0 = integer(a[5]);
        const int32_t b = narrow(B), h = narrow(H), inverse = PyObject_IsTrue(a[6]);
        if (inverse < 0) throw Raised();
        void *const stream = stream_on(a[7], dev);
        return without_gil([&] {
            return rotary_call(cfg, table, type == at::kBFloat16 ? VECINFER_BF16 : VECINFER_F16, px, xs, po, os, b, h, T, pos, pos0, inverse, stream);
        });
    });
}

// paged_append(pages, device, rot or None, table or None, k_new, v_new, q or None, q_out or None, block_table, seq_lens,
//              new_lens or None, positions or None, weights or None, stream)
PyObject *paged_append(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&] {
        if (n != 14) throw Refused();
        const Pool pool(a[0], a[1]);
        const int64_t dev = pool.device;
        const vecinfer_rotary_cfg *const rot = a[2] == Py_None ? nullptr : static_cast<const vecinfer_rotary_cfg *>(address(a[2]));
        const uint64_t *const table =
            rot ? reinterpret_cast<const uint64_t *>(flat<int64_t>(a[3], dev, at::kLong, {(int64_t)(rot->rot_dim / 2)})) : nullptr;
        const at::Tensor &k = tensor(a[4]), &v = tensor(a[5]), &bt = tensor(a[8]);
        const int64_t B = extent(k, 4, 0), T = k.size(2), cols = extent(bt, 2, 1);
        int64_t ks[3], vs[3], qs[3], os[3], Hq = 0, w_cap = 0;
        const void *const pk = rows(k, dev, pool.type, {B, pool.Hkv, T, pool.D}, ks), *const pv = rows(v, dev, pool.type, {B, pool.Hkv, T, pool.D}, vs);
        if ((a[6] == Py_None) != (a[7] == Py_None)) throw Refused();
        const void *pq = nullptr;
        void *po = nullptr;
        if (a[6] != Py_None) {
            const at::Tensor &q = tensor(a[6]);
            Hq = extent(q, 4, 1);
            pq = rows(q, dev, pool.type, {B, Hq, T, pool.D}, qs);
            po = rows(tensor(a[7]), dev, pool.type, {B, Hq, T, pool.D}, os, true);
        }
        const int32_t *const pages = flat<int32_t>(a[8], dev, at::kInt, {B, cols}), *const lens = flat<int32_t>(a[9], dev, at::kInt, {B});
        const int32_t *const fresh = flat<int32_t>(a[10], dev, at::kInt, {B}), *const pos = flat<int32_t>(a[11], dev, at::kInt, {B, T});
        if (a[12] != Py_None) w_cap = extent(tensor(a[12]), 3, 2);
        float *const w = flat<float>(a[12], dev, at::kFloat, {B, pool.Hkv, w_cap});
        const int32_t b = narrow(B), hq = narrow(Hq);
        void *const stream = stream_on(a[13], dev);
        return without_gil([&] {
            return paged_append_call(pool.p, rot, table, pk, ks, pv, vs, pq, qs, po, os, hq, pages, cols, lens, fresh, pos, b, T, w, w_cap, stream);
        });
    });
}

// paged_attention(pages, device, q, block_table, workspace, out, lse or None, seq_lens or None, N or None, scale or None,
//                 num_splits, weights_in or None, weights_out or None, stream)
PyObject *paged_attention(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&] {
        if (n != 14) throw Refused();
        const Pool pool(a[0], a[1]);
        const int64_t dev = pool.device;
        const at::Tensor &q = tensor(a[2]), &bt = tensor(a[3]), &ws = tensor(a[4]);
        const int64_t B = extent(q, 3, 0), Hq = q.size(1), cols = extent(bt, 2, 1);
        int64_t qs[2], w_cap = 0;
        const void *const pq = rows(q, dev, pool.type, {B, Hq, pool.D}, qs);
        const int32_t *const pages = flat<int32_t>(a[3], dev, at::kInt, {B, cols});
        on(ws, dev);
        if (!ws.is_contiguous()) throw Refused();
        void *const wp = ws.data_ptr();
        const size_t wb = (size_t)ws.numel() * ws.element_size();
        if (a[5] == Py_None) throw Refused();
        void *const out = flat<void>(a[5], dev, pool.type, {B, Hq, pool.D});
        float *const lse = flat<float>(a[6], dev, at::kFloat, {B, Hq});
        const int32_t *const lens = flat<int32_t>(a[7], dev, at::kInt, {B});
        const int64_t N = a[8] == Py_None ? cols * pool.p->page_size : integer(a[8]);
        double scale = 0;
        if (a[9] == Py_None)
            scale = pool.D == 64 ? 0.125 : 0.08838834764831845;            // 1 / sqrt(D)
        else if (PyFloat_CheckExact(a[9]))
            scale = PyFloat_AS_DOUBLE(a[9]);
        else
            throw Refused();
        const int32_t splits = integer32(a[10]);
        if (a[12] == Py_None && a[11] != Py_None) throw Refused();
        if (a[12] != Py_None) w_cap = extent(tensor(a[12]), 3, 2);
        const float *const w_in = flat<float>(a[11], dev, at::kFloat, {B, pool.Hkv, w_cap});
        float *const w_out = flat<float>(a[12], dev, at::kFloat, {B, pool.Hkv, w_cap});
        const int32_t b = narrow(B), hq = narrow(Hq);
        void *const stream = stream_on(a[13], dev);
        return without_gil([&] {
            return paged_attention_call(pool.p, pq, qs, hq, pages, cols, lens, b, N, (float)scale, splits, wp, wb, out, lse, w_in, w_out, w_cap, stream);
        });
    });
}

// paged_evict(pages, device, weights, block_table, dst_pages, dst_device, dst_table, dst_lens, workspace, keep, first, recent,
//             seq_lens or None, N or None, dst_weights or None, kept or None, stream)
PyObject *paged_evict(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&] {
        if (n != 17) throw Refused();
        const Pool src(a[0], a[1]), dst(a[4], a[5]);
        const int64_t dev = src.device;
        if (dst.device != dev) throw Refused();
        const at::Tensor &w = tensor(a[2]), &bt = tensor(a[3]), &dt = tensor(a[6]), &ws = tensor(a[8]);
        const int64_t B = extent(bt, 2, 0), cols = bt.size(1), dcols = extent(dt, 2, 1), w_cap = extent(w, 3, 2);
        const float *const pw = flat<float>(a[2], dev, at::kFloat, {B, src.Hkv, w_cap});
        const int32_t *const pages = flat<int32_t>(a[3], dev, at::kInt, {B, cols}), *const dpages = flat<int32_t>(a[6], dev, at::kInt, {B, dcols});
        if (a[7] == Py_None) throw Refused();
        int32_t *const dlens = flat<int32_t>(a[7], dev, at::kInt, {B});
        on(ws, dev);
        if (!ws.is_contiguous()) throw Refused();
        void *const wp = ws.data_ptr();
        const size_t wb = (size_t)ws.numel() * ws.element_size();
        const int64_t keep = integer(a[9]), first = integer(a[10]), recent = integer(a[11]), all = cols * src.p->page_size;
        const int32_t *const lens = flat<int32_t>(a[12], dev, at::kInt, {B});
        const int64_t N = a[13] == Py_None ? (w_cap < all ? w_cap : all) : integer(a[13]);
        const int64_t dw_cap = a[14] == Py_None ? 0 : extent(tensor(a[14]), 3, 2);
        float *const dw = flat<float>(a[14], dev, at::kFloat, {B, src.Hkv, dw_cap});
        int32_t *const kept = flat<int32_t>(a[15], dev, at::kInt, {B, src.Hkv, keep});
        const int32_t b = narrow(B);
        void *const stream = stream_on(a[16], dev);
        return without_gil([&] {
            return paged_evict_call(src.p, pw, w_cap, pages, cols, lens, b, N, keep, first, recent, dst.p, dpages, dcols, dlens, dw, dw_cap, kept, wp, wb,
                                    stream);
        });
    });
}

// bind_paged(addresses of the library's functions, in the order of the variables above, then the function for streams and
// torch's for the current device and for its stream's handle, or None)
PyObject *bind_paged(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 7) {
        PyErr_SetString(PyExc_TypeError, "bind_paged: four addresses and three functions");
        return nullptr;
    }
    void *p[4];
    for (int i = 0; i < 4; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    PyObject **const held[3] = {&find_stream_on, &get_device, &get_stream};
    for (int i = 0; i < 3; ++i) {
        Py_INCREF(a[4 + i]);
        Py_XDECREF(*held[i]);
        *held[i] = a[4 + i];
    }
    rotary_call = reinterpret_cast<decltype(rotary_call)>(p[0]);
    paged_append_call = reinterpret_cast<decltype(paged_append_call)>(p[1]);
    paged_attention_call = reinterpret_cast<decltype(paged_attention_call)>(p[2]);
    paged_evict_call = reinterpret_cast<decltype(paged_evict_call)>(p[3]);
    Py_RETURN_NONE;
}

#define VECINFER_METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {VECINFER_METHOD(bind), VECINFER_METHOD(encode), VECINFER_METHOD(append), VECINFER_METHOD(decode),
                         VECINFER_METHOD(bind_paged), VECINFER_METHOD(rotary), VECINFER_METHOD(paged_append), VECINFER_METHOD(paged_attention),
                         VECINFER_METHOD(paged_evict),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

} // namespace

PyMODINIT_FUNC PyInit__fastcall()
{
    PyObject *const m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", TORCH_VERSION) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
