// Python side of the calls that a decode loop makes once per layer: argument marshalling only.
//
// A decode call on a short context takes the GPU 4 - 6 us, less than ctypes and torch.cuda.current_stream() took to
// prepare it (7 of 12.5 us a call).  These functions take the same objects — the ctypes structures of the C header
// through the buffer protocol, torch tensors through data_ptr() — and return the library's status; each tensor costs one
// method call and the stream two plain C++ calls into torch.  The interpreter lock is released around the library call.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "../../include/sa.h"

namespace {

PyObject *g_data_ptr, *g_nbytes, *g_get_device, *g_get_stream, *g_shape, *g_stride, *g_is_contiguous, *g_dtype, *g_device_of, *g_float16, *g_int16, *g_uint16, *g_int32, *g_bfloat16;

struct Args {
    PyObject* const* v;
    Py_ssize_t n, i = 0;
    bool bad = false;

    PyObject* next() {
        if (i >= n) {
            bad = true;
            PyErr_SetString(PyExc_TypeError, "too few arguments");
            return nullptr;
        }
        return v[i++];
    }
    // pointer of a ctypes structure (it outlives the call: the caller holds it)
    template <typename T>
    const T* structure() {
        PyObject* o = bad ? nullptr : next();
        Py_buffer b;
        if (!o || PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) {
            bad = true;
            return nullptr;
        }
        const bool fits = b.len == (Py_ssize_t)sizeof(T);
        const T* p = static_cast<const T*>(b.buf);
        PyBuffer_Release(&b);
        if (!fits) {
            bad = true;
            PyErr_SetString(PyExc_TypeError, "not the structure of the C header");
        }
        return p;
    }
    unsigned long long number_of(PyObject* o) {
        if (!o) {
            bad = true;
            return 0;
        }
        const unsigned long long x = PyLong_AsUnsignedLongLong(o);
        if (x == (unsigned long long)-1 && PyErr_Occurred()) bad = true;
        Py_DECREF(o);
        return x;
    }
    // address of a tensor; None is NULL
    template <typename T>
    T* tensor() {
        PyObject* o = bad ? nullptr : next();
        if (!o || o == Py_None) return nullptr;
        return reinterpret_cast<T*>(number_of(PyObject_CallMethodNoArgs(o, g_data_ptr)));
    }
    void* tensor_and_bytes(size_t* bytes) {
        PyObject* o = bad ? nullptr : next();
        *bytes = 0;
        if (!o) return nullptr;
        *bytes = (size_t)number_of(PyObject_GetAttr(o, g_nbytes));
        return bad ? nullptr : reinterpret_cast<void*>(number_of(PyObject_CallMethodNoArgs(o, g_data_ptr)));
    }
    bool fail(const char* what) {
        if (!bad) PyErr_SetString(PyExc_ValueError, what);
        bad = true;
        return false;
    }
    // What a tensor of n dimensions has to be, at a price that a call of a few microseconds can bear: each of these is one attribute or method.
    bool shape(PyObject* o, int n, long long* out) {
        PyObject* sh = bad ? nullptr : PyObject_GetAttr(o, g_shape);
        bool ok = sh && PyTuple_Check(sh) && PyTuple_GET_SIZE(sh) == n;
        for (int i = 0; ok && i < n; ++i) out[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(sh, i));
        Py_XDECREF(sh);
        return ok;
    }
    bool strides(PyObject* o, int n, long long* out) {        // in elements
        PyObject* st = bad ? nullptr : PyObject_CallMethodNoArgs(o, g_stride);
        bool ok = st && PyTuple_Check(st) && PyTuple_GET_SIZE(st) == n;
        for (int i = 0; ok && i < n; ++i) out[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(st, i));
        Py_XDECREF(st);
        return ok;
    }
    bool contiguous(PyObject* o) {
        PyObject* c = bad ? nullptr : PyObject_CallMethodNoArgs(o, g_is_contiguous);
        const bool ok = c == Py_True;
        Py_XDECREF(c);
        return ok;
    }
    bool on_device(PyObject* o, long long device) {           // (a tensor that is not on a CUDA device says -1)
        PyObject* d = bad ? nullptr : PyObject_CallMethodNoArgs(o, g_device_of);
        const bool ok = d && PyLong_AsLongLong(d) == device;
        Py_XDECREF(d);
        return ok;
    }
    bool typed(PyObject* o, PyObject* dtype) {
        PyObject* t = bad ? nullptr : PyObject_GetAttr(o, g_dtype);
        const bool ok = t && t == dtype;
        Py_XDECREF(t);
        return ok;
    }
    // binary16, or 16-bit integers as a container of its bits (other types of two bytes would read the bits as other numbers)
    bool binary16(PyObject* o) {
        PyObject* t = bad ? nullptr : PyObject_GetAttr(o, g_dtype);
        const bool ok = t && (t == g_float16 || t == g_int16 || t == g_uint16);
        Py_XDECREF(t);
        return ok;
    }
    template <typename T>
    T* address(PyObject* o) {
        return reinterpret_cast<T*>(bad ? 0 : number_of(PyObject_CallMethodNoArgs(o, g_data_ptr)));
    }
    // The current device, which tensors and streams of a call belong to.
    long long current_device() { return bad ? -1 : (long long)number_of(PyObject_CallNoArgs(g_get_device)); }
    int integer() {
        PyObject* o = bad ? nullptr : next();
        const long x = o ? PyLong_AsLong(o) : -1;
        if (o && x == -1 && PyErr_Occurred()) bad = true;
        return (int)x;
    }
    int integer_32(const char* what) {
        PyObject* o = bad ? nullptr : next();
        const long x = o ? PyLong_AsLong(o) : 0;
        if (o && x == -1 && PyErr_Occurred()) bad = true;
        if (!bad && x != (int)x) fail(what);
        return (int)x;
    }
    // torch's current stream on the current device
    sa_stream stream() {
        if (bad) return nullptr;
        PyObject* dev = PyObject_CallNoArgs(g_get_device);
        if (!dev) {
            bad = true;
            return nullptr;
        }
        PyObject* s = PyObject_CallOneArg(g_get_stream, dev);
        Py_DECREF(dev);
        return reinterpret_cast<sa_stream>(number_of(s));
    }
};

// CALL: an expression of type sa_status over what was unpacked
#define SA_RETURN(CALL)                 \
    do {                                \
        if (a.bad) return nullptr;      \
        sa_status st;                   \
        Py_BEGIN_ALLOW_THREADS          \
        st = (CALL);                    \
        Py_END_ALLOW_THREADS            \
        return PyLong_FromLong(st);     \
    } while (0)

// (cfg, cache, Q, O, workspace, dbg_scores, stages)
PyObject* decode_attention(PyObject*, PyObject* const* v, Py_ssize_t n) {
    Args a{v, n};
    const sa_config* cfg = a.structure<sa_config>();
    const sa_cache* cache = a.structure<sa_cache>();
    const uint16_t* Q = a.tensor<uint16_t>();
    float* O = a.tensor<float>();
    size_t bytes;
    void* ws = a.tensor_and_bytes(&bytes);
    int32_t* dbg = a.tensor<int32_t>();
    const int stages = a.integer();
    const sa_stream s = a.stream();
    SA_RETURN(sa_decode_attention_stages(cfg, cache, Q, O, ws, bytes, dbg, stages, s));
}

// (cfg, cache, Q, O, workspace, stages)
PyObject* decode_attention_fp16(PyObject*, PyObject* const* v, Py_ssize_t n) {
    Args a{v, n};
    const sa_config* cfg = a.structure<sa_config>();
    const sa_cache* cache = a.structure<sa_cache>();
    const uint16_t* Q = a.tensor<uint16_t>();
    float* O = a.tensor<float>();
    size_t bytes;
    void* ws = a.tensor_and_bytes(&bytes);
    const int stages = a.integer();
    const sa_stream s = a.stream();
    SA_RETURN(sa_decode_attention_fp16_stages(cfg, cache, Q, O, ws, bytes, stages, s));
}

// (cfg, cache, Q, K_new, V_new, O, workspace)
PyObject* decode_step(PyObject*, PyObject* const* v, Py_ssize_t n) {
    Args a{v, n};
    const sa_config* cfg = a.structure<sa_config>();
    const sa_cache* cache = a.structure<sa_cache>();
    const uint16_t* Q = a.tensor<uint16_t>();
    const uint16_t* K = a.tensor<uint16_t>();
    const uint16_t* V = a.tensor<uint16_t>();
    float* O = a.tensor<float>();
    size_t bytes;
    void* ws = a.tensor_and_bytes(&bytes);
    const sa_stream s = a.stream();
    SA_RETURN(sa_decode_step(cfg, cache, Q, K, V, O, ws, bytes, s));
}

// (cfg, cache, Q, K_new, V_new, O, staging, workspace), the four in the middle on the host
PyObject* decode_step_host(PyObject*, PyObject* const* v, Py_ssize_t n) {
    Args a{v, n};
    const sa_config* cfg = a.structure<sa_config>();
    const sa_cache* cache = a.structure<sa_cache>();
    const uint16_t* Q = a.tensor<uint16_t>();
    const uint16_t* K = a.tensor<uint16_t>();
    const uint16_t* V = a.tensor<uint16_t>();
    float* O = a.tensor<float>();
    size_t sbytes, bytes;
    void* staging = a.tensor_and_bytes(&sbytes);
    void* ws = a.tensor_and_bytes(&bytes);
    const sa_stream s = a.stream();
    SA_RETURN(sa_decode_step_host(cfg, cache, Q, K, V, O, staging, sbytes, ws, bytes, s));
}

// (cfg, cache, K_new, V_new, bump_lens)
PyObject* append_kv(PyObject*, PyObject* const* v, Py_ssize_t n) {
    Args a{v, n};
    const sa_config* cfg = a.structure<sa_config>();
    const sa_cache* cache = a.structure<sa_cache>();
    const uint16_t* K = a.tensor<uint16_t>();
    const uint16_t* V = a.tensor<uint16_t>();
    const int bump = a.integer();
    const sa_stream s = a.stream();
    SA_RETURN(sa_append_kv(cfg, cache, K, V, bump, s));
}

// (cfg, cache, K, V, cu_lens): cu_lens a contiguous host array of at least batch + 1 64-bit integers, which the library
// reads on the host
PyObject* fill_kv(PyObject*, PyObject* const* v, Py_ssize_t n) {
    Args a{v, n};
    const sa_config* cfg = a.structure<sa_config>();
    const sa_cache* cache = a.structure<sa_cache>();
    const uint16_t* K = a.tensor<uint16_t>();
    const uint16_t* V = a.tensor<uint16_t>();
    PyObject* o = a.bad ? nullptr : a.next();
    Py_buffer cu;
    if (a.bad || PyObject_GetBuffer(o, &cu, PyBUF_SIMPLE) != 0) return nullptr;
    if (cu.len / (Py_ssize_t)sizeof(int64_t) <= (Py_ssize_t)cache->batch) {
        a.bad = true;
        PyErr_Format(PyExc_ValueError, "cu_lens holds %zd bytes, not the batch + 1 = %zd numbers of 8", cu.len, (Py_ssize_t)cache->batch + 1);
    }
    const sa_stream s = a.stream();
    if (a.bad) {
        PyBuffer_Release(&cu);
        return nullptr;
    }
    sa_status st;
    Py_BEGIN_ALLOW_THREADS
    st = sa_fill_kv(cfg, cache, K, V, static_cast<const int64_t*>(cu.buf), s);
    Py_END_ALLOW_THREADS
    PyBuffer_Release(&cu);
    return PyLong_FromLong(st);
}

// A contiguous host array of at least `n` 64-bit integers; None (where it may be): null.
struct HostArray {
    Py_buffer b{};
    bool held = false;
    const int64_t* p = nullptr;
    HostArray(Args& a, Py_ssize_t n, bool may_be_none, const char* what) {
        PyObject* o = a.bad ? nullptr : a.next();
        if (a.bad || (may_be_none && o == Py_None)) return;
        if (PyObject_GetBuffer(o, &b, PyBUF_FORMAT | PyBUF_C_CONTIGUOUS) != 0) {
            a.bad = true;
            return;
        }
        held = true;
        const char* f = b.format ? b.format : "B";
        if (b.itemsize != 8 || (f[0] != 'l' && f[0] != 'q') || f[1] || b.len / (Py_ssize_t)sizeof(int64_t) < n) a.fail(what);
        else p = static_cast<const int64_t*>(b.buf);
    }
    ~HostArray() {
        if (held) PyBuffer_Release(&b);
    }
};

// (cfg, cache, starts, cu_lens, K, V)
PyObject* read_kv(PyObject*, PyObject* const* v, Py_ssize_t n) {
    Args a{v, n};
    const sa_config* cfg = a.structure<sa_config>();
    const sa_cache* cache = a.structure<sa_cache>();
    const Py_ssize_t batch = a.bad || cache->batch < 0 ? 0 : cache->batch;
    HostArray starts(a, batch, true, "starts holds at least batch 64-bit integers");
    HostArray cu(a, batch + 1, false, "cu_lens holds at least batch + 1 64-bit integers");
    const long long dev = a.current_device();
    uint16_t* out[2] = {nullptr, nullptr};
    for (int i = 0; i < 2 && !a.bad; ++i) {
        PyObject* o = a.next();
        if (a.bad || o == Py_None) continue;
        long long sh[3];
        if (!a.shape(o, 3, sh) || sh[1] != cfg->n_kv_heads || sh[2] != cfg->head_dim || sh[0] < cu.p[batch] || !a.binary16(o) || !a.contiguous(o) || !a.on_device(o, dev))
            a.fail("K and V are contiguous [rows, n_kv_heads, head_dim] of float16 (or int16, uint16 for its bits) on the current CUDA device, with a row for every token");
        out[i] = a.address<uint16_t>(o);
    }
    const sa_stream s = a.stream();
    SA_RETURN(sa_read_kv(cfg, cache, starts.p, cu.p, out[0], out[1], s));
}

// What rotate_qkv and append_qkv take of a layer's projections, and the positions.
struct Projections {
    const void* in[3] = {};
    long long stride[3] = {}, n = -1;                          // n: rows; -1: none is given
    const int32_t* positions = nullptr;
    void take(Args& a, const sa_config* cfg, PyObject* dtype, long long dev) {
        long long sh[3], step[3];
        const long long d = a.bad ? 0 : cfg->head_dim;
        for (int i = 0; i < 3 && !a.bad; ++i) {
            PyObject* o = a.next();
            if (a.bad || o == Py_None) continue;
            const long long H = i == 0 ? cfg->n_q_heads : cfg->n_kv_heads;
            if (!a.shape(o, 3, sh) || sh[1] != H || sh[2] != d || (n >= 0 && sh[0] != n) || !a.strides(o, 3, step) || (H > 1 && step[1] != d) || step[2] != 1 ||
                !a.typed(o, dtype) || !a.on_device(o, dev))
                a.fail("Q, K and V are [n, heads, head_dim] of the rotary's dtype on the current CUDA device, a token's heads one after another, n the same for all");
            n = sh[0];
            stride[i] = n > 1 ? step[0] : H * d;
            in[i] = a.address<const void>(o);
        }
    }
    void take_positions(Args& a, const sa_rotary* rot, long long dev) {
        long long sh[3];
        PyObject* pos = a.bad ? nullptr : a.next();
        if (a.bad || pos == Py_None) return;
        const bool two = a.shape(pos, 2, sh);
        if (two ? sh[0] != rot->n_axes || (n >= 0 && sh[1] != n) : rot->n_axes != 1 || !a.shape(pos, 1, sh) || (n >= 0 && sh[0] != n)) a.fail("positions are [n_axes, n]");
        else if (!a.typed(pos, g_int32) || !a.contiguous(pos) || !a.on_device(pos, dev)) a.fail("positions are contiguous int32 on the current CUDA device");
        positions = a.address<const int32_t>(pos);
    }
};

// (cfg, rotary, dtype, device of the tables, Q, K, V, positions, Q_out, K_out, V_out)
PyObject* rotate_qkv(PyObject*, PyObject* const* v, Py_ssize_t n_args) {
    Args a{v, n_args};
    const sa_config* cfg = a.structure<sa_config>();
    const sa_rotary* rot = a.structure<sa_rotary>();
    PyObject* dtype = a.bad ? nullptr : a.next();
    const long long tables = a.integer(), dev = a.current_device();
    if (!a.bad && tables >= 0 && tables != dev) a.fail("the tables lie on another device than the current one");
    uint16_t* out[3] = {};
    long long sh[3];
    const long long d = a.bad ? 0 : cfg->head_dim;
    Projections x;
    x.take(a, cfg, dtype, dev);
    x.take_positions(a, rot, dev);
    const long long n = x.n;
    for (int i = 0; i < 3 && !a.bad; ++i) {
        PyObject* o = a.next();
        if (a.bad || o == Py_None) continue;
        if (!a.shape(o, 3, sh) || sh[0] != n || sh[1] != (i == 0 ? cfg->n_q_heads : cfg->n_kv_heads) || sh[2] != d || !a.binary16(o) || !a.contiguous(o) || !a.on_device(o, dev))
            a.fail("the outputs are contiguous [n, heads, head_dim] of float16 (or int16, uint16 for its bits) on the current CUDA device, one for each of Q, K and V that is given");
        out[i] = a.address<uint16_t>(o);
    }
    // (a tensor without elements has no address, which would read as one that is not there)
    if (!a.bad && n == 0) return PyLong_FromLong(SA_OK);
    const sa_stream s = a.stream();
    SA_RETURN(sa_rotate_qkv(cfg, rot, x.in[0], x.stride[0], x.in[1], x.stride[1], x.in[2], x.stride[2], x.positions, n < 0 ? 0 : n, out[0], out[1], out[2], s));
}

// (cfg, rotary, dtype, device of the tables, cache, Q, K, V, positions, cu_lens, Q_out, bump_lens)
PyObject* append_qkv(PyObject*, PyObject* const* v, Py_ssize_t n_args) {
    Args a{v, n_args};
    const sa_config* cfg = a.structure<sa_config>();
    const sa_rotary* rot = a.structure<sa_rotary>();
    PyObject* dtype = a.bad ? nullptr : a.next();
    const long long tables = a.integer(), dev = a.current_device();
    if (!a.bad && tables >= 0 && tables != dev) a.fail("the tables lie on another device than the current one");
    const sa_cache* cache = a.structure<sa_cache>();
    Projections x;
    x.take(a, cfg, dtype, dev);
    x.take_positions(a, rot, dev);
    HostArray cu(a, a.bad || cache->batch < 0 ? 1 : (Py_ssize_t)cache->batch + 1, false, "cu_lens holds at least batch + 1 64-bit integers");
    PyObject* o = a.bad ? nullptr : a.next();
    uint16_t* out = nullptr;
    long long sh[3];
    if (!a.bad && o != Py_None) {
        if (!a.shape(o, 3, sh) || sh[0] != x.n || sh[1] != cfg->n_q_heads || sh[2] != cfg->head_dim || !a.binary16(o) || !a.contiguous(o) || !a.on_device(o, dev))
            a.fail("Q_out is contiguous [n, n_q_heads, head_dim] of float16 (or int16, uint16 for its bits) on the current CUDA device");
        out = a.address<uint16_t>(o);
    }
    const int bump = a.integer();
    // (a tensor without elements has no address, which would read as one that is not there)
    if (!a.bad && x.n == 0 && cache->batch >= 0 && cu.p[cache->batch] == 0 && cu.p[0] == 0) return PyLong_FromLong(SA_OK);
    const sa_stream s = a.stream();
    SA_RETURN(sa_append_qkv(cfg, cache, rot, x.in[0], x.stride[0], x.in[1], x.stride[1], x.in[2], x.stride[2], x.positions, x.n < 0 ? 0 : x.n, cu.p, out, bump, s));
}

// (cfg, cache, Q, O, workspace, cu_lens, window, sinks)
PyObject* chunk_attention(PyObject*, PyObject* const* v, Py_ssize_t n) {
    Args a{v, n};
    const sa_config* cfg = a.structure<sa_config>();
    const sa_cache* cache = a.structure<sa_cache>();
    PyObject *Q = a.bad ? nullptr : a.next(), *O = a.bad ? nullptr : a.next();
    size_t bytes;
    void* ws = a.tensor_and_bytes(&bytes);
    HostArray cu(a, a.bad || cache->batch < 0 ? 1 : (Py_ssize_t)cache->batch + 1, false, "cu_lens holds at least batch + 1 64-bit integers");
    const char* const range = "window and sinks are below 2^31";
    const int window = a.integer_32(range), sinks = a.integer_32(range);
    const long long dev = a.current_device(), rows = a.bad || cache->batch < 0 ? 0 : cu.p[cache->batch];
    int dtype = SA_F16;
    for (int i = 0; i < 2 && !a.bad; ++i) {
        PyObject* o = i ? O : Q;
        long long sh[3];
        if (i && a.typed(o, g_bfloat16)) dtype = SA_BF16;
        if (!a.shape(o, 3, sh) || sh[1] != cfg->n_q_heads || sh[2] != cfg->head_dim || sh[0] < rows || (dtype == SA_F16 && !a.binary16(o)) || !a.contiguous(o) || !a.on_device(o, dev))
            a.fail("Q and O are contiguous [rows, n_q_heads, head_dim] of float16 (or int16, uint16 for its bits; O also bfloat16) on the current CUDA device, with a row for every token");
    }
    const uint16_t* q = a.address<const uint16_t>(Q);
    void* o = a.address<void>(O);
    const sa_stream s = a.stream();
    SA_RETURN(sa_chunk_attention(cfg, cache, q, cu.p, window, sinks, o, dtype, ws, bytes, s));
}

PyMethodDef kMethods[] = {
    {"append_qkv", (PyCFunction)(void (*)(void))append_qkv, METH_FASTCALL, nullptr},
    {"chunk_attention", (PyCFunction)(void (*)(void))chunk_attention, METH_FASTCALL, nullptr},
    {"read_kv", (PyCFunction)(void (*)(void))read_kv, METH_FASTCALL, nullptr},
    {"rotate_qkv", (PyCFunction)(void (*)(void))rotate_qkv, METH_FASTCALL, nullptr},
    {"fill_kv", (PyCFunction)(void (*)(void))fill_kv, METH_FASTCALL, nullptr},
    {"decode_attention", (PyCFunction)(void (*)(void))decode_attention, METH_FASTCALL, nullptr},
    {"decode_attention_fp16", (PyCFunction)(void (*)(void))decode_attention_fp16, METH_FASTCALL, nullptr},
    {"decode_step", (PyCFunction)(void (*)(void))decode_step, METH_FASTCALL, nullptr},
    {"decode_step_host", (PyCFunction)(void (*)(void))decode_step_host, METH_FASTCALL, nullptr},
    {"append_kv", (PyCFunction)(void (*)(void))append_kv, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) {
    PyObject* c = PyImport_ImportModule("torch._C");
    if (!c) return nullptr;
    g_get_device = PyObject_GetAttrString(c, "_cuda_getDevice");
    g_get_stream = PyObject_GetAttrString(c, "_cuda_getCurrentRawStream");
    Py_DECREF(c);
    g_data_ptr = PyUnicode_InternFromString("data_ptr");
    g_nbytes = PyUnicode_InternFromString("nbytes");
    g_shape = PyUnicode_InternFromString("shape");
    g_stride = PyUnicode_InternFromString("stride");
    g_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    PyObject* torch = PyImport_ImportModule("torch");
    g_float16 = torch ? PyObject_GetAttrString(torch, "float16") : nullptr;
    g_int16 = torch ? PyObject_GetAttrString(torch, "int16") : nullptr;
    g_uint16 = torch ? PyObject_GetAttrString(torch, "uint16") : nullptr;
    g_bfloat16 = torch ? PyObject_GetAttrString(torch, "bfloat16") : nullptr;
    g_int32 = torch ? PyObject_GetAttrString(torch, "int32") : nullptr;
    Py_XDECREF(torch);
    g_dtype = PyUnicode_InternFromString("dtype");
    g_device_of = PyUnicode_InternFromString("get_device");
    if (!g_get_device || !g_get_stream || !g_data_ptr || !g_nbytes || !g_shape || !g_stride || !g_is_contiguous || !g_float16 || !g_int16 || !g_uint16 || !g_int32 || !g_bfloat16 || !g_dtype || !g_device_of) return nullptr;
    return PyModule_Create(&kModule);
}
