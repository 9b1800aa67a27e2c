// Native half of the Python binding: tensor -> pointer marshalling, output allocation and the
// call into libgraft.so, one C function per entry point.
//
// A decoding round of a small model is bound by the host: the kernels of a call take 4 to 10 us.
// The same marshalling through ctypes cost 8 to 10 us per call (17 foreign-function arguments
// converted one by one, data_ptr() and is_contiguous() as Python method calls, torch.empty() at
// 1.5 us each, the current stream looked up through Python); here a call costs what its launches
// cost.  The library stays a plain C ABI without any knowledge of PyTorch: this file resolves its
// functions from the path the Python side hands to bind().
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <dlfcn.h>

#include <ATen/core/Tensor.h>
#include <ATen/hip/EmptyTensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "graft.h"

namespace {

// ---- the library's entry points ------------------------------------------------------------
#define GRAFT_ENTRY_POINTS(X)                                                                       \
    X(graft_retrieve) X(graft_build_tree_mask) X(graft_tree_attn_workspace_bytes) X(graft_tree_attn) \
    X(graft_accept_workspace_bytes) X(graft_accept) X(graft_accept_noalloc) X(graft_matrix_retrieve) \
    X(graft_matrix_update_workspace_bytes) X(graft_matrix_update) X(graft_kv_compact) X(graft_prune_select) \
    X(graft_kv_append) X(graft_kv_append_mx) X(graft_kv_gather_mx) X(graft_tree_attn_mx_workspace_bytes) X(graft_tree_attn_mx) \
    X(graft_kv_compact_mx) X(graft_prompt_attn_workspace_bytes) X(graft_prompt_attn) X(graft_token_counts) \
    X(graft_logits_adjust_workspace_bytes) X(graft_logits_adjust) X(graft_last_hip_error)
struct Library {
#define X(name) decltype(&::name) name = nullptr;
    GRAFT_ENTRY_POINTS(X)
#undef X
};
Library lib;
PyObject* graft_error = nullptr;         // the GraftError class
PyObject *s_page, *s_token, *s_head, *s_cuda_stream;

// Thrown after a Python error has been set.
struct PythonError {};

// ---- arguments -----------------------------------------------------------------------------
const at::Tensor& tensor(PyObject* o) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "expected a torch.Tensor, got %s", Py_TYPE(o)->tp_name);
        throw PythonError();
    }
    return THPVariable_Unpack(o);
}

template <class T> T* ptr(const at::Tensor& t) {
    if (!t.is_contiguous()) {
        PyErr_SetString(PyExc_AssertionError, "tensors cross the C ABI as dense row-major arrays");
        throw PythonError();
    }
    return static_cast<T*>(t.data_ptr());
}
template <class T> T* ptr(PyObject* o) { return o == Py_None ? nullptr : ptr<T>(tensor(o)); }

int32_t to_i32(PyObject* o) {
    const unsigned long v = PyLong_AsUnsignedLongMask(o);
    if (v == static_cast<unsigned long>(-1) && PyErr_Occurred()) throw PythonError();
    return static_cast<int32_t>(v);
}
int64_t to_i64(PyObject* o) {
    PyObject* i = PyNumber_Long(o);
    if (!i) throw PythonError();
    const long long v = PyLong_AsLongLong(i);
    Py_DECREF(i);
    if (v == -1 && PyErr_Occurred()) throw PythonError();
    return v;
}

void sizes2(const at::Tensor& t, int32_t& a, int32_t& b) {
    if (t.dim() != 2) {
        PyErr_Format(PyExc_ValueError, "expected a tensor of 2 dimensions, got %d", static_cast<int>(t.dim()));
        throw PythonError();
    }
    a = static_cast<int32_t>(t.size(0));
    b = static_cast<int32_t>(t.size(1));
}
int32_t size_at(const at::Tensor& t, int64_t dim) {
    if (t.dim() <= dim) {
        PyErr_SetString(PyExc_IndexError, "a tensor argument has too few dimensions");
        throw PythonError();
    }
    return static_cast<int32_t>(t.size(dim));
}

// A reference held for as long as the object is looked at.
struct Ref {
    PyObject* o;
    explicit Ref(PyObject* owned) : o(owned) {}
    ~Ref() { Py_XDECREF(o); }
    Ref(const Ref&) = delete;
    operator PyObject*() const { return o; }
};

// KeyError if the key is missing.  The reference is held: a mapping other than a dict may make its
// values on the fly.
Ref item(PyObject* dict, PyObject* key) {
    PyObject* v;
    if (PyDict_CheckExact(dict)) {
        v = PyDict_GetItemWithError(dict, key);
        Py_XINCREF(v);
        if (!v && !PyErr_Occurred()) PyErr_SetObject(PyExc_KeyError, key);
    } else v = PyObject_GetItem(dict, key);
    if (!v) throw PythonError();
    return Ref(v);
}

struct Strides { int64_t page, token, head; };
Strides strides_of(PyObject* d) {
    return {to_i64(item(d, s_page)), to_i64(item(d, s_token)), to_i64(item(d, s_head))};
}

at::Tensor empty_bytes(size_t n, const at::Device& dev);

// The stream a call launches on: the given one (an object with a cuda_stream attribute, or the handle
// itself), else the current stream of the current device.
class LaunchStream {
public:
    LaunchStream(PyObject* given, const at::Device& dev) : dev_(dev), given_(given != Py_None) {
        if (!given_) {
            handle_ = c10::hip::getCurrentHIPStream().stream();
            return;
        }
        PyObject* h = PyObject_GetAttr(given, s_cuda_stream);
        if (!h) {
            PyErr_Clear();
            handle_ = reinterpret_cast<void*>(to_i64(given));
            return;
        }
        PyObject* i = PyNumber_Long(h);
        Py_DECREF(h);
        if (!i) throw PythonError();
        handle_ = PyLong_AsVoidPtr(i);
        Py_DECREF(i);
    }
    void* handle() const { return handle_; }
    // Scratch memory of the call.  It is given back when the call returns, with its kernels still to run, so
    // it has to belong to the stream they run on: the allocator hands a block out again in the order of the
    // stream it was taken for.  Taken for the current stream, two calls on two other streams get the
    // same block, and so does whatever is allocated next.
    at::Tensor scratch(size_t n) const {
        if (!given_ || !dev_.is_cuda()) return empty_bytes(n, dev_);
        struct Restore {
            c10::hip::HIPStream before;
            ~Restore() { c10::hip::setCurrentHIPStream(before); }
        } restore{c10::hip::getCurrentHIPStream(dev_.index())};
        c10::hip::setCurrentHIPStream(c10::hip::getStreamFromExternal(static_cast<hipStream_t>(handle_), dev_.index()));
        return empty_bytes(n, dev_);
    }

private:
    at::Device dev_;
    bool given_;
    void* handle_;
};

// ---- results -------------------------------------------------------------------------------
at::Tensor empty(at::IntArrayRef shape, at::ScalarType type, const at::Device& dev) {
    if (dev.is_cuda()) return at::Tensor(at::detail::empty_cuda(shape, type, dev, std::nullopt));
    return at::empty(shape, at::TensorOptions().dtype(type).device(dev));
}
at::Tensor empty_i32(at::IntArrayRef shape, const at::Device& dev) { return empty(shape, at::kInt, dev); }
at::Tensor empty_bytes(size_t n, const at::Device& dev) { return empty({static_cast<int64_t>(n)}, at::kByte, dev); }

// A dict of result tensors: either the caller's (no allocation) or a new one.
class Outputs {
public:
    Outputs(PyObject* given, const at::Device& dev) : dev_(dev) {
        if (given != Py_None) {
            Py_INCREF(given);
            dict_ = given;
        } else {
            dict_ = PyDict_New();
            fresh_ = true;
            if (!dict_) throw PythonError();
        }
    }
    ~Outputs() { Py_XDECREF(dict_); }
    Outputs(const Outputs&) = delete;
    template <class T = int32_t> T* get(PyObject* key, at::IntArrayRef shape, at::ScalarType type = at::kInt) {
        if (!fresh_) return ptr<T>(item(dict_, key));
        at::Tensor t = empty(shape, type, dev_);
        T* p = static_cast<T*>(t.data_ptr());
        put(key, THPVariable_Wrap(std::move(t)));
        return p;
    }
    // The same, and a caller's tensor has to be of the type, the shape and on the device that a new one would be.
    template <class T = int32_t> T* get_checked(PyObject* key, at::IntArrayRef shape, at::ScalarType type = at::kInt) {
        if (fresh_) return get<T>(key, shape, type);
        const Ref o(item(dict_, key));
        const at::Tensor& t = tensor(o);
        if (t.sizes() != shape || t.scalar_type() != type || t.device() != dev_) {
            PyErr_Format(PyExc_ValueError, "the output %R does not have the shape, the type or the device of this call's results", key);
            throw PythonError();
        }
        return ptr<T>(t);
    }
    void put(PyObject* key, PyObject* value) {                     // steals value
        const int bad = value ? PyObject_SetItem(dict_, key, value) : -1;
        Py_XDECREF(value);
        if (bad) throw PythonError();
    }
    bool fresh() const { return fresh_; }
    PyObject* release() {
        PyObject* d = dict_;
        dict_ = nullptr;
        return d;
    }

private:
    PyObject* dict_ = nullptr;
    bool fresh_ = false;
    at::Device dev_;
};

// GraftError on a return code other than GRAFT_OK.
void check(const char* fn, int32_t rc) {
    if (rc == GRAFT_OK) return;
    PyObject* e = PyObject_CallFunction(graft_error, "sii", fn, rc, lib.graft_last_hip_error());
    if (e) {
        PyErr_SetObject(graft_error, e);
        Py_DECREF(e);
    }
    throw PythonError();
}

// The library call, without the GIL (a launch waits when the stream's queue is full).
template <class F> int32_t unlocked(F&& f) {
    PyThreadState* st = PyEval_SaveThread();
    const int32_t rc = f();
    PyEval_RestoreThread(st);
    return rc;
}

void need_args(Py_ssize_t got, Py_ssize_t want) {
    if (!graft_error) {
        PyErr_SetString(PyExc_RuntimeError, "the library has not been bound");
        throw PythonError();
    }
    if (got != want) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, got);
        throw PythonError();
    }
}

// ---- one function per entry point; arguments are those of the Python function, in order, all given
#define GRAFT_PY(name, n)                                                                 \
    PyObject* name##_body(PyObject* const* a);                                             \
    PyObject* name(PyObject*, PyObject* const* a, Py_ssize_t n_args) {                     \
        try {                                                                              \
            need_args(n_args, n);                                                          \
            return name##_body(a);                                                         \
        } catch (const PythonError&) {                                                     \
            return nullptr;                                                                \
        } catch (...) { /* as torch raises it: out of memory is torch.OutOfMemoryError */  \
            torch::translate_exception_to_python(std::current_exception());                \
            return nullptr;                                                                \
        }                                                                                  \
    }                                                                                      \
    PyObject* name##_body(PyObject* const* a)
#define GRAFT_KEY(name) static PyObject* const k_##name = PyUnicode_InternFromString(#name)

// ctx, ctx_len, n_min, n_max, C, m, tail, tail_len, out, stream
GRAFT_PY(py_retrieve, 10) {
    GRAFT_KEY(chain_tok); GRAFT_KEY(chain_len); GRAFT_KEY(chain_pos); GRAFT_KEY(chain_match); GRAFT_KEY(n_hits); GRAFT_KEY(status);
    const at::Tensor& ctx = tensor(a[0]);
    int32_t B, L_max;
    sizes2(ctx, B, L_max);
    const int32_t n_min = to_i32(a[2]), n_max = to_i32(a[3]), C = to_i32(a[4]), m = to_i32(a[5]);
    Outputs out(a[8], ctx.device());
    int32_t* tok = out.get(k_chain_tok, {B, C, m});
    int32_t* len = out.get(k_chain_len, {B, C});
    int32_t* pos = out.get(k_chain_pos, {B, C});
    int32_t* match = out.get(k_chain_match, {B, C});
    int32_t* hits = out.get(k_n_hits, {B});
    int32_t* status = out.get(k_status, {B});
    const int32_t tail_max = a[6] == Py_None ? 0 : size_at(tensor(a[6]), 1);
    const int32_t *c = ptr<int32_t>(ctx), *cl = ptr<int32_t>(a[1]), *t = ptr<int32_t>(a[6]), *tl = ptr<int32_t>(a[7]);
    void* s = LaunchStream(a[9], ctx.device()).handle();
    check("graft_retrieve", unlocked([&] {
        return lib.graft_retrieve(c, cl, B, L_max, t, tl, tail_max, n_min, n_max, C, m, tok, len, pos, match, hits, status, s);
    }));
    return out.release();
}

// parent, n_nodes, prefix_len, n_leaf_max, depth_cap, out, stream
GRAFT_PY(py_build_tree_mask, 7) {
    GRAFT_KEY(mask); GRAFT_KEY(pos); GRAFT_KEY(depth); GRAFT_KEY(paths); GRAFT_KEY(status);
    const at::Tensor& parent = tensor(a[0]);
    int32_t B, K;
    sizes2(parent, B, K);
    const int32_t n_leaf_max = to_i32(a[3]), depth_cap = to_i32(a[4]);
    Outputs out(a[5], parent.device());
    uint64_t* mask = out.get<uint64_t>(k_mask, {B, K, GRAFT_MASK_WORDS}, at::kLong);
    int32_t* pos = out.get(k_pos, {B, K});
    int32_t* depth = out.get(k_depth, {B, K});
    int32_t* paths = nullptr;
    if (!out.fresh() || n_leaf_max > 0) paths = out.get(k_paths, {B, n_leaf_max, depth_cap + 1});
    else {
        Py_INCREF(Py_None);
        out.put(k_paths, Py_None);
    }
    int32_t* status = out.get(k_status, {B});
    const int32_t *p = ptr<int32_t>(parent), *n = ptr<int32_t>(a[1]), *pl = ptr<int32_t>(a[2]);
    void* s = LaunchStream(a[6], parent.device()).handle();
    check("graft_build_tree_mask", unlocked([&] {
        return lib.graft_build_tree_mask(p, n, pl, B, K, mask, pos, depth, paths, n_leaf_max, depth_cap, status, s);
    }));
    return out.release();
}

// q, k_cache, v_cache, strides, block_table, prefix_len, n_nodes, mask, Hkv, scale, out, workspace, stream
GRAFT_PY(py_tree_attn, 13) {
    const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]), &v = tensor(a[2]), &table = tensor(a[4]);
    if (q.dim() != 4) {
        PyErr_Format(PyExc_ValueError, "expected a query tensor of 4 dimensions, got %d", static_cast<int>(q.dim()));
        throw PythonError();
    }
    const at::ScalarType type = q.scalar_type();
    if ((type != at::kFloat && type != at::kBFloat16) || k.scalar_type() != type || v.scalar_type() != type) {
        PyErr_SetString(PyExc_AssertionError, "queries, keys and values are all float32 or all bfloat16");
        throw PythonError();
    }
    const int32_t dtype = type == at::kFloat ? GRAFT_F32 : GRAFT_BF16;
    const int32_t B = static_cast<int32_t>(q.size(0)), K = static_cast<int32_t>(q.size(1)),
                  Hq = static_cast<int32_t>(q.size(2)), D = static_cast<int32_t>(q.size(3));
    const int32_t max_pages = size_at(table, 1), Hkv = to_i32(a[8]);
    const double scale = PyFloat_AsDouble(a[9]);
    if (scale == -1.0 && PyErr_Occurred()) throw PythonError();
    const Strides st = strides_of(a[3]);
    const LaunchStream stream(a[12], q.device());
    at::Tensor new_out, new_ws;
    void* out;
    if (a[10] == Py_None) {
        new_out = empty(q.sizes(), type, q.device());
        out = new_out.data_ptr();
    } else out = ptr<void>(a[10]);
    void* ws = nullptr;
    size_t ws_bytes = 0;
    if (a[11] == Py_None) {
        ws_bytes = lib.graft_tree_attn_workspace_bytes(B, K, Hq, Hkv, D, max_pages, dtype);
        if (ws_bytes > 0) {
            new_ws = stream.scratch(ws_bytes);
            ws = new_ws.data_ptr();
        }
    } else {
        const at::Tensor& w = tensor(a[11]);
        ws = ptr<void>(w);
        ws_bytes = static_cast<size_t>(w.numel());
    }
    const void *qp = ptr<void>(q), *kp = ptr<void>(k), *vp = ptr<void>(v);
    const int32_t *tp = ptr<int32_t>(table), *pl = ptr<int32_t>(a[5]), *n = ptr<int32_t>(a[6]);
    const uint64_t* mask = ptr<uint64_t>(a[7]);
    void* s = stream.handle();
    check("graft_tree_attn", unlocked([&] {
        return lib.graft_tree_attn(qp, kp, vp, st.page, st.token, st.head, tp, max_pages, pl, n, mask, B, K, Hq, Hkv, D,
                                   GRAFT_PAGE_SIZE, static_cast<float>(scale), dtype, out, ws, ws_bytes, s);
    }));
    if (new_out.defined()) return THPVariable_Wrap(std::move(new_out));
    Py_INCREF(a[10]);
    return a[10];
}

// parent, tokens, n_nodes, depth_cap, target_ids, logits, out, workspace, stream
GRAFT_PY(py_accept, 9) {
    GRAFT_KEY(accept_len); GRAFT_KEY(best_node); GRAFT_KEY(path); GRAFT_KEY(out_tokens); GRAFT_KEY(status); GRAFT_KEY(target_ids);
    const at::Tensor& parent = tensor(a[0]);
    int32_t B, K, V = 0;
    sizes2(parent, B, K);
    const int32_t depth_cap = to_i32(a[3]);
    const at::Device dev = parent.device();
    const LaunchStream stream(a[8], dev);
    const float* logits = nullptr;
    int32_t* ids;
    PyObject* ids_obj = a[4];
    at::Tensor new_ws;
    void* ws = nullptr;
    size_t ws_bytes = 0;
    if (a[5] != Py_None) {
        const at::Tensor& lg = tensor(a[5]);
        V = size_at(lg, 2);
        logits = ptr<float>(lg);
        at::Tensor t = empty_i32({B, K}, dev);
        ids = static_cast<int32_t*>(t.data_ptr());
        ids_obj = THPVariable_Wrap(std::move(t));
        if (!ids_obj) throw PythonError();
    } else {
        ids = ptr<int32_t>(a[4]);
        Py_INCREF(ids_obj);
    }
    const Ref ids_held(ids_obj);
    Outputs out(a[6], dev);
    int32_t* len = out.get(k_accept_len, {B});
    int32_t* best = out.get(k_best_node, {B});
    int32_t* path = out.get(k_path, {B, depth_cap + 1});
    int32_t* toks = out.get(k_out_tokens, {B, depth_cap + 1});
    int32_t* status = out.get(k_status, {B});
    Py_INCREF(ids_obj);
    out.put(k_target_ids, ids_obj);
    if (a[7] != Py_None) {
        const at::Tensor& w = tensor(a[7]);
        ws = ptr<void>(w);
        ws_bytes = static_cast<size_t>(w.numel());
    } else if (logits) {
        ws_bytes = lib.graft_accept_workspace_bytes(B, K, V);
        new_ws = stream.scratch(ws_bytes);
        ws = new_ws.data_ptr();
    }
    const int32_t *p = ptr<int32_t>(parent), *tk = ptr<int32_t>(a[1]), *n = ptr<int32_t>(a[2]);
    void* s = stream.handle();
    check("graft_accept", unlocked([&] {
        return lib.graft_accept(p, tk, n, logits, V, ids, B, K, depth_cap, len, best, path, toks, status, ws, ws_bytes, s);
    }));
    return out.release();
}

// parent, tokens, n_nodes, depth_cap, out, target_ids, logits, stream
GRAFT_PY(py_accept_noalloc, 8) {
    GRAFT_KEY(accept_len); GRAFT_KEY(best_node); GRAFT_KEY(path); GRAFT_KEY(out_tokens); GRAFT_KEY(status);
    const at::Tensor& parent = tensor(a[0]);
    int32_t B, K;
    sizes2(parent, B, K);
    const int32_t depth_cap = to_i32(a[3]), V = a[6] == Py_None ? 0 : size_at(tensor(a[6]), 2);
    const float* logits = ptr<float>(a[6]);
    int32_t* ids = ptr<int32_t>(a[5]);
    int32_t *len = ptr<int32_t>(item(a[4], k_accept_len)), *best = ptr<int32_t>(item(a[4], k_best_node)),
            *path = ptr<int32_t>(item(a[4], k_path)), *toks = ptr<int32_t>(item(a[4], k_out_tokens)),
            *status = ptr<int32_t>(item(a[4], k_status));
    const int32_t *p = ptr<int32_t>(parent), *tk = ptr<int32_t>(a[1]), *n = ptr<int32_t>(a[2]);
    void* s = LaunchStream(a[7], parent.device()).handle();
    check("graft_accept_noalloc", unlocked([&] {
        return lib.graft_accept_noalloc(p, tk, n, logits, V, ids, B, K, depth_cap, len, best, path, toks, status, s);
    }));
    Py_INCREF(a[4]);
    return a[4];
}

// M, tpl_parent, tpl_rank, n_ret, tokens, parent, n_nodes, status, stream
GRAFT_PY(py_matrix_retrieve, 9) {
    int32_t V, k, B, K;
    sizes2(tensor(a[0]), V, k);
    const at::Tensor& tokens = tensor(a[4]);
    sizes2(tokens, B, K);
    at::Tensor fresh;
    int32_t* status;
    if (a[7] == Py_None) {
        fresh = empty_i32({B}, tokens.device());
        status = static_cast<int32_t*>(fresh.data_ptr());
    } else status = ptr<int32_t>(a[7]);
    const int32_t *M = ptr<int32_t>(a[0]), *tp = ptr<int32_t>(a[1]), *tr = ptr<int32_t>(a[2]), *nr = ptr<int32_t>(a[3]);
    const int32_t N = size_at(tensor(a[1]), 0);
    int32_t *tk = ptr<int32_t>(tokens), *p = ptr<int32_t>(a[5]), *n = ptr<int32_t>(a[6]);
    void* s = LaunchStream(a[8], tokens.device()).handle();
    check("graft_matrix_retrieve", unlocked([&] {
        return lib.graft_matrix_retrieve(M, V, k, tp, tr, N, nr, B, K, tk, p, n, status, s);
    }));
    if (fresh.defined()) return THPVariable_Wrap(std::move(fresh));
    Py_INCREF(a[7]);
    return a[7];
}

// tokens, n_nodes, logits, M, target_ids, workspace, stream
GRAFT_PY(py_matrix_update, 7) {
    const at::Tensor &lg = tensor(a[2]), &M = tensor(a[3]);
    if (lg.dim() != 3) {
        PyErr_Format(PyExc_ValueError, "expected logits of 3 dimensions, got %d", static_cast<int>(lg.dim()));
        throw PythonError();
    }
    const int32_t B = size_at(lg, 0), K = size_at(lg, 1), V = size_at(lg, 2), k = size_at(M, 1);
    const LaunchStream stream(a[6], lg.device());
    at::Tensor fresh, new_ws;
    int32_t* ids;
    if (a[4] == Py_None) {
        fresh = empty_i32({B, K}, lg.device());
        ids = static_cast<int32_t*>(fresh.data_ptr());
    } else ids = ptr<int32_t>(a[4]);
    void* ws;
    size_t ws_bytes;
    if (a[5] == Py_None) {
        ws_bytes = lib.graft_matrix_update_workspace_bytes(B, K, V, k);
        ws_bytes = ws_bytes > 8 ? ws_bytes : 8;
        new_ws = stream.scratch(ws_bytes);
        ws = new_ws.data_ptr();
    } else {
        const at::Tensor& w = tensor(a[5]);
        ws = ptr<void>(w);
        ws_bytes = static_cast<size_t>(w.numel());
    }
    const int32_t *tk = ptr<int32_t>(a[0]), *n = ptr<int32_t>(a[1]);
    const float* logits = ptr<float>(lg);
    int32_t* Mp = ptr<int32_t>(M);
    void* s = stream.handle();
    check("graft_matrix_update", unlocked([&] {
        return lib.graft_matrix_update(tk, n, logits, V, B, K, Mp, k, ids, ws, ws_bytes, s);
    }));
    if (fresh.defined()) return THPVariable_Wrap(std::move(fresh));
    Py_INCREF(a[4]);
    return a[4];
}

// k_cache, v_cache, layer_stride, n_layers, strides, block_table, prefix_len, path, accept_len, K_max, Hkv, D, out, stream
GRAFT_PY(py_kv_compact, 14) {
    GRAFT_KEY(new_prefix_len); GRAFT_KEY(status);
    const at::Tensor &k = tensor(a[0]), &v = tensor(a[1]), &table = tensor(a[5]), &path = tensor(a[7]);
    int32_t B, width;
    sizes2(path, B, width);
    const at::ScalarType type = k.scalar_type();
    if ((type != at::kFloat && type != at::kBFloat16) || v.scalar_type() != type) {
        PyErr_SetString(PyExc_AssertionError, "the caches are both float32 or both bfloat16");
        throw PythonError();
    }
    const int64_t layer_stride = to_i64(a[2]);
    const int32_t n_layers = to_i32(a[3]), K = to_i32(a[9]), Hkv = to_i32(a[10]), D = to_i32(a[11]);
    const Strides st = strides_of(a[4]);
    Outputs out(a[12], path.device());
    int32_t* new_len = out.get(k_new_prefix_len, {B});
    int32_t* status = out.get(k_status, {B});
    void *kp = ptr<void>(k), *vp = ptr<void>(v);
    const int32_t *tp = ptr<int32_t>(table), *pl = ptr<int32_t>(a[6]), *pp = ptr<int32_t>(path), *al = ptr<int32_t>(a[8]);
    const int32_t max_pages = size_at(table, 1);
    void* s = LaunchStream(a[13], path.device()).handle();
    check("graft_kv_compact", unlocked([&] {
        return lib.graft_kv_compact(kp, vp, layer_stride, n_layers, st.page, st.token, st.head, tp, max_pages, pl, pp, al, B,
                                    width - 1, K, Hkv, D, type == at::kFloat ? GRAFT_F32 : GRAFT_BF16, new_len, status, s);
    }));
    return out.release();
}

// parent, tokens, logq, n_nodes, chk_depth, chk_log_tau, chk_keep, chk_ret, out, stream
GRAFT_PY(py_prune_select, 10) {
    GRAFT_KEY(parent); GRAFT_KEY(tokens); GRAFT_KEY(index); GRAFT_KEY(n_nodes); GRAFT_KEY(stage); GRAFT_KEY(n_ret); GRAFT_KEY(status);
    const at::Tensor& parent = tensor(a[0]);
    int32_t B, K;
    sizes2(parent, B, K);
    Outputs out(a[8], parent.device());
    int32_t* op = out.get(k_parent, {B, K});
    int32_t* ot = out.get(k_tokens, {B, K});
    int32_t* oi = out.get(k_index, {B, K});
    int32_t* on = out.get(k_n_nodes, {B});
    int32_t* stage = out.get(k_stage, {B});
    int32_t* nr = out.get(k_n_ret, {B});
    int32_t* status = out.get(k_status, {B});
    const int32_t *p = ptr<int32_t>(parent), *tk = ptr<int32_t>(a[1]), *n = ptr<int32_t>(a[3]), *cd = ptr<int32_t>(a[4]),
                  *ck = ptr<int32_t>(a[6]), *cr = ptr<int32_t>(a[7]);
    const float *lq = ptr<float>(a[2]), *ct = ptr<float>(a[5]);
    const int32_t n_chk = size_at(tensor(a[4]), 0);
    void* s = LaunchStream(a[9], parent.device()).handle();
    check("graft_prune_select", unlocked([&] {
        return lib.graft_prune_select(p, tk, lq, n, B, K, cd, ct, ck, cr, n_chk, op, ot, oi, on, stage, nr, status, s);
    }));
    return out.release();
}

// ---- rotation and append, and the 4-bit cache ------------------------------------------------------
[[noreturn]] void fail(PyObject* type, const char* what) {
    PyErr_SetString(type, what);
    throw PythonError();
}

// A whole number that fits 32 bits.
int32_t whole(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw PythonError();
    if (v != static_cast<int32_t>(v)) fail(PyExc_OverflowError, "a size of more than 32 bits");
    return static_cast<int32_t>(v);
}

// All tensors of a call have to be on one GPU; the call runs with that GPU as the current one.
struct OnDevice {
    explicit OnDevice(const at::Tensor& t) : dev(t.device()) {}
    at::Device dev;
    void same(const at::Tensor& t) const {
        if (t.device() != dev) fail(PyExc_ValueError, "the tensors of a call have to be on one device");
    }
    void gpu() const {
        if (!dev.is_cuda()) fail(PyExc_ValueError, "the tensors of this call have to be on the GPU");
    }
    // A dense array of the given type and shape; None is NULL where the call allows it.
    template <class T> T* dense(PyObject* o, at::IntArrayRef shape, at::ScalarType type, const char* what, bool optional = false) const {
        if (o == Py_None && optional) return nullptr;
        const at::Tensor& t = tensor(o);
        same(t);
        if (t.sizes() != shape || t.scalar_type() != type) {
            PyErr_Format(PyExc_ValueError, "%s does not have the shape or the type of this call", what);
            throw PythonError();
        }
        return ptr<T>(t);
    }
    unsigned char* cache(PyObject* o) const {
        const at::Tensor& t = tensor(o);
        same(t);
        if (t.scalar_type() != at::kByte) fail(PyExc_ValueError, "a 4-bit cache is a tensor of uint8");
        return ptr<unsigned char>(t);
    }
};
struct StridesMx { int64_t page, head; };
StridesMx strides_mx_of(PyObject* d) { return {to_i64(item(d, s_page)), to_i64(item(d, s_head))}; }

// Rows [B,T,H,D] whose tokens lie a constant number of elements apart, as a slice of a fused projection has them; that number.
int64_t token_stride_of(const at::Tensor& t) {
    if (t.dim() != 4) {
        PyErr_Format(PyExc_ValueError, "expected rows of 4 dimensions, got %d", static_cast<int>(t.dim()));
        throw PythonError();
    }
    const int64_t B = t.size(0), T = t.size(1), H = t.size(2), D = t.size(3);
    const int64_t stride = T > 1 ? t.stride(1) : B > 1 ? t.stride(0) : H * D;
    if ((D > 1 && t.stride(3) != 1) || (H > 1 && t.stride(2) != D) || (B > 1 && t.stride(0) != T * stride))
        fail(PyExc_ValueError, "a token's heads have to be dense and tokens a constant stride apart");
    return stride;
}

// q, k, v, cos_sin, pos, k_cache, v_cache, strides, block_table, prefix_len, n_nodes, interleaved, out, stream
PyObject* append(PyObject* const* a, bool mx) {
    GRAFT_KEY(q); GRAFT_KEY(status);
    const at::Tensor &k = tensor(a[1]), &v = tensor(a[2]), &table = tensor(a[8]);
    const OnDevice on(k);
    const int64_t k_stride = token_stride_of(k), v_stride = token_stride_of(v);
    const at::ScalarType type = k.scalar_type();
    if (type != at::kFloat && type != at::kBFloat16) fail(PyExc_AssertionError, "queries, keys and values are all float32 or all bfloat16");
    const int64_t B = k.size(0), T = k.size(1), Hkv = k.size(2), D = k.size(3);
    auto rows_of = [&](const at::Tensor& t) {
        on.same(t);
        if (t.scalar_type() != type) fail(PyExc_AssertionError, "queries, keys and values are all float32 or all bfloat16");
        if (t.size(0) != B || t.size(1) != T || t.size(3) != D) fail(PyExc_ValueError, "queries, keys and values are of different shapes");
    };
    rows_of(v);
    if (v.size(2) != Hkv) fail(PyExc_ValueError, "queries, keys and values are of different shapes");
    int64_t q_stride = 0, Hq = 0;
    const void* q = nullptr;
    if (a[0] != Py_None) {
        const at::Tensor& t = tensor(a[0]);
        q_stride = token_stride_of(t);
        rows_of(t);
        Hq = t.size(2);
        q = t.data_ptr();
    }
    int32_t n_pos = 0, R = 0;
    const float* angles = nullptr;
    if (a[3] != Py_None) {
        const at::Tensor& t = tensor(a[3]);
        on.same(t);
        if (t.scalar_type() != at::kFloat) fail(PyExc_ValueError, "cosines and sines are float32");
        sizes2(t, n_pos, R);
        angles = ptr<float>(t);
    }
    int32_t table_B, max_pages;
    sizes2(table, table_B, max_pages);
    const int32_t* pages = on.dense<int32_t>(a[8], {B, max_pages}, at::kInt, "block_table");
    const int32_t *pl = on.dense<int32_t>(a[9], {B}, at::kInt, "prefix_len"), *n = on.dense<int32_t>(a[10], {B}, at::kInt, "n_nodes"),
                  *pos = on.dense<int32_t>(a[4], {B, T}, at::kInt, "pos", true);
    void *kc, *vc;
    Strides st{0, 0, 0};
    if (mx) {
        kc = on.cache(a[5]);
        vc = on.cache(a[6]);
        const StridesMx two = strides_mx_of(a[7]);
        st = {two.page, 0, two.head};
    } else {
        const at::Tensor &x = tensor(a[5]), &y = tensor(a[6]);
        on.same(x);
        on.same(y);
        if (x.scalar_type() != type || y.scalar_type() != type) fail(PyExc_AssertionError, "the caches are of the rows' type");
        kc = ptr<void>(x);
        vc = ptr<void>(y);
        st = strides_of(a[7]);
    }
    const int interleaved = PyObject_IsTrue(a[11]);
    if (interleaved < 0) throw PythonError();
    on.gpu();
    const c10::DeviceGuard guard(on.dev);
    const LaunchStream stream(a[13], on.dev);
    Outputs out(a[12], on.dev);
    void* q_out = q ? out.get_checked<void>(k_q, {B, T, Hq, D}, type) : nullptr;
    int32_t* status = out.get_checked(k_status, {B});
    const int32_t dtype = type == at::kFloat ? GRAFT_F32 : GRAFT_BF16, Bi = static_cast<int32_t>(B), Ti = static_cast<int32_t>(T);
    const int32_t Hqi = static_cast<int32_t>(Hq), Hkvi = static_cast<int32_t>(Hkv), Di = static_cast<int32_t>(D);
    const void *kp = k.data_ptr(), *vp = v.data_ptr();
    void* s = stream.handle();
    check(mx ? "graft_kv_append_mx" : "graft_kv_append", unlocked([&] {
        return mx ? lib.graft_kv_append_mx(q, kp, vp, q_stride, k_stride, v_stride, angles, n_pos, R, interleaved, pos, kc, vc, st.page, st.head, pages,
                                           max_pages, pl, n, Bi, Ti, Hqi, Hkvi, Di, GRAFT_PAGE_SIZE, dtype, q_out, status, s)
                  : lib.graft_kv_append(q, kp, vp, q_stride, k_stride, v_stride, angles, n_pos, R, interleaved, pos, kc, vc, st.page, st.token, st.head,
                                        pages, max_pages, pl, n, Bi, Ti, Hqi, Hkvi, Di, GRAFT_PAGE_SIZE, dtype, q_out, status, s);
    }));
    return out.release();
}
GRAFT_PY(py_kv_append, 14) { return append(a, false); }
GRAFT_PY(py_kv_append_mx, 14) { return append(a, true); }

// k_cache, v_cache, layer_stride, n_layers, strides, block_table, start, count, T, Hkv, D, bf16, out, stream
GRAFT_PY(py_kv_gather_mx, 14) {
    GRAFT_KEY(k); GRAFT_KEY(v); GRAFT_KEY(status);
    const at::Tensor& table = tensor(a[5]);
    const OnDevice on(table);
    const unsigned char *kc = on.cache(a[0]), *vc = on.cache(a[1]);
    const int64_t layer_stride = to_i64(a[2]);
    const int32_t n_layers = whole(a[3]), T = whole(a[8]), Hkv = whole(a[9]), D = whole(a[10]);
    const StridesMx st = strides_mx_of(a[4]);
    int32_t B, max_pages;
    sizes2(table, B, max_pages);
    const int32_t* pages = on.dense<int32_t>(a[5], {B, max_pages}, at::kInt, "block_table");
    const int32_t *start = on.dense<int32_t>(a[6], {B}, at::kInt, "start", true), *count = on.dense<int32_t>(a[7], {B}, at::kInt, "count");
    const int bf16 = PyObject_IsTrue(a[11]);
    if (bf16 < 0) throw PythonError();
    if (n_layers < 1 || T < 1 || Hkv < 1 || D < 1) fail(PyExc_ValueError, "n_layers, T, Hkv and D are positive");
    on.gpu();
    const c10::DeviceGuard guard(on.dev);
    const LaunchStream stream(a[13], on.dev);
    Outputs out(a[12], on.dev);
    const at::ScalarType type = bf16 ? at::kBFloat16 : at::kFloat;
    void* ko = out.get_checked<void>(k_k, {n_layers, B, T, Hkv, D}, type);
    void* vo = out.get_checked<void>(k_v, {n_layers, B, T, Hkv, D}, type);
    int32_t* status = out.get_checked(k_status, {B});
    void* s = stream.handle();
    check("graft_kv_gather_mx", unlocked([&] {
        return lib.graft_kv_gather_mx(kc, vc, layer_stride, n_layers, st.page, st.head, pages, max_pages, start, count, B, T, Hkv, D,
                                      bf16 ? GRAFT_BF16 : GRAFT_F32, ko, vo, status, s);
    }));
    return out.release();
}

// q, k_cache, v_cache, strides, block_table, prefix_len, n_nodes, mask, Hkv, scale, softcap, window, pos, out, workspace, stream
GRAFT_PY(py_tree_attn_mx, 16) {
    const at::Tensor &q = tensor(a[0]), &table = tensor(a[4]);
    const OnDevice on(q);
    if (q.dim() != 4) {
        PyErr_Format(PyExc_ValueError, "expected a query tensor of 4 dimensions, got %d", static_cast<int>(q.dim()));
        throw PythonError();
    }
    if (q.scalar_type() != at::kBFloat16) fail(PyExc_AssertionError, "queries over a 4-bit cache are bfloat16");
    const int32_t B = size_at(q, 0), K = size_at(q, 1), Hq = size_at(q, 2), D = size_at(q, 3), Hkv = whole(a[8]), window = whole(a[11]);
    const unsigned char *kc = on.cache(a[1]), *vc = on.cache(a[2]);
    const StridesMx st = strides_mx_of(a[3]);
    int32_t table_B, max_pages;
    sizes2(table, table_B, max_pages);
    const int32_t* pages = on.dense<int32_t>(a[4], {B, max_pages}, at::kInt, "block_table");
    const int32_t *pl = on.dense<int32_t>(a[5], {B}, at::kInt, "prefix_len"), *n = on.dense<int32_t>(a[6], {B}, at::kInt, "n_nodes"),
                  *pos = on.dense<int32_t>(a[12], {B, K}, at::kInt, "pos", true);
    const uint64_t* mask = on.dense<uint64_t>(a[7], {B, K, GRAFT_MASK_WORDS}, at::kLong, "mask", true);
    const double scale = PyFloat_AsDouble(a[9]);
    if (scale == -1.0 && PyErr_Occurred()) throw PythonError();
    const double cap = PyFloat_AsDouble(a[10]);
    if (cap == -1.0 && PyErr_Occurred()) throw PythonError();
    const void* qp = ptr<void>(q);
    on.gpu();
    const c10::DeviceGuard guard(on.dev);
    const LaunchStream stream(a[15], on.dev);
    at::Tensor new_out, new_ws;
    void* out;
    if (a[13] == Py_None) {
        new_out = empty(q.sizes(), at::kBFloat16, on.dev);
        out = new_out.data_ptr();
    } else out = on.dense<void>(a[13], q.sizes(), at::kBFloat16, "out");
    void* ws = nullptr;
    size_t ws_bytes = 0;
    if (a[14] == Py_None) {
        ws_bytes = lib.graft_tree_attn_mx_workspace_bytes(B, K, Hq, Hkv, D, max_pages);
        if (ws_bytes > 0) {
            new_ws = stream.scratch(ws_bytes);
            ws = new_ws.data_ptr();
        }
    } else {
        const at::Tensor& w = tensor(a[14]);
        on.same(w);
        ws = ptr<void>(w);
        ws_bytes = w.nbytes();
    }
    void* s = stream.handle();
    check("graft_tree_attn_mx", unlocked([&] {
        return lib.graft_tree_attn_mx(qp, kc, vc, st.page, st.head, pages, max_pages, pl, n, mask, pos, B, K, Hq, Hkv, D, GRAFT_PAGE_SIZE,
                                      static_cast<float>(scale), static_cast<float>(cap), window, out, ws, ws_bytes, s);
    }));
    if (new_out.defined()) return THPVariable_Wrap(std::move(new_out));
    Py_INCREF(a[13]);
    return a[13];
}

// k_cache, v_cache, layer_stride, n_layers, strides, block_table, prefix_len, path, accept_len, K_max, Hkv, D, out, stream
GRAFT_PY(py_kv_compact_mx, 14) {
    GRAFT_KEY(new_prefix_len); GRAFT_KEY(status);
    const at::Tensor &table = tensor(a[5]), &path = tensor(a[7]);
    const OnDevice on(path);
    int32_t B, width, table_B, max_pages;
    sizes2(path, B, width);
    sizes2(table, table_B, max_pages);
    unsigned char *kc = on.cache(a[0]), *vc = on.cache(a[1]);
    const int64_t layer_stride = to_i64(a[2]);
    const int32_t n_layers = whole(a[3]), K = whole(a[9]), Hkv = whole(a[10]), D = whole(a[11]);
    const StridesMx st = strides_mx_of(a[4]);
    const int32_t* pages = on.dense<int32_t>(a[5], {B, max_pages}, at::kInt, "block_table");
    const int32_t *pl = on.dense<int32_t>(a[6], {B}, at::kInt, "prefix_len"), *pp = on.dense<int32_t>(a[7], {B, width}, at::kInt, "path"),
                  *al = on.dense<int32_t>(a[8], {B}, at::kInt, "accept_len");
    on.gpu();
    const c10::DeviceGuard guard(on.dev);
    const LaunchStream stream(a[13], on.dev);
    Outputs out(a[12], on.dev);
    int32_t* new_len = out.get_checked(k_new_prefix_len, {B});
    int32_t* status = out.get_checked(k_status, {B});
    void* s = stream.handle();
    check("graft_kv_compact_mx", unlocked([&] {
        return lib.graft_kv_compact_mx(kc, vc, layer_stride, n_layers, st.page, st.head, pages, max_pages, pl, pp, al, B, width - 1, K, Hkv, D,
                                       new_len, status, s);
    }));
    return out.release();
}

// ---- prompts, and rules on logits -------------------------------------------------------------------
// q, k_cache, v_cache, strides, block_table, prefix_len, n_nodes, Hkv, scale, softcap, window, out, workspace, stream
GRAFT_PY(py_prompt_attn, 14) {
    const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]), &v = tensor(a[2]), &table = tensor(a[4]);
    const OnDevice on(q);
    if (q.dim() != 4) {
        PyErr_Format(PyExc_ValueError, "expected a query tensor of 4 dimensions, got %d", static_cast<int>(q.dim()));
        throw PythonError();
    }
    const at::ScalarType type = q.scalar_type();
    if ((type != at::kFloat && type != at::kBFloat16) || k.scalar_type() != type || v.scalar_type() != type)
        fail(PyExc_AssertionError, "queries, keys and values are all float32 or all bfloat16");
    on.same(k);
    on.same(v);
    const int32_t B = size_at(q, 0), T = size_at(q, 1), Hq = size_at(q, 2), D = size_at(q, 3), Hkv = whole(a[7]), window = whole(a[10]);
    const void *qp = ptr<void>(q), *kp = ptr<void>(k), *vp = ptr<void>(v);
    const Strides st = strides_of(a[3]);
    int32_t table_B, max_pages;
    sizes2(table, table_B, max_pages);
    const int32_t* pages = on.dense<int32_t>(a[4], {B, max_pages}, at::kInt, "block_table");
    const int32_t *pl = on.dense<int32_t>(a[5], {B}, at::kInt, "prefix_len"), *n = on.dense<int32_t>(a[6], {B}, at::kInt, "n_nodes");
    const double scale = PyFloat_AsDouble(a[8]);
    if (scale == -1.0 && PyErr_Occurred()) throw PythonError();
    const double cap = PyFloat_AsDouble(a[9]);
    if (cap == -1.0 && PyErr_Occurred()) throw PythonError();
    on.gpu();
    const c10::DeviceGuard guard(on.dev);
    const LaunchStream stream(a[13], on.dev);
    const int32_t dtype = type == at::kFloat ? GRAFT_F32 : GRAFT_BF16;
    at::Tensor new_out, new_ws;
    void* out;
    if (a[11] == Py_None) {
        new_out = empty(q.sizes(), type, on.dev);
        out = new_out.data_ptr();
    } else out = on.dense<void>(a[11], q.sizes(), type, "out");
    void* ws = nullptr;
    size_t ws_bytes = 0;
    if (a[12] == Py_None) {
        ws_bytes = lib.graft_prompt_attn_workspace_bytes(B, T, Hq, Hkv, D, max_pages, window, dtype);
        if (ws_bytes > 0) {
            new_ws = stream.scratch(ws_bytes);
            ws = new_ws.data_ptr();
        }
    } else {
        const at::Tensor& w = tensor(a[12]);
        on.same(w);
        ws = ptr<void>(w);
        ws_bytes = w.nbytes();
    }
    void* s = stream.handle();
    check("graft_prompt_attn", unlocked([&] {
        return lib.graft_prompt_attn(qp, kp, vp, st.page, st.token, st.head, pages, max_pages, pl, n, B, T, Hq, Hkv, D, GRAFT_PAGE_SIZE,
                                     static_cast<float>(scale), static_cast<float>(cap), window, dtype, out, ws, ws_bytes, s);
    }));
    if (new_out.defined()) return THPVariable_Wrap(std::move(new_out));
    Py_INCREF(a[11]);
    return a[11];
}

// ctx, ctx_len, prompt_len, counts, start, status, stream
GRAFT_PY(py_token_counts, 7) {
    const at::Tensor &ctx = tensor(a[0]), &counts = tensor(a[3]);
    const OnDevice on(ctx);
    int32_t B, L_max, counts_B, V;
    sizes2(ctx, B, L_max);
    sizes2(counts, counts_B, V);
    const int32_t* c = on.dense<int32_t>(a[0], {B, L_max}, at::kInt, "ctx");
    int32_t* to = on.dense<int32_t>(a[3], {B, V}, at::kInt, "counts");
    const int32_t *len = on.dense<int32_t>(a[1], {B}, at::kInt, "ctx_len"), *prompt = on.dense<int32_t>(a[2], {B}, at::kInt, "prompt_len", true),
                  *start = on.dense<int32_t>(a[4], {B}, at::kInt, "start", true);
    on.gpu();
    const c10::DeviceGuard guard(on.dev);
    const LaunchStream stream(a[6], on.dev);
    at::Tensor fresh;
    int32_t* status;
    if (a[5] == Py_None) {
        fresh = empty_i32({B}, on.dev);
        status = static_cast<int32_t*>(fresh.data_ptr());
    } else status = on.dense<int32_t>(a[5], {B}, at::kInt, "status");
    void* s = stream.handle();
    check("graft_token_counts", unlocked([&] { return lib.graft_token_counts(c, len, prompt, start, B, L_max, V, to, status, s); }));
    if (fresh.defined()) return THPVariable_Wrap(std::move(fresh));
    Py_INCREF(a[5]);
    return a[5];
}

// logits, n_nodes, tokens, mask, counts, repetition, frequency, presence, bias, allow, allow_index, result, out, workspace, stream
GRAFT_PY(py_logits_adjust, 15) {
    GRAFT_KEY(target_ids); GRAFT_KEY(status);
    const at::Tensor& logits = tensor(a[0]);
    const OnDevice on(logits);
    if (logits.dim() != 3) {
        PyErr_Format(PyExc_ValueError, "expected logits of 3 dimensions, got %d", static_cast<int>(logits.dim()));
        throw PythonError();
    }
    const int32_t B = size_at(logits, 0), K = size_at(logits, 1), V = size_at(logits, 2);
    const float* l = on.dense<float>(a[0], {B, K, V}, at::kFloat, "logits");
    const int32_t *n = on.dense<int32_t>(a[1], {B}, at::kInt, "n_nodes"), *tokens = on.dense<int32_t>(a[2], {B, K}, at::kInt, "tokens", true),
                  *counts = on.dense<int32_t>(a[4], {B, V}, at::kInt, "counts", true);
    const uint64_t* mask = on.dense<uint64_t>(a[3], {B, K, GRAFT_MASK_WORDS}, at::kLong, "mask", true);
    const float *rep = on.dense<float>(a[5], {B}, at::kFloat, "repetition", true), *freq = on.dense<float>(a[6], {B}, at::kFloat, "frequency", true),
                *pres = on.dense<float>(a[7], {B}, at::kFloat, "presence", true);
    const float* bias = nullptr;
    int32_t bias_rows = 0;
    if (a[8] != Py_None) {
        const bool each = tensor(a[8]).dim() == 2;
        bias = each ? on.dense<float>(a[8], {B, V}, at::kFloat, "bias") : on.dense<float>(a[8], {V}, at::kFloat, "bias");
        bias_rows = each ? B : 1;
    }
    const uint32_t* allow = nullptr;
    int32_t n_allow = 0;
    if (a[9] != Py_None) {
        n_allow = size_at(tensor(a[9]), 0);
        allow = on.dense<uint32_t>(a[9], {n_allow, (static_cast<int64_t>(V) + 31) / 32}, at::kInt, "allow");
    }
    const int32_t* index = on.dense<int32_t>(a[10], {B, K}, at::kInt, "allow_index", true);
    float* result = on.dense<float>(a[11], {B, K, V}, at::kFloat, "result", true);
    on.gpu();
    const c10::DeviceGuard guard(on.dev);
    const LaunchStream stream(a[14], on.dev);
    Outputs out(a[12], on.dev);
    int32_t* ids = out.get_checked(k_target_ids, {B, K});
    int32_t* status = out.get_checked(k_status, {B});
    at::Tensor new_ws;
    void* ws;
    size_t ws_bytes;
    if (a[13] == Py_None) {
        ws_bytes = lib.graft_logits_adjust_workspace_bytes(B, K, V);
        new_ws = stream.scratch(ws_bytes);
        ws = new_ws.data_ptr();
    } else {
        const at::Tensor& w = tensor(a[13]);
        on.same(w);
        ws = ptr<void>(w);
        ws_bytes = w.nbytes();
    }
    void* s = stream.handle();
    check("graft_logits_adjust", unlocked([&] {
        return lib.graft_logits_adjust(l, n, tokens, mask, B, K, V, counts, rep, freq, pres, bias, bias_rows, allow, n_allow, index, result, ids, status, ws,
                                       ws_bytes, s);
    }));
    return out.release();
}

// path of the library, GraftError
PyObject* py_bind(PyObject*, PyObject* args) {
    const char* path;
    PyObject* error;
    if (!PyArg_ParseTuple(args, "sO", &path, &error)) return nullptr;
    void* h = dlopen(path, RTLD_NOW | RTLD_LOCAL);
    if (!h) return PyErr_Format(PyExc_OSError, "%s", dlerror());
    Library l;
#define X(name)                                                                      \
    l.name = reinterpret_cast<decltype(&::name)>(dlsym(h, #name));                    \
    if (!l.name) return PyErr_Format(PyExc_OSError, "%s does not export " #name, path);
    GRAFT_ENTRY_POINTS(X)
#undef X
    lib = l;
    Py_INCREF(error);
    Py_XDECREF(graft_error);
    graft_error = error;
    Py_RETURN_NONE;
}

#define GRAFT_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_##name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"bind", py_bind, METH_VARARGS, "bind(path, error_class): resolve the library's entry points"},
    GRAFT_METHOD(retrieve), GRAFT_METHOD(build_tree_mask), GRAFT_METHOD(tree_attn), GRAFT_METHOD(accept),
    GRAFT_METHOD(accept_noalloc), GRAFT_METHOD(matrix_retrieve), GRAFT_METHOD(matrix_update), GRAFT_METHOD(kv_compact),
    GRAFT_METHOD(prune_select), GRAFT_METHOD(kv_append), GRAFT_METHOD(kv_append_mx), GRAFT_METHOD(kv_gather_mx),
    GRAFT_METHOD(tree_attn_mx), GRAFT_METHOD(kv_compact_mx), GRAFT_METHOD(prompt_attn), GRAFT_METHOD(token_counts),
    GRAFT_METHOD(logits_adjust), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_native", "Marshalling of the graft_* calls.", -1, methods,
                          nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() {
    s_page = PyUnicode_InternFromString("page");
    s_token = PyUnicode_InternFromString("token");
    s_head = PyUnicode_InternFromString("head");
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    return PyModule_Create(&module_def);
}
