// The binding's host path in native code: what happens between a Python call and the C entry point.
//
// The functions of binding.py that enqueue work take torch tensors and pass device pointers, sizes
// and the current stream to libsepattn.  At the small end of the range (one conversation, one decode
// step) the kernels last a few microseconds, so what a call costs on the host decides how fast a
// generation loop runs: in Python (ctypes argument objects, current_stream(), torch.empty) it was
// about 5.5 us per call on top of the kernel launches, here it is well under 1 us.  Nothing is
// computed here: checks on the tensors, allocation of outputs and workspaces that the caller did not
// pass (through torch's allocator), one call into the library.
//
// The module does not link libsepattn: bind(path) opens the library the binding uses and looks the
// entry points up, so that SEPATTN_LIB selects another build for this path as well.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <dlfcn.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <vector>

#include "sepattn.h"

namespace {

#define LIB_FUNCTIONS(X)                                                                                               \
    X(sepattn_mark_separators) X(sepattn_compact_workspace_bytes) X(sepattn_compact_indices)  \
    X(sepattn_mark_compact) X(sepattn_forward_workspace_bytes) X(sepattn_forward) X(sepattn_forward_headwise)          \
    X(sepattn_backward_headwise_workspace_bytes) X(sepattn_backward_headwise) X(sepattn_doc_bounds)                    \
    X(sepattn_forward_packed) X(sepattn_backward_packed) X(sepattn_backward_workspace_bytes) X(sepattn_backward)       \
    X(sepattn_decode_workspace_bytes) X(sepattn_decode) X(sepattn_decode_noalloc) X(sepkv_evict_window)                \
    X(sepkv_fill_from_prefill) X(sepattn_decode_rope) X(sepkv_append)
// what some of them call where the outputs are their own, fresh ones
#define LIB_FRESH_FUNCTIONS(F) F(sepattn_compact_indices_filled) F(sepattn_mark_compact_filled) F(sepkv_fill_from_prefill_zeroed)
// rotary positions in front of the attention, shared prompts
#define LIB_POSITION_FUNCTIONS(P)                                                                                      \
    P(sepattn_rope) P(sepattn_rope_backward) P(sepkv_append_rope) P(sepkv_group_sequences) P(sepkv_rope_cache)          \
    P(sepattn_decode_shared_workspace_bytes) P(sepattn_decode_shared) P(sepattn_decode_shared_rope)
// norms in front of them, the cache in 4 bits
#define LIB_NORM_FP4_FUNCTIONS(N)                                                                                      \
    N(sepattn_norm_rope) N(sepattn_norm_rope_backward_workspace_bytes) N(sepattn_norm_rope_backward) N(sepkv_append_norm_rope) \
    N(sepkv_fill_from_prefill_mx) N(sepkv_fill_from_prefill_mx_zeroed) N(sepkv_append_mx) N(sepkv_append_rope_mx)      \
    N(sepkv_append_norm_rope_mx) N(sepkv_evict_window_mx) N(sepkv_expand_mx) N(sepattn_decode_mx_workspace_bytes)      \
    N(sepattn_decode_mx) N(sepattn_decode_rope_mx)
struct Lib {
#define X(name) decltype(&::name) name;
    LIB_FUNCTIONS(X)
    LIB_FRESH_FUNCTIONS(X)
    LIB_POSITION_FUNCTIONS(X)
    LIB_NORM_FP4_FUNCTIONS(X)
#undef X
} lib;
PyObject *g_raise = nullptr;  // Python callable: raises SepattnError(function, status)

// A failed check: the Python error is set, the caller returns nullptr.
struct Failed {};
[[noreturn]] void fail(PyObject *type, const char *msg) {
    PyErr_SetString(type, msg);
    throw Failed{};
}
void require(bool ok, const char *msg) {
    if (!ok) fail(PyExc_AssertionError, msg);
}

// a tensor argument (borrowed from the caller for the duration of the call)
const at::Tensor &tensor(PyObject *o) {
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, "a torch tensor is expected");
    return THPVariable_Unpack(o);
}
// ... that must live on the GPU and be contiguous
const at::Tensor &dev(PyObject *o) {
    const at::Tensor &t = tensor(o);
    if (!t.is_cuda()) fail(PyExc_ValueError, "libsepattn works on GPU tensors only");
    if (!t.is_contiguous()) fail(PyExc_ValueError, "tensors must be contiguous");
    return t;
}
void *ptr(const at::Tensor &t) { return t.data_ptr(); }
void *ptr(PyObject *o) { return o == Py_None ? nullptr : tensor(o).data_ptr(); }
const int32_t *i32(const at::Tensor &t) { return static_cast<const int32_t *>(t.data_ptr()); }

void *stream_of(const at::Tensor &t) { return c10::hip::getCurrentHIPStream(t.device().index()).stream(); }

int dtype_code(const at::Tensor &t) {
    const auto s = t.scalar_type();
    if (s == at::kBFloat16) return SEPATTN_BF16;
    if (s == at::kFloat) return SEPATTN_FP32;
    fail(PyExc_TypeError, "unsupported dtype: bf16 or fp32 expected");
}
at::Tensor empty(c10::IntArrayRef shape, at::ScalarType type, const at::Device &device) {
    return at::detail::empty_cuda(shape, type, device, std::nullopt);
}
at::Tensor fresh_like(const at::Tensor &t) { return empty(t.sizes(), t.scalar_type(), t.device()); }

long as_long(PyObject *o) {
    if (PyLong_CheckExact(o)) {
        const long v = PyLong_AsLong(o);
        if (v == -1 && PyErr_Occurred()) throw Failed{};
        return v;
    }
    PyObject *n = PyNumber_Long(o);  // what int(o) gives
    if (!n) throw Failed{};
    const long v = PyLong_AsLong(n);
    Py_DECREF(n);
    if (v == -1 && PyErr_Occurred()) throw Failed{};
    return v;
}
int as_int(PyObject *o) {
    const long v = as_long(o);
    if (v < INT32_MIN || v > INT32_MAX) fail(PyExc_OverflowError, "argument does not fit 32 bits");
    return (int)v;
}
float as_float(PyObject *o) {
    if (PyFloat_CheckExact(o)) return (float)PyFloat_AS_DOUBLE(o);
    PyObject *n = PyNumber_Float(o);  // what float(o) gives
    if (!n) throw Failed{};
    const double v = PyFloat_AS_DOUBLE(n);
    Py_DECREF(n);
    return (float)v;
}
bool as_bool(PyObject *o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Failed{};
    return v != 0;
}
// a reference that this call owns
struct Owned {
    PyObject *o;
    explicit Owned(PyObject *x) : o(x) {
        if (!o) throw Failed{};
    }
    ~Owned() { Py_DECREF(o); }
    Owned(const Owned &) = delete;
    Owned &operator=(const Owned &) = delete;
};
std::vector<int32_t> int_list(PyObject *o) {
    if (PyObject_Size(o) < 0) throw Failed{};    // an iterator is refused
    const Owned items(PySequence_Tuple(o));      // items of its own: int() of one may run code that changes the list
    const Py_ssize_t n = PyTuple_GET_SIZE(items.o);
    std::vector<int32_t> v((size_t)n);
    for (Py_ssize_t k = 0; k < n; ++k) v[(size_t)k] = (int32_t)as_long(PyTuple_GET_ITEM(items.o, k));
    return v;
}
// The N tensors of an `out` argument, which may be any iterable; None: the call allocates its own.  The items
// are held until the call has returned: an iterator that made them is no longer their owner.
template <int N>
struct Out {
    PyObject *items = nullptr;  // a tuple
    explicit Out(PyObject *o) {
        if (o == Py_None) return;
        items = PySequence_Tuple(o);
        if (!items) throw Failed{};
        if (PyTuple_GET_SIZE(items) == N) return;
        Py_DECREF(items);
        fail(PyExc_ValueError, "out: wrong number of tensors");
    }
    ~Out() { Py_XDECREF(items); }
    Out(const Out &) = delete;
    Out &operator=(const Out &) = delete;
    bool given() const { return items != nullptr; }
    PyObject *operator[](int k) const { return PyTuple_GET_ITEM(items, k); }
};
void check(const char *fn, int rc) {
    if (rc == SEPATTN_OK) return;
    PyObject *r = PyObject_CallFunction(g_raise, "si", fn, rc);
    Py_XDECREF(r);
    throw Failed{};
}
// What a call allocates and enqueues runs without the interpreter lock: the allocator may wait for the device, a
// launch for a place in a full queue, and other Python threads go on meanwhile.  Arguments are taken apart before
// (no Python object is touched inside), results wrapped afterwards.
template <typename F>
auto unlocked(F f) {
    struct Lock {
        PyThreadState *state = PyEval_SaveThread();
        ~Lock() { PyEval_RestoreThread(state); }
    } lock;
    return f();
}
// the caller's workspace, or one from torch's allocator that goes back when the call returns (the
// allocator hands it out again in stream order)
struct Workspace {
    at::Tensor own;
    void *p = nullptr;
    size_t bytes = 0;
    bool given;
    explicit Workspace(PyObject *ws) : given(ws != Py_None) {
        if (!given) return;
        const at::Tensor &t = tensor(ws);
        p = t.data_ptr();
        bytes = (size_t)t.numel();
    }
    void allocate(size_t need, const at::Device &device) {
        bytes = need < 256 ? 256 : need;
        own = empty({(int64_t)bytes}, at::kByte, device);
        p = own.data_ptr();
    }
};
PyObject *wrap(at::Tensor t) { return THPVariable_Wrap(std::move(t)); }
PyObject *keep(PyObject *o) {
    Py_INCREF(o);
    return o;
}
template <typename... P>
PyObject *tuple_of(P *...items) {  // takes over the references
    PyObject *t = PyTuple_New(sizeof...(items));
    Py_ssize_t k = 0;
    (PyTuple_SET_ITEM(t, k++, items), ...);
    return t;
}

sepattn_params attn_params(const at::Tensor &Q, const at::Tensor &K, int a, int n, float scale, const at::Tensor &idx) {
    if (Q.dim() != 4 || K.dim() < 2) fail(PyExc_ValueError, "Q [B,Hq,L,d] and K [B,Hkv,L,d] are expected");
    sepattn_params p;
    p.B = (int)Q.size(0);
    p.Hq = (int)Q.size(1);
    p.Hkv = (int)K.size(1);
    p.L = (int)Q.size(2);
    p.d = (int)Q.size(3);
    p.a = a;
    p.n = n;
    p.scale = scale;
    p.dtype = dtype_code(Q);
    p.cap = (int)idx.size(1);
    return p;
}

// ---- marking and compaction ----------------------------------------------------------------------
// mark_separators(token_ids, sep_ids, out)
PyObject *mark_separators(PyObject *const *a) {
    const at::Tensor &tok = dev(a[0]);
    if (a[2] != Py_None) dev(a[2]);
    require(tok.scalar_type() == at::kInt && tok.dim() == 2, "token_ids: int32 [B, L]");
    const int B = (int)tok.size(0), L = (int)tok.size(1);
    const std::vector<int32_t> ids = int_list(a[1]);
    at::Tensor out;
    if (a[2] != Py_None) out = tensor(a[2]);
    check("sepattn_mark_separators", unlocked([&] {
              if (!out.defined()) out = empty({B, L}, at::kByte, tok.device());
              return lib.sepattn_mark_separators(i32(tok), B, L, ids.data(), (int)ids.size(), (uint8_t *)ptr(out), stream_of(tok));
          }));
    return a[2] == Py_None ? wrap(std::move(out)) : keep(a[2]);
}

// Index arrays, the caller's or (`allocate`) the call's own, where every entry of the list behind the last separator is
// `fill` (the _filled entry points write it).  Arguments: the last three of `out`, cap, want_prefix, fill.
struct IndexOut {
    at::Tensor idx, cnt, pre;
    int cap = 0, fill = 0;
    bool want_prefix = false;
    int32_t *idx_p = nullptr, *cnt_p = nullptr, *pre_p = nullptr;
    template <int N>
    IndexOut(const Out<N> &out, int L, PyObject *cap_o, PyObject *want_prefix_o, PyObject *fill_o) {
        if (out.given()) {
            const at::Tensor &i = dev(out[N - 3]);
            cap = (int)i.size(1);
            idx_p = (int32_t *)ptr(i);
            cnt_p = (int32_t *)ptr(dev(out[N - 2]));
            pre_p = out[N - 1] == Py_None ? nullptr : (int32_t *)ptr(dev(out[N - 1]));
        } else {
            cap = cap_o == Py_None ? L : as_int(cap_o);
            want_prefix = as_bool(want_prefix_o);
            fill = as_int(fill_o);
        }
    }
    void allocate(int B, int L, const at::Device &device) {
        idx = empty({B, cap > 1 ? cap : 1}, at::kInt, device);
        cnt = empty({B}, at::kInt, device);
        idx_p = (int32_t *)ptr(idx), cnt_p = (int32_t *)ptr(cnt);
        if (!want_prefix) return;
        pre = empty({B, L + 1}, at::kInt, device);
        pre_p = (int32_t *)ptr(pre);
    }
    PyObject *prefix_object() const { return pre.defined() ? wrap(pre) : keep(Py_None); }
};

// compact_indices(is_sep, cap, want_prefix, fill, out, ws)
PyObject *compact_indices(PyObject *const *a) {
    const at::Tensor &sep = dev(a[0]);
    require(sep.scalar_type() == at::kByte && sep.dim() == 2, "is_sep: uint8 [B, L]");
    const int B = (int)sep.size(0), L = (int)sep.size(1);
    const Out<3> out(a[4]);
    IndexOut o(out, L, a[1], a[2], a[3]);
    Workspace ws(a[5]);
    check("sepattn_compact_indices", unlocked([&] {
              if (!ws.given) ws.allocate(lib.sepattn_compact_workspace_bytes(B, L), sep.device());
              if (!out.given()) o.allocate(B, L, sep.device());
              if (!out.given())
                  return lib.sepattn_compact_indices_filled((const uint8_t *)ptr(sep), B, L, o.idx_p, o.cap, o.cnt_p, o.pre_p, o.fill,
                                                            ws.p, ws.bytes, stream_of(sep));
              return lib.sepattn_compact_indices((const uint8_t *)ptr(sep), B, L, o.idx_p, o.cap, o.cnt_p, o.pre_p, ws.p, ws.bytes,
                                                 stream_of(sep));
          }));
    if (out.given()) return tuple_of(keep(out[0]), keep(out[1]), keep(out[2]));
    return tuple_of(wrap(o.idx), wrap(o.cnt), o.prefix_object());
}

// mark_compact(token_ids, sep_ids, cap, want_prefix, fill, out, ws)
PyObject *mark_compact(PyObject *const *a) {
    const at::Tensor &tok = dev(a[0]);
    require(tok.scalar_type() == at::kInt && tok.dim() == 2, "token_ids: int32 [B, L]");
    const int B = (int)tok.size(0), L = (int)tok.size(1);
    const std::vector<int32_t> ids = int_list(a[1]);
    const Out<4> out(a[5]);
    at::Tensor sep;
    if (out.given()) sep = dev(out[0]);
    IndexOut o(out, L, a[2], a[3], a[4]);
    Workspace ws(a[6]);
    check("sepattn_mark_compact", unlocked([&] {
              if (!ws.given) ws.allocate(lib.sepattn_compact_workspace_bytes(B, L), tok.device());
              if (!out.given()) {
                  sep = empty({B, L}, at::kByte, tok.device());
                  o.allocate(B, L, tok.device());
                  return lib.sepattn_mark_compact_filled(i32(tok), B, L, ids.data(), (int)ids.size(), (uint8_t *)ptr(sep), o.idx_p,
                                                         o.cap, o.cnt_p, o.pre_p, o.fill, ws.p, ws.bytes, stream_of(tok));
              }
              return lib.sepattn_mark_compact(i32(tok), B, L, ids.data(), (int)ids.size(), (uint8_t *)ptr(sep), o.idx_p, o.cap,
                                              o.cnt_p, o.pre_p, ws.p, ws.bytes, stream_of(tok));
          }));
    if (out.given()) return tuple_of(keep(out[0]), keep(out[1]), keep(out[2]), keep(out[3]));
    return tuple_of(wrap(std::move(sep)), wrap(o.idx), wrap(o.cnt), o.prefix_object());
}

// doc_bounds(cu_seqlens, L, a, is_sep_row, out)
PyObject *doc_bounds(PyObject *const *a) {
    const at::Tensor &cu = dev(a[0]);
    if (a[3] != Py_None) dev(a[3]);
    require(cu.scalar_type() == at::kInt && cu.dim() == 1, "cu_seqlens: int32 [n_docs + 1]");
    const int L = as_int(a[1]);
    const int n_docs = (int)cu.numel() - 1, init = as_int(a[2]);
    // `out` itself is returned, so it has to be a sequence; items beyond the two are left alone
    const Out<2> out(Owned(a[4] == Py_None ? keep(Py_None) : PySequence_GetSlice(a[4], 0, 2)).o);
    at::Tensor s, e;
    if (out.given()) {
        s = dev(out[0]);
        e = dev(out[1]);
    }
    uint8_t *row = (uint8_t *)ptr(a[3]);
    check("sepattn_doc_bounds", unlocked([&] {
              if (!out.given()) {
                  s = empty({L}, at::kInt, cu.device());
                  e = empty({L}, at::kInt, cu.device());
              }
              return lib.sepattn_doc_bounds(i32(cu), n_docs, L, init, (int32_t *)ptr(s), (int32_t *)ptr(e), row, stream_of(cu));
          }));
    if (out.given()) return keep(a[4]);
    return tuple_of(wrap(std::move(s)), wrap(std::move(e)));
}

// ---- attention -------------------------------------------------------------------------------------
// The three forms of a call differ in what stands between the sizes and the tensors: nothing, the
// heads' windows, or the documents' bounds (nh / ds, de).
enum Form { kPlain, kHeadwise, kPacked };

// the documents' bounds of a packed call: the kernels read a row of L entries for every row of the batch
struct DocBounds {
    const int32_t *start, *end;
    DocBounds(PyObject *so, PyObject *eo, const sepattn_params &p) {
        const at::Tensor &s = dev(so), &e = dev(eo);
        require(s.scalar_type() == at::kInt && e.scalar_type() == at::kInt && s.dim() == 2 && s.size(0) == p.B &&
                    s.size(1) == p.L && e.sizes() == s.sizes(), "doc_start, doc_end: int32 [B, L]");
        start = i32(s);
        end = i32(e);
    }
};

// forward(Q, K, V, sep_idx, sep_count, sep_prefix, a, n | n_per_head, scale, out, ws [, doc_start, doc_end])
template <Form F>
PyObject *forward(PyObject *const *a) {
    const at::Tensor &Q = dev(a[0]), &K = dev(a[1]), &V = dev(a[2]), &idx = dev(a[3]), &cnt = dev(a[4]), &pre = dev(a[5]);
    require(K.sizes() == V.sizes() && Q.scalar_type() == K.scalar_type() && K.scalar_type() == V.scalar_type(),
            "K and V of one shape, Q, K, V of one dtype");
    const sepattn_params p = attn_params(Q, K, as_int(a[6]), F == kHeadwise ? 1 : as_int(a[7]), as_float(a[8]), idx);
    std::vector<int32_t> nh;
    const int32_t *ds = nullptr, *de = nullptr;
    if constexpr (F == kHeadwise) {
        nh = int_list(a[7]);
        require((int)nh.size() == p.Hq, "n_per_head: one window per query head");
    }
    if constexpr (F == kPacked) {
        const DocBounds d(a[11], a[12], p);
        ds = d.start, de = d.end;
    }
    const Out<2> out(a[9]);
    at::Tensor O, LSE;
    void *optr = nullptr, *lptr = nullptr;
    if (out.given()) optr = ptr(out[0]), lptr = ptr(out[1]);
    Workspace ws(a[10]);
    constexpr const char *name = F == kPlain ? "sepattn_forward" : (F == kHeadwise ? "sepattn_forward_headwise" : "sepattn_forward_packed");
    check(name, unlocked([&] {
              if (!out.given()) {
                  O = fresh_like(Q);
                  LSE = empty({p.B, p.Hq, p.L}, at::kFloat, Q.device());
                  optr = ptr(O), lptr = ptr(LSE);
              }
              // (the forward needs no workspace; the query keeps this right if that changes)
              const size_t need = lib.sepattn_forward_workspace_bytes(&p);
              if (!ws.given && need > 0) ws.allocate(need, Q.device());
              float *lse = (float *)lptr;
              void *st = stream_of(Q);
              if constexpr (F == kPlain)
                  return lib.sepattn_forward(&p, ptr(Q), ptr(K), ptr(V), i32(idx), i32(cnt), i32(pre), optr, lse, ws.p, ws.bytes, st);
              else if constexpr (F == kHeadwise)
                  return lib.sepattn_forward_headwise(&p, nh.data(), ptr(Q), ptr(K), ptr(V), i32(idx), i32(cnt), i32(pre), optr, lse,
                                                      ws.p, ws.bytes, st);
              else
                  return lib.sepattn_forward_packed(&p, ds, de, ptr(Q), ptr(K), ptr(V), i32(idx), i32(cnt), i32(pre), optr, lse, ws.p,
                                                    ws.bytes, st);
          }));
    if (out.given()) return tuple_of(keep(out[0]), keep(out[1]));
    return tuple_of(wrap(std::move(O)), wrap(std::move(LSE)));
}

// backward(Q, K, V, O, LSE, dO, sep_idx, sep_count, sep_prefix, a, n | n_per_head, scale, out, ws [, doc_start, doc_end])
template <Form F>
PyObject *backward(PyObject *const *a) {
    const at::Tensor &Q = dev(a[0]), &K = dev(a[1]), &V = dev(a[2]), &O = dev(a[3]), &LSE = dev(a[4]), &dO = dev(a[5]),
                     &idx = dev(a[6]), &cnt = dev(a[7]), &pre = dev(a[8]);
    const sepattn_params p = attn_params(Q, K, as_int(a[9]), F == kHeadwise ? 1 : as_int(a[10]), as_float(a[11]), idx);
    std::vector<int32_t> nh;
    const int32_t *ds = nullptr, *de = nullptr;
    if constexpr (F == kHeadwise) {
        nh = int_list(a[10]);
        require((int)nh.size() == p.Hq, "n_per_head: one window per query head");
    }
    if constexpr (F == kPacked) {
        const DocBounds d(a[14], a[15], p);
        ds = d.start, de = d.end;
    }
    const Out<3> out(a[12]);
    at::Tensor g[3];
    void *gp[3];
    for (int k = 0; out.given() && k < 3; ++k) gp[k] = ptr(out[k]);
    Workspace ws(a[13]);
    constexpr const char *name = F == kPlain ? "sepattn_backward" : (F == kHeadwise ? "sepattn_backward_headwise" : "sepattn_backward_packed");
    check(name, unlocked([&] {
              if (!out.given()) {
                  g[0] = fresh_like(Q);
                  g[1] = fresh_like(K);
                  g[2] = fresh_like(V);
                  for (int k = 0; k < 3; ++k) gp[k] = ptr(g[k]);
              }
              if (!ws.given)
                  ws.allocate(F == kHeadwise ? lib.sepattn_backward_headwise_workspace_bytes(&p, nh.data())
                                             : lib.sepattn_backward_workspace_bytes(&p), Q.device());
              const float *lse = (const float *)ptr(LSE);
              void *st = stream_of(Q);
              if constexpr (F == kPlain)
                  return lib.sepattn_backward(&p, ptr(Q), ptr(K), ptr(V), ptr(O), lse, ptr(dO), i32(idx), i32(cnt), i32(pre), gp[0],
                                              gp[1], gp[2], ws.p, ws.bytes, st);
              else if constexpr (F == kHeadwise)
                  return lib.sepattn_backward_headwise(&p, nh.data(), ptr(Q), ptr(K), ptr(V), ptr(O), lse, ptr(dO), i32(idx), i32(cnt),
                                                       i32(pre), gp[0], gp[1], gp[2], ws.p, ws.bytes, st);
              else
                  return lib.sepattn_backward_packed(&p, ds, de, ptr(Q), ptr(K), ptr(V), ptr(O), lse, ptr(dO), i32(idx), i32(cnt),
                                                     i32(pre), gp[0], gp[1], gp[2], ws.p, ws.bytes, st);
          }));
    if (out.given()) return tuple_of(keep(out[0]), keep(out[1]), keep(out[2]));
    return tuple_of(wrap(std::move(g[0])), wrap(std::move(g[1])), wrap(std::move(g[2])));
}

// ---- the streaming cache ---------------------------------------------------------------------------
const at::Tensor &sizes_arg(PyObject *o) {
    const at::Tensor &t = dev(o);
    require(t.scalar_type() == at::kInt && t.dim() == 2 && t.size(1) == SEPKV_SIZES_COLS, "sizes: int32 [S, 6]");
    return t;
}
sepkv_params kv_params(const at::Tensor &Kc, int S, int Hq, int a, int s, int w, float scale) {
    if (Kc.dim() != 4) fail(PyExc_ValueError, "Kc [S,Hkv,c,d] is expected");
    sepkv_params p;
    p.S = S;
    p.Hq = Hq;
    p.Hkv = (int)Kc.size(1);
    p.d = (int)Kc.size(3);
    p.a = a;
    p.s = s;
    p.w = w;
    p.c = (int)Kc.size(2);
    p.scale = scale;
    p.dtype = dtype_code(Kc);
    return p;
}

enum Decode { kKept, kRope, kNoAlloc };  // positions as the keys hold them, by place in the cache; no allocation

// decode(q, Kc, Vc, sizes, rope_table, a, s, w, scale, out, ws): the table is looked at with kRope only; kNoAlloc: out is
// required, ws unused
template <Decode F>
PyObject *decode(PyObject *const *a) {
    const at::Tensor &q = dev(a[0]), &Kc = dev(a[1]), &Vc = dev(a[2]);
    const at::Tensor *table = F == kRope ? &dev(a[4]) : nullptr;
    const at::Tensor &sizes = sizes_arg(a[3]);
    if (q.dim() != 3) fail(PyExc_ValueError, "q [S,Hq,d] is expected");
    if (F == kRope)
        require(table->scalar_type() == at::kFloat && table->dim() == 3 && table->size(1) == 2 && table->size(2) * 2 == q.size(2),
                "rope_table: fp32 [n_pos, 2, d/2]");
    sepkv_params p = kv_params(Kc, (int)q.size(0), (int)q.size(1), as_int(a[5]), as_int(a[6]), as_int(a[7]), as_float(a[8]));
    p.d = (int)q.size(2);
    const Out<2> out(a[9]);
    if (F == kNoAlloc && !out.given()) fail(PyExc_TypeError, "out is required");
    at::Tensor o, lse;
    void *optr = nullptr, *lptr = nullptr;
    if (out.given()) optr = ptr(out[0]), lptr = ptr(out[1]);  // an item None: no LSE wanted
    Workspace ws(F == kNoAlloc ? Py_None : a[10]);
    check(F == kNoAlloc ? "sepattn_decode_noalloc" : (F == kRope ? "sepattn_decode_rope" : "sepattn_decode"), unlocked([&] {
              if (!out.given()) {
                  o = fresh_like(q);
                  lse = empty({p.S, p.Hq}, at::kFloat, q.device());
                  optr = ptr(o), lptr = ptr(lse);
              }
              if (F != kNoAlloc && !ws.given) ws.allocate(lib.sepattn_decode_workspace_bytes(&p), q.device());
              void *st = stream_of(q);
              if constexpr (F == kNoAlloc)
                  return lib.sepattn_decode_noalloc(&p, ptr(q), ptr(Kc), ptr(Vc), i32(sizes), optr, (float *)lptr, st);
              else if constexpr (F == kRope)
                  return lib.sepattn_decode_rope(&p, ptr(q), ptr(Kc), ptr(Vc), i32(sizes), (const float *)ptr(*table),
                                                 (int)table->size(0), optr, (float *)lptr, ws.p, ws.bytes, st);
              else
                  return lib.sepattn_decode(&p, ptr(q), ptr(Kc), ptr(Vc), i32(sizes), optr, (float *)lptr, ws.p, ws.bytes, st);
          }));
    if (out.given()) return tuple_of(keep(out[0]), keep(out[1]));
    return tuple_of(wrap(std::move(o)), wrap(std::move(lse)));
}

// append(k_new, v_new, is_sep_new, Kc, Vc, win_is_sep, sizes, Hq, a, s, w)
PyObject *append(PyObject *const *a) {
    const at::Tensor &k = dev(a[0]), &v = dev(a[1]), &sep = dev(a[2]), &Kc = dev(a[3]), &Vc = dev(a[4]), &flags = dev(a[5]);
    const at::Tensor &sizes = sizes_arg(a[6]);
    require(sep.scalar_type() == at::kByte && flags.scalar_type() == at::kByte, "is_sep_new, win_is_sep: uint8");
    const sepkv_params p = kv_params(Kc, (int)Kc.size(0), as_int(a[7]), as_int(a[8]), as_int(a[9]), as_int(a[10]), 1.0f);
    const int64_t want[3] = {p.S, p.Hkv, p.d};
    require(k.sizes() == c10::IntArrayRef(want, 3) && v.sizes() == k.sizes() && k.scalar_type() == Kc.scalar_type(),
            "k_new, v_new: [S, Hkv, d] in the cache's dtype");
    check("sepkv_append", unlocked([&] {
              return lib.sepkv_append(&p, ptr(k), ptr(v), (const uint8_t *)ptr(sep), ptr(Kc), ptr(Vc), (uint8_t *)ptr(flags),
                                      (int32_t *)ptr(sizes), stream_of(Kc));
          }));
    return keep(Py_None);
}

// evict_window(Kc, Vc, win_is_sep, sizes, Hq, a, s, w, ws)
PyObject *evict_window(PyObject *const *a) {
    const at::Tensor &Kc = dev(a[0]), &Vc = dev(a[1]), &flags = dev(a[2]);
    const at::Tensor &sizes = sizes_arg(a[3]);
    const sepkv_params p = kv_params(Kc, (int)Kc.size(0), as_int(a[4]), as_int(a[5]), as_int(a[6]), as_int(a[7]), 1.0f);
    // the step needs no scratch memory: a workspace is passed on if the caller has one, NULL otherwise
    const Workspace ws(a[8]);
    check("sepkv_evict_window", unlocked([&] {
              return lib.sepkv_evict_window(&p, ptr(Kc), ptr(Vc), (const uint8_t *)ptr(flags), (int32_t *)ptr(sizes), ws.p, ws.bytes,
                                            stream_of(Kc));
          }));
    return keep(Py_None);
}

// fill_from_prefill(K, V, is_sep, sep_idx, sep_prefix, Hq, a, s, w, c, nw, out)
PyObject *fill_from_prefill(PyObject *const *a) {
    const at::Tensor &K = dev(a[0]), &V = dev(a[1]), &sep = dev(a[2]), &idx = dev(a[3]), &pre = dev(a[4]);
    const int L = K.dim() == 4 ? (int)K.size(2) : 0, nw = as_int(a[10]);
    sepkv_params p = kv_params(K, (int)K.size(0), as_int(a[5]), as_int(a[6]), as_int(a[7]), as_int(a[8]), 1.0f);
    p.c = as_int(a[9]);
    const Out<4> out(a[11]);
    at::Tensor Kc, Vc, flags, sizes;
    if (out.given()) {
        Kc = dev(out[0]);
        Vc = dev(out[1]);
        flags = dev(out[2]);
        sizes = dev(out[3]);
        require(sizes.scalar_type() == at::kInt && sizes.dim() == 2 && sizes.size(0) == p.S && sizes.size(1) == SEPKV_SIZES_COLS,
                "sizes: int32 [S, 6]");
    }
    check("sepkv_fill_from_prefill", unlocked([&] {
              if (!out.given()) {
                  Kc = empty({p.S, p.Hkv, p.c, p.d}, K.scalar_type(), K.device());
                  Vc = empty({p.S, p.Hkv, p.c, p.d}, K.scalar_type(), K.device());
                  flags = empty({p.S, p.c - p.a - p.s}, at::kByte, K.device());
                  sizes = empty({p.S, SEPKV_SIZES_COLS}, at::kInt, K.device());
              }
              const auto fill = out.given() ? lib.sepkv_fill_from_prefill : lib.sepkv_fill_from_prefill_zeroed;
              return fill(&p, L, nw, ptr(K), ptr(V), (const uint8_t *)ptr(sep), i32(idx), (int)idx.size(1),
                          i32(pre), ptr(Kc), ptr(Vc), (uint8_t *)ptr(flags), (int32_t *)ptr(sizes), stream_of(K));
          }));
    if (out.given()) return tuple_of(keep(out[0]), keep(out[1]), keep(out[2]), keep(out[3]));
    return tuple_of(wrap(std::move(Kc)), wrap(std::move(Vc)), wrap(std::move(flags)), wrap(std::move(sizes)));
}

// ---- rotary positions ------------------------------------------------------------------------------
// The tensors of a call live on one device, which is the current one while the library is called.
template <typename... T>
void one_device(const at::Tensor &first, const T &...others) {
    const bool same[] = {true, (!others.defined() || others.device() == first.device())...};
    for (const bool s : same)
        if (!s) fail(PyExc_ValueError, "tensors on different devices");
}
// an optional tensor: undefined for None
at::Tensor dev_or_none(PyObject *o) { return o == Py_None ? at::Tensor() : dev(o); }
void *ptr_or_null(const at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }

// [B, H, L, d] on the GPU with any strides, d innermost
const at::Tensor &rows_arg(PyObject *o) {
    const at::Tensor &t = tensor(o);
    if (!t.is_cuda()) fail(PyExc_ValueError, "libsepattn works on GPU tensors only");
    if (t.dim() != 4) fail(PyExc_ValueError, "[B, H, L, d] is expected");
    if (t.size(3) != 1 && t.stride(3) != 1) fail(PyExc_ValueError, "the head dimension must be contiguous");
    for (const int64_t n : t.sizes()) require(n <= INT_MAX, "sizes of 32 bits are expected");
    return t;
}
struct Rows {  // one of q, k, v and what becomes of it
    at::Tensor from, to;
    sepattn_strides from_strides, to_strides;
    static sepattn_strides strides_of(const at::Tensor &t) { return {t.stride(0), t.stride(1), t.stride(2)}; }
    void finish() {
        if (!from.defined()) return;
        from_strides = strides_of(from);
        to_strides = strides_of(to);
    }
    const sepattn_strides *from_s() const { return from.defined() ? &from_strides : nullptr; }
    const sepattn_strides *to_s() const { return from.defined() ? &to_strides : nullptr; }
};
const double *freqs_arg(const at::Tensor &f) {
    require(f.scalar_type() == at::kDouble && f.dim() == 1, "freqs: float64 [rotary_dim / 2]");
    return static_cast<const double *>(f.data_ptr());
}

// three outputs, the caller's, of the shapes of `like` (r[i].from)
template <int N>
void rows_out(const Out<N> &out, Rows (&r)[3]) {
    for (int i = 0; out.given() && i < 3; ++i) {
        if (!r[i].from.defined()) {
            require(out[i] == Py_None, "out: no values were given");
            continue;
        }
        r[i].to = rows_arg(out[i]);
        require(r[i].to.sizes() == r[i].from.sizes() && r[i].to.scalar_type() == r[i].from.scalar_type(), "out: shapes and dtype of the inputs");
    }
}
// as one fused projection puts them out: [B, L, q heads | k heads | v heads, d]
void fused_rows(Rows (&r)[3], const at::Tensor &q, int B, int L, int Hq, int Hkv, int64_t d) {
    const int64_t Hv = r[2].from.defined() ? Hkv : 0;
    const at::Tensor dx = empty({B, L, Hq + Hkv + Hv, d}, q.scalar_type(), q.device());
    const at::AutoDispatchBelowADInplaceOrView plain;
    const int64_t l = (Hq + Hkv + Hv) * d, first[3] = {0, Hq * d, (Hq + Hkv) * d};
    for (int i = 0; i < (Hv ? 3 : 2); ++i) r[i].to = dx.as_strided({B, i == 0 ? Hq : Hkv, L, d}, {L * l, d, l, 1}, first[i]);
}

// rope(q, k, v, freqs, positions, doc_start, interleaved, out)
template <bool BACKWARD>
PyObject *rope(PyObject *const *a) {
    Rows r[3];
    for (int i = 0; i < 3; ++i)
        if (i < 2 || a[i] != Py_None) r[i].from = rows_arg(a[i]);
    const at::Tensor &q = r[0].from, &k = r[1].from, &v = r[2].from;
    const at::Tensor &f = dev(a[3]);
    const at::Tensor pos = dev_or_none(a[4]), doc = dev_or_none(a[5]);
    const int64_t want[4] = {q.size(0), k.size(1), q.size(2), q.size(3)};
    require(k.sizes() == c10::IntArrayRef(want, 4) && (!v.defined() || v.sizes() == k.sizes()) && k.scalar_type() == q.scalar_type() &&
                (!v.defined() || v.scalar_type() == q.scalar_type()), "q [B, Hq, L, d], k and v [B, Hkv, L, d] of one dtype");
    const double *freqs = freqs_arg(f);
    for (const at::Tensor *t : {&pos, &doc})
        require(!t->defined() || (t->scalar_type() == at::kInt && t->dim() == 2 && t->size(0) == q.size(0) && t->size(1) == q.size(2)),
                "positions, doc_start: int32 [B, L]");
    sepattn_rope_params p;
    p.B = (int)q.size(0), p.Hq = (int)q.size(1), p.Hkv = (int)k.size(1), p.L = (int)q.size(2), p.d = (int)q.size(3);
    p.rotary_dim = (int)(2 * f.numel());
    p.interleaved = as_bool(a[6]);
    p.dtype = dtype_code(q);
    const Out<3> out(a[7]);
    rows_out(out, r);
    one_device(q, k, v, f, pos, doc, r[0].to, r[1].to, r[2].to);
    check(BACKWARD ? "sepattn_rope_backward" : "sepattn_rope", unlocked([&] {
              const c10::DeviceGuard guard(q.device());
              if (!out.given()) {
                  if constexpr (BACKWARD) {
                      fused_rows(r, q, p.B, p.L, p.Hq, p.Hkv, p.d);
                  } else {
                      for (Rows &x : r)
                          if (x.from.defined()) x.to = fresh_like(x.from);
                  }
              }
              for (Rows &x : r) x.finish();
              return (BACKWARD ? lib.sepattn_rope_backward : lib.sepattn_rope)(
                  &p, freqs, (const int32_t *)ptr_or_null(pos), (const int32_t *)ptr_or_null(doc), ptr(q), r[0].from_s(), ptr(k), r[1].from_s(),
                  ptr_or_null(v), r[2].from_s(), ptr(r[0].to), r[0].to_s(), ptr(r[1].to), r[1].to_s(), ptr_or_null(r[2].to), r[2].to_s(),
                  stream_of(q));
          }));
    if (out.given()) return tuple_of(keep(out[0]), keep(out[1]), keep(out[2]));
    return tuple_of(wrap(r[0].to), wrap(r[1].to), v.defined() ? wrap(r[2].to) : keep(Py_None));
}

// How a token's query and key are changed on their way into a cache: arguments positions, [q_weight, k_weight,] freqs[, eps]
struct Turn {
    at::Tensor pos, qw, kw, f;
    const double *freqs = nullptr;
    int rotary_dim = 0, weight_dtype = SEPATTN_FP32;
    float eps = 0.f;
    const int32_t *positions() const { return (const int32_t *)ptr_or_null(pos); }
};
// weights [d] of one dtype, each may be None
void weights_arg(Turn &t, PyObject *q, PyObject *k, int64_t d) {
    t.qw = dev_or_none(q), t.kw = dev_or_none(k);
    for (const at::Tensor *w : {&t.qw, &t.kw}) {
        if (!w->defined()) continue;
        require(w->dim() == 1 && w->size(0) == d, "q_weight, k_weight: [d]");
        t.weight_dtype = dtype_code(*w);
    }
    require(!t.qw.defined() || !t.kw.defined() || t.qw.scalar_type() == t.kw.scalar_type(), "q_weight, k_weight: one dtype");
}

// What the forms of a token's append share: its tensors, those of the cache's bookkeeping, and the turned query.
struct Token {
    at::Tensor q, k, v, sep, flags, sizes, out;
    PyObject *out_arg;
    Token(PyObject *q_, PyObject *k_, PyObject *v_, PyObject *sep_, PyObject *flags_, PyObject *sizes_, PyObject *out_)
        : q(q_ ? dev(q_) : at::Tensor()), k(dev(k_)), v(dev(v_)), sep(dev(sep_)), flags(dev(flags_)), sizes(sizes_arg(sizes_)), out_arg(out_) {
        if (q_ && q.dim() != 3) fail(PyExc_ValueError, "q [S,Hq,d] is expected");
    }
    // `type`: of all rows
    void match(const sepkv_params &p, at::ScalarType type) {
        const int64_t want[3] = {p.S, p.Hkv, p.d};
        require(k.sizes() == c10::IntArrayRef(want, 3) && v.sizes() == k.sizes() && k.scalar_type() == type && v.scalar_type() == type,
                "k_new, v_new: [S, Hkv, d] in the cache's dtype");
        require(!q.defined() || (q.size(2) == p.d && q.scalar_type() == type), "q: [S, Hq, d] in the cache's dtype");
        require(sep.scalar_type() == at::kByte && flags.scalar_type() == at::kByte && sep.numel() == p.S && flags.dim() == 2 &&
                    flags.size(0) == p.S && flags.size(1) == (int64_t)p.c - p.a - p.s, "is_sep_new: uint8 [S], win_is_sep: uint8 [S, c-a-s]");
        require(sizes.size(0) == p.S, "sizes: int32 [S, 6]");
        if (!out_arg || out_arg == Py_None) return;
        out = dev(out_arg);
        require(out.sizes() == q.sizes() && out.scalar_type() == q.scalar_type(), "out: like q");
    }
    void match_turn(const Turn &t, const sepkv_params &p) const {
        require(!t.pos.defined() || (t.pos.scalar_type() == at::kInt && t.pos.dim() == 1 && t.pos.size(0) == p.S), "positions: int32 [S]");
    }
    void allocate() {
        if (!out.defined()) out = fresh_like(q);
    }
    PyObject *result() { return out_arg == Py_None ? wrap(std::move(out)) : keep(out_arg); }
    const uint8_t *is_sep() const { return (const uint8_t *)ptr(sep); }
    uint8_t *win() const { return (uint8_t *)ptr(flags); }
    int32_t *sz() const { return (int32_t *)ptr(sizes); }
};
// the frequencies, and with NORM eps and the weights in front of them
template <bool NORM>
Turn turn_args(PyObject *positions, PyObject *q_weight, PyObject *k_weight, PyObject *freqs, PyObject *eps, int64_t d) {
    Turn t;
    t.pos = NORM ? dev_or_none(positions) : at::Tensor(dev(positions));
    t.f = NORM ? dev_or_none(freqs) : at::Tensor(dev(freqs));
    if (t.f.defined()) {
        t.freqs = freqs_arg(t.f);
        t.rotary_dim = (int)(2 * t.f.numel());
    }
    if (NORM) {
        weights_arg(t, q_weight, k_weight, d);
        t.eps = as_float(eps);
    }
    return t;
}

// append_rope(q, k_new, v_new, is_sep_new, positions, freqs, Kc, Vc, win_is_sep, sizes, a, s, w, interleaved, out)
// append_norm_rope(q, k_new, v_new, is_sep_new, positions, q_weight, k_weight, freqs, eps, Kc, Vc, win_is_sep, sizes, a, s, w, interleaved, out)
template <bool NORM>
PyObject *append_turned(PyObject *const *a) {
    PyObject *const *b = a + (NORM ? 9 : 6);  // the cache and what follows
    Token x(a[0], a[1], a[2], a[3], b[2], b[3], b[8]);
    const at::Tensor &Kc = dev(b[0]), &Vc = dev(b[1]);
    const sepkv_params p = kv_params(Kc, (int)x.q.size(0), (int)x.q.size(1), as_int(b[4]), as_int(b[5]), as_int(b[6]), 1.0f);
    x.match(p, Kc.scalar_type());
    require(Kc.size(0) == p.S && Vc.sizes() == Kc.sizes() && Vc.scalar_type() == Kc.scalar_type(), "Kc, Vc: [S, Hkv, c, d] of one dtype");
    const Turn t = turn_args<NORM>(a[4], NORM ? a[5] : nullptr, NORM ? a[6] : nullptr, a[NORM ? 7 : 5], NORM ? a[8] : nullptr, p.d);
    x.match_turn(t, p);
    const int interleaved = as_bool(b[7]);
    one_device(x.q, x.k, x.v, x.sep, t.pos, t.f, t.qw, t.kw, Kc, Vc, x.flags, x.sizes, x.out);
    check(NORM ? "sepkv_append_norm_rope" : "sepkv_append_rope", unlocked([&] {
              const c10::DeviceGuard guard(x.q.device());
              x.allocate();
              if constexpr (NORM)
                  return lib.sepkv_append_norm_rope(&p, t.rotary_dim, interleaved, t.eps, t.weight_dtype, ptr_or_null(t.qw), ptr_or_null(t.kw), t.freqs,
                                                    t.positions(), ptr(x.q), ptr(x.k), ptr(x.v), x.is_sep(), ptr(x.out), ptr(Kc), ptr(Vc), x.win(),
                                                    x.sz(), stream_of(x.q));
              else
                  return lib.sepkv_append_rope(&p, t.rotary_dim, interleaved, t.freqs, t.positions(), ptr(x.q), ptr(x.k), ptr(x.v), x.is_sep(),
                                               ptr(x.out), ptr(Kc), ptr(Vc), x.win(), x.sz(), stream_of(x.q));
          }));
    return x.result();
}

// ---- norms in front of the rotary positions --------------------------------------------------------
// What forward and backward share: q, k (and v, or the three gradients) with weights, frequencies and positions
struct NormRope {
    Turn t;
    at::Tensor doc;
    sepattn_norm_rope_params p;
    NormRope(const at::Tensor &q, const at::Tensor &k, const at::Tensor &v, PyObject *q_weight, PyObject *k_weight, PyObject *freqs, PyObject *eps,
             PyObject *positions, PyObject *doc_start, PyObject *interleaved) {
        t = turn_args<true>(positions, q_weight, k_weight, freqs, eps, q.size(3));
        doc = dev_or_none(doc_start);
        const int64_t want[4] = {q.size(0), k.size(1), q.size(2), q.size(3)};
        require(k.sizes() == c10::IntArrayRef(want, 4) && (!v.defined() || v.sizes() == k.sizes()) && k.scalar_type() == q.scalar_type() &&
                    (!v.defined() || v.scalar_type() == q.scalar_type()), "q [B, Hq, L, d], k and v [B, Hkv, L, d] of one dtype");
        for (const at::Tensor *x : {&t.pos, &doc})
            require(!x->defined() || (x->scalar_type() == at::kInt && x->dim() == 2 && x->size(0) == q.size(0) && x->size(1) == q.size(2)),
                    "positions, doc_start: int32 [B, L]");
        p.B = (int)q.size(0), p.Hq = (int)q.size(1), p.Hkv = (int)k.size(1), p.L = (int)q.size(2), p.d = (int)q.size(3);
        p.rotary_dim = t.rotary_dim, p.interleaved = as_bool(interleaved), p.dtype = dtype_code(q), p.weight_dtype = t.weight_dtype, p.eps = t.eps;
    }
    const int32_t *doc_start() const { return (const int32_t *)ptr_or_null(doc); }
};
// norm_rope(q, k, v, q_weight, k_weight, freqs, eps, positions, doc_start, interleaved, out)
PyObject *norm_rope(PyObject *const *a) {
    Rows r[3];
    for (int i = 0; i < 3; ++i)
        if (i < 2 || a[i] != Py_None) r[i].from = rows_arg(a[i]);
    const at::Tensor &q = r[0].from, &k = r[1].from, &v = r[2].from;
    const NormRope n(q, k, v, a[3], a[4], a[5], a[6], a[7], a[8], a[9]);
    const Out<3> out(a[10]);
    rows_out(out, r);
    one_device(q, k, v, n.t.f, n.t.qw, n.t.kw, n.t.pos, n.doc, r[0].to, r[1].to, r[2].to);
    check("sepattn_norm_rope", unlocked([&] {
              const c10::DeviceGuard guard(q.device());
              for (Rows &x : r) {
                  if (!out.given() && x.from.defined()) x.to = fresh_like(x.from);
                  x.finish();
              }
              return lib.sepattn_norm_rope(&n.p, ptr_or_null(n.t.qw), ptr_or_null(n.t.kw), n.t.freqs, n.t.positions(), n.doc_start(), ptr(q), r[0].from_s(),
                                           ptr(k), r[1].from_s(), ptr_or_null(v), r[2].from_s(), ptr(r[0].to), r[0].to_s(), ptr(r[1].to), r[1].to_s(),
                                           ptr_or_null(r[2].to), r[2].to_s(), stream_of(q));
          }));
    if (out.given()) return tuple_of(keep(out[0]), keep(out[1]), keep(out[2]));
    return tuple_of(wrap(r[0].to), wrap(r[1].to), v.defined() ? wrap(r[2].to) : keep(Py_None));
}

// norm_rope_backward(q, k, dQ, dK, dV, q_weight, k_weight, freqs, eps, positions, doc_start, interleaved, out, out_weights, ws)
PyObject *norm_rope_backward(PyObject *const *a) {
    const at::Tensor &q = rows_arg(a[0]), &k = rows_arg(a[1]);
    Rows r[3];
    for (int i = 0; i < 3; ++i)
        if (i < 2 || a[2 + i] != Py_None) r[i].from = rows_arg(a[2 + i]);
    const at::Tensor &dQ = r[0].from, &dK = r[1].from, &dV = r[2].from;
    const NormRope n(dQ, dK, dV, a[5], a[6], a[7], a[8], a[9], a[10], a[11]);
    require(q.sizes() == dQ.sizes() && k.sizes() == dK.sizes() && q.scalar_type() == dQ.scalar_type() && k.scalar_type() == dK.scalar_type(),
            "q like dQ, k like dK");
    const Out<3> out(a[12]);
    rows_out(out, r);
    const Out<2> out_w(a[13]);
    at::Tensor w[2];
    for (int i = 0; out_w.given() && i < 2; ++i) {
        w[i] = dev_or_none(out_w[i]);  // None: not wanted
        require(!w[i].defined() || (w[i].scalar_type() == at::kFloat && w[i].dim() == 1 && w[i].size(0) == n.p.d), "out_weights: fp32 [d]");
    }
    Workspace ws(a[14]);
    at::Tensor given_ws;
    if (ws.given) {
        given_ws = dev(a[14]);
        ws.bytes = (size_t)given_ws.nbytes();
    }
    one_device(q, k, dQ, dK, dV, n.t.f, n.t.qw, n.t.kw, n.t.pos, n.doc, r[0].to, r[1].to, r[2].to, w[0], w[1], given_ws);
    const sepattn_strides qs = Rows::strides_of(q), ks = Rows::strides_of(k);
    check("sepattn_norm_rope_backward", unlocked([&] {
              const c10::DeviceGuard guard(q.device());
              if (!out.given()) fused_rows(r, q, n.p.B, n.p.L, n.p.Hq, n.p.Hkv, n.p.d);
              if (!out_w.given())
                  for (at::Tensor &x : w) x = empty({n.p.d}, at::kFloat, q.device());
              if (!ws.given && (w[0].defined() || w[1].defined())) ws.allocate(lib.sepattn_norm_rope_backward_workspace_bytes(&n.p), q.device());
              for (Rows &x : r) x.finish();
              return lib.sepattn_norm_rope_backward(&n.p, ptr_or_null(n.t.qw), ptr_or_null(n.t.kw), n.t.freqs, n.t.positions(), n.doc_start(), ptr(q), &qs,
                                                    ptr(k), &ks, ptr(dQ), r[0].from_s(), ptr(dK), r[1].from_s(), ptr_or_null(dV), r[2].from_s(),
                                                    ptr(r[0].to), r[0].to_s(), ptr(r[1].to), r[1].to_s(), ptr_or_null(r[2].to), r[2].to_s(),
                                                    static_cast<float *>(ptr_or_null(w[0])), static_cast<float *>(ptr_or_null(w[1])), ws.p, ws.bytes,
                                                    stream_of(q));
          }));
    PyObject *dx[3], *dw[2];
    for (int i = 0; i < 3; ++i) dx[i] = out.given() ? keep(out[i]) : r[i].to.defined() ? wrap(r[i].to) : keep(Py_None);
    for (int i = 0; i < 2; ++i) dw[i] = out_w.given() ? keep(out_w[i]) : wrap(w[i]);
    return tuple_of(dx[0], dx[1], dx[2], dw[0], dw[1]);
}

// ---- the cache in 4 bits -----------------------------------------------------------------------------
// Kc, Ks, Vc, Vs: uint8 [S, Hkv, c, d/2] and [S, Hkv, c, d/32]
struct Fp4Args {
    at::Tensor Kc, Ks, Vc, Vs;
    explicit Fp4Args(PyObject *const *a) : Kc(dev(a[0])), Ks(dev(a[1])), Vc(dev(a[2])), Vs(dev(a[3])) {
        for (const at::Tensor *t : {&Kc, &Ks, &Vc, &Vs}) {
            require(t->scalar_type() == at::kByte && t->dim() == 4, "Kc, Ks, Vc, Vs: uint8 [S, Hkv, c, d/2] and [S, Hkv, c, d/32]");
            for (const int64_t n : t->sizes()) require(n <= INT_MAX / 2, "sizes of 32 bits are expected");
        }
        const int64_t want[4] = {Kc.size(0), Kc.size(1), Kc.size(2), Kc.size(3) / 16};
        require(Vc.sizes() == Kc.sizes() && Ks.sizes() == c10::IntArrayRef(want, 4) && Vs.sizes() == Ks.sizes(),
                "Kc, Ks, Vc, Vs: uint8 [S, Hkv, c, d/2] and [S, Hkv, c, d/32]");
    }
    sepkv_params params(int Hq, PyObject *const *blocks, float scale, int dtype) const {
        sepkv_params p;
        p.S = (int)Kc.size(0), p.Hq = Hq, p.Hkv = (int)Kc.size(1), p.d = (int)Kc.size(3) * 2, p.c = (int)Kc.size(2);
        p.a = as_int(blocks[0]), p.s = as_int(blocks[1]), p.w = as_int(blocks[2]);
        p.scale = scale, p.dtype = dtype;
        return p;
    }
};

// append_fp4(k_new, v_new, is_sep_new, Kc, Ks, Vc, Vs, win_is_sep, sizes, Hq, a, s, w)
PyObject *append_fp4(PyObject *const *a) {
    Token x(nullptr, a[0], a[1], a[2], a[7], a[8], nullptr);
    const Fp4Args c(a + 3);
    const sepkv_params p = c.params(as_int(a[9]), a + 10, 1.0f, dtype_code(x.k));
    x.match(p, x.k.scalar_type());
    one_device(x.k, x.v, x.sep, c.Kc, c.Ks, c.Vc, c.Vs, x.flags, x.sizes);
    check("sepkv_append_mx", unlocked([&] {
              const c10::DeviceGuard guard(x.k.device());
              return lib.sepkv_append_mx(&p, ptr(x.k), ptr(x.v), x.is_sep(), ptr(c.Kc), ptr(c.Ks), ptr(c.Vc), ptr(c.Vs), x.win(), x.sz(), stream_of(x.k));
          }));
    return keep(Py_None);
}

// append_rope_fp4, append_norm_rope_fp4: as append_rope, append_norm_rope, with Kc, Ks, Vc, Vs in the place of Kc, Vc
template <bool NORM>
PyObject *append_turned_fp4(PyObject *const *a) {
    PyObject *const *b = a + (NORM ? 9 : 6);
    Token x(a[0], a[1], a[2], a[3], b[4], b[5], b[10]);
    const Fp4Args c(b);
    const sepkv_params p = c.params((int)x.q.size(1), b + 6, 1.0f, dtype_code(x.q));
    require(x.q.size(0) == p.S, "q: [S, Hq, d]");
    x.match(p, x.q.scalar_type());
    const Turn t = turn_args<NORM>(a[4], NORM ? a[5] : nullptr, NORM ? a[6] : nullptr, a[NORM ? 7 : 5], NORM ? a[8] : nullptr, p.d);
    x.match_turn(t, p);
    const int interleaved = as_bool(b[9]);
    one_device(x.q, x.k, x.v, x.sep, t.pos, t.f, t.qw, t.kw, c.Kc, c.Ks, c.Vc, c.Vs, x.flags, x.sizes, x.out);
    check(NORM ? "sepkv_append_norm_rope_mx" : "sepkv_append_rope_mx", unlocked([&] {
              const c10::DeviceGuard guard(x.q.device());
              x.allocate();
              if constexpr (NORM)
                  return lib.sepkv_append_norm_rope_mx(&p, t.rotary_dim, interleaved, t.eps, t.weight_dtype, ptr_or_null(t.qw), ptr_or_null(t.kw), t.freqs,
                                                        t.positions(), ptr(x.q), ptr(x.k), ptr(x.v), x.is_sep(), ptr(x.out), ptr(c.Kc), ptr(c.Ks),
                                                        ptr(c.Vc), ptr(c.Vs), x.win(), x.sz(), stream_of(x.q));
              else
                  return lib.sepkv_append_rope_mx(&p, t.rotary_dim, interleaved, t.freqs, t.positions(), ptr(x.q), ptr(x.k), ptr(x.v), x.is_sep(),
                                                   ptr(x.out), ptr(c.Kc), ptr(c.Ks), ptr(c.Vc), ptr(c.Vs), x.win(), x.sz(), stream_of(x.q));
          }));
    return x.result();
}

void window_args(const at::Tensor &flags, const at::Tensor &sizes, const sepkv_params &p) {
    require(flags.scalar_type() == at::kByte && flags.dim() == 2 && flags.size(0) == p.S && flags.size(1) == (int64_t)p.c - p.a - p.s,
            "win_is_sep: uint8 [S, c-a-s]");
    require(sizes.size(0) == p.S, "sizes: int32 [S, 6]");
}

// evict_window_fp4(Kc, Ks, Vc, Vs, win_is_sep, sizes, Hq, a, s, w)
PyObject *evict_window_fp4(PyObject *const *a) {
    const Fp4Args c(a);
    const at::Tensor &flags = dev(a[4]), &sizes = sizes_arg(a[5]);
    const sepkv_params p = c.params(as_int(a[6]), a + 7, 1.0f, SEPATTN_BF16);
    window_args(flags, sizes, p);
    one_device(c.Kc, c.Ks, c.Vc, c.Vs, flags, sizes);
    check("sepkv_evict_window_mx", unlocked([&] {
              const c10::DeviceGuard guard(c.Kc.device());
              return lib.sepkv_evict_window_mx(&p, ptr(c.Kc), ptr(c.Ks), ptr(c.Vc), ptr(c.Vs), (const uint8_t *)ptr(flags), (int32_t *)ptr(sizes),
                                                stream_of(c.Kc));
          }));
    return keep(Py_None);
}

// fill_from_prefill_fp4(K, V, is_sep, sep_idx, sep_prefix, Hq, a, s, w, c, nw, out)
PyObject *fill_from_prefill_fp4(PyObject *const *a) {
    const at::Tensor &K = dev(a[0]), &V = dev(a[1]), &sep = dev(a[2]), &idx = dev(a[3]), &pre = dev(a[4]);
    if (K.dim() != 4) fail(PyExc_ValueError, "K [S,Hkv,L,d] is expected");
    for (const int64_t n : K.sizes()) require(n < INT_MAX, "sizes of 32 bits are expected");
    const int64_t S = K.size(0), L = K.size(2);
    const int nw = as_int(a[10]);
    sepkv_params p = {(int)S, as_int(a[5]), (int)K.size(1), (int)K.size(3), as_int(a[6]), as_int(a[7]), as_int(a[8]), as_int(a[9]), 1.0f, dtype_code(K)};
    require(V.sizes() == K.sizes() && V.scalar_type() == K.scalar_type(), "V like K");
    require(sep.scalar_type() == at::kByte && sep.dim() == 2 && sep.size(0) == S && sep.size(1) == L, "is_sep: uint8 [S, L]");
    require(idx.scalar_type() == at::kInt && idx.dim() == 2 && idx.size(0) == S && pre.scalar_type() == at::kInt && pre.dim() == 2 && pre.size(0) == S &&
                pre.size(1) == L + 1, "sep_idx: int32 [S, cap], sep_prefix: int32 [S, L+1]");
    require(p.d == 64 || p.d == 128, "d: 64 or 128");
    require(p.a >= 0 && p.s >= 0 && p.c > 0 && (int64_t)p.a + p.s < p.c, "blocks: a + s + w < c");
    const Out<6> out(a[11]);
    at::Tensor x[4], flags, sizes;
    if (out.given()) {
        PyObject *const four[4] = {out[0], out[1], out[2], out[3]};
        const Fp4Args c(four);
        x[0] = c.Kc, x[1] = c.Ks, x[2] = c.Vc, x[3] = c.Vs;
        const int64_t want[4] = {S, p.Hkv, p.c, p.d / 2};
        require(c.Kc.sizes() == c10::IntArrayRef(want, 4), "out: Kc, Ks, Vc, Vs: uint8 [S, Hkv, c, d/2] and [S, Hkv, c, d/32]");
        flags = dev(out[4]), sizes = sizes_arg(out[5]);
        window_args(flags, sizes, p);
    }
    one_device(K, V, sep, idx, pre, x[0], x[1], x[2], x[3], flags, sizes);
    check("sepkv_fill_from_prefill_mx", unlocked([&] {
              const c10::DeviceGuard guard(K.device());
              if (!out.given()) {
                  for (int i = 0; i < 4; ++i) x[i] = empty({p.S, p.Hkv, p.c, p.d / (i % 2 ? 32 : 2)}, at::kByte, K.device());
                  flags = empty({p.S, p.c - p.a - p.s}, at::kByte, K.device());
                  sizes = empty({p.S, SEPKV_SIZES_COLS}, at::kInt, K.device());
              }
              return (out.given() ? lib.sepkv_fill_from_prefill_mx : lib.sepkv_fill_from_prefill_mx_zeroed)(
                  &p, (int)L, nw, ptr(K), ptr(V), (const uint8_t *)ptr(sep), i32(idx), (int)idx.size(1), i32(pre), ptr(x[0]), ptr(x[1]), ptr(x[2]), ptr(x[3]),
                  (uint8_t *)ptr(flags), (int32_t *)ptr(sizes), stream_of(K));
          }));
    if (out.given()) return tuple_of(keep(out[0]), keep(out[1]), keep(out[2]), keep(out[3]), keep(out[4]), keep(out[5]));
    return tuple_of(wrap(x[0]), wrap(x[1]), wrap(x[2]), wrap(x[3]), wrap(flags), wrap(sizes));
}

// expand_fp4(Kc, Ks, Vc, Vs, sizes, a, s, w, fp32, out)
PyObject *expand_fp4(PyObject *const *a) {
    const Fp4Args c(a);
    const at::Tensor &sizes = sizes_arg(a[4]);
    const Out<2> out(a[9]);
    at::Tensor K, V;
    if (out.given()) K = dev(out[0]), V = dev(out[1]);
    const auto type = K.defined() ? K.scalar_type() : as_bool(a[8]) ? at::kFloat : at::kBFloat16;
    const sepkv_params p = c.params((int)c.Kc.size(1), a + 5, 1.0f, K.defined() ? dtype_code(K) : type == at::kFloat ? SEPATTN_FP32 : SEPATTN_BF16);
    require(sizes.size(0) == p.S, "sizes: int32 [S, 6]");
    if (out.given()) {
        const int64_t want[4] = {p.S, p.Hkv, p.c, p.d};
        require(K.sizes() == c10::IntArrayRef(want, 4) && V.sizes() == K.sizes() && V.scalar_type() == type, "out: K, V [S, Hkv, c, d] of one dtype");
    }
    one_device(c.Kc, c.Ks, c.Vc, c.Vs, sizes, K, V);
    check("sepkv_expand_mx", unlocked([&] {
              const c10::DeviceGuard guard(c.Kc.device());
              if (!out.given()) {
                  K = empty({p.S, p.Hkv, p.c, p.d}, type, c.Kc.device());
                  V = empty({p.S, p.Hkv, p.c, p.d}, type, c.Kc.device());
              }
              return lib.sepkv_expand_mx(&p, i32(sizes), ptr(c.Kc), ptr(c.Ks), ptr(c.Vc), ptr(c.Vs), ptr(K), ptr(V), stream_of(c.Kc));
          }));
    if (out.given()) return tuple_of(keep(out[0]), keep(out[1]));
    return tuple_of(wrap(std::move(K)), wrap(std::move(V)));
}

// ---- shared prompts ----------------------------------------------------------------------------------
// group_sequences(prefix_of, n_prefixes, out)
PyObject *group_sequences(PyObject *const *a) {
    const at::Tensor &of = dev(a[0]);
    require(of.scalar_type() == at::kInt && of.dim() == 1 && of.numel() <= INT_MAX, "prefix_of: int32 [S]");
    const int S = (int)of.numel(), G = as_int(a[1]);
    const Out<2> out(a[2]);
    at::Tensor start, seq;
    if (out.given()) {
        start = dev(out[0]);
        seq = dev(out[1]);
        require(start.scalar_type() == at::kInt && start.numel() == (int64_t)G + 1 && seq.scalar_type() == at::kInt && seq.numel() == S,
                "out: int32 [n_prefixes + 1], int32 [S]");
    }
    one_device(of, start, seq);
    check("sepkv_group_sequences", unlocked([&] {
              const c10::DeviceGuard guard(of.device());
              if (!out.given()) {
                  start = empty({G > 0 ? (int64_t)G + 1 : 1}, at::kInt, of.device());
                  seq = empty({S}, at::kInt, of.device());
              }
              return lib.sepkv_group_sequences(i32(of), S, G, (int32_t *)ptr(start), (int32_t *)ptr(seq), stream_of(of));
          }));
    if (out.given()) return tuple_of(keep(out[0]), keep(out[1]));
    return tuple_of(wrap(std::move(start)), wrap(std::move(seq)));
}

void table_arg(const at::Tensor &table, int64_t d) {
    require(table.scalar_type() == at::kFloat && table.dim() == 3 && table.size(1) == 2 && table.size(2) * 2 == d, "rope_table: fp32 [n_pos, 2, d/2]");
}

// rope_cache(Kc, sizes, rope_table, a, s, w, out): out None: in place
PyObject *rope_cache(PyObject *const *a) {
    const at::Tensor &Kc = dev(a[0]), &sizes = sizes_arg(a[1]), &table = dev(a[2]);
    if (Kc.dim() != 4) fail(PyExc_ValueError, "Kc [S,Hkv,c,d] is expected");
    const sepkv_params p = kv_params(Kc, (int)Kc.size(0), (int)Kc.size(1), as_int(a[3]), as_int(a[4]), as_int(a[5]), 1.0f);
    table_arg(table, p.d);
    require(sizes.size(0) == p.S, "sizes: int32 [S, 6]");
    const at::Tensor &o = a[6] == Py_None ? Kc : dev(a[6]);
    require(o.sizes() == Kc.sizes() && o.scalar_type() == Kc.scalar_type(), "out: like Kc");
    one_device(Kc, sizes, table, o);
    check("sepkv_rope_cache", unlocked([&] {
              const c10::DeviceGuard guard(Kc.device());
              return lib.sepkv_rope_cache(&p, i32(sizes), (const float *)ptr(table), (int)table.size(0), ptr(Kc), ptr(o), stream_of(Kc));
          }));
    return keep(a[6] == Py_None ? a[0] : a[6]);
}

// Own and prefix caches of a shared decode: q, Kc, a, s, w, Kp, pa, ps, pw, scale
struct SharedParams {
    sepkv_params p, pp;
    SharedParams(const at::Tensor &q, const at::Tensor &Kc, PyObject *const *own, const at::Tensor &Kp, PyObject *const *prefix, float scale) {
        if (q.dim() != 3) fail(PyExc_ValueError, "q [S,Hq,d] is expected");
        p = kv_params(Kc, (int)q.size(0), (int)q.size(1), as_int(own[0]), as_int(own[1]), as_int(own[2]), scale);
        pp = kv_params(Kp, (int)Kp.size(0), (int)q.size(1), as_int(prefix[0]), as_int(prefix[1]), as_int(prefix[2]), scale);
        require(q.size(2) == p.d && q.scalar_type() == Kc.scalar_type() && Kc.size(0) == p.S, "q [S, Hq, d], Kc [S, Hkv, c, d] of one dtype");
        require(Kp.size(1) == p.Hkv && Kp.size(3) == p.d && Kp.scalar_type() == Kc.scalar_type(), "Kp: [G, Hkv, prefix_c, d] in the cache's dtype");
    }
};

// decode_shared(q, Kc, Vc, sizes, a, s, w, Kp, Vp, prefix_sizes, pa, ps, pw, prefix_of, group_start, group_seq, rope_table, scale, out, ws)
template <bool ROPE>
PyObject *decode_shared(PyObject *const *a) {
    const at::Tensor &q = dev(a[0]), &Kc = dev(a[1]), &Vc = dev(a[2]), &sizes = sizes_arg(a[3]), &Kp = dev(a[7]), &Vp = dev(a[8]),
                     &psizes = sizes_arg(a[9]), &of = dev(a[13]), &start = dev(a[14]), &seq = dev(a[15]);
    const at::Tensor table = ROPE ? dev(a[16]) : at::Tensor();
    const SharedParams x(q, Kc, a + 4, Kp, a + 10, as_float(a[17]));
    const int S = x.p.S, G = x.pp.S;
    require(Vc.sizes() == Kc.sizes() && Vc.scalar_type() == Kc.scalar_type() && Vp.sizes() == Kp.sizes() && Vp.scalar_type() == Kp.scalar_type(),
            "Vc like Kc, Vp like Kp");
    require(sizes.size(0) == S && psizes.size(0) == G, "sizes: int32 [S, 6], prefix_sizes: int32 [G, 6]");
    require(of.scalar_type() == at::kInt && of.numel() == S && start.scalar_type() == at::kInt && start.numel() == (int64_t)G + 1 &&
                seq.scalar_type() == at::kInt && seq.numel() == S, "prefix_of, group_seq: int32 [S], group_start: int32 [G + 1]");
    if (ROPE) table_arg(table, x.p.d);
    const Out<2> out(a[18]);
    at::Tensor o, lse;
    if (out.given()) {
        o = dev(out[0]);
        lse = dev_or_none(out[1]);  // None: no LSE wanted
        require(o.sizes() == q.sizes() && o.scalar_type() == q.scalar_type() &&
                    (!lse.defined() || (lse.scalar_type() == at::kFloat && lse.numel() == (int64_t)S * x.p.Hq)), "out: like q, lse: fp32 [S, Hq]");
    }
    Workspace ws(a[19]);
    at::Tensor given_ws;
    if (ws.given) {
        given_ws = dev(a[19]);
        ws.bytes = (size_t)given_ws.nbytes();
    }
    one_device(q, Kc, Vc, sizes, Kp, Vp, psizes, of, start, seq, table, o, lse, given_ws);
    check(ROPE ? "sepattn_decode_shared_rope" : "sepattn_decode_shared", unlocked([&] {
              const c10::DeviceGuard guard(q.device());
              if (!out.given()) {
                  o = fresh_like(q);
                  lse = empty({S, x.p.Hq}, at::kFloat, q.device());
              }
              if (!ws.given) ws.allocate(lib.sepattn_decode_shared_workspace_bytes(&x.p, &x.pp), q.device());
              float *l = static_cast<float *>(ptr_or_null(lse));
              void *st = stream_of(q);
              if constexpr (ROPE)
                  return lib.sepattn_decode_shared_rope(&x.p, &x.pp, ptr(q), ptr(Kc), ptr(Vc), i32(sizes), ptr(Kp), ptr(Vp), i32(psizes), i32(of),
                                                        i32(start), i32(seq), (const float *)ptr(table), (int)table.size(0), ptr(o), l, ws.p, ws.bytes, st);
              else
                  return lib.sepattn_decode_shared(&x.p, &x.pp, ptr(q), ptr(Kc), ptr(Vc), i32(sizes), ptr(Kp), ptr(Vp), i32(psizes), i32(of),
                                                   i32(start), i32(seq), ptr(o), l, ws.p, ws.bytes, st);
          }));
    if (out.given()) return tuple_of(keep(out[0]), keep(out[1]));
    return tuple_of(wrap(std::move(o)), wrap(std::move(lse)));
}

// decode_shared_workspace_bytes(q, Kc, a, s, w, Kp, pa, ps, pw)
PyObject *decode_shared_workspace_bytes(PyObject *const *a) {
    const at::Tensor &q = tensor(a[0]);
    const SharedParams x(q, tensor(a[1]), a + 2, tensor(a[5]), a + 6, 1.0f);
    const c10::DeviceGuard guard(q.device());
    return PyLong_FromSize_t(lib.sepattn_decode_shared_workspace_bytes(&x.p, &x.pp));
}

// decode_fp4(q, Kc, Ks, Vc, Vs, sizes, rope_table, a, s, w, scale, out, ws)
template <bool ROPE>
PyObject *decode_fp4(PyObject *const *a) {
    const at::Tensor &q = dev(a[0]), &sizes = sizes_arg(a[5]);
    const Fp4Args c(a + 1);
    const at::Tensor table = ROPE ? at::Tensor(dev(a[6])) : at::Tensor();
    if (q.dim() != 3) fail(PyExc_ValueError, "q [S,Hq,d] is expected");
    const sepkv_params p = c.params((int)q.size(1), a + 7, as_float(a[10]), dtype_code(q));
    require(q.size(0) == p.S && q.size(2) == p.d && sizes.size(0) == p.S, "q [S, Hq, d], sizes int32 [S, 6], Kc [S, Hkv, c, d/2]");
    if (ROPE) table_arg(table, p.d);
    const Out<2> out(a[11]);
    at::Tensor o, lse;
    if (out.given()) {
        o = dev(out[0]);
        lse = dev_or_none(out[1]);  // None: no LSE wanted
        require(o.sizes() == q.sizes() && o.scalar_type() == q.scalar_type() &&
                    (!lse.defined() || (lse.scalar_type() == at::kFloat && lse.numel() == (int64_t)p.S * p.Hq)), "out: like q, lse: fp32 [S, Hq]");
    }
    Workspace ws(a[12]);
    at::Tensor given_ws;
    if (ws.given) {
        given_ws = dev(a[12]);
        ws.bytes = (size_t)given_ws.nbytes();
    }
    one_device(q, c.Kc, c.Ks, c.Vc, c.Vs, sizes, table, o, lse, given_ws);
    check(ROPE ? "sepattn_decode_rope_mx" : "sepattn_decode_mx", unlocked([&] {
              const c10::DeviceGuard guard(q.device());
              if (!out.given()) {
                  o = fresh_like(q);
                  lse = empty({p.S, p.Hq}, at::kFloat, q.device());
              }
              if (!ws.given) ws.allocate(lib.sepattn_decode_mx_workspace_bytes(&p), q.device());
              float *l = static_cast<float *>(ptr_or_null(lse));
              if constexpr (ROPE)
                  return lib.sepattn_decode_rope_mx(&p, ptr(q), ptr(c.Kc), ptr(c.Ks), ptr(c.Vc), ptr(c.Vs), i32(sizes), (const float *)ptr(table),
                                                     (int)table.size(0), ptr(o), l, ws.p, ws.bytes, stream_of(q));
              else
                  return lib.sepattn_decode_mx(&p, ptr(q), ptr(c.Kc), ptr(c.Ks), ptr(c.Vc), ptr(c.Vs), i32(sizes), ptr(o), l, ws.p, ws.bytes,
                                                stream_of(q));
          }));
    if (out.given()) return tuple_of(keep(out[0]), keep(out[1]));
    return tuple_of(wrap(std::move(o)), wrap(std::move(lse)));
}

// ---- module ------------------------------------------------------------------------------------------
typedef PyObject *(*Body)(PyObject *const *);
template <Body F, int N>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "%d arguments expected, got %zd", N, n);
        return nullptr;
    }
    try {
        return F(args);
    } catch (const Failed &) {
        return nullptr;
    } catch (...) {  // torch's own errors as the Python classes it gives them (OutOfMemoryError, IndexError, ...)
        torch::translate_exception_to_python(std::current_exception());
        return nullptr;
    }
}

// bind(path, raise_error): open the library and look its entry points up
PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 2) {
        PyErr_SetString(PyExc_TypeError, "bind(path, raise_error)");
        return nullptr;
    }
    const char *path = PyUnicode_AsUTF8(args[0]);
    if (!path) return nullptr;
    void *h = dlopen(path, RTLD_NOW | RTLD_LOCAL);
    if (!h) {
        PyErr_SetString(PyExc_OSError, dlerror());
        return nullptr;
    }
#define X(name)                                                            \
    lib.name = reinterpret_cast<decltype(lib.name)>(dlsym(h, #name));      \
    if (!lib.name) {                                                       \
        PyErr_SetString(PyExc_OSError, #name " is missing in the library"); \
        return nullptr;                                                    \
    }
    LIB_FUNCTIONS(X)
    LIB_FRESH_FUNCTIONS(X)
    LIB_POSITION_FUNCTIONS(X)
    LIB_NORM_FP4_FUNCTIONS(X)
#undef X
    Py_INCREF(args[1]);
    Py_XSETREF(g_raise, args[1]);
    Py_RETURN_NONE;
}

#define METHOD(name, body, count) \
    {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(&entry<body, count>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(&bind)), METH_FASTCALL, nullptr},
    METHOD("mark_separators", mark_separators, 3),
    METHOD("compact_indices", compact_indices, 6),
    METHOD("mark_compact", mark_compact, 7),
    METHOD("doc_bounds", doc_bounds, 5),
    METHOD("forward", forward<kPlain>, 11),
    METHOD("forward_headwise", forward<kHeadwise>, 11),
    METHOD("forward_packed", forward<kPacked>, 13),
    METHOD("backward", backward<kPlain>, 14),
    METHOD("backward_headwise", backward<kHeadwise>, 14),
    METHOD("backward_packed", backward<kPacked>, 16),
    METHOD("decode", decode<kKept>, 11),
    METHOD("decode_rope", decode<kRope>, 11),
    METHOD("decode_noalloc", decode<kNoAlloc>, 11),
    METHOD("append", append, 11),
    METHOD("evict_window", evict_window, 9),
    METHOD("fill_from_prefill", fill_from_prefill, 12),
    METHOD("rope", rope<false>, 8),
    METHOD("rope_backward", rope<true>, 8),
    METHOD("append_rope", append_turned<false>, 15),
    METHOD("append_norm_rope", append_turned<true>, 18),
    METHOD("norm_rope", norm_rope, 11),
    METHOD("norm_rope_backward", norm_rope_backward, 15),
    METHOD("append_fp4", append_fp4, 13),
    METHOD("append_rope_fp4", append_turned_fp4<false>, 17),
    METHOD("append_norm_rope_fp4", append_turned_fp4<true>, 20),
    METHOD("evict_window_fp4", evict_window_fp4, 10),
    METHOD("fill_from_prefill_fp4", fill_from_prefill_fp4, 12),
    METHOD("expand_fp4", expand_fp4, 10),
    METHOD("decode_fp4", decode_fp4<false>, 13),
    METHOD("decode_rope_fp4", decode_fp4<true>, 13),
    METHOD("group_sequences", group_sequences, 3),
    METHOD("rope_cache", rope_cache, 7),
    METHOD("decode_shared", decode_shared<false>, 20),
    METHOD("decode_shared_rope", decode_shared<true>, 20),
    METHOD("decode_shared_workspace_bytes", decode_shared_workspace_bytes, 9),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&module); }
