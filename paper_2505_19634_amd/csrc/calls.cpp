// The host side of the calls that are shorter on the GPU than in Python: argument checks, the descriptor and the library call of
// verify_attention (and its _noalloc form), spec_accept, majority_vote and skinny_gemm, and of the paged cache's and the microscaled calls, as a CPython extension on torch's tensors.  binding.py keeps
// the signatures, makes what a caller leaves out and holds the workspaces; a call that finds its workspace missing or too small
// says how much it needs and is made again.
// Measured (2 branches, fp32, vocabulary 1000): a step's three calls through ctypes are 6.5 + 6.5 + 4.1 us of host time for
// three launches of 2.7 us each, and their kernels take 11 us together; through here 4.1 + 4.0 + 3.4 us, the step 16.7 -> 12.7.
#include <Python.h>
#include <algorithm>
#include <torch/csrc/autograd/python_variable.h>

#include "lotts.h"

namespace {

// entry points of the liblotts build in use, bound by address: the extension itself links against none
using attn_ws_fn = decltype(&verify_attention_workspace_bytes);
using attn_fn = decltype(&verify_attention);
using attn_noalloc_fn = decltype(&verify_attention_noalloc);
using accept_ws_fn = decltype(&spec_accept_workspace_bytes);
using accept_fn = decltype(&spec_accept);
using vote_fn = decltype(&majority_vote);
using gemm_ws_fn = decltype(&skinny_gemm_workspace_bytes);
using gemm_fn = decltype(&skinny_gemm);

struct Calls {
    PyObject_HEAD
    attn_ws_fn attn_ws;
    attn_fn attn;
    accept_ws_fn accept_ws;
    accept_fn accept;
    vote_fn vote;
    gemm_ws_fn gemm_ws;
    gemm_fn gemm;
    attn_noalloc_fn attn_noalloc;
};

struct Error {  // a Python exception to raise
    PyObject* type;
    const char* text;
};

const at::Tensor& tensor(PyObject* o, const char* what) {
    if (!THPVariable_Check(o)) throw Error{PyExc_TypeError, what};
    return THPVariable_Unpack(o);
}
bool is(const at::Tensor& t, at::ScalarType type) { return t.scalar_type() == type && t.is_contiguous(); }

// The workspace of a call: the caller's as it is, or the cached one if it is large enough; false if that is not there.
bool workspace(PyObject* own, PyObject* cached, size_t need, void** ptr, size_t* bytes) {
    PyObject* o = own != Py_None ? own : cached;
    if (o == Py_None) return false;
    const at::Tensor& t = tensor(o, "the workspace must be a tensor");
    *ptr = t.data_ptr();
    *bytes = t.nbytes();
    return own != Py_None || *bytes >= need;
}

// Status of a call, 0 or negative; a positive number asks for that many bytes of workspace.
template <typename F>
PyObject* guarded(F body) {
    try {
        return PyLong_FromSsize_t(body());
    } catch (const Error& e) {
        PyErr_SetString(e.type, e.text);
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}
template <typename F>
Py_ssize_t released(F call) {
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return rc;
}
void* address(PyObject* o) { return PyLong_AsVoidPtr(o); }
void expect(Py_ssize_t n, Py_ssize_t want) {
    if (n != want) throw Error{PyExc_TypeError, "wrong number of arguments"};
}
constexpr Py_ssize_t kNoWorkspaceQuery = -2;  // a size of 0: the geometry cannot be served

// At least as large in every dimension: what a kernel addresses by the other tensor's sizes lies inside this one.
bool covers(const at::Tensor& t, at::IntArrayRef wanted) {
    const at::IntArrayRef sizes = t.sizes();
    if (sizes.size() != wanted.size()) return false;
    for (size_t i = 0; i < sizes.size(); ++i)
        if (sizes[i] < wanted[i]) return false;
    return true;
}
bool expanded(const at::Tensor& t) {
    const at::IntArrayRef sizes = t.sizes(), strides = t.strides();
    for (size_t i = 0; i < sizes.size(); ++i)
        if (strides[i] == 0 && sizes[i] > 1) return true;
    return false;
}
// One of the outputs with a number for each row: dense and long enough.
template <typename T>
T* rows_of(PyObject* o, at::ScalarType type, int64_t rows, const char* what) {
    const at::Tensor& t = tensor(o, what);
    if (!is(t, type)) throw Error{PyExc_TypeError, what};
    if (t.numel() < rows) throw Error{PyExc_ValueError, what};
    return static_cast<T*>(t.data_ptr());
}

struct Attention {  // the descriptor and the pointers of a call
    lotts_attn_desc d = {};
    const void *q, *kpre = nullptr, *vpre = nullptr, *kpriv, *vpriv;
    const int32_t* len;
    void* out;
    float* lse = nullptr;
};
// a: Q, Kpre, Vpre, Kpriv, Vpriv, priv_len, scale, out, lse.  Whatever the kernels address lies inside the tensors: they know pointers and
// strides alone, and a stride of 0 means the dense layout to them.
Attention attention(PyObject* const* a) {
    const at::Tensor &Q = tensor(a[0], "Q must be a tensor"), &Kpriv = tensor(a[3], "Kpriv must be a tensor"),
                     &Vpriv = tensor(a[4], "Vpriv must be a tensor"), &len = tensor(a[5], "priv_len must be a tensor"),
                     &O = tensor(a[7], "out must be a tensor");
    const at::Tensor *Kpre = nullptr, *Vpre = nullptr;
    if (a[1] != Py_None) {
        Kpre = &tensor(a[1], "Kpre must be a tensor");
        if (Kpre->dim() != 3) throw Error{PyExc_ValueError, "Kpre must be [Hkv][P][D]"};
        if (Kpre->size(1) == 0) Kpre = nullptr;
        else Vpre = &tensor(a[2], "Vpre must be a tensor");
    }
    if (Q.dim() != 4 || Kpriv.dim() != 4 || O.dim() != 4) throw Error{PyExc_ValueError, "Q and out must be [B][k+1][Hq][D], Kpriv [B][Hkv][Lmax][D]"};
    if (Vpriv.strides() != Kpriv.strides() || (Kpre && Vpre->strides() != Kpre->strides()))
        throw Error{PyExc_ValueError, "K and V of a segment must share strides"};
    if (len.scalar_type() != at::kInt) throw Error{PyExc_TypeError, "priv_len must be int32"};
    if (Kpriv.sizes()[0] != Q.sizes()[0] || Kpriv.sizes()[3] != Q.sizes()[3]) throw Error{PyExc_ValueError, "Q and Kpriv disagree"};
    Attention c;
    lotts_attn_desc& d = c.d;
    if (Q.scalar_type() == at::kBFloat16) d.dtype = LOTTS_BF16;
    else if (Q.scalar_type() == at::kFloat) d.dtype = LOTTS_F32;
    else throw Error{PyExc_TypeError, "Q/K/V must be bfloat16 or float32"};
    const at::ScalarType type = Q.scalar_type();
    for (const at::Tensor* t : {&Q, &Kpriv, &O, Kpre}) {
        if (!t) continue;
        if (t->strides().back() != 1) throw Error{PyExc_ValueError, "the head dimension must be contiguous"};
        if (expanded(*t)) throw Error{PyExc_ValueError, "expanded tensors are not supported"};
    }
    for (const at::Tensor* t : {&Kpriv, &Vpriv, &O, Kpre, Vpre})
        if (t && t->scalar_type() != type) throw Error{PyExc_TypeError, "Q, K, V and out share one dtype"};
    const at::IntArrayRef q = Q.sizes(), own = Kpriv.sizes();
    if (!covers(O, q)) throw Error{PyExc_ValueError, "out must be [B][k+1][Hq][D]"};
    if (!covers(Vpriv, own)) throw Error{PyExc_ValueError, "Vpriv must be [B][Hkv][Lmax][D]"};
    if (Kpre) {
        const int64_t prefix[] = {own[1], Kpre->sizes()[1], q[3]};
        if (!covers(*Kpre, prefix) || !covers(*Vpre, prefix)) throw Error{PyExc_ValueError, "Kpre and Vpre must be [Hkv][P][D]"};
    }
    if (!len.is_contiguous() || len.numel() < q[0]) throw Error{PyExc_ValueError, "priv_len must be contiguous [B]"};
    d.B = (int32_t)q[0];
    d.k = (int32_t)q[1] - 1;
    d.Hq = (int32_t)q[2];
    d.D = (int32_t)q[3];
    d.Hkv = (int32_t)own[1];
    d.Lmax = (int32_t)own[2];
    d.scale = (float)PyFloat_AsDouble(a[6]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        throw Error{PyExc_TypeError, "scale must be a number"};
    }
    const at::IntArrayRef qs = Q.strides(), os = O.strides(), ks = Kpriv.strides();
    d.q_stride_b = qs[0], d.q_stride_r = qs[1], d.q_stride_h = qs[2];
    d.o_stride_b = os[0], d.o_stride_r = os[1], d.o_stride_h = os[2];
    d.kpriv_stride_b = ks[0], d.kpriv_stride_h = ks[1], d.kpriv_stride_t = ks[2];
    c.q = Q.data_ptr(), c.kpriv = Kpriv.data_ptr(), c.vpriv = Vpriv.data_ptr(), c.out = O.data_ptr();
    c.len = static_cast<const int32_t*>(len.data_ptr());
    if (Kpre) {
        d.P = (int32_t)Kpre->sizes()[1];
        d.kpre_stride_h = Kpre->strides()[0], d.kpre_stride_t = Kpre->strides()[1];
        c.kpre = Kpre->data_ptr(), c.vpre = Vpre->data_ptr();
    }
    if (a[8] != Py_None) c.lse = rows_of<float>(a[8], at::kFloat, q[0] * q[1] * q[2], "lse must be contiguous float32 [B][k+1][Hq]");
    return c;
}

// Q, Kpre, Vpre, Kpriv, Vpriv, priv_len, scale, out, lse, workspace, cached workspace, stream
PyObject* call_attention(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    const Calls* c = reinterpret_cast<Calls*>(self);
    return guarded([&]() -> Py_ssize_t {
        expect(n, 12);
        const Attention t = attention(a);
        const size_t need = c->attn_ws(&t.d);
        if (need == 0) return kNoWorkspaceQuery;
        void* ws;
        size_t bytes;
        if (!workspace(a[9], a[10], need, &ws, &bytes)) return (Py_ssize_t)need;
        void* stream = address(a[11]);
        return released([&] { return c->attn(&t.d, t.q, t.kpre, t.vpre, t.kpriv, t.vpriv, t.len, t.out, t.lse, ws, bytes, stream); });
    });
}

// Q, Kpre, Vpre, Kpriv, Vpriv, priv_len, scale, out, lse, stream
PyObject* call_attention_noalloc(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    const Calls* c = reinterpret_cast<Calls*>(self);
    return guarded([&]() -> Py_ssize_t {
        expect(n, 10);
        const Attention t = attention(a);
        void* stream = address(a[9]);
        return released([&] { return c->attn_noalloc(&t.d, t.q, t.kpre, t.vpre, t.kpriv, t.vpriv, t.len, t.out, t.lse, stream); });
    });
}

// p, q, draft, u, accept_len, next_token, workspace, cached workspace, stream
PyObject* call_accept(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    const Calls* c = reinterpret_cast<Calls*>(self);
    return guarded([&]() -> Py_ssize_t {
        expect(n, 9);
        const at::Tensor &p = tensor(a[0], "p must be a tensor"), &u = tensor(a[3], "u must be a tensor");
        if (p.dim() != 3) throw Error{PyExc_ValueError, "p must be [B][k+1][V]"};
        const int64_t B = p.size(0), R = p.size(1), V = p.size(2), k = R - 1;
        if (!is(p, at::kFloat) || !is(u, at::kFloat)) throw Error{PyExc_TypeError, "p and u must be contiguous float32"};
        if (u.dim() != 2 || u.size(0) != B || u.size(1) != R) throw Error{PyExc_ValueError, "u must be [B][k+1]"};
        const float* q = nullptr;
        const int32_t* draft = nullptr;
        if (k > 0) {
            if (a[1] == Py_None || a[2] == Py_None) throw Error{PyExc_ValueError, "q must be [B][k][V] and draft [B][k]"};
            const at::Tensor &tq = tensor(a[1], "q must be a tensor"), &td = tensor(a[2], "draft must be a tensor");
            if (tq.dim() != 3 || tq.size(0) != B || tq.size(1) != k || tq.size(2) != V || td.dim() != 2 || td.size(0) != B || td.size(1) != k)
                throw Error{PyExc_ValueError, "q must be [B][k][V] and draft [B][k]"};
            if (!is(tq, at::kFloat) || !is(td, at::kInt)) throw Error{PyExc_TypeError, "q must be contiguous float32 and draft contiguous int32"};
            q = static_cast<const float*>(tq.data_ptr());
            draft = static_cast<const int32_t*>(td.data_ptr());
        }
        const size_t need = c->accept_ws((int32_t)B, (int32_t)k, (int32_t)V);
        if (need == 0) return kNoWorkspaceQuery;
        void* ws;
        size_t bytes;
        if (!workspace(a[6], a[7], need, &ws, &bytes)) return (Py_ssize_t)need;
        const float *pp = static_cast<const float*>(p.data_ptr()), *up = static_cast<const float*>(u.data_ptr());
        int32_t* len = rows_of<int32_t>(a[4], at::kInt, B, "accept_len must be contiguous int32 [B]");
        int32_t* next = rows_of<int32_t>(a[5], at::kInt, B, "next_token must be contiguous int32 [B]");
        void* stream = address(a[8]);
        return released([&] { return c->accept((int32_t)B, (int32_t)k, (int32_t)V, pp, q, draft, up, len, next, ws, bytes, stream); });
    });
}

// answers [N][B], winner, winner_count, stream
PyObject* call_vote(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    const Calls* c = reinterpret_cast<Calls*>(self);
    return guarded([&]() -> Py_ssize_t {
        expect(n, 4);
        const at::Tensor& answers = tensor(a[0], "answers must be a tensor");
        if (!is(answers, at::kInt)) throw Error{PyExc_TypeError, "answers must be contiguous int32"};
        if (answers.dim() != 2) throw Error{PyExc_ValueError, "answers must be [N][B]"};
        const int32_t N = (int32_t)answers.size(0), B = (int32_t)answers.size(1);
        const int32_t* src = static_cast<const int32_t*>(answers.data_ptr());
        int32_t* winner = rows_of<int32_t>(a[1], at::kInt, N, "winner must be contiguous int32 [N]");
        int32_t* count = rows_of<int32_t>(a[2], at::kInt, N, "winner_count must be contiguous int32 [N]");
        void* stream = address(a[3]);
        return released([&] { return c->vote(N, B, src, winner, count, stream); });
    });
}

// X, W, out, workspace, cached workspace, stream
PyObject* call_gemm(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    const Calls* c = reinterpret_cast<Calls*>(self);
    return guarded([&]() -> Py_ssize_t {
        expect(n, 6);
        const at::Tensor &X = tensor(a[0], "X must be a tensor"), &W = tensor(a[1], "W must be a tensor"), &Y = tensor(a[2], "out must be a tensor");
        if (X.dim() != 2 || W.dim() != 2 || W.size(1) != X.size(1) || X.stride(1) != 1 || W.stride(1) != 1)
            throw Error{PyExc_ValueError, "X [M][K] and W [N][K] must share K and have contiguous rows"};
        const int64_t shape[] = {X.size(0), W.size(0)};
        if (Y.scalar_type() != at::kBFloat16) throw Error{PyExc_TypeError, "out must be bfloat16"};
        int64_t row = 1;  // elements of a row of out that lie next to each other
        for (int64_t i = Y.dim() - 1; i > 0 && (Y.size(i) == 1 || Y.stride(i) == row); --i) row *= Y.size(i);
        if (Y.dim() < 2 || Y.size(0) < shape[0] || row < shape[1]) throw Error{PyExc_ValueError, "out must be [M][N] with contiguous rows"};
        const int32_t M = (int32_t)X.size(0), N = (int32_t)W.size(0), K = (int32_t)X.size(1);
        const size_t need = c->gemm_ws(M, N, K);
        if (need == 0) return kNoWorkspaceQuery;
        void* ws;
        size_t bytes;
        if (!workspace(a[3], a[4], need, &ws, &bytes)) return (Py_ssize_t)need;
        const void *x = X.data_ptr(), *w = W.data_ptr();
        void* y = Y.data_ptr();
        const int64_t ldx = X.stride(0), ldw = W.stride(0), ldy = Y.stride(0);
        void* stream = address(a[5]);
        return released([&] { return c->gemm(M, N, K, x, ldx, w, ldw, y, ldy, ws, bytes, stream); });
    });
}

// Calls(address of verify_attention_workspace_bytes, verify_attention, spec_accept_workspace_bytes, spec_accept, majority_vote,
// skinny_gemm_workspace_bytes, skinny_gemm, verify_attention_noalloc)
PyObject* calls_new(PyTypeObject* type, PyObject* args, PyObject*) {
    void* f[8];
    if (PyTuple_GET_SIZE(args) != 8) {
        PyErr_SetString(PyExc_TypeError, "eight addresses");
        return nullptr;
    }
    for (int i = 0; i < 8; ++i) {
        f[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(args, i));
        if (!f[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an address is 0");
            return nullptr;
        }
    }
    Calls* c = reinterpret_cast<Calls*>(type->tp_alloc(type, 0));
    if (!c) return nullptr;
    c->attn_ws = reinterpret_cast<attn_ws_fn>(f[0]);
    c->attn = reinterpret_cast<attn_fn>(f[1]);
    c->accept_ws = reinterpret_cast<accept_ws_fn>(f[2]);
    c->accept = reinterpret_cast<accept_fn>(f[3]);
    c->vote = reinterpret_cast<vote_fn>(f[4]);
    c->gemm_ws = reinterpret_cast<gemm_ws_fn>(f[5]);
    c->gemm = reinterpret_cast<gemm_fn>(f[6]);
    c->attn_noalloc = reinterpret_cast<attn_noalloc_fn>(f[7]);
    return reinterpret_cast<PyObject*>(c);
}

// ---- the paged cache ----------------------------------------------------------------------------------------------------
using paged_ws_fn = decltype(&verify_attention_paged_workspace_bytes);
using paged_fn = decltype(&verify_attention_paged);
using append_fn = decltype(&kv_append_paged);
using reserve_fn = decltype(&kv_pages_reserve);
using fork_fn = decltype(&kv_pages_fork);
using free_fn = decltype(&kv_pages_free);
using compact_fn = decltype(&kv_pages_compact);
using copy_fn = decltype(&kv_pages_copy);

struct PagedCalls {
    PyObject_HEAD
    paged_ws_fn attn_ws;
    paged_fn attn;
    append_fn append;
    reserve_fn reserve;
    fork_fn fork;
    free_fn release;
    compact_fn compact;
    copy_fn copy;
};

// The tensors of a call lie on one GPU, the first one's, and it is the current one (`device`, negative: not looked at).
struct OneDevice {
    long device;
    const at::Tensor& operator()(PyObject* o, const char* what) const {
        const at::Tensor& t = tensor(o, what);
        if (device >= 0 && (!t.is_cuda() || t.get_device() != device)) throw Error{PyExc_ValueError, "all tensors lie on the current GPU"};
        return t;
    }
};
long device_of(PyObject* o) {
    const long d = PyLong_AsLong(o);
    if (d == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Error{PyExc_TypeError, "the device must be a number"};
    }
    return d;
}
int32_t page_of(PyObject* o) {
    const long n = PyLong_AsLong(o);
    if (n == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Error{PyExc_TypeError, "page_tokens must be a number"};
    }
    if (n != (int32_t)n) throw Error{PyExc_ValueError, "page_tokens must be a power of two from 16 to 1024"};
    return (int32_t)n;
}
// Whole numbers: dense, at least n of them.
int32_t* numbers(const at::Tensor& t, int64_t n, const char* what) {
    if (!is(t, at::kInt)) throw Error{PyExc_TypeError, what};
    if (t.numel() < n) throw Error{PyExc_ValueError, what};
    return static_cast<int32_t*>(t.data_ptr());
}
struct Table {
    int32_t *entries, B, columns;
    int64_t stride;
};
Table table_of(const at::Tensor& t) {
    if (t.scalar_type() != at::kInt) throw Error{PyExc_TypeError, "page_table must be int32"};
    if (t.dim() != 2 || t.stride(1) != 1 || (t.size(0) > 1 && t.stride(0) < t.size(1))) throw Error{PyExc_ValueError, "page_table must be [B][columns] with rows apart"};
    if (t.size(0) > 0x7fffffff || t.size(1) > 0x7fffffff) throw Error{PyExc_ValueError, "page_table is too large"};
    return {static_cast<int32_t*>(t.data_ptr()), (int32_t)t.size(0), (int32_t)t.size(1), t.size(0) > 1 ? t.stride(0) : std::max<int64_t>(t.stride(0), t.size(1))};
}
int32_t paged_dtype(const at::Tensor& t) {
    if (t.scalar_type() == at::kBFloat16) return LOTTS_BF16;
    if (t.scalar_type() == at::kFloat) return LOTTS_F32;
    throw Error{PyExc_TypeError, "Q, K and V must be bfloat16 or float32"};
}
void rows_apart(const at::Tensor& t) {
    if (t.strides().back() != 1) throw Error{PyExc_ValueError, "the head dimension must be contiguous"};
    if (expanded(t)) throw Error{PyExc_ValueError, "expanded tensors are not supported"};
}
void same_pages(const at::Tensor& K, const at::Tensor& V) {
    if (K.dim() != 4 || V.sizes() != K.sizes() || V.strides() != K.strides())
        throw Error{PyExc_ValueError, "Kpages and Vpages must be [pages][Hkv][page_tokens][D] with shared strides"};
    if (V.scalar_type() != K.scalar_type()) throw Error{PyExc_TypeError, "Kpages and Vpages share one dtype"};
    rows_apart(K);
}
// Rows of tokens: [T][H][D], or [B][n][H][D] whose tokens lie evenly apart where every branch has as many.
struct Tokens {
    int64_t T, H, D, stride_t, stride_h;
};
Tokens tokens_of(const at::Tensor& t, int64_t B, bool uniform) {
    if (t.dim() == 4 && uniform) {
        if (t.size(0) != B || (B > 1 && t.size(1) > 1 && t.stride(0) != t.size(1) * t.stride(1))) throw Error{PyExc_ValueError, "[B][n][H][D]: the tokens must lie evenly apart"};
        rows_apart(t);
        return {B * t.size(1), t.size(2), t.size(3), t.size(1) > 1 ? t.stride(1) : t.stride(0), t.stride(2)};
    }
    if (t.dim() != 3) throw Error{PyExc_ValueError, uniform ? "rows of tokens must be [T][H][D] or [B][n][H][D]" : "rows of tokens must be [T][H][D]"};
    rows_apart(t);
    return {t.size(0), t.size(1), t.size(2), t.stride(0), t.stride(1)};
}
int64_t pitch(int64_t n, int64_t stride, int64_t dense) { return n > 1 ? stride : std::max(stride, dense); }

// What verify_attention_paged and verify_attention_paged_mxfp8 share: the rows of Q and out, lengths, first rows, lse, and the numbers of the call.
struct Rows {
    Tokens q, o;
    const int32_t *lens, *start;
    int32_t most, dtype;
    float scale;
    float* lse;
};
Rows rows_of_call(const OneDevice& on, const at::Tensor& Q, const at::Tensor& O, const at::Tensor& K, const Table& tab, const at::Tensor& len, PyObject* q_start, bool uniform,
                  PyObject* max_new, PyObject* softmax_scale, PyObject* lse) {
    Rows r;
    r.q = tokens_of(Q, tab.B, uniform), r.o = tokens_of(O, tab.B, uniform);
    if (O.sizes() != Q.sizes()) throw Error{PyExc_ValueError, "out must have Q's shape"};
    if (O.scalar_type() != Q.scalar_type()) throw Error{PyExc_TypeError, "Q and out share one dtype"};
    if (K.size(3) != r.q.D) throw Error{PyExc_ValueError, "Q and Kpages disagree"};
    if (r.q.T > 0x7fffffff) throw Error{PyExc_ValueError, "too many tokens"};
    r.lens = numbers(len, tab.B, "kv_len must be contiguous int32 [B]");
    r.start = uniform ? nullptr : numbers(on(q_start, "q_start must be a tensor"), (int64_t)tab.B + 1, "q_start must be contiguous int32 [B+1]");
    long most = max_new == Py_None ? (uniform ? std::max<long>(1, r.q.T / std::max(1, tab.B)) : (long)r.q.T) : PyLong_AsLong(max_new);
    const double scale = PyFloat_AsDouble(softmax_scale);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        throw Error{PyExc_TypeError, "max_new and scale must be numbers"};
    }
    if (scale != 0.0 && (float)scale == 0.0f) throw Error{PyExc_ValueError, "the scale is nothing in float32"};  // (where 0 selects 1 / sqrt(D))
    if (most < 0 || most > 0x7fffffff) most = 0;
    if (uniform && most * tab.B != r.q.T) throw Error{PyExc_ValueError, "without q_start every branch has T / B new tokens"};
    r.most = (int32_t)most, r.scale = (float)scale, r.dtype = paged_dtype(Q);
    r.lse = nullptr;
    if (lse != Py_None) {
        on(lse, "lse must be a tensor");
        r.lse = rows_of<float>(lse, at::kFloat, r.q.T * r.q.H, "lse must be contiguous float32 [T][Hq]");
    }
    return r;
}
lotts_paged_desc paged_geometry(const Rows& r, const at::Tensor& K, const Table& tab) {
    return {tab.B, (int32_t)r.q.T, r.most, (int32_t)r.q.H, (int32_t)K.size(1), (int32_t)r.q.D, (int32_t)K.size(2), (int32_t)K.size(0), tab.columns,
            r.dtype, r.scale, pitch(r.q.T, r.q.stride_t, r.q.H * r.q.D), pitch(r.q.H, r.q.stride_h, r.q.D), K.stride(0), K.stride(1),
            pitch(K.size(2), K.stride(2), r.q.D), tab.stride, pitch(r.o.T, r.o.stride_t, r.q.H * r.q.D), pitch(r.o.H, r.o.stride_h, r.q.D)};
}

// Q, Kpages, Vpages, page_table, kv_len, q_start, max_new, scale, out, lse, workspace, cached workspace, device, stream
PyObject* call_paged(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    const PagedCalls* c = reinterpret_cast<PagedCalls*>(self);
    return guarded([&]() -> Py_ssize_t {
        expect(n, 14);
        const OneDevice on{device_of(a[12])};
        const at::Tensor &Q = on(a[0], "Q must be a tensor"), &K = on(a[1], "Kpages must be a tensor"), &V = on(a[2], "Vpages must be a tensor"),
                         &table = on(a[3], "page_table must be a tensor"), &len = on(a[4], "kv_len must be a tensor"), &O = on(a[8], "out must be a tensor");
        const bool uniform = a[5] == Py_None;
        const Table tab = table_of(table);
        same_pages(K, V);
        if (K.scalar_type() != Q.scalar_type()) throw Error{PyExc_TypeError, "Q, K, V and out share one dtype"};
        const Rows r = rows_of_call(on, Q, O, K, tab, len, a[5], uniform, a[6], a[7], a[9]);
        const lotts_paged_desc d = paged_geometry(r, K, tab);
        const size_t need = c->attn_ws(&d);
        if (need == 0) return kNoWorkspaceQuery;
        void* ws;
        size_t bytes;
        if (a[10] != Py_None) on(a[10], "the workspace must be a tensor");
        if (!workspace(a[10], a[11], need, &ws, &bytes)) return (Py_ssize_t)need;
        const void *qp = Q.data_ptr(), *kp = K.data_ptr(), *vp = V.data_ptr();
        void *op = O.data_ptr(), *stream = address(a[13]);
        return released([&] { return c->attn(&d, qp, kp, vp, tab.entries, r.lens, r.start, op, r.lse, ws, bytes, stream); });
    });
}

// Knew, Vnew, Kpages, Vpages, page_table, kv_len, q_start, device, stream
PyObject* call_append(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    const PagedCalls* c = reinterpret_cast<PagedCalls*>(self);
    return guarded([&]() -> Py_ssize_t {
        expect(n, 9);
        const OneDevice on{device_of(a[7])};
        const at::Tensor &Kn = on(a[0], "Knew must be a tensor"), &Vn = on(a[1], "Vnew must be a tensor"), &K = on(a[2], "Kpages must be a tensor"),
                         &V = on(a[3], "Vpages must be a tensor"), &table = on(a[4], "page_table must be a tensor"), &len = on(a[5], "kv_len must be a tensor");
        const bool uniform = a[6] == Py_None;
        const Table tab = table_of(table);
        same_pages(K, V);
        if (Vn.sizes() != Kn.sizes() || Vn.strides() != Kn.strides()) throw Error{PyExc_ValueError, "Knew and Vnew must share shape and strides"};
        const Tokens k = tokens_of(Kn, tab.B, uniform);
        if (Vn.scalar_type() != Kn.scalar_type() || K.scalar_type() != Kn.scalar_type()) throw Error{PyExc_TypeError, "all four buffers share one dtype"};
        if (K.size(1) != k.H || K.size(3) != k.D) throw Error{PyExc_ValueError, "Knew and Kpages disagree"};
        if (k.T > 0x7fffffff) throw Error{PyExc_ValueError, "too many tokens"};
        const int32_t* lens = numbers(len, tab.B, "kv_len must be contiguous int32 [B]");
        const int32_t* start = uniform ? nullptr : numbers(on(a[6], "q_start must be a tensor"), (int64_t)tab.B + 1, "q_start must be contiguous int32 [B+1]");
        const void *kn = Kn.data_ptr(), *vn = Vn.data_ptr();
        void *kp = K.data_ptr(), *vp = V.data_ptr(), *stream = address(a[8]);
        const lotts_dtype dt = (lotts_dtype)paged_dtype(Kn);
        return released([&] {
            return c->append(tab.B, (int32_t)k.T, (int32_t)k.H, (int32_t)k.D, (int32_t)K.size(2), (int32_t)K.size(0), tab.columns, dt, kn, vn, k.stride_t,
                             pitch(k.H, k.stride_h, k.D), kp, vp, K.stride(0), K.stride(1), pitch(K.size(2), K.stride(2), k.D), tab.entries, tab.stride, lens, start, stream);
        });
    });
}

struct Upkeep {
    Table tab;
    int32_t *refs, pages;
};
Upkeep upkeep_of(const OneDevice& on, PyObject* table, PyObject* refs) {
    Upkeep u;
    u.tab = table_of(on(table, "page_table must be a tensor"));
    const at::Tensor& r = on(refs, "refs must be a tensor");
    u.refs = numbers(r, 1, "refs must be contiguous int32 [pages]");
    if (r.numel() > 0x7fffffff) throw Error{PyExc_ValueError, "too many pages"};
    u.pages = (int32_t)r.numel();
    return u;
}

// page_table, refs, kv_len, new_tokens, page_tokens, copies, missing, workspace, cached workspace, device, stream
PyObject* call_reserve(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    const PagedCalls* c = reinterpret_cast<PagedCalls*>(self);
    return guarded([&]() -> Py_ssize_t {
        expect(n, 11);
        const OneDevice on{device_of(a[9])};
        const Upkeep u = upkeep_of(on, a[0], a[1]);
        int32_t* len = numbers(on(a[2], "kv_len must be a tensor"), u.tab.B, "kv_len must be contiguous int32 [B]");
        const int32_t* more = numbers(on(a[3], "new_tokens must be a tensor"), u.tab.B, "new_tokens must be contiguous int32 [B]");
        const int32_t page = page_of(a[4]);
        int32_t* copies = numbers(on(a[5], "copies must be a tensor"), 2 * (int64_t)u.tab.B, "copies must be contiguous int32 [B][2]");
        int32_t* missing = numbers(on(a[6], "missing must be a tensor"), 1, "missing must be contiguous int32 [1]");
        const size_t need = 4 * (size_t)u.pages;
        void* ws;
        size_t bytes;
        if (a[7] != Py_None) on(a[7], "the workspace must be a tensor");
        if (!workspace(a[7], a[8], need, &ws, &bytes)) return (Py_ssize_t)need;
        void* stream = address(a[10]);
        return released([&] { return c->reserve(u.tab.B, u.tab.columns, u.pages, page, u.tab.entries, u.tab.stride, u.refs, len, more, copies, missing, ws, bytes, stream); });
    });
}

// page_table, refs, kv_len, parent, device, stream
PyObject* call_fork(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    const PagedCalls* c = reinterpret_cast<PagedCalls*>(self);
    return guarded([&]() -> Py_ssize_t {
        expect(n, 6);
        const OneDevice on{device_of(a[4])};
        const Upkeep u = upkeep_of(on, a[0], a[1]);
        int32_t* len = numbers(on(a[2], "kv_len must be a tensor"), u.tab.B, "kv_len must be contiguous int32 [B]");
        const int32_t* parent = numbers(on(a[3], "parent must be a tensor"), u.tab.B, "parent must be contiguous int32 [B]");
        void* stream = address(a[5]);
        return released([&] { return c->fork(u.tab.B, u.tab.columns, u.pages, u.tab.entries, u.tab.stride, u.refs, len, parent, stream); });
    });
}

// page_table, refs, kv_len, page_tokens, keep, device, stream
PyObject* call_free(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    const PagedCalls* c = reinterpret_cast<PagedCalls*>(self);
    return guarded([&]() -> Py_ssize_t {
        expect(n, 7);
        const OneDevice on{device_of(a[5])};
        const Upkeep u = upkeep_of(on, a[0], a[1]);
        int32_t* len = numbers(on(a[2], "kv_len must be a tensor"), u.tab.B, "kv_len must be contiguous int32 [B]");
        const int32_t page = page_of(a[3]);
        const int32_t* keep = a[4] == Py_None ? nullptr : numbers(on(a[4], "keep must be a tensor"), u.tab.B, "keep must be contiguous int32 [B]");
        void* stream = address(a[6]);
        return released([&] { return c->release(u.tab.B, u.tab.columns, u.pages, page, u.tab.entries, u.tab.stride, u.refs, len, keep, stream); });
    });
}

// page_table, refs, moves, counts, workspace, cached workspace, device, stream
PyObject* call_compact(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    const PagedCalls* c = reinterpret_cast<PagedCalls*>(self);
    return guarded([&]() -> Py_ssize_t {
        expect(n, 8);
        const OneDevice on{device_of(a[6])};
        const Upkeep u = upkeep_of(on, a[0], a[1]);
        int32_t* moves = numbers(on(a[2], "moves must be a tensor"), 2 * std::max<int64_t>(1, u.pages / 2), "moves must be contiguous int32 [max(1, pages / 2)][2]");
        int32_t* counts = numbers(on(a[3], "counts must be a tensor"), 2, "counts must be contiguous int32 [2]");
        const size_t need = 4 * (size_t)u.pages;
        void* ws;
        size_t bytes;
        if (a[4] != Py_None) on(a[4], "the workspace must be a tensor");
        if (!workspace(a[4], a[5], need, &ws, &bytes)) return (Py_ssize_t)need;
        void* stream = address(a[7]);
        return released([&] { return c->compact(u.tab.B, u.tab.columns, u.pages, u.tab.entries, u.tab.stride, u.refs, moves, counts, ws, bytes, stream); });
    });
}

// pool, pairs, count, device, stream
PyObject* call_copy(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    const PagedCalls* c = reinterpret_cast<PagedCalls*>(self);
    return guarded([&]() -> Py_ssize_t {
        expect(n, 5);
        const OneDevice on{device_of(a[3])};
        const at::Tensor &pool = on(a[0], "pool must be a tensor"), &pairs = on(a[1], "pairs must be a tensor");
        int64_t page = 1;  // elements of a page, dense
        bool dense = pool.dim() >= 3 && pool.numel() > 0;
        for (int64_t i = pool.dim() - 1; dense && i >= 2; --i) {
            dense = pool.size(i) == 1 || pool.stride(i) == page;
            page *= pool.size(i);
        }
        if (!dense) throw Error{PyExc_ValueError, "pool must be [planes][pages][...] with dense pages"};
        if (expanded(pool)) throw Error{PyExc_ValueError, "expanded tensors are not supported"};
        if (pairs.dim() != 2 || pairs.size(1) != 2 || pairs.size(0) > 0x7fffffff || pool.size(0) > 0x7fffffff || pool.size(1) > 0x7fffffff)
            throw Error{PyExc_ValueError, "pairs must be [n][2]"};
        const int32_t* from_to = numbers(pairs, 2, "pairs must be contiguous int32 [n][2]");
        const int32_t* count = a[2] == Py_None ? nullptr : numbers(on(a[2], "count must be a tensor"), 1, "count must be contiguous int32");
        const int64_t size = (int64_t)pool.element_size();
        void *base = pool.data_ptr(), *stream = address(a[4]);
        return released([&] {
            return c->copy(base, (int32_t)pool.size(0), (int32_t)pool.size(1), pool.stride(0) * size, (pool.size(1) > 1 ? pool.stride(1) : page) * size, page * size, from_to,
                           (int32_t)pairs.size(0), count, stream);
        });
    });
}

// PagedCalls(address of verify_attention_paged_workspace_bytes, verify_attention_paged, kv_append_paged, kv_pages_reserve, kv_pages_fork,
// kv_pages_free, kv_pages_compact, kv_pages_copy)
PyObject* paged_new(PyTypeObject* type, PyObject* args, PyObject*) {
    void* f[8];
    if (PyTuple_GET_SIZE(args) != 8) {
        PyErr_SetString(PyExc_TypeError, "eight addresses");
        return nullptr;
    }
    for (int i = 0; i < 8; ++i) {
        f[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(args, i));
        if (!f[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an address is 0");
            return nullptr;
        }
    }
    PagedCalls* c = reinterpret_cast<PagedCalls*>(type->tp_alloc(type, 0));
    if (!c) return nullptr;
    c->attn_ws = reinterpret_cast<paged_ws_fn>(f[0]);
    c->attn = reinterpret_cast<paged_fn>(f[1]);
    c->append = reinterpret_cast<append_fn>(f[2]);
    c->reserve = reinterpret_cast<reserve_fn>(f[3]);
    c->fork = reinterpret_cast<fork_fn>(f[4]);
    c->release = reinterpret_cast<free_fn>(f[5]);
    c->compact = reinterpret_cast<compact_fn>(f[6]);
    c->copy = reinterpret_cast<copy_fn>(f[7]);
    return reinterpret_cast<PyObject*>(c);
}

PyMethodDef paged_methods[] = {
    {"verify_attention_paged", (PyCFunction)(void (*)(void))call_paged, METH_FASTCALL, nullptr},
    {"kv_append_paged", (PyCFunction)(void (*)(void))call_append, METH_FASTCALL, nullptr},
    {"kv_pages_reserve", (PyCFunction)(void (*)(void))call_reserve, METH_FASTCALL, nullptr},
    {"kv_pages_fork", (PyCFunction)(void (*)(void))call_fork, METH_FASTCALL, nullptr},
    {"kv_pages_free", (PyCFunction)(void (*)(void))call_free, METH_FASTCALL, nullptr},
    {"kv_pages_compact", (PyCFunction)(void (*)(void))call_compact, METH_FASTCALL, nullptr},
    {"kv_pages_copy", (PyCFunction)(void (*)(void))call_copy, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyTypeObject paged_type = {PyVarObject_HEAD_INIT(nullptr, 0)};

// ---- microscaled numbers -------------------------------------------------------------------------------------------------
using quantize_fn = decltype(&mxfp4_quantize);
using dequantize_fn = decltype(&mxfp4_dequantize);
using gemm4_ws_fn = decltype(&skinny_gemm_mxfp4_workspace_bytes);
using gemm4_fn = decltype(&skinny_gemm_mxfp4);
using append8_fn = decltype(&kv_append_paged_mxfp8);
using paged8_ws_fn = decltype(&verify_attention_paged_mxfp8_workspace_bytes);
using paged8_fn = decltype(&verify_attention_paged_mxfp8);

struct MxCalls {
    PyObject_HEAD
    quantize_fn quantize;
    dequantize_fn dequantize;
    gemm4_ws_fn gemm_ws;
    gemm4_fn gemm;
    append8_fn append;
    paged8_ws_fn attn_ws;
    paged8_fn attn;
};

constexpr int64_t kBlock = 32;  // values that share a scale

void scale_type(const at::Tensor& t) {
    if (t.scalar_type() != at::kByte && t.scalar_type() != at::kFloat8_e8m0fnu) throw Error{PyExc_TypeError, "scales must be float8_e8m0fnu or uint8"};
}
// Rows that lie apart, the elements of a row next to each other.
void dense_rows(const at::Tensor& t, const char* what) {
    if (t.dim() != 2 || (t.size(1) > 1 && t.stride(1) != 1)) throw Error{PyExc_ValueError, what};
    if (expanded(t)) throw Error{PyExc_ValueError, "expanded tensors are not supported"};
}
struct Matrix4 {  // codes and scales of [N][K]
    int64_t N, K, ld_codes, ld_scales;
    void *codes, *scales;
};
Matrix4 matrix4(const OneDevice& on, PyObject* c, PyObject* s) {
    const at::Tensor &codes = on(c, "codes must be a tensor"), &scales = on(s, "scales must be a tensor");
    dense_rows(codes, "codes must be [N][K / 2] with contiguous rows");
    dense_rows(scales, "scales must be [N][K / 32] with contiguous rows");
    if (codes.scalar_type() != at::kByte) throw Error{PyExc_TypeError, "codes must be uint8"};
    scale_type(scales);
    const int64_t N = codes.size(0), K = 2 * codes.size(1);
    if (scales.size(0) != N || scales.size(1) * kBlock != K) throw Error{PyExc_ValueError, "codes [N][K / 2] and scales [N][K / 32] disagree"};
    if (N > 0x7fffffff || K > 0x7fffffff) throw Error{PyExc_ValueError, "the matrix is too large"};
    return {N, K, pitch(N, codes.stride(0), K / 2), pitch(N, scales.stride(0), K / kBlock), codes.data_ptr(), scales.data_ptr()};
}

// values, codes, scales, device, stream: mxfp4_quantize reads the first, mxfp4_dequantize writes it
template <typename F>
PyObject* convert4(PyObject* const* a, Py_ssize_t n, F call) {
    return guarded([&]() -> Py_ssize_t {
        expect(n, 5);
        const OneDevice on{device_of(a[3])};
        const at::Tensor& W = on(a[0], "the matrix must be a tensor");
        dense_rows(W, "the matrix must be [N][K] with contiguous rows");
        if (W.scalar_type() != at::kBFloat16 && W.scalar_type() != at::kFloat) throw Error{PyExc_TypeError, "the matrix must be bfloat16 or float32"};
        const Matrix4 m = matrix4(on, a[1], a[2]);
        if (W.size(0) != m.N || W.size(1) != m.K) throw Error{PyExc_ValueError, "the matrix [N][K] and codes [N][K / 2] disagree"};
        void *values = W.data_ptr(), *stream = address(a[4]);
        const int64_t ld = pitch(m.N, W.stride(0), m.K);
        const lotts_dtype type = W.scalar_type() == at::kBFloat16 ? LOTTS_BF16 : LOTTS_F32;
        return released([&] { return call(m, type, values, ld, stream); });
    });
}
PyObject* call_quantize(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    const MxCalls* c = reinterpret_cast<MxCalls*>(self);
    return convert4(a, n, [c](const Matrix4& m, lotts_dtype type, void* values, int64_t ld, void* stream) {
        return c->quantize((int32_t)m.N, (int32_t)m.K, type, values, ld, m.codes, m.ld_codes, m.scales, m.ld_scales, stream);
    });
}
PyObject* call_dequantize(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    const MxCalls* c = reinterpret_cast<MxCalls*>(self);
    return convert4(a, n, [c](const Matrix4& m, lotts_dtype type, void* values, int64_t ld, void* stream) {
        return c->dequantize((int32_t)m.N, (int32_t)m.K, type, m.codes, m.ld_codes, m.scales, m.ld_scales, values, ld, stream);
    });
}

// X, codes, scales, out, workspace, cached workspace, device, stream
PyObject* call_gemm4(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    const MxCalls* c = reinterpret_cast<MxCalls*>(self);
    return guarded([&]() -> Py_ssize_t {
        expect(n, 8);
        const OneDevice on{device_of(a[6])};
        const at::Tensor &X = on(a[0], "X must be a tensor"), &Y = on(a[3], "out must be a tensor");
        dense_rows(X, "X must be [M][K] with contiguous rows");
        dense_rows(Y, "out must be [M][N] with contiguous rows");
        if (X.scalar_type() != at::kBFloat16 || Y.scalar_type() != at::kBFloat16) throw Error{PyExc_TypeError, "X and out must be bfloat16"};
        const Matrix4 w = matrix4(on, a[1], a[2]);
        const int64_t M = X.size(0);
        if (X.size(1) != w.K) throw Error{PyExc_ValueError, "X [M][K] and codes [N][K / 2] disagree"};
        if (Y.size(0) != M || Y.size(1) != w.N) throw Error{PyExc_ValueError, "out must be [M][N]"};
        if (M > 0x7fffffff) throw Error{PyExc_ValueError, "too many tokens"};
        const size_t need = c->gemm_ws((int32_t)M, (int32_t)w.N, (int32_t)w.K);
        if (need == 0) return kNoWorkspaceQuery;
        void* ws;
        size_t bytes;
        if (a[4] != Py_None) on(a[4], "the workspace must be a tensor");
        if (!workspace(a[4], a[5], need, &ws, &bytes)) return (Py_ssize_t)need;
        const void* x = X.data_ptr();
        void *y = Y.data_ptr(), *stream = address(a[7]);
        const int64_t ldx = pitch(M, X.stride(0), w.K), ldy = pitch(M, Y.stride(0), w.N);
        return released([&] { return c->gemm((int32_t)M, (int32_t)w.N, (int32_t)w.K, x, ldx, w.codes, w.ld_codes, w.scales, w.ld_scales, y, ldy, ws, bytes, stream); });
    });
}

struct Scales {
    void *K, *V;
    int64_t p, h, t;
};
Scales scales_of(const at::Tensor& K, const at::Tensor& V, const at::Tensor& Ks, const at::Tensor& Vs) {
    same_pages(K, V);
    if (K.scalar_type() != at::kByte && K.scalar_type() != at::kFloat8_e4m3fn) throw Error{PyExc_TypeError, "Kpages and Vpages must be float8_e4m3fn or uint8"};
    if (Ks.dim() != 4 || Vs.sizes() != Ks.sizes() || Vs.strides() != Ks.strides() || Ks.size(0) != K.size(0) || Ks.size(1) != K.size(1) || Ks.size(2) != K.size(2) ||
        Ks.size(3) * kBlock != K.size(3))
        throw Error{PyExc_ValueError, "Kscales and Vscales must be [pages][Hkv][page_tokens][D / 32] with shared strides"};
    scale_type(Ks);
    if (Vs.scalar_type() != Ks.scalar_type()) throw Error{PyExc_TypeError, "Kscales and Vscales share one dtype"};
    if (Ks.size(3) > 1 && Ks.stride(3) != 1) throw Error{PyExc_ValueError, "the scales of a row must be contiguous"};
    if (expanded(Ks)) throw Error{PyExc_ValueError, "expanded tensors are not supported"};
    return {Ks.data_ptr(), Vs.data_ptr(), Ks.stride(0), Ks.stride(1), pitch(Ks.size(2), Ks.stride(2), Ks.size(3))};
}

// Q, Kpages, Vpages, Kscales, Vscales, page_table, kv_len, q_start, max_new, scale, out, lse, workspace, cached workspace, device, stream
PyObject* call_paged8(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    const MxCalls* c = reinterpret_cast<MxCalls*>(self);
    return guarded([&]() -> Py_ssize_t {
        expect(n, 16);
        const OneDevice on{device_of(a[14])};
        const at::Tensor &Q = on(a[0], "Q must be a tensor"), &K = on(a[1], "Kpages must be a tensor"), &V = on(a[2], "Vpages must be a tensor"),
                         &Ks = on(a[3], "Kscales must be a tensor"), &Vs = on(a[4], "Vscales must be a tensor"), &table = on(a[5], "page_table must be a tensor"),
                         &len = on(a[6], "kv_len must be a tensor"), &O = on(a[10], "out must be a tensor");
        const bool uniform = a[7] == Py_None;
        const Table tab = table_of(table);
        const Scales sc = scales_of(K, V, Ks, Vs);
        const Rows r = rows_of_call(on, Q, O, K, tab, len, a[7], uniform, a[8], a[9], a[11]);
        lotts_paged_mx_desc d = {paged_geometry(r, K, tab), sc.p, sc.h, sc.t};
        const size_t need = c->attn_ws(&d);
        if (need == 0) return kNoWorkspaceQuery;
        void* ws;
        size_t bytes;
        if (a[12] != Py_None) on(a[12], "the workspace must be a tensor");
        if (!workspace(a[12], a[13], need, &ws, &bytes)) return (Py_ssize_t)need;
        const void *qp = Q.data_ptr(), *kp = K.data_ptr(), *vp = V.data_ptr();
        void *op = O.data_ptr(), *stream = address(a[15]);
        return released([&] { return c->attn(&d, qp, kp, vp, sc.K, sc.V, tab.entries, r.lens, r.start, op, r.lse, ws, bytes, stream); });
    });
}

// Knew, Vnew, Kpages, Vpages, Kscales, Vscales, page_table, kv_len, q_start, device, stream
PyObject* call_append8(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    const MxCalls* c = reinterpret_cast<MxCalls*>(self);
    return guarded([&]() -> Py_ssize_t {
        expect(n, 11);
        const OneDevice on{device_of(a[9])};
        const at::Tensor &Kn = on(a[0], "Knew must be a tensor"), &Vn = on(a[1], "Vnew must be a tensor"), &K = on(a[2], "Kpages must be a tensor"),
                         &V = on(a[3], "Vpages must be a tensor"), &Ks = on(a[4], "Kscales must be a tensor"), &Vs = on(a[5], "Vscales must be a tensor"),
                         &table = on(a[6], "page_table must be a tensor"), &len = on(a[7], "kv_len must be a tensor");
        const bool uniform = a[8] == Py_None;
        const Table tab = table_of(table);
        const Scales sc = scales_of(K, V, Ks, Vs);
        if (Vn.sizes() != Kn.sizes() || Vn.strides() != Kn.strides()) throw Error{PyExc_ValueError, "Knew and Vnew must share shape and strides"};
        const Tokens k = tokens_of(Kn, tab.B, uniform);
        const lotts_dtype dt = (lotts_dtype)paged_dtype(Kn);
        if (Vn.scalar_type() != Kn.scalar_type()) throw Error{PyExc_TypeError, "Knew and Vnew share one dtype"};
        if (K.size(1) != k.H || K.size(3) != k.D) throw Error{PyExc_ValueError, "Knew and Kpages disagree"};
        if (k.T > 0x7fffffff) throw Error{PyExc_ValueError, "too many tokens"};
        const int32_t* lens = numbers(len, tab.B, "kv_len must be contiguous int32 [B]");
        const int32_t* start = uniform ? nullptr : numbers(on(a[8], "q_start must be a tensor"), (int64_t)tab.B + 1, "q_start must be contiguous int32 [B+1]");
        const void *kn = Kn.data_ptr(), *vn = Vn.data_ptr();
        void *kp = K.data_ptr(), *vp = V.data_ptr(), *stream = address(a[10]);
        return released([&] {
            return c->append(tab.B, (int32_t)k.T, (int32_t)k.H, (int32_t)k.D, (int32_t)K.size(2), (int32_t)K.size(0), tab.columns, dt, kn, vn, k.stride_t,
                             pitch(k.H, k.stride_h, k.D), kp, vp, K.stride(0), K.stride(1), pitch(K.size(2), K.stride(2), k.D), sc.K, sc.V, sc.p, sc.h, sc.t,
                             tab.entries, tab.stride, lens, start, stream);
        });
    });
}

// MxCalls(address of mxfp4_quantize, mxfp4_dequantize, skinny_gemm_mxfp4_workspace_bytes, skinny_gemm_mxfp4, kv_append_paged_mxfp8,
// verify_attention_paged_mxfp8_workspace_bytes, verify_attention_paged_mxfp8)
PyObject* mx_new(PyTypeObject* type, PyObject* args, PyObject*) {
    void* f[7];
    if (PyTuple_GET_SIZE(args) != 7) {
        PyErr_SetString(PyExc_TypeError, "seven addresses");
        return nullptr;
    }
    for (int i = 0; i < 7; ++i) {
        f[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(args, i));
        if (!f[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an address is 0");
            return nullptr;
        }
    }
    MxCalls* c = reinterpret_cast<MxCalls*>(type->tp_alloc(type, 0));
    if (!c) return nullptr;
    c->quantize = reinterpret_cast<quantize_fn>(f[0]);
    c->dequantize = reinterpret_cast<dequantize_fn>(f[1]);
    c->gemm_ws = reinterpret_cast<gemm4_ws_fn>(f[2]);
    c->gemm = reinterpret_cast<gemm4_fn>(f[3]);
    c->append = reinterpret_cast<append8_fn>(f[4]);
    c->attn_ws = reinterpret_cast<paged8_ws_fn>(f[5]);
    c->attn = reinterpret_cast<paged8_fn>(f[6]);
    return reinterpret_cast<PyObject*>(c);
}

PyMethodDef mx_methods[] = {
    {"mxfp4_quantize", (PyCFunction)(void (*)(void))call_quantize, METH_FASTCALL, nullptr},
    {"mxfp4_dequantize", (PyCFunction)(void (*)(void))call_dequantize, METH_FASTCALL, nullptr},
    {"skinny_gemm_mxfp4", (PyCFunction)(void (*)(void))call_gemm4, METH_FASTCALL, nullptr},
    {"kv_append_paged_mxfp8", (PyCFunction)(void (*)(void))call_append8, METH_FASTCALL, nullptr},
    {"verify_attention_paged_mxfp8", (PyCFunction)(void (*)(void))call_paged8, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyTypeObject mx_type = {PyVarObject_HEAD_INIT(nullptr, 0)};

PyMethodDef calls_methods[] = {
    {"verify_attention", (PyCFunction)(void (*)(void))call_attention, METH_FASTCALL, nullptr},
    {"verify_attention_noalloc", (PyCFunction)(void (*)(void))call_attention_noalloc, METH_FASTCALL, nullptr},
    {"spec_accept", (PyCFunction)(void (*)(void))call_accept, METH_FASTCALL, nullptr},
    {"majority_vote", (PyCFunction)(void (*)(void))call_vote, METH_FASTCALL, nullptr},
    {"skinny_gemm", (PyCFunction)(void (*)(void))call_gemm, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyTypeObject calls_type = {PyVarObject_HEAD_INIT(nullptr, 0)};
PyModuleDef calls_module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls(void) {
    calls_type.tp_name = "_calls.Calls";
    calls_type.tp_basicsize = sizeof(Calls);
    calls_type.tp_flags = Py_TPFLAGS_DEFAULT;
    calls_type.tp_new = calls_new;
    calls_type.tp_methods = calls_methods;
    paged_type.tp_name = "_calls.PagedCalls";
    paged_type.tp_basicsize = sizeof(PagedCalls);
    paged_type.tp_flags = Py_TPFLAGS_DEFAULT;
    paged_type.tp_new = paged_new;
    paged_type.tp_methods = paged_methods;
    mx_type.tp_name = "_calls.MxCalls";
    mx_type.tp_basicsize = sizeof(MxCalls);
    mx_type.tp_flags = Py_TPFLAGS_DEFAULT;
    mx_type.tp_new = mx_new;
    mx_type.tp_methods = mx_methods;
    if (PyType_Ready(&calls_type) < 0 || PyType_Ready(&paged_type) < 0 || PyType_Ready(&mx_type) < 0) return nullptr;
    PyObject* m = PyModule_Create(&calls_module);
    if (!m) return nullptr;
    for (PyTypeObject* type : {&calls_type, &paged_type, &mx_type}) {
        Py_INCREF(type);
        if (PyModule_AddObject(m, type == &calls_type ? "Calls" : type == &paged_type ? "PagedCalls" : "MxCalls", reinterpret_cast<PyObject*>(type)) < 0) {
            Py_DECREF(type);
            Py_DECREF(m);
            return nullptr;
        }
    }
    if (PyModule_AddStringConstant(m, "built_for_torch", LOTTS_TORCH) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
