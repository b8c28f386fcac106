// The operators on a cache kept in pages on torch tensors: argument checks, allocation of outputs and the calls of include/sdv.h, for paged.py.  A call
// takes the host 5.2 us (an append) to 8.4 (an attention with its workspace and two launches); through Python checks and ctypes it took 11.2 to 14 (0.4 a tensor checked, 0.7 to 1.4 a tensor
// allocated).  Called on the current device and stream.  What shapes and types do not allow raises
// ValueError; a status of the library other than SDV_OK is handed back as an int.
#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/core/InferenceMode.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstring>
#include <initializer_list>

#include "../../include/sdv.h"

namespace {

// The library's entry points (set by bind()).
struct Library {
    decltype(&sdv_paged_slots) slots;
    decltype(&sdv_rope_append) rope;
    decltype(&sdv_tree_attention_workspace_bytes) workspace_bytes;
    decltype(&sdv_tree_attention) attention, attention_fresh;
    decltype(&sdv_verify_sampled) verify;
};
Library g_lib{};

struct Raised {};   // a Python exception is set
[[noreturn]] void refuse(const char* text) {
    PyErr_SetString(PyExc_ValueError, text);
    throw Raised{};
}
[[noreturn]] void refuse(const char* what, const char* text) {
    PyErr_Format(PyExc_ValueError, "%s: %s", what, text);
    throw Raised{};
}

bool given(PyObject* o) { return o != Py_None; }
const at::Tensor& tensor(PyObject* o, const char* what) {
    if (!THPVariable_Check(o)) refuse(what, "a tensor expected");
    return THPVariable_Unpack(o);
}
long long whole(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    return v;
}
double real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Raised{};
    return v;
}
int int_of(int64_t n, const char* what) {
    if (n > INT32_MAX) refuse(what, "more than 2^31 - 1 entries");
    return (int)n;
}

// Other Python threads run while torch allocates (it may wait for the device) and while the library launches (it waits when the device's queue is full).
struct Released {
    PyThreadState* state = PyEval_SaveThread();
    ~Released() { PyEval_RestoreThread(state); }
};

template <typename F>
int released(F call) {
    const Released r;
    return call();
}

struct Call {
    int device;
    void* stream;
    Call() {
        const c10::cuda::CUDAStream s = c10::cuda::getCurrentCUDAStream();
        device = s.device_index();
        stream = s.stream();
    }
    void here(const at::Tensor& t, const char* what) const {
        if (!t.is_cuda() || t.get_device() != device) refuse(what, "not on the current CUDA device");
    }
    // A contiguous vector of 32-bit integers; n < 0: of any length.
    int32_t* vector(PyObject* o, int64_t n, const char* what) const {
        const at::Tensor& t = tensor(o, what);
        if (t.scalar_type() != at::kInt || t.dim() != 1 || (n >= 0 && t.size(0) != n) || !t.is_contiguous()) refuse(what, "a contiguous int32 vector of the right length expected");
        here(t, what);
        return t.data_ptr<int32_t>();
    }
    int32_t* vector_or_null(PyObject* o, int64_t n, const char* what) const { return given(o) ? vector(o, n, what) : nullptr; }
    at::Tensor empty(at::IntArrayRef size, at::ScalarType type) const {
        const Released r;
        return at::detail::empty_cuda(size, type, at::Device(at::kCUDA, (at::DeviceIndex)device), c10::nullopt);
    }
};

// int32 vectors in one allocation, each from a 256-byte boundary on (slots of five trees 6.2 us a call, with four allocations 7.8).
class Vectors {
public:
    Vectors(const Call& c, std::initializer_list<int64_t> lengths) {
        int64_t total = 0;
        for (const int64_t n : lengths) total += padded(n);
        memory_ = c.empty({total}, at::kInt);
    }
    at::Tensor next(int64_t n, int32_t*& p) {
        at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(memory_.storage()), c10::DispatchKeySet(c10::DispatchKey::CUDA), memory_.dtype());
        t.unsafeGetTensorImpl()->set_storage_offset(at_);
        t.unsafeGetTensorImpl()->set_sizes_contiguous({n});
        p = n ? memory_.data_ptr<int32_t>() + at_ : nullptr;
        at_ += padded(n);
        return t;
    }

private:
    static int64_t padded(int64_t n) { return (n + 63) / 64 * 64; }
    at::Tensor memory_;
    int64_t at_ = 0;
};

int type_of(const at::Tensor& t, const char* what) {
    if (t.scalar_type() == at::kBFloat16) return SDV_BF16;
    if (t.scalar_type() == at::kHalf) return SDV_FP16;
    refuse(what, "bfloat16 or float16 expected");
}
int64_t length(PyObject* o, const char* what) {
    const at::Tensor& t = tensor(o, what);
    if (t.dim() != 1) refuse(what, "a vector expected");
    return t.size(0);
}

PyObject* const* four(PyObject* o, const char* text) {
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4) refuse(text);
    return ((PyTupleObject*)o)->ob_item;
}

// Block tables of n sequences.
int32_t* table(const Call& c, PyObject* o, int64_t n, int& width, long long& stride) {
    const at::Tensor& t = tensor(o, "block_table");
    if (t.scalar_type() != at::kInt || t.dim() != 2 || t.size(0) != n || (t.size(1) > 1 && t.stride(1) != 1)) refuse("block_table: int32 [sequences][width] with contiguous rows expected");
    c.here(t, "block_table");
    width = int_of(t.size(1), "block_table");
    stride = n > 1 ? t.stride(0) : width;
    return t.data_ptr<int32_t>();
}

// [pages][KV heads][tokens of a page][head dim], any strides with contiguous head elements.
sdv_pages pool(const Call& c, PyObject* ko, PyObject* vo) {
    const at::Tensor &k = tensor(ko, "k_pages"), &v = tensor(vo, "v_pages");
    if (k.dim() != 4 || v.sizes() != k.sizes() || v.strides() != k.strides() || v.scalar_type() != k.scalar_type())
        refuse("k_pages and v_pages: two tensors [pages][KV heads][page size][head dim] of the same shape, strides and type expected");
    c.here(k, "k_pages");
    c.here(v, "v_pages");
    if (k.size(3) > 1 && k.stride(3) != 1) refuse("k_pages: the elements of a head have to be contiguous");
    sdv_pages p;
    std::memset(&p, 0, sizeof(p));
    p.k = k.data_ptr();
    p.v = v.data_ptr();
    p.dtype = type_of(k, "k_pages");
    p.n_pages = int_of(k.size(0), "k_pages");
    p.n_kv_heads = int_of(k.size(1), "k_pages");
    p.page_size = int_of(k.size(2), "k_pages");
    p.head_dim = int_of(k.size(3), "k_pages");
    p.page_stride = p.n_pages > 1 ? k.stride(0) : 0;   // the stride of a dimension of one says nothing
    p.head_stride = p.n_kv_heads > 1 ? k.stride(1) : 0;
    p.token_stride = p.page_size > 1 ? k.stride(2) : 0;
    return p;
}

// Row and head stride of [rows][heads][head dim].
void rows_of(const Call& c, const at::Tensor& t, const char* what, long long& row, long long& head) {
    if (t.dim() != 3) refuse(what, "[rows][heads][head dim] expected");
    c.here(t, what);
    if (t.size(2) > 1 && t.stride(2) != 1) refuse(what, "the elements of a head have to be contiguous");
    row = t.size(0) > 1 ? t.stride(0) : 0;
    head = t.size(1) > 1 ? t.stride(1) : 0;
}

// A given output (rows of the shape and type of `like`), or a fresh one.
at::Tensor output(const Call& c, PyObject* o, const at::Tensor& like, const char* what, long long& row, long long& head) {
    at::Tensor out;
    if (given(o)) {
        out = tensor(o, what);
        rows_of(c, out, what, row, head);
        if (out.sizes() != like.sizes() || out.scalar_type() != like.scalar_type()) refuse(what, "shape and type of q expected");
    } else {
        out = c.empty(like.sizes(), like.scalar_type());
        row = like.size(1) * like.size(2);
        head = like.size(2);
    }
    return out;
}

// float32 [rows][vocab].
const float* probabilities(const Call& c, PyObject* o, int64_t n, int64_t vocab, const char* what, long long& stride) {
    const at::Tensor& t = tensor(o, what);
    if (t.scalar_type() != at::kFloat || t.dim() != 2 || t.size(0) != n || t.size(1) != vocab || (vocab > 1 && t.stride(1) != 1)) refuse(what, "float32 [rows][vocab] with contiguous rows expected");
    c.here(t, what);
    stride = n > 1 ? t.stride(0) : vocab;
    return t.data_ptr<float>();
}

// The caller's tensors among those that a call wrote to: autograd learns of it, as of torch's own writes in place.
void wrote(std::initializer_list<PyObject*> os) {
    for (PyObject* o : os) {
        if (!given(o)) continue;
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();   // (those have no counter)
    }
}

// A whole tensor to one value, as a call would write it: any tensor of the caller's, whatever mode it is from.
void fill(const at::Tensor& t, int value) {
    if (!t.defined() || !t.numel()) return;
    const c10::InferenceMode mode(t.is_inference() || c10::InferenceMode::is_enabled());
    const c10::NoGradGuard plain;
    t.fill_(value);
}

PyObject* result(int rc, std::initializer_list<PyObject*> written, std::initializer_list<at::Tensor> ts) {
    if (rc != SDV_OK) return PyLong_FromLong(rc);
    wrote(written);
    PyObject* out = PyTuple_New((Py_ssize_t)ts.size());
    if (!out) return nullptr;
    Py_ssize_t i = 0;
    for (const at::Tensor& t : ts) {
        PyObject* o = t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None);
        if (!o) {
            Py_DECREF(out);
            return nullptr;
        }
        PyTuple_SET_ITEM(out, i++, o);
    }
    return out;
}

// (kv_len, cu_rows, block_table, n_held, free_pages, free_state, page_size, n_rows, parent, out)
PyObject* slots(PyObject* const* a) {
    const Call c;
    sdv_slots_args s;
    std::memset(&s, 0, sizeof(s));
    const int64_t n = length(a[0], "kv_len"), n_rows = whole(a[7]);
    if (n_rows < 0 || length(a[5], "free_state") < 1) refuse("paged_slots: n_rows >= 0 and a free_state of at least one entry expected");
    s.n_seqs = int_of(n, "kv_len");
    s.n_rows = int_of(n_rows, "n_rows");
    s.n_free = int_of(length(a[4], "free_pages"), "free_pages");
    const long long page = whole(a[6]);
    s.page_size = page < 1 || page > INT32_MAX ? 0 : (int)page;
    s.kv_len = c.vector(a[0], n, "kv_len");
    s.cu_rows = c.vector(a[1], n + 1, "cu_rows");
    s.block_table = table(c, a[2], n, s.table_width, s.table_stride);
    s.n_held = c.vector(a[3], n, "n_held");
    s.free_pages = c.vector(a[4], -1, "free_pages");
    s.free_state = c.vector(a[5], -1, "free_state");
    s.parent = c.vector_or_null(a[8], n_rows, "parent");
    at::Tensor slots, positions, held, state;
    PyObject *const none[4] = {Py_None, Py_None, Py_None, Py_None}, *const* o = none;
    if (given(a[9])) {
        o = four(a[9], "out: the four tensors slots, positions, n_held and free_state expected");
        s.slots = c.vector(o[0], n_rows, "slots");
        s.positions = c.vector(o[1], n_rows, "positions");
        s.n_held_out = c.vector(o[2], n, "n_held (out)");
        s.free_state_out = c.vector(o[3], 2, "free_state (out)");
        slots = tensor(o[0], "slots"), positions = tensor(o[1], "positions"), held = tensor(o[2], "n_held (out)"), state = tensor(o[3], "free_state (out)");
    } else {
        Vectors v(c, {n_rows, n_rows, n, 2});
        slots = v.next(n_rows, s.slots);
        positions = v.next(n_rows, s.positions);
        held = v.next(n, s.n_held_out);
        state = v.next(2, s.free_state_out);
    }
    return result(released([&] { return g_lib.slots(&s, c.stream); }), {a[2], o[0], o[1], o[2], o[3]}, {slots, positions, held, state});
}

// (positions, frequencies, q, k, v, k_pages, v_pages, slots, interleaved, factor, q_out)
PyObject* rope(PyObject* const* a) {
    const Call c;
    sdv_rope_args s;
    std::memset(&s, 0, sizeof(s));
    sdv_pages p;
    std::memset(&p, 0, sizeof(p));
    const int64_t n = length(a[0], "positions");
    s.n_rows = int_of(n, "positions");
    s.positions = c.vector(a[0], n, "positions");
    const at::Tensor& f = tensor(a[1], "frequencies");
    if (f.scalar_type() != at::kDouble || f.dim() != 1 || !f.is_contiguous() || f.size(0) > INT32_MAX / 2) refuse("frequencies: contiguous float64 [rot_dim / 2] expected");
    c.here(f, "frequencies");
    s.frequencies = f.data_ptr<double>();
    s.rot_dim = 2 * (int)f.size(0);
    const bool has_q = given(a[2]), has_k = given(a[3]);
    if ((!has_q && !has_k) || has_k != given(a[4])) refuse("rope_append: q, or k and v, expected");
    s.interleaved = PyObject_IsTrue(a[8]);
    if (s.interleaved < 0) throw Raised{};
    s.factor = (float)real(a[9]);
    if (has_k) {
        if (!given(a[5]) || !given(a[6]) || !given(a[7])) refuse("rope_append: k and v need k_pages, v_pages and slots");
        p = pool(c, a[5], a[6]);
        const at::Tensor &k = tensor(a[3], "k"), &v = tensor(a[4], "v");
        rows_of(c, k, "k", s.k_row_stride, s.k_head_stride);
        rows_of(c, v, "v", s.v_row_stride, s.v_head_stride);
        const at::ScalarType type = THPVariable_Unpack(a[5]).scalar_type();
        if (k.size(0) != n || k.size(1) != p.n_kv_heads || k.size(2) != p.head_dim || v.sizes() != k.sizes() || k.scalar_type() != type || v.scalar_type() != type)
            refuse("k, v: [rows][KV heads][head dim] of the pages' type expected");
        s.k = k.data_ptr();
        s.v = v.data_ptr();
        s.slots = c.vector(a[7], n, "slots");
        s.n_kv_heads = p.n_kv_heads;
        s.head_dim = p.head_dim;
        s.dtype = p.dtype;
    }
    at::Tensor out;
    if (has_q) {
        const at::Tensor& q = tensor(a[2], "q");
        rows_of(c, q, "q", s.q_row_stride, s.q_head_stride);
        const int type = type_of(q, "q");
        if (q.size(0) != n || (has_k && (q.size(2) != s.head_dim || type != s.dtype))) refuse("q: a row for every position, with the head dim and type of k, expected");
        s.dtype = type;
        s.n_q_heads = int_of(q.size(1), "q");
        s.head_dim = int_of(q.size(2), "q");
        out = output(c, a[10], q, "q_out", s.out_row_stride, s.out_head_stride);
        s.q = q.data_ptr();
        s.q_out = out.data_ptr();
    }
    if (!n) return result(SDV_OK, {}, {out});
    return result(released([&] { return g_lib.rope(&s, has_k ? &p : nullptr, c.stream); }), {has_k ? a[5] : Py_None, has_k ? a[6] : Py_None, has_q ? a[10] : Py_None}, {out});
}

// (q, k_pages, v_pages, block_table, kv_len, cu_rows, parent, scale, out, workspace, status)
PyObject* attention(PyObject* const* a) {
    const Call c;
    sdv_attention_args s;
    std::memset(&s, 0, sizeof(s));
    const sdv_pages p = pool(c, a[1], a[2]);
    const at::Tensor& q = tensor(a[0], "q");
    rows_of(c, q, "q", s.q_row_stride, s.q_head_stride);
    if (q.scalar_type() != THPVariable_Unpack(a[1]).scalar_type() || q.size(2) != p.head_dim) refuse("q: type and head dim of the pages expected");
    const int64_t n = q.size(0), seqs = length(a[4], "kv_len");
    s.q = q.data_ptr();
    s.n_rows = int_of(n, "q");
    s.n_q_heads = int_of(q.size(1), "q");
    s.n_seqs = int_of(seqs, "kv_len");
    s.block_table = table(c, a[3], seqs, s.table_width, s.table_stride);
    s.kv_len = c.vector(a[4], seqs, "kv_len");
    s.cu_rows = c.vector(a[5], seqs + 1, "cu_rows");
    s.parent = c.vector_or_null(a[6], n, "parent");
    s.scale = given(a[7]) ? (float)real(a[7]) : (float)(1.0 / std::sqrt((double)p.head_dim));
    at::Tensor out = output(c, a[8], q, "out", s.out_row_stride, s.out_head_stride), workspace;
    s.out = out.data_ptr();
    if (given(a[9])) {
        workspace = tensor(a[9], "workspace");
        c.here(workspace, "workspace");
        if (!workspace.is_contiguous()) refuse("workspace: contiguous memory expected");
    } else {
        workspace = c.empty({(int64_t)g_lib.workspace_bytes(s.n_seqs, p.head_dim)}, at::kByte);
    }
    s.workspace = workspace.data_ptr();
    s.workspace_bytes = workspace.nbytes();
    s.status = c.vector_or_null(a[10], 1, "status");
    const bool fresh = !given(a[8]);   // memory of the allocator's is not handed out as it is
    if (!n || !seqs || !s.table_width) {   // the library does nothing: no row sees a token
        if (fresh) fill(out, 0);
        return result(SDV_OK, {}, {out});
    }
    return result(released([&] { return (fresh ? g_lib.attention_fresh : g_lib.attention)(&s, &p, c.stream); }), {a[8], a[10]}, {out});
}

// (target_probs, tokens, cu_rows, uniforms, draft_probs, parent, slots, out)
PyObject* verify(PyObject* const* a) {
    const Call c;
    sdv_verify_args s;
    std::memset(&s, 0, sizeof(s));
    const int64_t n = length(a[1], "tokens"), seqs = length(a[2], "cu_rows") - 1;
    const at::Tensor& target = tensor(a[0], "target_probs");
    if (target.dim() != 2 || seqs < 0) refuse("verify_sampled: target_probs [rows][vocab] and cu_rows [sequences + 1] expected");
    const int64_t vocab = target.size(1);
    s.target = probabilities(c, a[0], n, vocab, "target_probs", s.target_stride);
    if (given(a[4])) {
        if (given(a[5])) refuse("verify_sampled: drafts with probabilities are chains");
        s.draft = probabilities(c, a[4], n, vocab, "draft_probs", s.draft_stride);
    }
    const at::Tensor& u = tensor(a[3], "uniforms");
    if (u.scalar_type() != at::kFloat || u.dim() != 1 || u.size(0) != n || !u.is_contiguous()) refuse("uniforms: contiguous float32 [rows] expected");
    c.here(u, "uniforms");
    s.uniforms = u.data_ptr<float>();
    s.n_seqs = int_of(seqs, "cu_rows");
    s.n_rows = int_of(n, "tokens");
    s.vocab = int_of(vocab, "target_probs");
    s.tokens = c.vector(a[1], n, "tokens");
    s.cu_rows = c.vector(a[2], seqs + 1, "cu_rows");
    s.parent = c.vector_or_null(a[5], n, "parent");
    const bool has_slots = given(a[6]);   // (a vector of no rows has no address)
    s.slots = c.vector_or_null(a[6], n, "slots");
    at::Tensor accept, words, rows, moved;
    PyObject *const none[4] = {Py_None, Py_None, Py_None, Py_None}, *const* o = none;
    if (given(a[7])) {
        o = four(a[7], "out: the four tensors accept_len, tokens, rows and slots (None without slots) expected");
        s.accept_len = c.vector(o[0], seqs, "accept_len");
        s.out_tokens = c.vector(o[1], n, "tokens (out)");
        s.out_rows = c.vector(o[2], n, "rows (out)");
        accept = tensor(o[0], "accept_len"), words = tensor(o[1], "tokens (out)"), rows = tensor(o[2], "rows (out)");
        if (has_slots) {
            s.out_slots = c.vector(o[3], n, "slots (out)");
            moved = tensor(o[3], "slots (out)");
        }
    } else {
        Vectors v(c, {seqs, n, n, has_slots ? n : 0});
        accept = v.next(seqs, s.accept_len);
        words = v.next(n, s.out_tokens);
        rows = v.next(n, s.out_rows);
        if (has_slots) moved = v.next(n, s.out_slots);
    }
    if (!n || !seqs) {   // the library does nothing: no sequence has rows, no row a sequence
        for (const at::Tensor* t : {&accept, &words, &rows, &moved}) fill(*t, -1);
        return result(SDV_OK, {}, {accept, words, rows, moved});
    }
    return result(released([&] { return g_lib.verify(&s, c.stream); }), {o[0], o[1], o[2], has_slots ? o[3] : Py_None}, {accept, words, rows, moved});
}

template <PyObject* (*F)(PyObject* const*), Py_ssize_t N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != N || !g_lib.slots) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments, or called before bind()");
        return nullptr;
    }
    HANDLE_TH_ERRORS
    try {
        return F(args);
    } catch (const Raised&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// The addresses of the library's six entry points, in the order of Library.
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
    void* p[6];
    if (n != 6) {
        PyErr_SetString(PyExc_TypeError, "six addresses expected");
        return nullptr;
    }
    for (int i = 0; i < 6; ++i) {
        p[i] = PyLong_AsVoidPtr(args[i]);
        if (!p[i] && PyErr_Occurred()) return nullptr;
    }
    g_lib.slots = (decltype(g_lib.slots))p[0];
    g_lib.rope = (decltype(g_lib.rope))p[1];
    g_lib.workspace_bytes = (decltype(g_lib.workspace_bytes))p[2];
    g_lib.attention = (decltype(g_lib.attention))p[3];
    g_lib.attention_fresh = (decltype(g_lib.attention_fresh))p[4];
    g_lib.verify = (decltype(g_lib.verify))p[5];
    Py_RETURN_NONE;
}

#define ENTRY(name, f, n) {name, (PyCFunction)(void*)(&entry<f, n>), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"bind", (PyCFunction)(void*)bind, METH_FASTCALL, nullptr},
                         ENTRY("paged_slots", slots, 10),
                         ENTRY("rope_append", rope, 11),
                         ENTRY("tree_attention", attention, 11),
                         ENTRY("verify_sampled", verify, 8),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_paged", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__paged() { return PyModule_Create(&module); }
