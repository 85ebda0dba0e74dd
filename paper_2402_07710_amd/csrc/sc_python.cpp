// CPython front of the calls a layer makes every frame: takes torch tensors, checks them, hands
// pointers and sizes to libsc's C functions and returns their status.  Argument marshalling only.
//
// A layer on a small cloud is three launches of 4-5 us of GPU time each, so the host's part of a call
// decides its pace.  The same marshalling in Python over ctypes costs 8.4-9.2 us per call (the current
// stream 2.7, seven to eight tensors 0.35 each, the ctypes conversion 0.8, the launch itself ~4); here
// everything but the launch is well under half a microsecond.
//
// The C functions are the ones of the library that binding.py has loaded: it passes their addresses
// to bind(), so both always use the same libsc.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <algorithm>
#include <initializer_list>

#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "sc.h"

namespace {

struct Lib {
    decltype(&sc_hash_build) hash_build;
    decltype(&sc_hash_rebuild) hash_rebuild;
    decltype(&sc_kmap_build) kmap_build;
    decltype(&sc_kmap_build_noalloc) kmap_build_noalloc;
    decltype(&sc_kmap_transpose) kmap_transpose;
    decltype(&sc_conv_fwd) conv_fwd;
    decltype(&sc_conv_fwd_packed) conv_fwd_packed;
    decltype(&sc_conv_up_fwd) conv_up_fwd;
    decltype(&sc_conv_fwd_grid) conv_fwd_grid;
    decltype(&sc_grid_build) grid_build;
    decltype(&sc_kmap_build_grid) kmap_build_grid;
} lib;

// the row layers, bound apart by bind_rows()
struct RowLib {
    decltype(&sc_linear_fwd) linear_fwd;
    decltype(&sc_linear_bwd) linear_bwd;
    decltype(&sc_grouped_fwd) grouped_fwd;
    decltype(&sc_grouped_bwd) grouped_bwd;
    decltype(&sc_qk_rope_fwd) qk_rope_fwd;
    decltype(&sc_qk_rope_bwd) qk_rope_bwd;
    decltype(&sc_attention_fwd) attention_fwd;
    decltype(&sc_attention_bwd) attention_bwd;
    decltype(&sc_group_norm_fwd) group_norm_fwd;
    decltype(&sc_group_norm_bwd) group_norm_bwd;
} row_lib;

struct PyFailure {};      // a Python exception is set

[[noreturn]] void fail(PyObject* kind, const char* what) {
    PyErr_SetString(kind, what);
    throw PyFailure{};
}

const at::Tensor& tensor(PyObject* o) {
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, "tensor expected");
    return THPVariable_Unpack(o);
}
// device pointer of a tensor argument; null for None
void* ptr(PyObject* o) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o);
    if (!t.is_cuda()) fail(PyExc_ValueError, "device tensor expected");
    if (!t.is_contiguous()) fail(PyExc_ValueError, "contiguous tensor expected");
    return t.data_ptr();
}
size_t nbytes(PyObject* o) { return o == Py_None ? 0 : tensor(o).nbytes(); }
int64_t size(PyObject* o, int dim) {
    const at::Tensor& t = tensor(o);
    if (dim >= t.dim()) fail(PyExc_IndexError, "tensor has too few dimensions");
    return t.size(dim);
}
int dtype(PyObject* o) {
    switch (tensor(o).scalar_type()) {
        case at::kFloat: return SC_F32;
        case at::kHalf: return SC_F16;
        case at::kBFloat16: return SC_BF16;
        default: fail(PyExc_KeyError, "dtype must be float32, float16 or bfloat16");
    }
}
long long integer(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw PyFailure{};
    return v;
}
int small_int(PyObject* o) {
    const long long v = integer(o);
    if (v < INT32_MIN || v > INT32_MAX) fail(PyExc_OverflowError, "integer out of range");
    return (int)v;
}
uint32_t epoch32(PyObject* o) {
    const long long v = integer(o);
    if (v < 0 || v > (long long)UINT32_MAX) fail(PyExc_OverflowError, "epoch out of range");
    return (uint32_t)v;
}
struct Dims {
    int32_t B, X, Y, Z;
};
Dims dims(PyObject* o) {
    PyObject* seq = PySequence_Fast(o, "dims must be (B, X, Y, Z)");
    if (seq == nullptr) throw PyFailure{};
    Dims d{};
    try {
        if (PySequence_Fast_GET_SIZE(seq) != 4) fail(PyExc_TypeError, "dims must be (B, X, Y, Z)");
        int32_t* v[4] = {&d.B, &d.X, &d.Y, &d.Z};
        for (int i = 0; i < 4; ++i) *v[i] = small_int(PySequence_Fast_GET_ITEM(seq, i));
    } catch (...) {
        Py_DECREF(seq);
        throw;
    }
    Py_DECREF(seq);
    return d;
}
// None: torch's current stream; a torch stream; or the stream itself as an integer
void* stream(PyObject* o) {
    if (o == Py_None) return (void*)c10::hip::getCurrentHIPStream().stream();
    if (PyLong_Check(o)) {
        void* p = PyLong_AsVoidPtr(o);
        if (p == nullptr && PyErr_Occurred()) throw PyFailure{};
        return p;
    }
    PyObject* raw = PyObject_GetAttrString(o, "cuda_stream");
    if (raw == nullptr) throw PyFailure{};
    void* p = PyLong_AsVoidPtr(raw);
    Py_DECREF(raw);
    if (p == nullptr && PyErr_Occurred()) throw PyFailure{};
    return p;
}
// [rows, channels] and no other number of dimensions: a row's channels are contiguous
void check_matrix(PyObject* o, const char* what) {
    if (tensor(o).dim() != 2) fail(PyExc_ValueError, what);
}
bool same_dtype(PyObject* a, PyObject* b) { return tensor(a).scalar_type() == tensor(b).scalar_type(); }
// weight must be [K^3, C_in, C_out] in the feature type
bool weight_fits(PyObject* weight, PyObject* feat, int K, int64_t C_in, int64_t C_out) {
    const at::Tensor& w = tensor(weight);
    return w.dim() == 3 && w.size(0) == (int64_t)K * K * K && w.size(1) == C_in && w.size(2) == C_out && same_dtype(weight, feat);
}

using Args = PyObject* const*;

// The library's call with the interpreter lock released: a launch may block (full queue, first load of a code
// object) and other Python threads go on meanwhile.  The arguments have been read under the lock, and the
// caller's frame holds the tensors they point into.
template <class F, class... A>
int unlocked(F function, A... arguments) {
    PyThreadState* const thread = PyEval_SaveThread();
    const int rc = function(arguments...);
    PyEval_RestoreThread(thread);
    return rc;
}

int hash_build(Args a) {                 // coords, table, counts, stream
    return unlocked(lib.hash_build, (const int32_t*)ptr(a[0]), size(a[0], 0), ptr(a[1]), nbytes(a[1]), (sc_counts*)ptr(a[2]), stream(a[3]));
}
int hash_rebuild(Args a) {               // coords, table, epoch, counts, stream
    return unlocked(lib.hash_rebuild, (const int32_t*)ptr(a[0]), size(a[0], 0), ptr(a[1]), nbytes(a[1]), small_int(a[2]), (sc_counts*)ptr(a[3]),
                            stream(a[4]));
}
int kmap_build(Args a) {                 // coords, table, K, stride, mode, out_coords, kmap, scratch, counts, stream
    return unlocked(lib.kmap_build, (const int32_t*)ptr(a[0]), size(a[0], 0), ptr(a[1]), small_int(a[2]), small_int(a[3]), small_int(a[4]),
                          (int32_t*)ptr(a[5]), ptr(a[6]), nbytes(a[6]), ptr(a[7]), nbytes(a[7]), (sc_counts*)ptr(a[8]), stream(a[9]));
}
int kmap_build_noalloc(Args a) {         // coords, table, K, stride, mode, out_coords, kmap, counts, stream
    return unlocked(lib.kmap_build_noalloc, (const int32_t*)ptr(a[0]), size(a[0], 0), ptr(a[1]), small_int(a[2]), small_int(a[3]), small_int(a[4]),
                                  (int32_t*)ptr(a[5]), ptr(a[6]), nbytes(a[6]), (sc_counts*)ptr(a[7]), stream(a[8]));
}
int kmap_transpose(Args a) {             // kmap, n, K, stride, counts, kmap_inv, stream
    return unlocked(lib.kmap_transpose, ptr(a[0]), integer(a[1]), small_int(a[2]), small_int(a[3]), (const sc_counts*)ptr(a[4]), ptr(a[5]),
                              nbytes(a[5]), stream(a[6]));
}
int grid_build(Args a) {                 // coords, grid, dims, epoch, counts, stream
    const Dims d = dims(a[2]);
    return unlocked(lib.grid_build, (const int32_t*)ptr(a[0]), size(a[0], 0), ptr(a[1]), nbytes(a[1]), d.B, d.X, d.Y, d.Z, epoch32(a[3]),
                          (sc_counts*)ptr(a[4]), stream(a[5]));
}
int kmap_build_grid(Args a) {            // coords, grid, dims, epoch, K, kmap, counts, stream
    const Dims d = dims(a[2]);
    return unlocked(lib.kmap_build_grid, (const int32_t*)ptr(a[0]), size(a[0], 0), ptr(a[1]), nbytes(a[1]), d.B, d.X, d.Y, d.Z, epoch32(a[3]),
                               small_int(a[4]), ptr(a[5]), nbytes(a[5]), (sc_counts*)ptr(a[6]), stream(a[7]));
}
int conv_fwd(Args a) {                   // feat_in, n_map, weight, feat_out, kmap, counts, K, stride, mode, workspace, stream
    const int K = small_int(a[6]);
    check_matrix(a[0], "feat_in must be [rows, C_in]");
    check_matrix(a[3], "feat_out must be [rows, C_out]");
    const int64_t n_in = size(a[0], 0), C_in = size(a[0], 1), n_out_cap = size(a[3], 0), C_out = size(a[3], 1);
    if (!weight_fits(a[2], a[0], K, C_in, C_out)) fail(PyExc_ValueError, "weight must be [K^3, C_in, C_out] in the feature dtype");
    return unlocked(lib.conv_fwd, ptr(a[0]), a[1] == Py_None ? n_in : integer(a[1]), ptr(a[2]), ptr(a[3]), n_out_cap, ptr(a[4]), nbytes(a[4]),
                        (const sc_counts*)ptr(a[5]), K, small_int(a[7]), small_int(a[8]), (int)C_in, (int)C_out, dtype(a[0]), dtype(a[3]),
                        ptr(a[9]), nbytes(a[9]), stream(a[10]));
}
int conv_fwd_packed(Args a) {            // feat_in, n_map, packed, C_out, feat_out, kmap, counts, K, stride, mode, stream
    check_matrix(a[0], "feat_in must be [rows, C_in]");
    check_matrix(a[4], "feat_out must be [rows, C_out]");
    const int64_t n_in = size(a[0], 0), C_in = size(a[0], 1), n_out_cap = size(a[4], 0), C_out = integer(a[3]);
    if (size(a[4], 1) != C_out) fail(PyExc_ValueError, "feat_out must have C_out columns");
    return unlocked(lib.conv_fwd_packed, ptr(a[0]), a[1] == Py_None ? n_in : integer(a[1]), ptr(a[2]), ptr(a[4]), n_out_cap, ptr(a[5]),
                               nbytes(a[5]), (const sc_counts*)ptr(a[6]), small_int(a[7]), small_int(a[8]), small_int(a[9]), (int)C_in,
                               (int)C_out, dtype(a[0]), dtype(a[4]), stream(a[10]));
}
int conv_up_fwd(Args a) {                // feat_coarse, n_map, weight, feat_fine, kmap, counts, K, stream
    const int K = small_int(a[6]);
    const int64_t n_map = integer(a[1]), C_in = size(a[2], 1), C_out = size(a[2], 2);
    if (!weight_fits(a[2], a[0], K, C_in, C_out) || tensor(a[0]).dim() != 2 || size(a[0], 1) != C_in || tensor(a[3]).dim() != 2 || size(a[3], 0) != n_map ||
        size(a[3], 1) != C_out)
        return SC_EINVAL;
    return unlocked(lib.conv_up_fwd, ptr(a[0]), n_map, ptr(a[2]), ptr(a[3]), ptr(a[4]), nbytes(a[4]), (const sc_counts*)ptr(a[5]), K, (int)C_in,
                           (int)C_out, dtype(a[0]), dtype(a[3]), stream(a[7]));
}
int conv_fwd_grid(Args a) {              // feat_in, coords, grid, dims, epoch, weight, feat_out, K, workspace, stream
    const Dims d = dims(a[3]);
    return unlocked(lib.conv_fwd_grid, ptr(a[0]), (const int32_t*)ptr(a[1]), size(a[1], 0), ptr(a[2]), nbytes(a[2]), d.B, d.X, d.Y, d.Z,
                             epoch32(a[4]), ptr(a[5]), ptr(a[6]), small_int(a[7]), (int)size(a[5], 1), (int)size(a[5], 2), dtype(a[0]),
                             dtype(a[6]), ptr(a[8]), nbytes(a[8]), stream(a[9]));
}

// A matrix whose rows may be a slice of wider ones: [n, C], a row's elements next to each other.
struct Rows {
    void* data = nullptr;
    int64_t n = 0, C = 0, ld = 0;
};
[[noreturn]] void fail_on(PyObject* kind, const char* name, const char* what) {
    PyErr_Format(kind, "%s %s", name, what);
    throw PyFailure{};
}
// Where a tensor's elements are.  One without elements has no address, but is not the same as none that is given, for which null stands: it gets one that
// nothing is read from or written to.
void* address(const at::Tensor& t) {
    alignas(64) static char nothing[64];
    return t.numel() == 0 ? nothing : t.data_ptr();
}
// every tensor among a call's arguments, behind the checks of their shapes
void all_on_device(Args a, int n) {
    for (int i = 0; i < n; ++i)
        if (THPVariable_Check(a[i]) && !THPVariable_Unpack(a[i]).is_cuda()) fail(PyExc_ValueError, "device tensor expected");
}
Rows rows_of(PyObject* o, const char* name) {
    if (o == Py_None) return Rows{};
    const at::Tensor& t = tensor(o);
    if (t.dim() != 2 || (t.size(1) > 1 && t.stride(1) != 1)) fail_on(PyExc_ValueError, name, "must be [rows, channels], a row's channels contiguous");
    Rows r;
    r.n = t.size(0);
    r.C = t.size(1);
    r.ld = r.n > 1 ? t.stride(0) : r.C;                // torch leaves the stride of a single row undefined
    if (r.ld < r.C) fail_on(PyExc_ValueError, name, "has rows that overlap");
    if (r.C > INT32_MAX) fail_on(PyExc_ValueError, name, "has too many channels");         // the library counts them in an int
    r.data = address(t);
    return r;
}
// a contiguous tensor of `dims` dimensions, sizes -1 unchecked
void check_block(PyObject* o, const char* name, std::initializer_list<int64_t> sizes) {
    if (o == Py_None) return;
    const at::Tensor& t = tensor(o);
    bool fits = t.dim() == (int64_t)sizes.size();
    int d = 0;
    for (const int64_t s : sizes) fits = fits && t.size(d++) == s;
    if (!fits) fail_on(PyExc_ValueError, name, "has the wrong shape");
    if (!t.is_contiguous()) fail_on(PyExc_ValueError, name, "must be contiguous");
}
void check_dtype(PyObject* o, const char* name, PyObject* like) {
    if (o != Py_None && !same_dtype(o, like)) fail_on(PyExc_ValueError, name, "has the wrong dtype");
}
// a count for the library, which holds it in an int; what does not fit is above every limit anyway
int count32(int64_t n) { return (int)std::min<int64_t>(n, INT32_MAX); }
const int32_t* list_of(PyObject* o, const char* name, int64_t n) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o);
    if (t.scalar_type() != at::kInt) fail_on(PyExc_ValueError, name, "must be int32");
    check_block(o, name, {n});
    return (const int32_t*)t.data_ptr();
}
void check_rows(const Rows& r, PyObject* o, const char* name, int64_t n, int64_t C) {
    if (o != Py_None && (r.n != n || r.C != C)) fail_on(PyExc_ValueError, name, "has the wrong shape");
}
void check_out_dtype(PyObject* out, PyObject* in) {
    if (!same_dtype(out, in) && tensor(out).scalar_type() != at::kFloat) fail(PyExc_ValueError, "out must be of the rows' dtype or float32");
}

// Without a list entry p reads row p.  (The library itself takes rows past the last for zeros.)
void check_entries(const Rows& x, PyObject* list, int64_t n) {
    if (list == Py_None && x.n < n) fail(PyExc_ValueError, "x has fewer rows than there are entries");
}

int linear_fwd(Args a) {                 // x, weight, out, bias, act, residual, pre, stream
    const Rows x = rows_of(a[0], "x"), out = rows_of(a[2], "out"), residual = rows_of(a[5], "residual"), pre = rows_of(a[6], "pre");
    const int64_t C_out = out.C;
    check_block(a[1], "weight", {x.C, C_out});
    check_block(a[3], "bias", {C_out});
    check_dtype(a[1], "weight", a[0]);
    check_dtype(a[3], "bias", a[0]);
    check_out_dtype(a[2], a[0]);
    check_dtype(a[5], "residual", a[2]);
    check_dtype(a[6], "pre", a[2]);
    check_rows(out, a[2], "out", x.n, C_out);
    check_rows(residual, a[5], "residual", x.n, C_out);
    check_rows(pre, a[6], "pre", x.n, C_out);
    all_on_device(a, 8);
    return unlocked(row_lib.linear_fwd, x.data, x.ld, x.n, ptr(a[1]), ptr(a[3]), small_int(a[4]), residual.data, residual.ld, out.data, out.ld, pre.data,
                    pre.ld, (int)x.C, (int)C_out, dtype(a[0]), dtype(a[2]), stream(a[7]));
}
int linear_bwd(Args a) {                 // grad, x, weight, grad_x, grad_weight, grad_bias, pre, act, workspace, stream
    const Rows grad = rows_of(a[0], "grad_out"), x = rows_of(a[1], "x"), grad_x = rows_of(a[3], "grad_x"), pre = rows_of(a[6], "pre");
    const int64_t C_in = a[1] == Py_None && a[2] != Py_None ? size(a[2], 0) : x.C;         // x is read for the weight's gradient only
    check_block(a[2], "weight", {C_in, grad.C});
    check_block(a[4], "grad_weight", {C_in, grad.C});
    check_block(a[5], "grad_bias", {grad.C});
    for (int i = 1; i <= 6; ++i) check_dtype(a[i], "an argument", a[0]);
    check_rows(x, a[1], "x", grad.n, C_in);
    check_rows(grad_x, a[3], "grad_x", grad.n, C_in);
    check_rows(pre, a[6], "pre", grad.n, grad.C);
    all_on_device(a, 10);
    return unlocked(row_lib.linear_bwd, grad.data, grad.ld, x.data, x.ld, grad.n, ptr(a[2]), pre.data, pre.ld, small_int(a[7]), grad_x.data, grad_x.ld,
                    ptr(a[4]), ptr(a[5]), count32(C_in), (int)grad.C, dtype(a[0]), ptr(a[8]), nbytes(a[8]), stream(a[9]));
}
int grouped_fwd(Args a) {                // x, weight, starts, out, rows, bias, act, pre, stream
    const Rows x = rows_of(a[0], "x"), out = rows_of(a[3], "out"), pre = rows_of(a[7], "pre");
    const int64_t groups = size(a[2], 0) - 1, n = out.n, C_out = out.C;
    check_block(a[1], "weight", {groups, x.C, C_out});
    check_block(a[5], "bias", {groups, C_out});
    check_dtype(a[1], "weight", a[0]);
    check_dtype(a[5], "bias", a[0]);
    check_out_dtype(a[3], a[0]);
    check_dtype(a[7], "pre", a[3]);
    check_rows(pre, a[7], "pre", n, C_out);
    const int32_t* starts = list_of(a[2], "starts", groups + 1);
    const int32_t* rows = list_of(a[4], "rows", n);
    check_entries(x, a[4], n);
    all_on_device(a, 9);
    return unlocked(row_lib.grouped_fwd, x.data, x.ld, x.n, rows, n, starts, count32(groups), ptr(a[1]), ptr(a[5]), small_int(a[6]), out.data, out.ld, pre.data,
                    pre.ld, (int)x.C, (int)C_out, dtype(a[0]), dtype(a[3]), stream(a[8]));
}
int grouped_bwd(Args a) {                // grad, x, weight, starts, grad_x, grad_weight, grad_bias, rows, grad_rows, pre, act, workspace, stream
    const Rows grad = rows_of(a[0], "grad_out"), x = rows_of(a[1], "x"), grad_x = rows_of(a[4], "grad_x"), pre = rows_of(a[9], "pre");
    const int64_t groups = size(a[3], 0) - 1;
    int64_t n = grad.n;                  // entries: as many as there are gradient rows, or as the list has
    if (a[8] != Py_None) n = size(a[8], 0);
    const int64_t C_in = a[1] == Py_None && a[2] != Py_None ? size(a[2], 1) : x.C;
    check_block(a[2], "weight", {groups, C_in, grad.C});
    check_block(a[5], "grad_weight", {groups, C_in, grad.C});
    check_block(a[6], "grad_bias", {groups, grad.C});
    for (const int i : {1, 2, 4, 5, 6, 9}) check_dtype(a[i], "an argument", a[0]);
    check_rows(grad_x, a[4], "grad_x", n, C_in);
    check_rows(pre, a[9], "pre", n, grad.C);
    const int32_t* starts = list_of(a[3], "starts", groups + 1);
    const int32_t* rows = list_of(a[7], "rows", n);
    if (a[5] != Py_None) check_entries(x, a[7], n);         // rows are read for weight gradients only
    const int32_t* grad_rows = list_of(a[8], "grad_rows", n);
    all_on_device(a, 13);
    return unlocked(row_lib.grouped_bwd, grad.data, grad.ld, grad.n, grad_rows, x.data, x.ld, x.n, rows, n, starts, count32(groups), ptr(a[2]), pre.data, pre.ld,
                    small_int(a[10]), grad_x.data, grad_x.ld, ptr(a[5]), ptr(a[6]), count32(C_in), (int)grad.C, dtype(a[0]), ptr(a[11]), nbytes(a[11]),
                    stream(a[12]));
}

// [rows, heads, D] in any order of rows and heads, a head's channels contiguous
sc_heads heads_of(PyObject* o, const char* name, int64_t rows, int64_t D) {
    sc_heads h{};
    if (o == Py_None) return h;
    const at::Tensor& t = tensor(o);
    if (t.dim() != 3 || t.size(0) != rows || t.size(2) != D) fail_on(PyExc_ValueError, name, "has the wrong shape");
    if (t.size(2) > 1 && t.stride(2) != 1) fail_on(PyExc_ValueError, name, "must have a head's channels contiguous");
    if (t.size(1) > INT32_MAX) fail_on(PyExc_ValueError, name, "has too many heads");
    h.row = t.size(0) > 1 ? t.stride(0) : 0;
    h.head = t.size(1) > 1 ? t.stride(1) : 0;
    h.heads = (int32_t)t.size(1);
    h.data = address(t);
    return h;
}
PyObject* tensor_given(PyObject* o, const char* name) {
    if (o == Py_None) fail_on(PyExc_ValueError, name, "is needed");
    return o;
}
struct Positions {
    const int32_t* data;
    int64_t ld;
    int axes;
};
Positions positions(PyObject* o, int64_t rows) {
    const at::Tensor& t = tensor(o);
    if (t.dim() != 2 || t.size(0) != rows || t.scalar_type() != at::kInt) fail(PyExc_ValueError, "pos must be int32 [rows, axes]");
    if (t.size(1) > 1 && t.stride(1) != 1) fail(PyExc_ValueError, "pos must have a row's coordinates contiguous");
    const int64_t ld = t.size(0) > 1 ? t.stride(0) : t.size(1);
    return Positions{(const int32_t*)address(t), ld, count32(t.size(1))};
}
float number(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw PyFailure{};
    return (float)v;
}
// Large enough, and with a coordinate for every axis: sc_rope_table leaves their number on the tensors it gives.  (Those from elsewhere are taken as they are.)
void check_table(PyObject* table, int64_t D, const Positions& pos) {
    if ((int64_t)nbytes(table) < 8 * D) fail(PyExc_ValueError, "table is not one of sc_rope_table for this head size");
    static PyObject* const name = PyUnicode_InternFromString("rope_axes");
    PyObject* const axes = PyObject_GetAttr(table, name);
    if (axes == nullptr) {
        if (!PyErr_ExceptionMatches(PyExc_AttributeError)) throw PyFailure{};
        PyErr_Clear();
        return;
    }
    const long n = PyLong_AsLong(axes);
    Py_DECREF(axes);
    if (n == -1 && PyErr_Occurred()) throw PyFailure{};
    if (n > pos.axes) fail(PyExc_ValueError, "table turns by more axes than pos has");
}
int qk_rope_fwd(Args a) {                // q, k, pos, table, q_out, k_out, gain_q, gain_k, eps, pairing, stream
    if (tensor(a[0]).dim() != 3) fail(PyExc_ValueError, "q must be [rows, heads, D]");
    const int64_t rows = size(a[0], 0), D = size(a[0], 2);
    const sc_heads q = heads_of(a[0], "q", rows, D), k = heads_of(a[1], "k", rows, D), q_out = heads_of(a[4], "q_out", rows, D),
                   k_out = heads_of(a[5], "k_out", rows, D);
    for (const int i : {1, 4, 5, 6, 7}) check_dtype(a[i], "an argument", a[0]);
    check_block(a[6], "gain_q", {D});
    check_block(a[7], "gain_k", {D});
    const Positions pos = positions(a[2], rows);
    check_table(a[3], D, pos);
    all_on_device(a, 11);
    return unlocked(row_lib.qk_rope_fwd, &q, a[1] == Py_None ? nullptr : &k, rows, count32(D), pos.data, pos.ld, pos.axes, (const void*)ptr(a[3]), small_int(a[9]),
                    ptr(a[6]), ptr(a[7]), number(a[8]), &q_out, a[5] == Py_None ? nullptr : &k_out, dtype(a[0]), stream(a[10]));
}
int qk_rope_bwd(Args a) {                // grad_q_out, grad_k_out, q, k, pos, table, grad_q, grad_k, gain_q, gain_k, grad_gain_q, grad_gain_k, eps, pairing, workspace, stream
    if (tensor(a[0]).dim() != 3) fail(PyExc_ValueError, "grad_q_out must be [rows, heads, D]");
    const int64_t rows = size(a[0], 0), D = size(a[0], 2);
    const sc_heads dq_out = heads_of(a[0], "grad_q_out", rows, D), dk_out = heads_of(a[1], "grad_k_out", rows, D), q = heads_of(a[2], "q", rows, D),
                   k = heads_of(a[3], "k", rows, D), dq = heads_of(a[6], "grad_q", rows, D), dk = heads_of(a[7], "grad_k", rows, D);
    for (const int i : {1, 2, 3, 6, 7, 8, 9, 10, 11}) check_dtype(a[i], "an argument", a[0]);
    const char* const names[4] = {"gain_q", "gain_k", "grad_gain_q", "grad_gain_k"};
    for (int i = 0; i < 4; ++i) check_block(a[8 + i], names[i], {D});
    const Positions pos = positions(a[4], rows);
    check_table(a[5], D, pos);
    all_on_device(a, 16);
    return unlocked(row_lib.qk_rope_bwd, &dq_out, a[1] == Py_None ? nullptr : &dk_out, &q, a[3] == Py_None ? nullptr : &k, rows, count32(D), pos.data, pos.ld,
                    pos.axes, (const void*)ptr(a[5]), small_int(a[13]), ptr(a[8]), ptr(a[9]), number(a[12]), &dq, a[7] == Py_None ? nullptr : &dk,
                    ptr(a[10]), ptr(a[11]), dtype(a[0]), ptr(a[14]), nbytes(a[14]), stream(a[15]));
}

// The scenes of attention's queries and keys: starts int32 [scenes + 1], lengths int32 [scenes], all of them optional.
struct Scenes {
    const int32_t *q_starts, *k_starts, *k_lens;
    int scenes;
};
Scenes scenes_of(PyObject* q_starts, PyObject* k_starts, PyObject* k_lens, int64_t q_rows, int64_t k_rows) {
    if (q_starts == Py_None && k_starts != Py_None) fail(PyExc_ValueError, "k_starts without q_starts");
    if (q_starts != Py_None && k_starts == Py_None && q_rows != k_rows) fail(PyExc_ValueError, "as many keys as queries, or k_starts");
    const int64_t scenes = q_starts == Py_None ? 1 : size(q_starts, 0) - 1;
    if (scenes < 1 || scenes > SC_SCENES_MAX) fail(PyExc_ValueError, "q_starts must be int32 [scenes + 1]");
    return Scenes{list_of(q_starts, "q_starts", scenes + 1), list_of(k_starts, "k_starts", scenes + 1), list_of(k_lens, "k_lens", scenes), (int)scenes};
}
float* floats_of(PyObject* o, const char* name, std::initializer_list<int64_t> sizes) {
    if (o == Py_None) return nullptr;
    if (tensor(o).scalar_type() != at::kFloat) fail_on(PyExc_ValueError, name, "must be float32");
    check_block(o, name, sizes);
    return (float*)address(tensor(o));
}
int attention_fwd(Args a) {              // q, k, v, out, q_starts, k_starts, k_lens, causal, scale, lse, workspace, stream
    if (tensor(a[0]).dim() != 3) fail(PyExc_ValueError, "q must be [rows, heads, D]");
    if (tensor(a[1]).dim() != 3) fail(PyExc_ValueError, "k must be [rows, heads, D]");
    const int64_t rows = size(a[0], 0), D = size(a[0], 2), keys = size(a[1], 0);
    const sc_heads q = heads_of(a[0], "q", rows, D), k = heads_of(a[1], "k", keys, D), v = heads_of(tensor_given(a[2], "v"), "v", keys, D),
                   out = heads_of(tensor_given(a[3], "out"), "out", rows, D);
    for (const int i : {1, 2, 3}) check_dtype(a[i], "an argument", a[0]);
    if (k.heads != v.heads) fail(PyExc_ValueError, "v has another number of heads than k");
    if (out.heads != q.heads) fail(PyExc_ValueError, "out has another number of heads than q");
    const Scenes s = scenes_of(a[4], a[5], a[6], rows, keys);
    float* lse = floats_of(a[9], "lse", {rows, q.heads});
    all_on_device(a, 12);
    return unlocked(row_lib.attention_fwd, &q, &k, &v, rows, keys, count32(D), s.q_starts, s.k_starts, s.k_lens, s.scenes, small_int(a[7]), number(a[8]), &out, lse,
                    dtype(a[0]), ptr(a[10]), nbytes(a[10]), stream(a[11]));
}
int attention_bwd(Args a) {              // grad_out, q, k, v, out, lse, grad_q, grad_k, grad_v, q_starts, k_starts, k_lens, causal, scale, workspace, stream
    if (tensor(a[1]).dim() != 3) fail(PyExc_ValueError, "q must be [rows, heads, D]");
    if (tensor(a[2]).dim() != 3) fail(PyExc_ValueError, "k must be [rows, heads, D]");
    const int64_t rows = size(a[1], 0), D = size(a[1], 2), keys = size(a[2], 0);
    const char* const names[9] = {"grad_out", "q", "k", "v", "out", "lse", "grad_q", "grad_k", "grad_v"};
    const bool of_keys[9] = {false, false, true, true, false, false, false, true, true};
    sc_heads h[9];
    for (int i = 0; i < 9; ++i) {
        tensor_given(a[i], names[i]);
        if (i == 5) continue;
        h[i] = heads_of(a[i], names[i], of_keys[i] ? keys : rows, D);
        check_dtype(a[i], names[i], a[1]);
        if (h[i].heads != size(a[of_keys[i] ? 2 : 1], 1)) fail_on(PyExc_ValueError, names[i], "has another number of heads");
    }
    const Scenes s = scenes_of(a[9], a[10], a[11], rows, keys);
    const float* lse = floats_of(a[5], "lse", {rows, size(a[1], 1)});
    all_on_device(a, 16);
    return unlocked(row_lib.attention_bwd, &h[0], &h[1], &h[2], &h[3], &h[4], lse, rows, keys, count32(D), s.q_starts, s.k_starts, s.k_lens, s.scenes, small_int(a[12]),
                    number(a[13]), &h[6], &h[7], &h[8], dtype(a[1]), ptr(a[14]), nbytes(a[14]), stream(a[15]));
}

int scenes_of_starts(PyObject* starts) {
    const int64_t scenes = starts == Py_None ? 1 : size(starts, 0) - 1;
    if (scenes < 1 || scenes > SC_SCENES_MAX) fail(PyExc_ValueError, "starts must be int32 [scenes + 1]");
    return (int)scenes;
}
int group_norm_fwd(Args a) {             // x, out, groups, starts, gain, bias, act, eps, stats, workspace, stream
    const Rows x = rows_of(tensor_given(a[0], "x"), "x"), out = rows_of(tensor_given(a[1], "out"), "out");
    const int scenes = scenes_of_starts(a[3]), groups = small_int(a[2]);
    check_rows(out, a[1], "out", x.n, x.C);
    check_block(a[4], "gain", {x.C});
    check_block(a[5], "bias", {x.C});
    for (const int i : {1, 4, 5}) check_dtype(a[i], "an argument", a[0]);
    const int32_t* starts = list_of(a[3], "starts", scenes + 1);
    float* stats = floats_of(a[8], "stats", {scenes, groups, 2});
    all_on_device(a, 11);
    return unlocked(row_lib.group_norm_fwd, x.data, x.ld, x.n, starts, scenes, (int)x.C, groups, ptr(a[4]), ptr(a[5]), number(a[7]), small_int(a[6]), out.data, out.ld,
                    stats, dtype(a[0]), ptr(a[9]), nbytes(a[9]), stream(a[10]));
}
int group_norm_bwd(Args a) {             // grad_out, x, stats, grad_x, groups, starts, gain, bias, act, grad_gain, grad_bias, workspace, stream
    const Rows grad = rows_of(tensor_given(a[0], "grad_out"), "grad_out"), x = rows_of(tensor_given(a[1], "x"), "x"), grad_x = rows_of(a[3], "grad_x");
    const int scenes = scenes_of_starts(a[5]), groups = small_int(a[4]);
    check_rows(grad, a[0], "grad_out", x.n, x.C);
    check_rows(grad_x, a[3], "grad_x", x.n, x.C);
    const char* const names[4] = {"gain", "bias", "grad_gain", "grad_bias"};
    const int of_channels[4] = {6, 7, 9, 10};
    for (int i = 0; i < 4; ++i) check_block(a[of_channels[i]], names[i], {x.C});
    for (const int i : {0, 3, 6, 7, 9, 10}) check_dtype(a[i], "an argument", a[1]);
    const int32_t* starts = list_of(a[5], "starts", scenes + 1);
    const float* stats = floats_of(tensor_given(a[2], "stats"), "stats", {scenes, groups, 2});
    all_on_device(a, 13);
    return unlocked(row_lib.group_norm_bwd, grad.data, grad.ld, x.data, x.ld, x.n, starts, scenes, (int)x.C, groups, ptr(a[6]), ptr(a[7]), small_int(a[8]), stats,
                    grad_x.data, grad_x.ld, ptr(a[9]), ptr(a[10]), dtype(a[1]), ptr(a[11]), nbytes(a[11]), stream(a[12]));
}

template <int (*F)(Args), int N>
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != N) {
        PyErr_Format(PyExc_TypeError, "%d arguments expected, %zd given", N, nargs);
        return nullptr;
    }
    try {
        return PyLong_FromLong(F(args));
    } catch (const PyFailure&) {
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// the addresses of the C functions, in the order of L's members
template <class L, L& TARGET>
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    void* addr[sizeof(L) / sizeof(void*)];
    if (nargs != (Py_ssize_t)(sizeof(L) / sizeof(void*))) {
        PyErr_SetString(PyExc_TypeError, "one address per function expected");
        return nullptr;
    }
    for (Py_ssize_t i = 0; i < nargs; ++i) {
        addr[i] = PyLong_AsVoidPtr(args[i]);
        if (addr[i] == nullptr) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null function address");
            return nullptr;
        }
    }
    memcpy(&TARGET, addr, sizeof TARGET);
    Py_RETURN_NONE;
}

#define SC_METHOD(name, nargs) {#name, (PyCFunction)(void (*)(void))call<name, nargs>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)(void))bind<Lib, lib>, METH_FASTCALL, nullptr},
    {"bind_rows", (PyCFunction)(void (*)(void))bind<RowLib, row_lib>, METH_FASTCALL, nullptr},
    SC_METHOD(hash_build, 4),
    SC_METHOD(hash_rebuild, 5),
    SC_METHOD(kmap_build, 10),
    SC_METHOD(kmap_build_noalloc, 9),
    SC_METHOD(kmap_transpose, 7),
    SC_METHOD(grid_build, 6),
    SC_METHOD(kmap_build_grid, 8),
    SC_METHOD(conv_fwd, 11),
    SC_METHOD(conv_fwd_packed, 11),
    SC_METHOD(conv_up_fwd, 8),
    SC_METHOD(conv_fwd_grid, 10),
    SC_METHOD(linear_fwd, 8),
    SC_METHOD(linear_bwd, 10),
    SC_METHOD(grouped_fwd, 9),
    SC_METHOD(grouped_bwd, 13),
    SC_METHOD(qk_rope_fwd, 11),
    SC_METHOD(qk_rope_bwd, 16),
    SC_METHOD(attention_fwd, 12),
    SC_METHOD(attention_bwd, 16),
    SC_METHOD(group_norm_fwd, 11),
    SC_METHOD(group_norm_bwd, 13),
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", "argument marshalling for libsc's calls", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&module); }
