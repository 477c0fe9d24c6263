// Native half of the Python binding: argument marshalling, output allocation and the call into libhalo's C ABI in one step.
//
// What it is for: a small layer's step is bound by the host.  Through ctypes one forward call cost 19.5 us, of which only
// 5 us are the two kernel launches: five torch.empty (1.7 us each), the current stream (2.9 us) and the conversion of the
// arguments make up the rest.  Here a tensor costs 0.4 us (the caching allocator called directly) and the stream 0.15 us.
//
// Every function takes positional arguments, tensors or None, and returns the outputs, or the halo_status of a failed call
// as an int.  binding.py holds the public signatures and documentation.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/EmptyTensor.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/Allocator.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <vector>

#include "halo.h"

namespace {

PyObject* g_get_device = nullptr;       // torch._C._cuda_getDevice
PyObject* g_get_raw_stream = nullptr;   // torch._C._cuda_getCurrentRawStream

PyObject* g_out_of_memory = nullptr;    // torch.OutOfMemoryError

struct Failed {};                       // a Python exception is set

const at::Tensor* tensor(PyObject* o) {
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) {
        PyErr_SetString(PyExc_TypeError, "expected a tensor or None");
        throw Failed();
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda()) {
        PyErr_SetString(PyExc_ValueError, "libhalo takes device tensors only");
        throw Failed();
    }
    return &t;
}

void require(bool ok, const char* what) {
    if (ok) return;
    PyErr_SetString(PyExc_AssertionError, what);
    throw Failed();
}

long integer(PyObject* o) {
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw Failed();
    return v;
}

double real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Failed();
    return v;
}

// A Python integer from 0 to 2^64 - 1.
uint64_t word64(PyObject* o) {
    const unsigned long long v = PyLong_AsUnsignedLongLong(o);
    if (v == (unsigned long long)-1 && PyErr_Occurred()) throw Failed();
    return v;
}

void* data(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
size_t bytes(const at::Tensor* t) { return t ? (size_t)t->numel() : 0; }      // workspaces are uint8

// True if at::empty would do nothing but allocate: no dispatch mode, functorch transform or tracer sees tensors being made.
bool plain_creation() {
    const c10::DispatchKeySet on = c10::impl::tls_local_dispatch_key_set().included_;
    return (on - c10::default_included_set - c10::autocast_dispatch_keyset).empty();
}

at::Tensor new_tensor(at::IntArrayRef size, at::ScalarType dtype, const at::Tensor& like, int current_device) {
    if (!plain_creation() || like.device().index() != current_device)
        return at::empty(size, at::TensorOptions().dtype(dtype).device(like.device()));
    // the allocator that torch.empty uses for device memory, taken from a tensor that it made
    static c10::Allocator* const allocator =
        at::empty({1}, at::TensorOptions().dtype(at::kByte).device(like.device())).storage().allocator();
    if (!allocator) return at::empty(size, at::TensorOptions().dtype(dtype).device(like.device()));
    return at::Tensor(at::detail::empty_generic(size, allocator, c10::DispatchKeySet(c10::DispatchKey::CUDA), dtype,
                                                std::nullopt));
}

// [rows, cols] whose row pitch is a multiple of 16 bytes (the ABI's alignment rule).
at::Tensor new_padded(int64_t rows, int64_t cols, at::ScalarType dtype, const at::Tensor& like, int device) {
    const int64_t per16 = 16 / (int64_t)c10::elementSize(dtype);
    int64_t ld = (cols + per16 - 1) / per16 * per16;
    if (ld < per16) ld = per16;
    at::Tensor t = new_tensor({rows, ld}, dtype, like, device);
    return ld == cols ? t : t.narrow(1, 0, cols);
}

struct Context {
    int device;
    void* stream;
    Context() {
        PyObject* d = PyObject_CallNoArgs(g_get_device);
        if (!d) throw Failed();
        PyObject* s = PyObject_CallOneArg(g_get_raw_stream, d);
        device = (int)PyLong_AsLong(d);
        Py_DECREF(d);
        if (!s) throw Failed();
        stream = PyLong_AsVoidPtr(s);
        Py_DECREF(s);
    }
};

// The halo_linear_desc inside a ctypes structure.
struct Desc {
    Py_buffer view;
    const halo_linear_desc* d;
    explicit Desc(PyObject* o) {
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw Failed();
        d = reinterpret_cast<const halo_linear_desc*>(view.buf);
        if ((size_t)view.len != sizeof(halo_linear_desc)) {
            PyBuffer_Release(&view);
            PyErr_SetString(PyExc_TypeError, "expected a LinearDesc");
            throw Failed();
        }
    }
    ~Desc() { PyBuffer_Release(&view); }
    Desc(const Desc&) = delete;
    at::ScalarType out_type() const { return d->out_dt == HALO_BF16 ? at::kBFloat16 : at::kFloat; }
};

PyObject* wrap(const at::Tensor& t) { return THPVariable_Wrap(t); }
PyObject* wrap_or_none(bool want, const at::Tensor& t) {
    if (want) return THPVariable_Wrap(t);
    Py_RETURN_NONE;
}

// None, or [rows, cols] of the type with contiguous rows.
bool matrix(const at::Tensor* t, int64_t rows, int64_t cols, at::ScalarType dtype) {
    return !t || (t->dim() == 2 && t->size(0) == rows && t->size(1) == cols && t->scalar_type() == dtype &&
                  (rows == 0 || cols <= 1 || t->stride(1) == 1));
}
// Elements from row to row; that of a matrix of one row does not matter.
int64_t pitch(const at::Tensor* t) { return !t ? 0 : t->size(0) > 1 ? t->stride(0) : (t->size(1) + 7) / 8 * 8; }

// The given output, or a new one.
at::Tensor output(const at::Tensor* given, bool want, at::IntArrayRef size, at::ScalarType dtype, const at::Tensor& like,
                  const Context& c) {
    if (given) return *given;
    return want ? new_tensor(size, dtype, like, c.device) : at::Tensor();
}
void* data(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

bool bf16(const at::Tensor* t) { return t->scalar_type() == at::kBFloat16; }

// f(args...) with the interpreter lock released.  The pointers are arguments, so they are taken before the release: a tensor
// without storage (inside a functorch transform) makes data_ptr() throw, and the handler in entry() needs the lock.
struct ReleaseGil {
    PyThreadState* state = PyEval_SaveThread();
    ~ReleaseGil() { PyEval_RestoreThread(state); }
};
template <class... P, class... A>
halo_status without_gil(halo_status (*f)(P...), A... args) {
    const ReleaseGil released;
    return f(args...);
}

// desc, X, W, Xq, s_x, Wq, s_w, Y, workspace, new_state.  new_state: the caller has no state, the codes and scales are made
// here; otherwise a missing member of its state goes to the C ABI as the null pointer that it is, and is refused there.
PyObject* linear_fwd(PyObject* const* a) {
    const Desc desc(a[0]);
    const halo_linear_desc& d = *desc.d;
    const at::Tensor *X = tensor(a[1]), *W = tensor(a[2]), *xq = tensor(a[3]), *sx = tensor(a[4]), *wq = tensor(a[5]),
                     *sw = tensor(a[6]), *y = tensor(a[7]), *ws = tensor(a[8]);
    const bool make = a[9] == Py_True;
    const at::Tensor* like = X ? X : xq;
    require(like != nullptr, "X or a state is needed");
    require((!X || (bf16(X) && X->is_contiguous())) && (!W || (bf16(W) && W->is_contiguous())), "X and W are contiguous bf16");
    const Context c;
    const at::Tensor Xq = output(xq, make, {d.b, d.m}, at::kChar, *like, c), s_x = output(sx, make, {d.b}, at::kFloat, *like, c),
                     Wq = output(wq, make, {d.n, d.m}, at::kChar, *like, c), s_w = output(sw, make, {d.n}, at::kFloat, *like, c),
                     Y = output(y, true, {d.b, d.n}, desc.out_type(), *like, c);
    at::Tensor scratch;
    if (!ws && d.scale_mode == HALO_SCALE_PER_TENSOR) {
        const size_t need = halo_linear_workspace_bytes(&d);
        scratch = new_tensor({(int64_t)(need > 16 ? need : 16)}, at::kByte, *like, c.device);
        ws = &scratch;
    }
    const halo_status st = without_gil(
        halo_linear_fwd, &d, data(X), data(W), data(Y), (int8_t*)data(Xq), (float*)data(s_x), (int8_t*)data(Wq),
        (float*)data(s_w), data(ws), bytes(ws), c.stream);
    if (st != HALO_OK) return PyLong_FromLong(st);
    return Py_BuildValue("(NNNNN)", wrap(Y), wrap(Xq), wrap(s_x), wrap(Wq), wrap(s_w));
}

// desc, E, Xq, s_x, Wq, s_w, want_ex, want_g, workspace, EX, G
PyObject* linear_bwd(PyObject* const* a) {
    const Desc desc(a[0]);
    const halo_linear_desc& d = *desc.d;
    const at::Tensor *E = tensor(a[1]), *Xq = tensor(a[2]), *s_x = tensor(a[3]), *Wq = tensor(a[4]), *s_w = tensor(a[5]),
                     *ws = tensor(a[8]), *ex = tensor(a[9]), *g = tensor(a[10]);
    const bool want_ex = a[6] == Py_True, want_g = a[7] == Py_True;
    require(E && bf16(E) && E->is_contiguous(), "E is contiguous bf16");
    const Context c;
    const at::Tensor EX = output(ex, want_ex, {d.b, d.m}, desc.out_type(), *E, c),
                     G = output(g, want_g, {d.n, d.m}, desc.out_type(), *E, c);
    at::Tensor scratch;
    if (!ws) {
        const size_t need = halo_linear_workspace_bytes(&d);
        scratch = new_tensor({(int64_t)(need > 1 ? need : 1)}, at::kByte, *E, c.device);
        ws = &scratch;
    }
    const halo_status st = without_gil(
        halo_linear_bwd, &d, data(E), (int8_t*)data(Xq), (float*)data(s_x), (int8_t*)data(Wq), (float*)data(s_w),
        want_ex ? data(EX) : nullptr, want_g ? data(G) : nullptr, data(ws), bytes(ws), c.stream);
    if (st != HALO_OK) return PyLong_FromLong(st);
    return Py_BuildValue("(NN)", wrap_or_none(want_ex, EX), wrap_or_none(want_g, G));
}

// desc, X, Wq, s_w, U, V, workspace, Y, T
PyObject* peft_fwd(PyObject* const* a) {
    const Desc desc(a[0]);
    const halo_linear_desc& d = *desc.d;
    const at::Tensor *X = tensor(a[1]), *Wq = tensor(a[2]), *s_w = tensor(a[3]), *U = tensor(a[4]), *V = tensor(a[5]),
                     *ws = tensor(a[6]), *y = tensor(a[7]), *t = tensor(a[8]);
    require(X && Wq && s_w && U && V && bf16(X) && bf16(U) && bf16(V), "X, U and V are bf16");
    require(X->is_contiguous() && U->is_contiguous() && V->is_contiguous() && Wq->is_contiguous(), "operands are contiguous");
    require(U->dim() == 2 && V->dim() == 2 && V->size(0) == d.n && V->size(1) == U->size(0) && U->size(1) == d.m,
            "U is [rank, m] and V [n, rank]");
    const int64_t rank = U->size(0);
    const Context c;
    const at::Tensor Y = output(y, true, {d.b, d.n}, desc.out_type(), *X, c), T = output(t, true, {d.b, rank}, at::kFloat, *X, c);
    at::Tensor scratch;
    if (!ws) {
        const size_t need = halo_peft_workspace_bytes(&d, (int32_t)rank);
        scratch = new_tensor({(int64_t)(need > 1 ? need : 1)}, at::kByte, *X, c.device);
        ws = &scratch;
    }
    const halo_status st = without_gil(
        halo_peft_fwd, &d, (int32_t)rank, data(X), (int8_t*)data(Wq), (float*)data(s_w), data(U), data(V), data(Y),
        (float*)data(T), data(ws), bytes(ws), c.stream);
    if (st != HALO_OK) return PyLong_FromLong(st);
    return Py_BuildValue("(NN)", wrap(Y), wrap(T));
}

// desc, E, X, T, Wq, s_w, U, V, want_ex, want_gu, want_gv, workspace, EX, GU, GV
PyObject* peft_bwd(PyObject* const* a) {
    const Desc desc(a[0]);
    const halo_linear_desc& d = *desc.d;
    const at::Tensor *E = tensor(a[1]), *X = tensor(a[2]), *T = tensor(a[3]), *Wq = tensor(a[4]), *s_w = tensor(a[5]),
                     *U = tensor(a[6]), *V = tensor(a[7]), *ws = tensor(a[11]), *ex = tensor(a[12]), *gu = tensor(a[13]),
                     *gv = tensor(a[14]);
    const bool want_ex = a[8] == Py_True, want_gu = a[9] == Py_True, want_gv = a[10] == Py_True;
    require(U && U->dim() == 2 && E && bf16(E) && E->is_contiguous(), "E is contiguous bf16");
    const int64_t rank = U->size(0);
    const Context c;
    const at::Tensor EX = output(ex, want_ex, {d.b, d.m}, desc.out_type(), *E, c),
                     GU = output(gu, want_gu, {rank, d.m}, at::kFloat, *E, c),
                     GV = output(gv, want_gv, {d.n, rank}, at::kFloat, *E, c);
    at::Tensor scratch;
    if (!ws) {
        const size_t need = halo_peft_workspace_bytes(&d, (int32_t)rank);
        scratch = new_tensor({(int64_t)(need > 1 ? need : 1)}, at::kByte, *E, c.device);
        ws = &scratch;
    }
    const halo_status st = without_gil(
        halo_peft_bwd, &d, (int32_t)rank, data(E), data(X), (float*)data(T), (int8_t*)data(Wq), (float*)data(s_w), data(U),
        data(V), want_ex ? data(EX) : nullptr, want_gu ? (float*)data(GU) : nullptr, want_gv ? (float*)data(GV) : nullptr,
        data(ws), bytes(ws), c.stream);
    if (st != HALO_OK) return PyLong_FromLong(st);
    return Py_BuildValue("(NNN)", wrap_or_none(want_ex, EX), wrap_or_none(want_gu, GU), wrap_or_none(want_gv, GV));
}

// x, had_block, out_codes, out_scales
PyObject* mx6_quant(PyObject* const* a) {
    const at::Tensor *x = tensor(a[0]), *codes = tensor(a[2]), *scales = tensor(a[3]);
    require(x && x->dim() == 2 && x->stride(1) == 1 && bf16(x), "x is a bf16 matrix with contiguous rows");
    const int64_t rows = x->size(0), cols = x->size(1);
    const int32_t block = (int32_t)integer(a[1]);
    const Context c;
    const at::Tensor q = output(codes, true, {rows, cols / 32 * 24}, at::kByte, *x, c),
                     s = output(scales, true, {rows, cols / 32}, at::kByte, *x, c);
    const halo_status st = without_gil(
        halo_mx6_quant, data(x), rows, cols, rows ? x->stride(0) : cols, block, (uint8_t*)data(q), rows ? q.stride(0) : 24,
        (uint8_t*)data(s), rows ? s.stride(0) : 1, c.stream);
    if (st != HALO_OK) return PyLong_FromLong(st);
    return Py_BuildValue("(NN)", wrap(q), wrap(s));
}

at::ScalarType out_dtype(long code) { return code == HALO_BF16 ? at::kBFloat16 : at::kFloat; }
halo_dtype dtype_code(const at::Tensor& t) {
    if (t.scalar_type() == at::kBFloat16) return HALO_BF16;
    if (t.scalar_type() == at::kFloat) return HALO_F32;
    PyErr_SetString(PyExc_TypeError, "HALO tensors are bf16 or fp32");
    throw Failed();
}

// a, sa, b, sb, dtype of a new output, out
PyObject* gemm_mx6(PyObject* const* a) {
    const at::Tensor *A = tensor(a[0]), *sa = tensor(a[1]), *B = tensor(a[2]), *sb = tensor(a[3]), *out = tensor(a[5]);
    require(A && sa && B && sb && A->dim() == 2 && B->dim() == 2 && sa->dim() == 2 && sb->dim() == 2, "operands are matrices");
    const int64_t M = A->size(0), N = B->size(0), K = sa->size(1) * 32;
    require(A->size(1) == K / 32 * 24 && B->size(1) == K / 32 * 24 && sb->size(1) * 32 == K, "codes and scales fit together");
    const long code = integer(a[4]);
    const Context c;
    const at::Tensor C = out ? *out : new_padded(M, N, out_dtype(code), *A, c.device);
    const halo_dtype dt = dtype_code(C);
    const halo_status st = without_gil(
        halo_gemm_mx6, (uint8_t*)data(A), M ? A->stride(0) : 24, (uint8_t*)data(sa), M ? sa->stride(0) : 4, (uint8_t*)data(B),
        N ? B->stride(0) : 24, (uint8_t*)data(sb), N ? sb->stride(0) : 4, M, N, K, data(C), dt, M ? C.stride(0) : N, c.stream);
    if (st != HALO_OK) return PyLong_FromLong(st);
    return wrap(C);
}

// x, axis, had_block, had_block_left, fold, out_q, out_scale, workspace
PyObject* hadamard_quant(PyObject* const* a) {
    const at::Tensor *x = tensor(a[0]), *fold = tensor(a[4]), *oq = tensor(a[5]), *os = tensor(a[6]), *ws = tensor(a[7]);
    require(x && x->dim() == 2 && x->stride(1) == 1, "x is a matrix with contiguous rows");
    const int64_t rows = x->size(0), cols = x->size(1);
    const halo_axis axis = (halo_axis)integer(a[1]);
    const int32_t block = (int32_t)integer(a[2]), left = (int32_t)integer(a[3]);
    const int64_t qr = axis == HALO_QUANT_ROWS ? rows : cols, qc = axis == HALO_QUANT_ROWS ? cols : rows;
    const halo_dtype dt = dtype_code(*x);
    const Context c;
    const at::Tensor q = oq ? *oq : new_padded(qr, qc, at::kChar, *x, c.device), s = output(os, true, {qr}, at::kFloat, *x, c);
    const size_t need = halo_hadamard_quant_workspace_bytes(rows, cols, axis, left);
    at::Tensor scratch;
    if (!ws && need) {
        scratch = new_tensor({(int64_t)need}, at::kByte, *x, c.device);
        ws = &scratch;
    }
    const halo_status st = without_gil(
        halo_hadamard_quant, data(x), dt, rows, cols, rows ? x->stride(0) : cols, axis, block, left, (float*)data(fold),
        (int8_t*)data(q), q.numel() ? q.stride(0) : qc, (float*)data(s), data(ws), bytes(ws), c.stream);
    if (st != HALO_OK) return PyLong_FromLong(st);
    return Py_BuildValue("(NN)", wrap(q), wrap(s));
}

// a, b, trans_b, row_scale, col_scale, dtype of a new output (-1: none), want_acc, out, acc_out
PyObject* gemm_i8(PyObject* const* a) {
    const at::Tensor *A = tensor(a[0]), *B = tensor(a[1]), *rs = tensor(a[3]), *cs = tensor(a[4]), *out = tensor(a[7]),
                     *acc = tensor(a[8]);
    require(A && B && A->scalar_type() == at::kChar && B->scalar_type() == at::kChar && A->dim() == 2 && B->dim() == 2,
            "operands are int8 matrices");
    const bool trans = PyObject_IsTrue(a[2]) != 0, want_acc = PyObject_IsTrue(a[6]) != 0;
    const int64_t M = A->size(0), K = A->size(1), N = B->size(trans ? 0 : 1);
    require(B->size(trans ? 1 : 0) == K, "operands fit together");
    const long code = integer(a[5]);
    const Context c;
    at::Tensor C = out ? *out : (code >= 0 ? new_padded(M, N, out_dtype(code), *A, c.device) : at::Tensor());
    at::Tensor S = acc ? *acc : (want_acc ? new_padded(M, N, at::kInt, *A, c.device) : at::Tensor());
    const halo_dtype dt = C.defined() ? dtype_code(C) : HALO_F32;
    const halo_status st = without_gil(
        halo_gemm_i8, (int8_t*)data(A), M ? A->stride(0) : K, (int8_t*)data(B), B->size(0) ? B->stride(0) : B->size(1),
        trans ? 1 : 0, M, N, K, (float*)data(rs), (float*)data(cs), data(C), dt, C.defined() ? (M ? C.stride(0) : N) : 0,
        (int32_t*)data(S), S.defined() ? (M ? S.stride(0) : N) : 0, c.stream);
    if (st != HALO_OK) return PyLong_FromLong(st);
    return Py_BuildValue("(NN)", wrap_or_none(C.defined(), C), wrap_or_none(S.defined(), S));
}

// x, p, seed, offset, residual, out
PyObject* dropout(PyObject* const* a) {
    const at::Tensor *x = tensor(a[0]), *res = tensor(a[4]), *out = tensor(a[5]);
    require(x && x->dim() == 2 && matrix(x, x->size(0), x->size(1), x->scalar_type()), "x is a matrix with contiguous rows");
    const int64_t rows = x->size(0), cols = x->size(1);
    require(matrix(res, rows, cols, x->scalar_type()) && matrix(out, rows, cols, x->scalar_type()),
            "residual and out are matrices like x, with contiguous rows");
    const double p = real(a[1]);
    const uint64_t seed = word64(a[2]), offset = word64(a[3]);
    const halo_dtype dt = dtype_code(*x);
    const Context c;
    const at::Tensor y = out ? *out : new_padded(rows, cols, x->scalar_type(), *x, c.device);
    const halo_status st = without_gil(halo_dropout, data(x), dt, rows, cols, pitch(x), data(res), pitch(res), p, seed, offset, data(y),
                                       pitch(&y), c.stream);
    if (st != HALO_OK) return PyLong_FromLong(st);
    return wrap(y);
}

// What both passes of the adapters take.
struct Adapters {
    const at::Tensor *U, *V, *of, *ranks, *scale;
    halo_adapters_desc d{};
    Adapters(PyObject* u, PyObject* v, PyObject* adapter_of, PyObject* rank, PyObject* s, const at::Tensor* rows, long out_code,
             PyObject* p, PyObject* seed, PyObject* offset)
        : U(tensor(u)), V(tensor(v)), of(tensor(adapter_of)), ranks(tensor(rank)), scale(tensor(s)) {
        require(U && V && of && rows, "U, V, adapter_of and the tokens are needed");
        require(bf16(U) && bf16(V) && U->is_contiguous() && V->is_contiguous() && U->dim() == 3 && V->dim() == 3 &&
                    U->size(0) == V->size(0) && U->size(1) == V->size(2),
                "U [slots, max_rank, m] and V [slots, n, max_rank] are contiguous bf16");
        d.b = rows->size(0); d.m = U->size(2); d.n = V->size(1);
        // the library does nothing without either, and what it has not written is no result
        require(d.m > 0 && d.n > 0, "U and V have in- and out-features");
        require(U->size(0) <= INT32_MAX && U->size(1) <= INT32_MAX, "the pool is too large");
        d.slots = (int32_t)U->size(0); d.max_rank = (int32_t)U->size(1);
        require(of->scalar_type() == at::kInt && of->is_contiguous() && of->dim() == 1 && of->size(0) == d.b, "adapter_of is int32 [b]");
        require(!ranks || (ranks->scalar_type() == at::kInt && ranks->is_contiguous() && ranks->numel() == d.slots), "ranks is int32 [slots]");
        require(!scale || (scale->scalar_type() == at::kFloat && scale->is_contiguous() && scale->numel() == d.slots), "scale is fp32 [slots]");
        d.out_dt = (int32_t)out_code;
        d.dropout_p = real(p); d.seed = word64(seed); d.offset = word64(offset);
    }
    at::ScalarType out_type() const { return out_dtype(d.out_dt); }
    at::Tensor workspace(const at::Tensor* given, size_t need, const Context& c) const {
        if (given) return *given;
        return new_tensor({(int64_t)(need > 16 ? need : 16)}, at::kByte, *U, c.device);
    }
};

// X, U, V, adapter_of, ranks, scale, base, dtype of Y, p, seed, offset, Y, T, workspace
PyObject* adapters_fwd(PyObject* const* a) {
    const at::Tensor *X = tensor(a[0]), *base = tensor(a[6]), *y = tensor(a[11]), *t = tensor(a[12]), *ws = tensor(a[13]);
    require(X && X->dim() == 2, "X is a bf16 matrix with contiguous rows");
    const Adapters f(a[1], a[2], a[3], a[4], a[5], X, integer(a[7]), a[8], a[9], a[10]);
    const halo_adapters_desc& d = f.d;
    require(matrix(X, d.b, d.m, at::kBFloat16), "X is a bf16 matrix with contiguous rows");
    require(matrix(base, d.b, d.n, f.out_type()) && matrix(y, d.b, d.n, f.out_type()), "base and Y are [b, n] of the output's type");
    require(!t || (matrix(t, d.b, d.max_rank, at::kFloat) && t->is_contiguous()), "T is fp32 [b, max_rank]");
    const Context c;
    const at::Tensor Y = output(y, true, {d.b, d.n}, f.out_type(), *X, c), T = output(t, true, {d.b, d.max_rank}, at::kFloat, *X, c),
                     W = f.workspace(ws, halo_adapters_fwd_workspace_bytes(&d), c);
    const halo_status st = without_gil(
        halo_adapters_fwd, &d, data(X), pitch(X), data(f.U), data(f.V), (int32_t*)data(f.ranks), (float*)data(f.scale),
        (int32_t*)data(f.of), data(base), pitch(base), data(Y), pitch(&Y), (float*)data(T), data(W), bytes(&W), c.stream);
    if (st != HALO_OK) return PyLong_FromLong(st);
    return Py_BuildValue("(NN)", wrap(Y), wrap(T));
}

// E, X, T, U, V, adapter_of, ranks, scale, base, dtype of EX, p, seed, offset, want_ex, want_gu, want_gv, EX, GU, GV, workspace
PyObject* adapters_bwd(PyObject* const* a) {
    const at::Tensor *E = tensor(a[0]), *X = tensor(a[1]), *T = tensor(a[2]), *base = tensor(a[8]), *ex = tensor(a[16]),
                     *gu = tensor(a[17]), *gv = tensor(a[18]), *ws = tensor(a[19]);
    const bool want_ex = a[13] == Py_True, want_gu = a[14] == Py_True, want_gv = a[15] == Py_True;
    require(E && E->dim() == 2, "E is a bf16 matrix with contiguous rows");
    const Adapters f(a[3], a[4], a[5], a[6], a[7], E, integer(a[9]), a[10], a[11], a[12]);
    const halo_adapters_desc& d = f.d;
    require(matrix(E, d.b, d.n, at::kBFloat16) && matrix(X, d.b, d.m, at::kBFloat16), "E and X are bf16 matrices with contiguous rows");
    require(!T || (matrix(T, d.b, d.max_rank, at::kFloat) && T->is_contiguous()), "T is fp32 [b, max_rank]");
    require(matrix(base, d.b, d.m, f.out_type()) && matrix(ex, d.b, d.m, f.out_type()), "base and EX are [b, m] of the output's type");
    require(!gu || (gu->scalar_type() == at::kFloat && gu->is_contiguous() && gu->sizes() == f.U->sizes()), "GU is fp32, shaped like U");
    require(!gv || (gv->scalar_type() == at::kFloat && gv->is_contiguous() && gv->sizes() == f.V->sizes()), "GV is fp32, shaped like V");
    const Context c;
    const at::Tensor EX = output(want_ex ? ex : nullptr, want_ex, {d.b, d.m}, f.out_type(), *E, c),
                     GU = output(want_gu ? gu : nullptr, want_gu, f.U->sizes(), at::kFloat, *E, c),
                     GV = output(want_gv ? gv : nullptr, want_gv, f.V->sizes(), at::kFloat, *E, c),
                     W = f.workspace(ws, halo_adapters_bwd_workspace_bytes(&d), c);
    const halo_status st = without_gil(
        halo_adapters_bwd, &d, data(E), pitch(E), data(X), pitch(X), (float*)data(T), data(f.U), data(f.V), (int32_t*)data(f.ranks),
        (float*)data(f.scale), (int32_t*)data(f.of), data(base), pitch(base), data(EX), want_ex ? pitch(&EX) : 0, (float*)data(GU),
        (float*)data(GV), data(W), bytes(&W), c.stream);
    if (st != HALO_OK) return PyLong_FromLong(st);
    return Py_BuildValue("(NNN)", wrap_or_none(want_ex, EX), wrap_or_none(want_gu, GU), wrap_or_none(want_gv, GV));
}

// What runs on the current device's stream has its memory there.
void on_current_device(const Context& c, std::initializer_list<const at::Tensor*> all) {
    for (const at::Tensor* t : all) {
        if (!t || t->device().index() == c.device) continue;
        PyErr_SetString(PyExc_ValueError, "tensors are on the current device");
        throw Failed();
    }
}
// None, or a dense vector of n elements, of one of the two types.
bool vector_of(const at::Tensor* t, int64_t n) {
    return !t || (t->dim() == 1 && t->size(0) == n && t->is_contiguous() &&
                  (t->scalar_type() == at::kBFloat16 || t->scalar_type() == at::kFloat));
}
bool floats(const at::Tensor* t, int64_t n) { return vector_of(t, n) && (!t || t->scalar_type() == at::kFloat); }
at::Tensor scratch_of(const at::Tensor* given, size_t need, const at::Tensor& like, const Context& c) {
    return given ? *given : new_tensor({(int64_t)(need > 16 ? need : 16)}, at::kByte, like, c.device);
}

// bias, activation, residual, want_z, Z of a product [M x N] of the type
struct Epilogue {
    const at::Tensor *bias, *residual;
    at::Tensor Z;
    halo_epilogue e{};
    bool want_z;
    Epilogue(PyObject* b, PyObject* act, PyObject* res, PyObject* want, PyObject* z, int64_t M, int64_t N, at::ScalarType type,
             const at::Tensor& like, const Context& c, bool padded)
        : bias(tensor(b)), residual(tensor(res)), want_z(want == Py_True || z != Py_None) {
        const at::Tensor* given = tensor(z);
        require(vector_of(bias, N), "bias is a bf16 or fp32 vector, one element for each column");
        require(matrix(residual, M, N, type) && matrix(given, M, N, type), "residual and Z are matrices like the output, with contiguous rows");
        if (given) Z = *given;
        else if (want_z) Z = padded ? new_padded(M, N, type, like, c.device) : new_tensor({M, N}, type, like, c.device);
        e.bias = data(bias); e.bias_dt = bias ? dtype_code(*bias) : HALO_F32;
        e.activation = (int32_t)integer(act);
        e.residual = data(residual); e.ld_res = pitch(residual);
        e.Z = data(Z); e.ld_z = Z.defined() ? pitch(&Z) : 0;
        on_current_device(c, {bias, residual, given});
    }
};

// a, b, row_scale, col_scale, bias, activation, residual, dtype of a new output, want_z, out, Z
PyObject* gemm_i8_epilogue(PyObject* const* a) {
    const at::Tensor *A = tensor(a[0]), *B = tensor(a[1]), *rs = tensor(a[2]), *cs = tensor(a[3]), *out = tensor(a[9]);
    require(A && B && A->dim() == 2 && B->dim() == 2 && A->size(1) == B->size(1), "operands are int8 matrices that fit together");
    const int64_t M = A->size(0), K = A->size(1), N = B->size(0);
    require(matrix(A, M, K, at::kChar) && matrix(B, N, K, at::kChar), "operands are int8 matrices with contiguous rows");
    require(floats(rs, M) && floats(cs, N), "row_scale is fp32 [M], col_scale fp32 [N]");
    const at::ScalarType type = out ? out->scalar_type() : out_dtype(integer(a[7]));
    require(matrix(out, M, N, type), "out is [M, N] with contiguous rows");
    const Context c;
    on_current_device(c, {A, B, rs, cs, out});
    const at::Tensor C = out ? *out : new_padded(M, N, type, *A, c.device);
    const Epilogue f(a[4], a[5], a[6], a[8], a[10], M, N, type, *A, c, true);
    // the pitch of a matrix of one row does not matter, but has to be one that int8 rows can have
    const int64_t lda = M > 1 ? A->stride(0) : (K + 15) / 16 * 16, ldb = N > 1 ? B->stride(0) : (K + 15) / 16 * 16;
    const halo_gemm_desc g{(int8_t*)data(A), lda, (int8_t*)data(B), ldb, 1, M, N, K, (float*)data(rs), (float*)data(cs), data(C),
                           (int32_t)dtype_code(C), pitch(&C), nullptr, 0, HALO_GEMM_AUTO};
    const halo_status st = without_gil(halo_gemm_i8_epilogue, &g, &f.e, c.stream);
    if (st != HALO_OK) return PyLong_FromLong(st);
    return Py_BuildValue("(NN)", wrap(C), wrap_or_none(f.want_z, f.Z));
}

// desc, X, W, Xq, s_x, Wq, s_w, Y, workspace, new_state, bias, activation, residual, want_z, Z
PyObject* linear_fwd_epilogue(PyObject* const* a) {
    const Desc desc(a[0]);
    const halo_linear_desc& d = *desc.d;
    const at::Tensor *X = tensor(a[1]), *W = tensor(a[2]), *xq = tensor(a[3]), *sx = tensor(a[4]), *wq = tensor(a[5]),
                     *sw = tensor(a[6]), *y = tensor(a[7]), *ws = tensor(a[8]);
    const bool make = a[9] == Py_True;
    const at::Tensor* like = X ? X : xq;
    require(like != nullptr, "X or a state is needed");
    require((!X || (matrix(X, d.b, d.m, at::kBFloat16) && X->is_contiguous())) && (!W || (matrix(W, d.n, d.m, at::kBFloat16) && W->is_contiguous())),
            "X [b, m] and W [n, m] are contiguous bf16");
    require(!y || (matrix(y, d.b, d.n, desc.out_type()) && y->is_contiguous()), "Y is [b, n] of the output's type, contiguous");
    const Context c;
    on_current_device(c, {X, W, xq, sx, wq, sw, y, ws});
    const at::Tensor Xq = output(xq, make, {d.b, d.m}, at::kChar, *like, c), s_x = output(sx, make, {d.b}, at::kFloat, *like, c),
                     Wq = output(wq, make, {d.n, d.m}, at::kChar, *like, c), s_w = output(sw, make, {d.n}, at::kFloat, *like, c),
                     Y = output(y, true, {d.b, d.n}, desc.out_type(), *like, c);
    const Epilogue f(a[10], a[11], a[12], a[13], a[14], d.b, d.n, desc.out_type(), *like, c, false);
    at::Tensor scratch;
    if (!ws && d.scale_mode == HALO_SCALE_PER_TENSOR) {
        scratch = scratch_of(nullptr, halo_linear_workspace_bytes(&d), *like, c);
        ws = &scratch;
    }
    const halo_status st = without_gil(
        halo_linear_fwd_epilogue, &d, data(X), data(W), data(Y), (int8_t*)data(Xq), (float*)data(s_x), (int8_t*)data(Wq),
        (float*)data(s_w), &f.e, data(ws), bytes(ws), c.stream);
    if (st != HALO_OK) return PyLong_FromLong(st);
    return Py_BuildValue("(NNNNNN)", wrap(Y), wrap(Xq), wrap(s_x), wrap(Wq), wrap(s_w), wrap_or_none(f.want_z, f.Z));
}

// E, Z, activation, want_ez, want_gb, EZ, GB, workspace
PyObject* activation_bwd(PyObject* const* a) {
    const at::Tensor *E = tensor(a[0]), *Z = tensor(a[1]), *ez = tensor(a[5]), *gb = tensor(a[6]), *ws = tensor(a[7]);
    const long act = integer(a[2]);
    const bool want_ez = a[3] == Py_True, want_gb = a[4] == Py_True;
    require(E && E->dim() == 2, "E is a matrix with contiguous rows");
    const int64_t rows = E->size(0), cols = E->size(1);
    const at::ScalarType type = E->scalar_type();
    const halo_dtype dt = dtype_code(*E);
    require(matrix(E, rows, cols, type) && matrix(Z, rows, cols, type) && matrix(ez, rows, cols, type),
            "E, Z and EZ are matrices of one shape and type, with contiguous rows");
    require(floats(gb, cols), "GB is fp32, one element for each column");
    const Context c;
    on_current_device(c, {E, Z, ez, gb, ws});
    const at::Tensor EZ = want_ez && !ez ? new_padded(rows, cols, type, *E, c.device) : output(want_ez ? ez : nullptr, false, {}, type, *E, c),
                     GB = output(want_gb ? gb : nullptr, want_gb, {cols}, at::kFloat, *E, c);
    at::Tensor W;
    if (want_gb) W = scratch_of(ws, halo_activation_bwd_workspace_bytes(rows, cols), *E, c);
    const halo_status st = without_gil(halo_activation_bwd, data(E), pitch(E), data(Z), pitch(Z), dt, rows, cols, (halo_activation)act, data(EZ),
                                       want_ez ? pitch(&EZ) : 0, (float*)data(GB), data(W), W.defined() ? bytes(&W) : 0, c.stream);
    if (st != HALO_OK) return PyLong_FromLong(st);
    return Py_BuildValue("(NN)", wrap_or_none(want_ez, EZ), wrap_or_none(want_gb, GB));
}

halo_norm_desc norm_desc(const at::Tensor& x, const at::Tensor* weight, const at::Tensor* bias, long kind, double eps) {
    require(vector_of(weight, x.size(1)) && vector_of(bias, x.size(1)) && (!weight || !bias || weight->scalar_type() == bias->scalar_type()),
            "weight and bias are vectors of one type, bf16 or fp32, one element for each column");
    const at::Tensor* w = weight ? weight : bias;
    return halo_norm_desc{x.size(0), x.size(1), (int32_t)kind, (int32_t)dtype_code(x), w ? (int32_t)dtype_code(*w) : (int32_t)HALO_F32, 0, eps};
}

// X, weight, bias, eps, kind, want_stats, Y, mean, rstd
PyObject* layer_norm_fwd(PyObject* const* a) {
    const at::Tensor *X = tensor(a[0]), *w = tensor(a[1]), *b = tensor(a[2]), *y = tensor(a[6]), *m = tensor(a[7]), *r = tensor(a[8]);
    require(X && X->dim() == 2, "X is a matrix with contiguous rows");
    const long kind = integer(a[4]);
    const halo_norm_desc d = norm_desc(*X, w, b, kind, real(a[3]));
    require(matrix(X, d.rows, d.cols, X->scalar_type()) && matrix(y, d.rows, d.cols, X->scalar_type()), "X and Y are matrices of one shape and type, with contiguous rows");
    require(floats(m, d.rows) && floats(r, d.rows), "mean and rstd are fp32, one element for each row");
    const bool stats = a[5] == Py_True, want_mean = (stats || m) && kind == HALO_NORM_LAYER, want_rstd = stats || r;
    require(d.cols > 0 || d.rows == 0 || !(want_mean || want_rstd), "rows without columns have no statistics");
    const Context c;
    on_current_device(c, {X, w, b, y, m, r});
    const at::Tensor Y = y ? *y : new_padded(d.rows, d.cols, X->scalar_type(), *X, c.device),
                     mean = output(want_mean ? m : nullptr, want_mean, {d.rows}, at::kFloat, *X, c),
                     rstd = output(r, want_rstd, {d.rows}, at::kFloat, *X, c);
    const halo_status st = without_gil(halo_layer_norm_fwd, &d, data(X), pitch(X), data(w), data(b), data(Y), pitch(&Y), (float*)data(mean),
                                       (float*)data(rstd), c.stream);
    if (st != HALO_OK) return PyLong_FromLong(st);
    return Py_BuildValue("(NNN)", wrap(Y), wrap_or_none(want_mean, mean), wrap_or_none(want_rstd, rstd));
}

// E, X, mean, rstd, weight, kind, base, want_ex, want_gw, want_gb, EX, GW, GB, workspace
PyObject* layer_norm_bwd(PyObject* const* a) {
    const at::Tensor *E = tensor(a[0]), *X = tensor(a[1]), *m = tensor(a[2]), *r = tensor(a[3]), *w = tensor(a[4]), *base = tensor(a[6]),
                     *ex = tensor(a[10]), *gw = tensor(a[11]), *gb = tensor(a[12]), *ws = tensor(a[13]);
    const bool want_ex = a[7] == Py_True, want_gw = a[8] == Py_True, want_gb = a[9] == Py_True;
    require(E && E->dim() == 2, "E is a matrix with contiguous rows");
    const halo_norm_desc d = norm_desc(*E, w, nullptr, integer(a[5]), 0.0);
    const at::ScalarType type = E->scalar_type();
    require(matrix(E, d.rows, d.cols, type) && matrix(X, d.rows, d.cols, type) && matrix(base, d.rows, d.cols, type) && matrix(ex, d.rows, d.cols, type),
            "E, X, base and EX are matrices of one shape and type, with contiguous rows");
    require(floats(m, d.rows) && floats(r, d.rows), "mean and rstd are fp32, one element for each row");
    require(floats(gw, d.cols) && floats(gb, d.cols), "GW and GB are fp32, one element for each column");
    const Context c;
    on_current_device(c, {E, X, m, r, w, base, ex, gw, gb, ws});
    const at::Tensor EX = want_ex && !ex ? new_padded(d.rows, d.cols, type, *E, c.device) : output(want_ex ? ex : nullptr, false, {}, type, *E, c),
                     GW = output(want_gw ? gw : nullptr, want_gw, {d.cols}, at::kFloat, *E, c),
                     GB = output(want_gb ? gb : nullptr, want_gb, {d.cols}, at::kFloat, *E, c);
    at::Tensor W;
    if (want_gw || want_gb) W = scratch_of(ws, halo_layer_norm_bwd_workspace_bytes(&d), *E, c);
    const halo_status st = without_gil(
        halo_layer_norm_bwd, &d, data(E), pitch(E), data(X), pitch(X), (float*)data(m), (float*)data(r), data(w), data(base), pitch(base), data(EX),
        want_ex ? pitch(&EX) : 0, (float*)data(GW), (float*)data(GB), data(W), W.defined() ? bytes(&W) : 0, c.stream);
    if (st != HALO_OK) return PyLong_FromLong(st);
    return Py_BuildValue("(NNN)", wrap_or_none(want_ex, EX), wrap_or_none(want_gw, GW), wrap_or_none(want_gb, GB));
}

// A list or tuple of tensors, or None (an empty one).
struct Tensors {
    PyObject* fast = nullptr;
    Py_ssize_t n = 0;
    explicit Tensors(PyObject* o) {
        if (o == Py_None) return;
        fast = PySequence_Fast(o, "expected a list of tensors");
        if (!fast) throw Failed();
        n = PySequence_Fast_GET_SIZE(fast);
    }
    ~Tensors() { Py_XDECREF(fast); }
    Tensors(const Tensors&) = delete;
    const at::Tensor* at(Py_ssize_t i) const { return fast ? tensor(PySequence_Fast_GET_ITEM(fast, i)) : nullptr; }
};
// A number, or a tensor of one element of the type: its address, and `none` for the number.
template <class T, class F>
const T* number_or_address(PyObject* o, at::ScalarType type, const Context& c, const F& number) {
    if (!THPVariable_Check(o)) {
        number();
        return nullptr;
    }
    const at::Tensor* t = tensor(o);
    require(t->numel() == 1 && t->scalar_type() == type, "step is int64, lr and grad_scale are fp32, of one element");
    on_current_device(c, {t});
    return (const T*)t->data_ptr();
}

// params, grads, m, v, masters, m_scales, v_scales, step, lr, beta1, beta2, eps, weight_decay, grad_scale, seed, offset
PyObject* adamw(PyObject* const* a) {
    const Tensors p(a[0]), g(a[1]), m(a[2]), v(a[3]), master(a[4]), ms(a[5]), vs(a[6]);
    require(g.n == p.n && m.n == p.n && v.n == p.n && (!master.fast || master.n == p.n) && (!ms.fast || ms.n == p.n) &&
                (!vs.fast || vs.n == p.n),
            "the lists have one entry for each parameter");
    const Context c;
    halo_adamw_desc d{};
    d.state_bits = 32;
    d.step = 1;
    d.step_ptr = number_or_address<int64_t>(a[7], at::kLong, c, [&] { d.step = integer(a[7]); });
    d.lr_ptr = number_or_address<float>(a[8], at::kFloat, c, [&] { d.lr = real(a[8]); });
    d.beta1 = real(a[9]); d.beta2 = real(a[10]); d.eps = real(a[11]); d.weight_decay = real(a[12]);
    d.grad_scale_ptr = number_or_address<float>(a[13], at::kFloat, c, [&] { d.grad_scale = real(a[13]); });
    d.seed = word64(a[14]); d.offset = word64(a[15]);
    std::vector<halo_adamw_tensor> list((size_t)p.n);
    for (Py_ssize_t i = 0; i < p.n; ++i) {
        const at::Tensor *P = p.at(i), *G = g.at(i), *M = m.at(i), *V = v.at(i), *R = master.at(i), *SM = ms.at(i), *SV = vs.at(i);
        require(P && G && M && V, "every parameter has a gradient, m and v");
        const int64_t n = P->numel(), blocks = (n + HALO_ADAMW_BLOCK - 1) / HALO_ADAMW_BLOCK;
        const bool eight = M->scalar_type() == at::kFloat8_e4m3fn;
        for (const at::Tensor* t : {P, G, M, V, R})
            require(!t || (t->numel() == n && t->is_contiguous()), "what belongs to a parameter has its number of elements and is contiguous");
        require(M->scalar_type() == V->scalar_type() && (eight || M->scalar_type() == at::kFloat), "m and v are fp32, or both float8_e4m3fn");
        require(!eight || (SM && SV && floats(SM, blocks) && floats(SV, blocks)), "states in 8 bits have fp32 scales, one for 256 elements");
        require(!R || R->scalar_type() == at::kFloat, "masters are fp32");
        const int32_t pd = dtype_code(*P), gd = dtype_code(*G), bits = eight ? 8 : 32;
        require(i == 0 || (pd == d.param_dt && gd == d.grad_dt && bits == d.state_bits), "all parameters, all gradients and all states have one type");
        d.param_dt = pd; d.grad_dt = gd; d.state_bits = bits;
        on_current_device(c, {P, G, M, V, R, eight ? SM : nullptr, eight ? SV : nullptr});
        list[(size_t)i] = halo_adamw_tensor{n, data(P), data(G), data(M), data(V), (float*)data(R), eight ? (float*)data(SM) : nullptr,
                                            eight ? (float*)data(SV) : nullptr};
    }
    const halo_status st = without_gil(halo_adamw, (const halo_adamw_desc*)&d, (const halo_adamw_tensor*)list.data(), (int32_t)p.n, c.stream);
    if (st != HALO_OK) return PyLong_FromLong(st);
    Py_RETURN_NONE;
}

template <PyObject* (*F)(PyObject* const*), Py_ssize_t N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t count) {
    if (count != N) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", N, count);
        return nullptr;
    }
    try {
        return F(args);
    } catch (const Failed&) {
        return nullptr;
    } catch (const c10::OutOfMemoryError& e) {
        PyErr_SetString(g_out_of_memory, e.what_without_backtrace());
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

#define HALO_ENTRY(F, N) {#F, (PyCFunction)(void (*)(void))entry<F, N>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {HALO_ENTRY(linear_fwd, 10), HALO_ENTRY(linear_bwd, 11), HALO_ENTRY(peft_fwd, 9), HALO_ENTRY(peft_bwd, 15),
                         HALO_ENTRY(mx6_quant, 4),  HALO_ENTRY(gemm_mx6, 6),    HALO_ENTRY(hadamard_quant, 8),
                         HALO_ENTRY(gemm_i8, 9),    HALO_ENTRY(dropout, 6),     HALO_ENTRY(adapters_fwd, 14),
                         HALO_ENTRY(adapters_bwd, 20), HALO_ENTRY(gemm_i8_epilogue, 11), HALO_ENTRY(linear_fwd_epilogue, 15),
                         HALO_ENTRY(activation_bwd, 8), HALO_ENTRY(layer_norm_fwd, 9), HALO_ENTRY(layer_norm_bwd, 14),
                         HALO_ENTRY(adamw, 16), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_halo_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__halo_native(void) {
    PyObject* c = PyImport_ImportModule("torch._C");
    if (!c) return nullptr;
    g_get_device = PyObject_GetAttrString(c, "_cuda_getDevice");
    g_get_raw_stream = PyObject_GetAttrString(c, "_cuda_getCurrentRawStream");
    g_out_of_memory = PyObject_GetAttrString(c, "OutOfMemoryError");
    Py_DECREF(c);
    if (!g_out_of_memory || !g_get_device || !g_get_raw_stream) return nullptr;
    return PyModule_Create(&module);
}
