// Argument marshalling of the calls a decode loop makes for every projection, as a CPython extension: tensors to pointers,
// the checks of binding.py, torch's current stream, and the C ABI call.  No arithmetic and no kernels.
//
// Why native: a small projection takes the GPU 2.6 us (256 x 512) and took the host 9.8 us per call, nearly all of it Python
// attribute look-ups, ctypes conversions and torch.cuda.current_stream().
#include <Python.h>

#include <ATen/cuda/EmptyTensor.h>
#include <ATen/detail/CUDAHooksInterface.h>
#include <ATen/ops/clone.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/vptq.h"

namespace {

PyObject *g_error_class = nullptr;       // binding.VptqError

// The memory of a ctypes structure (or array of them) of at least `bytes` bytes; it stays valid while the object lives.
template <typename T>
const T *struct_of(PyObject *o, Py_ssize_t count = 1)
{
    Py_buffer v;
    if (PyObject_GetBuffer(o, &v, PyBUF_SIMPLE) != 0) return nullptr;
    const T *p = static_cast<const T *>(v.buf);
    const Py_ssize_t len = v.len;
    PyBuffer_Release(&v);
    if (len < count * (Py_ssize_t)sizeof(T)) {
        PyErr_SetString(PyExc_TypeError, "descriptor or pointer structure too small");
        return nullptr;
    }
    return p;
}

const at::Tensor *tensor_of(PyObject *o)
{
    if (!THPVariable_Check(o)) {
        PyErr_SetString(PyExc_TypeError, "a torch tensor was expected");
        return nullptr;
    }
    return &THPVariable_Unpack(o);
}

PyObject *fail(int code)
{
    if (PyErr_Occurred()) return nullptr;
    PyObject *arg = PyLong_FromLong(code);
    PyObject *e = arg && g_error_class ? PyObject_CallOneArg(g_error_class, arg) : nullptr;
    if (e) {
        PyErr_SetObject(g_error_class, e);
        Py_DECREF(e);
    } else if (!PyErr_Occurred()) {
        PyErr_Format(PyExc_RuntimeError, "libvptq error %d", code);
    }
    Py_XDECREF(arg);
    return nullptr;
}

PyObject *assertion(const char *what)
{
    PyErr_SetString(PyExc_AssertionError, what);
    return nullptr;
}

at::ScalarType dtype_of(int32_t code)
{
    return code == VPTQ_DTYPE_FP16 ? at::kHalf : code == VPTQ_DTYPE_BF16 ? at::kBFloat16 : at::kFloat;
}

void *current_stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

// workspace argument: a tensor or None
bool workspace_of(PyObject *o, void **p, size_t *bytes)
{
    *p = nullptr; *bytes = 0;
    if (o == Py_None) return true;
    const at::Tensor *t = tensor_of(o);
    if (!t) return false;
    *p = t->data_ptr();
    *bytes = (size_t)t->nbytes();
    return true;
}

// out = x * W^T for one layer; the checks are those binding.vptq_linear documents
PyObject *call_linear(const vptq_layer_desc *d, const at::Tensor &x, const vptq_layer_ptrs *p, const at::Tensor &out,
                      PyObject *out_obj, void *ws, size_t ws_bytes)
{
    if (!x.is_cuda() || !x.is_contiguous() || !out.is_cuda() || !out.is_contiguous()) return assertion("contiguous CUDA tensors");
    if (x.scalar_type() != dtype_of(d->x_dtype) || out.scalar_type() != dtype_of(d->out_dtype)) return assertion("dtypes of the descriptor");
    if (x.dim() != 2 || out.dim() != 2 || x.size(1) != d->N || out.size(0) != x.size(0) || out.size(1) != d->M)
        return assertion("x [B][N] and out [B][M]");
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = vptq_linear(d, x.data_ptr(), (int32_t)x.size(0), p, out.data_ptr(), ws, ws_bytes, current_stream());
    Py_END_ALLOW_THREADS
    if (rc != VPTQ_OK) return fail(rc);
    Py_INCREF(out_obj);
    return out_obj;
}

// linear(desc, x, ptrs, out, workspace) -> out
PyObject *py_linear(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 5) { PyErr_SetString(PyExc_TypeError, "linear takes 5 arguments"); return nullptr; }
    const vptq_layer_desc *d = struct_of<vptq_layer_desc>(a[0]);
    const at::Tensor *x = d ? tensor_of(a[1]) : nullptr;
    const vptq_layer_ptrs *p = x ? struct_of<vptq_layer_ptrs>(a[2]) : nullptr;
    const at::Tensor *out = p ? tensor_of(a[3]) : nullptr;
    void *ws;
    size_t ws_bytes;
    if (!out || !workspace_of(a[4], &ws, &ws_bytes)) return nullptr;
    return call_linear(d, *x, p, *out, a[3], ws, ws_bytes);
}

// layer_linear(desc, ptrs, workspaces, x, out or None) -> out, or None when `workspaces` (a dict by batch size) has no entry
// for the batch of x
PyObject *py_layer_linear(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 5) { PyErr_SetString(PyExc_TypeError, "layer_linear takes 5 arguments"); return nullptr; }
    const vptq_layer_desc *d = struct_of<vptq_layer_desc>(a[0]);
    const vptq_layer_ptrs *p = d ? struct_of<vptq_layer_ptrs>(a[1]) : nullptr;
    const at::Tensor *x = p ? tensor_of(a[3]) : nullptr;
    if (!x) return nullptr;
    if (x->dim() != 2) return assertion("x [B][N] and out [B][M]");
    PyObject *key = PyLong_FromLongLong(x->size(0));
    PyObject *w = key ? PyDict_GetItemWithError(a[2], key) : nullptr;
    Py_XDECREF(key);
    if (!w) {
        if (PyErr_Occurred()) return nullptr;
        Py_RETURN_NONE;
    }
    void *ws;
    size_t ws_bytes;
    if (!workspace_of(w, &ws, &ws_bytes)) return nullptr;
    if (a[4] != Py_None) {
        const at::Tensor *out = tensor_of(a[4]);
        return out ? call_linear(d, *x, p, *out, a[4], ws, ws_bytes) : nullptr;
    }
    PyObject *out_obj = nullptr;
    try {
        out_obj = THPVariable_Wrap(at::empty({x->size(0), d->M}, x->options().dtype(dtype_of(d->out_dtype))));
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    if (!out_obj) return nullptr;
    PyObject *r = call_linear(d, *x, p, THPVariable_Unpack(out_obj), out_obj, ws, ws_bytes);
    Py_DECREF(out_obj);
    return r;
}

// fused_linear(descs, ptrs, n, workspaces, x, outs) -> outs, or None when `workspaces` has no entry for the batch of x
PyObject *py_fused_linear(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    if (n_args != 6) { PyErr_SetString(PyExc_TypeError, "fused_linear takes 6 arguments"); return nullptr; }
    const long n = PyLong_AsLong(a[2]);
    if (n < 1 || n > VPTQ_MAX_FUSED_LAYERS) return PyErr_Occurred() ? nullptr : fail(VPTQ_E_SHAPE);
    const vptq_layer_desc *d = struct_of<vptq_layer_desc>(a[0], n);
    const vptq_layer_ptrs *p = d ? struct_of<vptq_layer_ptrs>(a[1], n) : nullptr;
    const at::Tensor *x = p ? tensor_of(a[4]) : nullptr;
    if (!x) return nullptr;
    PyObject *key = PyLong_FromLongLong(x->size(0));
    PyObject *w = key ? PyDict_GetItemWithError(a[3], key) : nullptr;
    Py_XDECREF(key);
    if (!w) {
        if (PyErr_Occurred()) return nullptr;
        Py_RETURN_NONE;
    }
    void *ws;
    size_t ws_bytes;
    if (!workspace_of(w, &ws, &ws_bytes)) return nullptr;
    PyObject *outs = PySequence_Fast(a[5], "a sequence of output tensors was expected");
    if (!outs) return nullptr;
    void *op[VPTQ_MAX_FUSED_LAYERS];
    bool ok = PySequence_Fast_GET_SIZE(outs) == n;
    if (!ok) PyErr_SetString(PyExc_ValueError, "one output tensor per layer");
    for (long i = 0; ok && i < n; i++) {
        const at::Tensor *t = tensor_of(PySequence_Fast_GET_ITEM(outs, i));
        ok = t != nullptr;
        if (ok) op[i] = t->data_ptr();
    }
    Py_DECREF(outs);
    if (!ok) return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = vptq_linear_fused(d, p, (int32_t)n, x->data_ptr(), (int32_t)x->size(0), op, ws, ws_bytes, current_stream());
    Py_END_ALLOW_THREADS
    if (rc != VPTQ_OK) return fail(rc);
    Py_INCREF(a[5]);
    return a[5];
}

// dequant(desc, ptrs, W_out) -> W_out (a restored 256 x 256 weight: 11.8 us a call through ctypes, all of it host time)
PyObject *py_dequant(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 3) { PyErr_SetString(PyExc_TypeError, "dequant takes 3 arguments"); return nullptr; }
    const vptq_layer_desc *d = struct_of<vptq_layer_desc>(a[0]);
    const vptq_layer_ptrs *p = d ? struct_of<vptq_layer_ptrs>(a[1]) : nullptr;
    const at::Tensor *w = p ? tensor_of(a[2]) : nullptr;
    if (!w) return nullptr;
    if (!w->is_cuda() || !w->is_contiguous() || w->scalar_type() != at::kHalf) return assertion("a contiguous FP16 CUDA tensor");
    if (w->dim() != 2 || w->size(0) != d->M || w->size(1) != d->N) return assertion("W_out [M][N]");
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = vptq_dequant(d, p, w->data_ptr(), current_stream());
    Py_END_ALLOW_THREADS
    if (rc != VPTQ_OK) return fail(rc);
    Py_INCREF(a[2]);
    return a[2];
}

// ---- 8-bit floating point: these allocate their results (and workspaces) themselves, from torch's allocator -----------------

// a CUDA tensor on the device of the current stream, with memory and strides (a sparse one throws when asked for either), and a contiguous one
bool on_current_device(const at::Tensor &t) { return t.is_cuda() && t.layout() == at::kStrided && t.get_device() == c10::cuda::current_device(); }
bool plain(const at::Tensor &t) { return on_current_device(t) && t.is_contiguous(); }

// workspace argument: a contiguous tensor of the current device (its bytes are written) or None
bool room_of(PyObject *o, void **p, size_t *bytes)
{
    if (o != Py_None) {
        const at::Tensor *t = tensor_of(o);
        if (!t) return false;
        if (!plain(*t)) { assertion("workspace: a contiguous tensor of the current device"); return false; }
    }
    return workspace_of(o, p, bytes);
}

// whether an address that came without a tensor is memory of the current device
bool address_on_current_device(const void *p)
{
    try {
        return at::detail::getCUDAHooks().getDeviceFromPtr(const_cast<void *>(p)).index() == c10::cuda::current_device();
    } catch (const std::exception &) {                                           // (host memory, or no device)
        return false;
    }
}

// runs a call that may throw (torch's allocator, questions that a tensor does not answer) and turns what it throws into a Python error
template <typename F>
PyObject *guarded(F f)
{
    try {
        return f();
    } catch (const std::exception &e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

PyObject *pair_of(const at::Tensor &a, const at::Tensor &b)
{
    PyObject *x = THPVariable_Wrap(a), *y = THPVariable_Wrap(b);
    PyObject *r = x && y ? PyTuple_Pack(2, x, y) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    return r;
}

// tensors of an e4m3 matrix: [rows][pitch] and its scales
struct Fp8Tensors { at::Tensor q, scale; };
Fp8Tensors empty_fp8(int64_t rows, int64_t cols, int64_t block_rows, const at::TensorOptions &options)
{
    return {at::empty({rows, (cols + 15) / 16 * 16}, options.dtype(at::kFloat8_e4m3fn)),
            at::empty({(rows + block_rows - 1) / block_rows, (cols + 127) / 128}, options.dtype(at::kFloat))};
}

// [rows][pitch] e4m3 with [ceil(rows / block_rows)][ceil(pitch / 128)] FP32 scales
bool is_fp8(const at::Tensor &q, const at::Tensor &scale, int64_t rows, int64_t pitch, int64_t block_rows)
{
    return plain(q) && plain(scale) && q.scalar_type() == at::kFloat8_e4m3fn && scale.scalar_type() == at::kFloat && q.dim() == 2 && scale.dim() == 2 &&
           q.size(0) == rows && q.size(1) == pitch && scale.size(0) == (rows + block_rows - 1) / block_rows && scale.size(1) == (pitch + 127) / 128;
}

int32_t code_of(at::ScalarType t)
{
    return t == at::kHalf ? VPTQ_DTYPE_FP16 : t == at::kBFloat16 ? VPTQ_DTYPE_BF16 : t == at::kFloat ? VPTQ_DTYPE_FP32 : t == at::kFloat8_e4m3fn ? VPTQ_DTYPE_E4M3 : -1;
}

// Scales as the C ABI takes them, on a 16-byte boundary.  Part of a stack of them (an expert's, some tokens') starts at any multiple of
// four bytes: that part is copied, on the current stream.
at::Tensor aligned(const at::Tensor &scale)
{
    return (reinterpret_cast<uintptr_t>(scale.data_ptr()) & 15u) == 0 ? scale : scale.detach().clone();
}

constexpr int64_t MAX_INT = 0x7FFFFFFF;

// fp8_quantize(x, block_rows) -> (q, scale)
PyObject *py_fp8_quantize(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 2) { PyErr_SetString(PyExc_TypeError, "fp8_quantize takes 2 arguments"); return nullptr; }
    const at::Tensor *x = tensor_of(a[0]);
    const long block_rows = x ? PyLong_AsLong(a[1]) : -1;
    if (!x || (block_rows == -1 && PyErr_Occurred())) return nullptr;
    if (block_rows != 1 && block_rows != 128) return fail(VPTQ_E_SHAPE);
    if (!on_current_device(*x)) return assertion("a CUDA tensor of the current device");
    if (x->dim() != 2 || x->size(1) < 1 || x->size(0) > MAX_INT || x->size(1) > MAX_INT) return assertion("x [rows][cols]");
    const int64_t rows = x->size(0), cols = x->size(1), ld = rows > 1 ? x->stride(0) : cols;
    if ((cols > 1 && x->stride(1) != 1) || ld < cols) return assertion("a row's columns next to each other, rows apart");
    return guarded([&]() -> PyObject * {
        const Fp8Tensors r = empty_fp8(rows, cols, block_rows, x->options());
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = vptq_fp8_quantize(x->data_ptr(), code_of(x->scalar_type()), (int32_t)rows, (int32_t)cols, ld, (int32_t)block_rows,
                               static_cast<uint8_t *>(r.q.data_ptr()), static_cast<float *>(r.scale.data_ptr()), current_stream());
        Py_END_ALLOW_THREADS
        return rc != VPTQ_OK ? fail(rc) : pair_of(r.q, r.scale);
    });
}

// desc, ptrs, workspace or None -> (q, scale) of a layer restored to a narrow format: `empty` makes the two, `restore` is the C ABI's call
template <typename Empty, typename Restore>
PyObject *restored(PyObject *const *a, Empty empty, Restore restore)
{
    const vptq_layer_desc *d = struct_of<vptq_layer_desc>(a[0]);
    const vptq_layer_ptrs *p = d ? struct_of<vptq_layer_ptrs>(a[1]) : nullptr;
    void *ws = nullptr;
    size_t ws_bytes = 0;
    if (!p || !room_of(a[2], &ws, &ws_bytes)) return nullptr;
    const int64_t need = vptq_dequant_fp8_workspace_bytes(d);
    if (need < 0) return fail((int)need);
    for (const void *stream : {p->packed_idx, p->outlier_idx})                   // (a pointer that is missing is the C ABI's to refuse)
        if (stream && !address_on_current_device(stream)) return assertion("a layer in the current device's memory");
    return guarded([&]() -> PyObject * {
        const at::TensorOptions options = at::TensorOptions().device(at::kCUDA, c10::cuda::current_device());
        const auto r = empty(d, options);
        at::Tensor own;
        if (need > 0 && ws == nullptr) {
            own = at::empty({need}, options.dtype(at::kByte));
            ws = own.data_ptr();
            ws_bytes = (size_t)need;
        }
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = restore(d, p, r.q.data_ptr(), r.scale.data_ptr(), ws, ws_bytes);
        Py_END_ALLOW_THREADS
        return rc != VPTQ_OK ? fail(rc) : pair_of(r.q, r.scale);
    });
}

// dequant_fp8(desc, ptrs, workspace or None) -> (q, scale)
PyObject *py_dequant_fp8(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 3) { PyErr_SetString(PyExc_TypeError, "dequant_fp8 takes 3 arguments"); return nullptr; }
    return restored(a, [](const vptq_layer_desc *d, const at::TensorOptions &options) { return empty_fp8(d->M, d->N, 128, options); },
                    [](const vptq_layer_desc *d, const vptq_layer_ptrs *p, void *q, void *scale, void *ws, size_t ws_bytes) {
                        return vptq_dequant_fp8(d, p, static_cast<uint8_t *>(q), static_cast<float *>(scale), ws, ws_bytes, current_stream());
                    });
}

// linear_fp8(x, w, w_scale, x_scale or None, out dtype or None, out or None, workspace or None) -> out
PyObject *py_linear_fp8(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 7) { PyErr_SetString(PyExc_TypeError, "linear_fp8 takes 7 arguments"); return nullptr; }
    const at::Tensor *x = tensor_of(a[0]), *w = x ? tensor_of(a[1]) : nullptr, *ws_t = w ? tensor_of(a[2]) : nullptr;
    const at::Tensor *xs = nullptr, *out = nullptr;
    if (!ws_t || (a[3] != Py_None && !(xs = tensor_of(a[3]))) || (a[5] != Py_None && !(out = tensor_of(a[5])))) return nullptr;
    vptq_fp8_desc d = {};
    d.x_dtype = code_of(x->scalar_type());
    const bool e4m3 = d.x_dtype == VPTQ_DTYPE_E4M3;
    if (x->dim() != 2 || w->dim() != 2 || !plain(*x) || x->size(0) > MAX_INT || x->size(1) > MAX_INT || w->size(0) > MAX_INT)
        return assertion("x [B][N] and w [M][pitch], contiguous tensors of the current device");
    const int64_t B = x->size(0), N = x->size(1), M = w->size(0);
    if (!is_fp8(*w, *ws_t, M, (N + 15) / 16 * 16, 128)) return assertion("w e4m3 [M][N rounded up to 16] with FP32 scales [ceil(M / 128)][ceil(N / 128)]");
    if (e4m3 != (xs != nullptr)) return assertion("x_scale comes with e4m3 activations, and with no others");
    if (e4m3 && !is_fp8(*x, *xs, B, (N + 15) / 16 * 16, 1)) return assertion("x e4m3 [B][pitch] with FP32 scales [B][ceil(N / 128)]");
    d.M = (int32_t)M; d.N = (int32_t)N;
    if (a[4] != Py_None) {
        d.out_dtype = (int32_t)PyLong_AsLong(a[4]);
        if (PyErr_Occurred()) return nullptr;
    } else {
        d.out_dtype = out ? code_of(out->scalar_type()) : e4m3 ? VPTQ_DTYPE_BF16 : d.x_dtype;
    }
    if (out && (!plain(*out) || out->dim() != 2 || out->size(0) != B || out->size(1) != M || code_of(out->scalar_type()) != d.out_dtype))
        return assertion("out [B][M], contiguous, of the type asked for");
    void *ws;
    size_t ws_bytes;
    if (!room_of(a[6], &ws, &ws_bytes)) return nullptr;
    const int64_t need = vptq_linear_fp8_workspace_bytes(&d, B > 0 ? (int32_t)B : 1);
    if (need < 0) return fail((int)need);
    return guarded([&]() -> PyObject * {
        at::Tensor own, result = out ? *out : at::empty({B, M}, x->options().dtype(dtype_of(d.out_dtype)));
        if (B == 0) return out ? Py_NewRef(a[5]) : THPVariable_Wrap(result);           // no tokens: nothing to do
        if (need > 0 && ws == nullptr) {
            own = at::empty({need}, x->options().dtype(at::kByte));
            ws = own.data_ptr();
            ws_bytes = (size_t)need;
        }
        const at::Tensor w_scale = aligned(*ws_t), x_scale = xs ? aligned(*xs) : at::Tensor();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = vptq_linear_fp8(&d, x->data_ptr(), xs ? static_cast<const float *>(x_scale.data_ptr()) : nullptr, (int32_t)B,
                             static_cast<const uint8_t *>(w->data_ptr()), static_cast<const float *>(w_scale.data_ptr()), result.data_ptr(), ws, ws_bytes,
                             current_stream());
        Py_END_ALLOW_THREADS
        if (rc != VPTQ_OK) return fail(rc);
        if (out) { Py_INCREF(a[5]); return a[5]; }
        return THPVariable_Wrap(result);
    });
}

// an operand of all experts: [experts][rows][cols rounded up to 16] with [experts][ceil(rows / 128)][ceil(cols / 128)] FP32 scales
bool is_expert_operand(const at::Tensor &q, const at::Tensor &scale, int64_t experts, int64_t rows, int64_t cols)
{
    return plain(q) && plain(scale) && q.scalar_type() == at::kFloat8_e4m3fn && scale.scalar_type() == at::kFloat && q.dim() == 3 && scale.dim() == 3 &&
           q.size(0) == experts && q.size(1) == rows && q.size(2) == (cols + 15) / 16 * 16 && scale.size(0) == experts &&
           scale.size(1) == (rows + 127) / 128 && scale.size(2) == (cols + 127) / 128;
}

// moe_fp8(x, router, gate, gate_scale, up, up_scale, down, down_scale, top_k, renormalize, out or None, workspace or None) -> out
PyObject *py_moe_fp8(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 12) { PyErr_SetString(PyExc_TypeError, "moe_fp8 takes 12 arguments"); return nullptr; }
    const at::Tensor *t[8], *out = nullptr;
    for (int i = 0; i < 8; i++)
        if (!(t[i] = tensor_of(a[i]))) return nullptr;
    const long top = PyLong_AsLong(a[8]);
    const int renormalize = PyObject_IsTrue(a[9]);
    if ((top == -1 && PyErr_Occurred()) || renormalize < 0 || (a[10] != Py_None && !(out = tensor_of(a[10])))) return nullptr;
    const at::Tensor &x = *t[0], &router = *t[1], &gate = *t[2];
    if (!plain(x) || !plain(router) || x.dim() != 2 || router.dim() != 2 || gate.dim() != 3 || router.scalar_type() != x.scalar_type() || router.size(1) != x.size(1))
        return assertion("x [T][hidden], router [experts][hidden] of one type, gate [experts][inner][pitch], contiguous tensors of the current device");
    const int64_t T = x.size(0), hidden = x.size(1), experts = router.size(0), inner = gate.size(1);
    if (T > MAX_INT || hidden > MAX_INT || experts > MAX_INT || inner > MAX_INT) return fail(VPTQ_E_SHAPE);
    if (!is_expert_operand(gate, *t[3], experts, inner, hidden) || !is_expert_operand(*t[4], *t[5], experts, inner, hidden) ||
        !is_expert_operand(*t[6], *t[7], experts, hidden, inner))
        return assertion("gate, up [experts][inner][pitch(hidden)], down [experts][hidden][pitch(inner)] in e4m3 with their FP32 block scales");
    vptq_moe_desc d = {(int32_t)hidden, (int32_t)inner, (int32_t)experts, (int32_t)(top > MAX_INT || top < 0 ? 0 : top), code_of(x.scalar_type()),
                       code_of(out ? out->scalar_type() : x.scalar_type()), renormalize ? VPTQ_FLAG_MOE_RENORMALIZE : 0};
    if (out && (!plain(*out) || out->dim() != 2 || out->size(0) != T || out->size(1) != hidden)) return assertion("out [T][hidden], contiguous");
    void *ws;
    size_t ws_bytes;
    if (!room_of(a[11], &ws, &ws_bytes)) return nullptr;
    const int64_t need = vptq_moe_fp8_workspace_bytes(&d, T > 0 ? (int32_t)T : 1);
    if (need < 0) return fail((int)need);
    return guarded([&]() -> PyObject * {
        at::Tensor own, result = out ? *out : at::empty({T, hidden}, x.options());
        if (T == 0) return out ? Py_NewRef(a[10]) : THPVariable_Wrap(result);
        const at::Tensor gate_scale = aligned(*t[3]), up_scale = aligned(*t[5]), down_scale = aligned(*t[7]);
        const vptq_moe_ptrs p = {router.data_ptr(), static_cast<const uint8_t *>(gate.data_ptr()), static_cast<const uint8_t *>(t[4]->data_ptr()),
                                 static_cast<const uint8_t *>(t[6]->data_ptr()), static_cast<const float *>(gate_scale.data_ptr()),
                                 static_cast<const float *>(up_scale.data_ptr()), static_cast<const float *>(down_scale.data_ptr())};
        if (ws == nullptr) {
            own = at::empty({need}, x.options().dtype(at::kByte));
            ws = own.data_ptr();
            ws_bytes = (size_t)need;
        }
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = vptq_moe_fp8(&d, &p, x.data_ptr(), (int32_t)T, result.data_ptr(), ws, ws_bytes, current_stream());
        Py_END_ALLOW_THREADS
        if (rc != VPTQ_OK) return fail(rc);
        if (out) { Py_INCREF(a[10]); return a[10]; }
        return THPVariable_Wrap(result);
    });
}

// ---- 4-bit floating point ---------------------------------------------------------------------------------------------------

// at::empty on the options' device, without the dispatcher: 0.2 us less of a call's 4 or 5 for every tensor
at::Tensor new_tensor(at::IntArrayRef sizes, const at::TensorOptions &options)
{
    return at::Tensor(at::detail::empty_cuda(sizes, options.dtype().toScalarType(), options.device(), std::nullopt));
}

int64_t fp4_pitch(int64_t cols) { return (cols + 31) / 32 * 16; }

// tensors of an e2m1 matrix: [rows][pitch] and its tiles of scales
struct Fp4Tensors { at::Tensor q, scale; };
Fp4Tensors empty_fp4(int64_t rows, int64_t cols, const at::TensorOptions &options)
{
    return {new_tensor({rows, fp4_pitch(cols)}, options.dtype(at::kByte)), new_tensor({(rows + 127) / 128, (cols + 127) / 128, 32, 16}, options.dtype(at::kByte))};
}

// [rows][pitch] e2m1 codes with tiles of scales
bool is_fp4(const at::Tensor &q, const at::Tensor &scale, int64_t rows, int64_t cols)
{
    return plain(q) && plain(scale) && q.scalar_type() == at::kByte && scale.scalar_type() == at::kByte && q.dim() == 2 && scale.dim() == 4 &&
           q.size(0) == rows && q.size(1) == fp4_pitch(cols) && scale.size(0) == (rows + 127) / 128 && scale.size(1) == (cols + 127) / 128 &&
           scale.size(2) == 32 && scale.size(3) == 16;
}

// a type argument: a code, or None (then `otherwise`); false with a Python error
bool dtype_argument(PyObject *o, int32_t otherwise, int32_t *code)
{
    *code = otherwise;
    if (o == Py_None) return true;
    *code = (int32_t)PyLong_AsLong(o);
    return !PyErr_Occurred();
}

// Memory for one call, from torch's allocator as a tensor's is (and so from a graph's pool while one is captured), without the tensor: 0.4 us of
// a call's 6.
struct CallMemory {
    void *p = nullptr;
    void take(int64_t bytes) { p = c10::cuda::CUDACachingAllocator::raw_alloc_with_stream((size_t)bytes, c10::cuda::getCurrentCUDAStream().stream()); }
    ~CallMemory() { if (p) c10::cuda::CUDACachingAllocator::raw_delete(p); }
};

// fp4_quantize(x) -> (q, scale)
PyObject *py_fp4_quantize(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 1) { PyErr_SetString(PyExc_TypeError, "fp4_quantize takes 1 argument"); return nullptr; }
    const at::Tensor *x = tensor_of(a[0]);
    if (!x) return nullptr;
    if (!on_current_device(*x)) return assertion("a CUDA tensor of the current device");
    if (x->dim() != 2 || x->size(1) < 1 || x->size(0) > MAX_INT || x->size(1) > MAX_INT) return assertion("x [rows][cols]");
    const int64_t rows = x->size(0), cols = x->size(1), ld = rows > 1 ? x->stride(0) : cols;
    if ((cols > 1 && x->stride(1) != 1) || ld < cols) return assertion("a row's columns next to each other, rows apart");
    return guarded([&]() -> PyObject * {
        const Fp4Tensors r = empty_fp4(rows, cols, x->options());
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = vptq_fp4_quantize(x->data_ptr(), code_of(x->scalar_type()), (int32_t)rows, (int32_t)cols, ld, static_cast<uint8_t *>(r.q.data_ptr()),
                               static_cast<uint8_t *>(r.scale.data_ptr()), current_stream());
        Py_END_ALLOW_THREADS
        return rc != VPTQ_OK ? fail(rc) : pair_of(r.q, r.scale);
    });
}

// fp4_values(q, scale, cols, out dtype or None, out or None) -> out
PyObject *py_fp4_values(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 5) { PyErr_SetString(PyExc_TypeError, "fp4_values takes 5 arguments"); return nullptr; }
    const at::Tensor *q = tensor_of(a[0]), *scale = q ? tensor_of(a[1]) : nullptr, *out = nullptr;
    const long cols = scale ? PyLong_AsLong(a[2]) : -1;
    int32_t dtype;
    if (!scale || (cols == -1 && PyErr_Occurred()) || (a[4] != Py_None && !(out = tensor_of(a[4])))) return nullptr;
    if (!dtype_argument(a[3], out ? code_of(out->scalar_type()) : VPTQ_DTYPE_BF16, &dtype)) return nullptr;
    if (cols < 1 || cols > MAX_INT || q->dim() != 2 || q->size(0) > MAX_INT) return fail(VPTQ_E_SHAPE);
    const int64_t rows = q->size(0);
    if (!is_fp4(*q, *scale, rows, cols)) return assertion("q uint8 [rows][16 * ceil(cols / 32)] with scales uint8 [ceil(rows / 128)][ceil(cols / 128)][32][16]");
    if (out && (!plain(*out) || out->dim() != 2 || out->size(0) != rows || out->size(1) != cols || code_of(out->scalar_type()) != dtype))
        return assertion("out [rows][cols], contiguous, of the type asked for");
    return guarded([&]() -> PyObject * {
        at::Tensor result = out ? *out : new_tensor({rows, cols}, q->options().dtype(dtype_of(dtype)));
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = vptq_fp4_values(static_cast<const uint8_t *>(q->data_ptr()), static_cast<const uint8_t *>(scale->data_ptr()), (int32_t)rows, (int32_t)cols, dtype,
                             result.data_ptr(), current_stream());
        Py_END_ALLOW_THREADS
        if (rc != VPTQ_OK) return fail(rc);
        return out ? Py_NewRef(a[4]) : THPVariable_Wrap(result);
    });
}

// dequant_fp4(desc, ptrs, workspace or None) -> (q, scale)
PyObject *py_dequant_fp4(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 3) { PyErr_SetString(PyExc_TypeError, "dequant_fp4 takes 3 arguments"); return nullptr; }
    return restored(a, [](const vptq_layer_desc *d, const at::TensorOptions &options) { return empty_fp4(d->M, d->N, options); },
                    [](const vptq_layer_desc *d, const vptq_layer_ptrs *p, void *q, void *scale, void *ws, size_t ws_bytes) {
                        return vptq_dequant_fp4(d, p, static_cast<uint8_t *>(q), static_cast<uint8_t *>(scale), ws, ws_bytes, current_stream());
                    });
}

// linear_fp4(x, w, w_scale, x_scale or None, out dtype or None, out or None, workspace or None) -> out
PyObject *py_linear_fp4(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 7) { PyErr_SetString(PyExc_TypeError, "linear_fp4 takes 7 arguments"); return nullptr; }
    const at::Tensor *x = tensor_of(a[0]), *w = x ? tensor_of(a[1]) : nullptr, *w_scale = w ? tensor_of(a[2]) : nullptr;
    const at::Tensor *x_scale = nullptr, *out = nullptr;
    if (!w_scale || (a[3] != Py_None && !(x_scale = tensor_of(a[3]))) || (a[5] != Py_None && !(out = tensor_of(a[5])))) return nullptr;
    const bool e2m1 = x->scalar_type() == at::kByte;
    vptq_fp4_desc d = {};
    d.x_dtype = e2m1 ? VPTQ_DTYPE_E2M1 : code_of(x->scalar_type());
    if (x->dim() != 2 || w->dim() != 2 || !plain(*x) || x->size(0) > MAX_INT || x->size(1) > MAX_INT / 2 || w->size(0) > MAX_INT)
        return assertion("x [B][N] and w [M][pitch], contiguous tensors of the current device");
    const int64_t B = x->size(0), N = e2m1 ? 2 * x->size(1) : x->size(1), M = w->size(0);
    if (!is_fp4(*w, *w_scale, M, N)) return assertion("w uint8 [M][16 * ceil(N / 32)] with scales uint8 [ceil(M / 128)][ceil(N / 128)][32][16]");
    if (e2m1 != (x_scale != nullptr)) return assertion("x_scale comes with e2m1 activations, and with no others");
    if (e2m1 && !is_fp4(*x, *x_scale, B, N)) return assertion("x uint8 [B][pitch] with scales uint8 [ceil(B / 128)][ceil(N / 128)][32][16]");
    d.M = (int32_t)M; d.N = (int32_t)N;
    if (!dtype_argument(a[4], out ? code_of(out->scalar_type()) : e2m1 ? VPTQ_DTYPE_BF16 : d.x_dtype, &d.out_dtype)) return nullptr;
    if (out && (!plain(*out) || out->dim() != 2 || out->size(0) != B || out->size(1) != M || code_of(out->scalar_type()) != d.out_dtype))
        return assertion("out [B][M], contiguous, of the type asked for");
    void *ws;
    size_t ws_bytes;
    if (!room_of(a[6], &ws, &ws_bytes)) return nullptr;
    const int64_t need = vptq_linear_fp4_workspace_bytes(&d, B > 0 ? (int32_t)B : 1);
    if (need < 0) return fail((int)need);
    return guarded([&]() -> PyObject * {
        CallMemory own;
        const at::Tensor result = out ? *out : new_tensor({B, M}, x->options().dtype(dtype_of(d.out_dtype)));
        if (B == 0) return out ? Py_NewRef(a[5]) : THPVariable_Wrap(result);           // no tokens: nothing to do
        if (need > 0 && ws == nullptr) {
            own.take(need);
            ws = own.p;
            ws_bytes = (size_t)need;
        }
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = vptq_linear_fp4(&d, x->data_ptr(), x_scale ? static_cast<const uint8_t *>(x_scale->data_ptr()) : nullptr, (int32_t)B,
                             static_cast<const uint8_t *>(w->data_ptr()), static_cast<const uint8_t *>(w_scale->data_ptr()), result.data_ptr(), ws, ws_bytes,
                             current_stream());
        Py_END_ALLOW_THREADS
        if (rc != VPTQ_OK) return fail(rc);
        return out ? Py_NewRef(a[5]) : THPVariable_Wrap(result);
    });
}

// ---- caches of keys and values ----------------------------------------------------------------------------------------------

// The cache's four tensors and the three of its sequences, a[0..6], checked against one another and a row's columns; false with a Python error.
bool cache_of(PyObject *const *a, int64_t heads, int64_t dim, vptq_cache_desc *d, vptq_cache_ptrs *p)
{
    const at::Tensor *t[7];
    for (int i = 0; i < 7; i++)
        if (!(t[i] = tensor_of(a[i]))) return false;
    const at::Tensor &k = *t[0], &k_scale = *t[1], &v = *t[2], &v_scale = *t[3], &table = *t[4], &start = *t[5], &cu = *t[6];
    for (int i = 0; i < 7; i++)
        if (!plain(*t[i])) { assertion("contiguous tensors of the current device"); return false; }
    const bool e4m3 = k.scalar_type() == at::kFloat8_e4m3fn;
    if ((!e4m3 && k.scalar_type() != at::kByte) || v.scalar_type() != k.scalar_type() || k_scale.scalar_type() != (e4m3 ? at::kFloat : at::kByte) ||
        v_scale.scalar_type() != k_scale.scalar_type()) {
        assertion("codes float8_e4m3fn with FP32 scales, or uint8 with uint8 scales");
        return false;
    }
    if (dim < 1 || dim > VPTQ_CACHE_MAX_DIM || k.dim() != 4 || k_scale.dim() != 4) { fail(VPTQ_E_SHAPE); return false; }
    d->cache_dtype = e4m3 ? VPTQ_DTYPE_E4M3 : VPTQ_DTYPE_E2M1;
    if (k.sizes() != v.sizes() || k_scale.sizes() != v_scale.sizes() || k.sizes().slice(0, 3) != k_scale.sizes().slice(0, 3) || (heads >= 0 && k.size(1) != heads) ||
        k.size(3) != vptq_cache_row_bytes((int32_t)dim, d->cache_dtype) || k_scale.size(3) != vptq_cache_row_scales((int32_t)dim, d->cache_dtype)) {
        assertion("codes [pages][heads][page][row bytes] and scales [pages][heads][page][row scales], keys' and values' alike, for this head size");
        return false;
    }
    if (table.scalar_type() != at::kInt || start.scalar_type() != at::kInt || cu.scalar_type() != at::kInt || table.dim() != 2 || start.dim() != 1 || cu.dim() != 1 ||
        start.size(0) != table.size(0) || cu.size(0) != table.size(0) + 1) {
        assertion("table [sequences][width], start [sequences], cu [sequences + 1], int32");
        return false;
    }
    for (const int64_t n : {k.size(0), k.size(1), k.size(2), table.size(0), table.size(1)})
        if (n > MAX_INT) { fail(VPTQ_E_SHAPE); return false; }
    d->n_pages = (int32_t)k.size(0); d->n_heads = (int32_t)k.size(1); d->page_size = (int32_t)k.size(2); d->head_dim = (int32_t)dim;
    d->n_seqs = (int32_t)table.size(0); d->table_width = (int32_t)table.size(1);
    *p = {static_cast<uint8_t *>(k.data_ptr()), static_cast<uint8_t *>(v.data_ptr()), k_scale.data_ptr(), v_scale.data_ptr(), static_cast<const int32_t *>(table.data_ptr()),
          static_cast<const int32_t *>(start.data_ptr()), static_cast<const int32_t *>(cu.data_ptr())};
    return true;
}

// cache_write(k, v, k_cache, k_scale, v_cache, v_scale, table, start, cu)
PyObject *py_cache_write(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 9) { PyErr_SetString(PyExc_TypeError, "cache_write takes 9 arguments"); return nullptr; }
    const at::Tensor *k = tensor_of(a[0]), *v = k ? tensor_of(a[1]) : nullptr;
    if (!v) return nullptr;
    if (!on_current_device(*k) || !on_current_device(*v)) return assertion("CUDA tensors of the current device");
    if (k->dim() != 3 || k->sizes() != v->sizes() || k->scalar_type() != v->scalar_type() || (k->size(2) > 1 && (k->stride(2) != 1 || v->stride(2) != 1)))
        return assertion("k and v [tokens][heads][dim] of one type, a head's columns next to each other");
    if (k->size(0) > MAX_INT) return fail(VPTQ_E_SHAPE);
    vptq_cache_desc d = {};
    vptq_cache_ptrs p;
    if (!cache_of(a + 2, k->size(1), k->size(2), &d, &p)) return nullptr;
    d.x_dtype = code_of(k->scalar_type());
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = vptq_cache_write(&d, &p, k->data_ptr(), v->data_ptr(), (int32_t)k->size(0), k->stride(0), k->stride(1), v->stride(0), v->stride(1), current_stream());
    Py_END_ALLOW_THREADS
    if (rc != VPTQ_OK) return fail(rc);
    Py_RETURN_NONE;
}

// cache_read(k_cache, k_scale, v_cache, v_scale, table, start, cu, n_tokens, head_dim, out dtype or None, k or None, v or None) -> (k, v)
PyObject *py_cache_read(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 12) { PyErr_SetString(PyExc_TypeError, "cache_read takes 12 arguments"); return nullptr; }
    const long tokens = PyLong_AsLong(a[7]);
    if (tokens == -1 && PyErr_Occurred()) return nullptr;
    const long dim = PyLong_AsLong(a[8]);
    if (dim == -1 && PyErr_Occurred()) return nullptr;
    const at::Tensor *k = nullptr, *v = nullptr;
    if ((a[10] != Py_None && !(k = tensor_of(a[10]))) || (a[11] != Py_None && !(v = tensor_of(a[11])))) return nullptr;
    vptq_cache_desc d = {};
    vptq_cache_ptrs p;
    if (!cache_of(a, -1, dim, &d, &p)) return nullptr;
    if (tokens < 0 || tokens > MAX_INT) return fail(VPTQ_E_SHAPE);
    const at::Tensor *given = k ? k : v;
    if (!dtype_argument(a[9], given ? code_of(given->scalar_type()) : VPTQ_DTYPE_BF16, &d.x_dtype)) return nullptr;
    for (const at::Tensor *t : {k, v})
        if (t && (!plain(*t) || t->dim() != 3 || t->size(0) != tokens || t->size(1) != d.n_heads || t->size(2) != dim || code_of(t->scalar_type()) != d.x_dtype))
            return assertion("k and v [tokens][heads][dim], contiguous, of the type asked for");
    return guarded([&]() -> PyObject * {
        const at::TensorOptions options = THPVariable_Unpack(a[0]).options().dtype(dtype_of(d.x_dtype));
        at::Tensor k_out = k ? *k : new_tensor({tokens, d.n_heads, dim}, options), v_out = v ? *v : new_tensor({tokens, d.n_heads, dim}, options);
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = vptq_cache_read(&d, &p, k_out.data_ptr(), v_out.data_ptr(), (int32_t)tokens, current_stream());
        Py_END_ALLOW_THREADS
        return rc != VPTQ_OK ? fail(rc) : pair_of(k_out, v_out);
    });
}

PyObject *py_set_error_class(PyObject *, PyObject *cls)
{
    Py_INCREF(cls);
    Py_XSETREF(g_error_class, cls);
    Py_RETURN_NONE;
}

// A method as the table takes it.  Nothing that its C++ throws gets past it: in the interpreter's C frames that would end the process.
template <PyObject *(*CALL)(PyObject *, PyObject *const *, Py_ssize_t)>
PyObject *entry(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() { return CALL(self, a, n); });
}
template <PyObject *(*CALL)(PyObject *, PyObject *const *, Py_ssize_t)>
PyCFunction method() { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(entry<CALL>)); }

PyMethodDef methods[] = {
    {"linear", method<py_linear>(), METH_FASTCALL, "vptq_linear on torch tensors"},
    {"dequant", method<py_dequant>(), METH_FASTCALL, "vptq_dequant on torch tensors"},
    {"layer_linear", method<py_layer_linear>(), METH_FASTCALL, "DeviceLayer.linear"},
    {"fused_linear", method<py_fused_linear>(), METH_FASTCALL, "FusedLayers.linear"},
    {"fp8_quantize", method<py_fp8_quantize>(), METH_FASTCALL, "vptq_fp8_quantize on torch tensors"},
    {"dequant_fp8", method<py_dequant_fp8>(), METH_FASTCALL, "vptq_dequant_fp8 on torch tensors"},
    {"linear_fp8", method<py_linear_fp8>(), METH_FASTCALL, "vptq_linear_fp8 on torch tensors"},
    {"moe_fp8", method<py_moe_fp8>(), METH_FASTCALL, "vptq_moe_fp8 on torch tensors"},
    {"fp4_quantize", method<py_fp4_quantize>(), METH_FASTCALL, "vptq_fp4_quantize on torch tensors"},
    {"fp4_values", method<py_fp4_values>(), METH_FASTCALL, "vptq_fp4_values on torch tensors"},
    {"dequant_fp4", method<py_dequant_fp4>(), METH_FASTCALL, "vptq_dequant_fp4 on torch tensors"},
    {"linear_fp4", method<py_linear_fp4>(), METH_FASTCALL, "vptq_linear_fp4 on torch tensors"},
    {"cache_write", method<py_cache_write>(), METH_FASTCALL, "vptq_cache_write on torch tensors"},
    {"cache_read", method<py_cache_read>(), METH_FASTCALL, "vptq_cache_read on torch tensors"},
    {"set_error_class", py_set_error_class, METH_O, "exception raised for VPTQ_E_* codes"},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&module); }
