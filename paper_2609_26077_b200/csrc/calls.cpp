// The usual calls of `fp8` and `gradients` from Python without Python in between: arguments are read from the tensors themselves, outputs allocated, and
// the library's entry point called.  What a call of a small layer takes is the host's time (a product from Python 10.6 us, 3 of them in the library;
// 45 ns for each property of each tensor of a list).
//
// Every function returns None where anything about its arguments is not as it expects (types, devices, strides, a refusal by the library), without having
// enqueued anything but what a refused call may have left in its own workspace; the caller then goes the general way, which says what is wrong or does what
// is unusual.  Any other failure of the library's is raised here: its work may have been enqueued, and must not be a second time.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>
#include <c10/cuda/CUDAStream.h>
#include <algorithm>
#include <vector>
#include "../../include/fmm_fp8.h"
#include "../../include/fmm_gradients.h"

namespace {

typedef fmm_status_t (*Quantize)(const fmm_fp8_quantize_t*, void*);
typedef fmm_status_t (*Product)(const fmm_fp8_product_t*, void*);
typedef fmm_status_t (*WorkspaceBytes)(int64_t, size_t*);
typedef fmm_status_t (*Norm)(const fmm_gradients_t*, float*, void*, size_t, void*);
typedef fmm_status_t (*Clip)(const fmm_gradients_t*, double, float*, void*, size_t, void*);
enum { QUANTIZE, MATMUL, GRAD_INPUT, GRAD_WEIGHT, WORKSPACE_BYTES, NORM, CLIP, COUNT };
void* entry[COUNT];

constexpr at::ScalarType CODES = at::kFloat8_e4m3fn;

int type_of(at::ScalarType t) { return t == at::kFloat ? FMM_TYPE_F32 : t == at::kBFloat16 ? FMM_TYPE_BF16 : t == at::kHalf ? FMM_TYPE_F16 : -1; }
const at::Tensor* tensor(PyObject* o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }
int64_t up(int64_t n, int64_t a) { return (n + a - 1) / a * a; }
int64_t blocks(int64_t n) { return (n + 127) / 128; }

// A tensor on the current device; its stream.
struct Place { int device; void* stream; };
bool place_of(const at::Tensor* t, Place& p)
{
    if (!t || !t->is_cuda()) return false;
    p.device = t->get_device();
    if (p.device != c10::cuda::current_device()) return false;
    p.stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)p.device).stream();
    return true;
}
bool here(const at::Tensor* t, const Place& p, at::ScalarType type) { return t && t->is_cuda() && t->get_device() == p.device && t->scalar_type() == type; }
// rows x cols with contiguous columns, rows `step` elements apart (or a multiple); codes and scales on 16-byte boundaries
bool matrix(const at::Tensor* t, const Place& p, at::ScalarType type, int64_t rows, int64_t cols, int64_t step, int64_t& ld)
{
    if (!here(t, p, type) || t->dim() != 2 || t->size(0) != rows || t->size(1) != cols || t->stride(1) != 1) return false;
    ld = t->stride(0);
    return ld >= cols && ld >= 1 && ld % step == 0 && (step == 1 || ((uintptr_t)t->data_ptr() & 15) == 0);
}
// scales along rows or columns, rows x cols; loose: rows that start anywhere but on 16-byte boundaries
bool scales_of(const at::Tensor* t, const Place& p, int64_t rows, int64_t cols, int64_t& ld, int64_t& loose)
{
    if (!matrix(t, p, at::kFloat, rows, cols, 1, ld)) return false;
    if (rows == 1) ld = up(cols, 4);
    loose |= (ld & 3) != 0 || ((uintptr_t)t->data_ptr() & 15) != 0;
    return true;
}
bool dense(const at::Tensor* t, const Place& p, at::ScalarType type, at::IntArrayRef shape) { return here(t, p, type) && t->sizes() == shape && t->is_contiguous(); }
// codes of a weight, or of one for each group
bool weight(const at::Tensor* t, const Place& p, int64_t groups, int64_t& ld, int64_t& step)
{
    if (!here(t, p, CODES) || t->dim() != (groups ? 3 : 2)) return false;
    const int64_t d = groups ? 1 : 0, rows = t->size(d), cols = t->size(d + 1);
    ld = t->stride(d);
    step = groups > 1 ? t->stride(0) : 0;
    return (!groups || t->size(0) == groups) && t->stride(d + 1) == 1 && rows > 0 && cols > 0 && ld >= cols && (groups <= 1 || step >= (rows - 1) * ld + cols) &&
           ((ld | step | (int64_t)(uintptr_t)t->data_ptr()) & 15) == 0;
}
// number of groups of `offsets`, 0 for None, -1 where they are not usual
int64_t groups_of(PyObject* o, const Place& p, const int32_t*& offsets)
{
    offsets = nullptr;
    if (o == Py_None) return 0;
    const at::Tensor* t = tensor(o);
    if (!here(t, p, at::kInt) || t->dim() != 1 || t->size(0) < 2 || t->size(0) > FMM_FP8_MAX_GROUPS + 1 || !t->is_contiguous()) return -1;
    offsets = static_cast<const int32_t*>(t->data_ptr());
    return t->size(0) - 1;
}
at::Tensor empty(at::IntArrayRef size, at::ScalarType type, const Place& p) { return at::empty(size, at::TensorOptions().dtype(type).device(at::kCUDA, (c10::DeviceIndex)p.device)); }
// rows a multiple of `step` elements apart
at::Tensor spaced(int64_t rows, int64_t cols, int64_t step, at::ScalarType type, const Place& p)
{
    if (cols % step == 0) return empty({rows, cols}, type, p);
    return at::empty_strided({rows, cols}, {up(cols, step), 1}, at::TensorOptions().dtype(type).device(at::kCUDA, (c10::DeviceIndex)p.device));
}
// An output: the one that is given, in `t`, or of which type one has to be allocated (t undefined), dense
bool output(PyObject* out, PyObject* dtype, at::IntArrayRef shape, const Place& p, at::Tensor& t, at::ScalarType& type, int64_t& ld, int64_t& step)
{
    if (out == Py_None) {
        if (!THPDtype_Check(dtype)) return false;
        type = reinterpret_cast<THPDtype*>(dtype)->scalar_type;
        ld = shape.back();
        step = shape.size() == 3 && shape[0] > 1 ? shape[1] * shape[2] : 0;
        return type_of(type) >= 0;
    }
    const at::Tensor* o = tensor(out);
    if (!o || type_of(type = o->scalar_type()) < 0 || !here(o, p, type) || o->sizes() != shape) return false;
    t = *o;
    const int64_t d = (int64_t)shape.size() - 2, rows = shape[d], cols = shape[d + 1];
    ld = t.stride(d);
    step = d && shape[0] > 1 ? t.stride(0) : 0;
    return t.stride(d + 1) == 1 && ld >= cols && (!step || step >= (rows - 1) * ld + cols);
}

// While one lives, other Python threads run: an allocation may wait for the device, a launch for its queue, and what the device waits for may be another
// thread's to do.  Nothing of Python is touched meanwhile; the tensors are those of the caller's frame (lists: its own), which holds on to them.
struct OthersRun {
    PyThreadState* state = PyEval_SaveThread();
    ~OthersRun() { PyEval_RestoreThread(state); }
};

#define NOT_USUAL(condition) if (condition) { PyErr_Clear(); Py_RETURN_NONE; }

// What a function returns for a status that is not FMM_OK
PyObject* failed(fmm_status_t status, const char* what)
{
    NOT_USUAL(status == FMM_ERR_INVALID_ARG || status == FMM_ERR_SHAPE || status == FMM_ERR_WORKSPACE);
    PyErr_Clear();
    PyObject* fmm = PyImport_ImportModule("paper_2609_26077_b200.fmm");
    PyObject* r = fmm ? PyObject_CallMethod(fmm, "_check", "is", (int)status, what) : nullptr;      // raises FmmError
    Py_XDECREF(fmm);
    Py_XDECREF(r);
    return nullptr;
}
// What it returns for a C++ exception, before or after the library has been called
PyObject* thrown(bool called)
{
    NOT_USUAL(!called);
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "the call was made, its result could not be handed over");
    return nullptr;
}

// quantize(x, offsets or None, pow2, forms): forms 1: along the rows, 2: along the columns, 3: both
PyObject* quantize(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    bool called = false;
    try {
        NOT_USUAL(n != 4 || !entry[QUANTIZE]);
        const at::Tensor* x = tensor(args[0]);
        Place p;
        NOT_USUAL(!place_of(x, p) || x->dim() != 2);
        const int type = type_of(x->scalar_type()), pow2 = PyObject_IsTrue(args[2]);
        const long forms = PyLong_AsLong(args[3]);
        const int32_t* offsets;
        const int64_t groups = groups_of(args[1], p, offsets), rows = x->size(0), cols = x->size(1);
        int64_t ldx;
        NOT_USUAL(type < 0 || pow2 < 0 || groups < 0 || rows == 0 || cols == 0 || !matrix(x, p, x->scalar_type(), rows, cols, 1, ldx));
        fmm_fp8_quantize_t a = {};
        a.type = (fmm_type_t)type; a.scale_mode = pow2 ? FMM_FP8_SCALE_POW2 : FMM_FP8_SCALE_AMAX_DIV_448;
        a.rows = rows; a.cols = cols; a.x = x->data_ptr(); a.ldx = ldx; a.groups = groups; a.offsets = offsets;
        at::Tensor out[4];
        fmm_status_t status;
        {
            const OthersRun others;
            if (forms & 1) {
                out[0] = spaced(rows, cols, 16, CODES, p);
                out[1] = spaced(blocks(cols), rows, 4, at::kFloat, p);
                a.codes = static_cast<uint8_t*>(out[0].data_ptr()); a.ldc = out[0].stride(0);
                a.scales = static_cast<float*>(out[1].data_ptr()); a.lds = out[1].stride(0);
            }
            if (forms & 2) {
                const int64_t padded = (rows + 127 * std::max<int64_t>(groups, 1)) / 128 * 128;
                out[2] = spaced(padded, cols, 16, CODES, p);
                out[3] = spaced(padded / 128, cols, 4, at::kFloat, p);
                a.column_codes = static_cast<uint8_t*>(out[2].data_ptr()); a.ldcc = out[2].stride(0);
                a.column_scales = static_cast<float*>(out[3].data_ptr()); a.ldcs = out[3].stride(0);
            }
            called = true;
            status = reinterpret_cast<Quantize>(entry[QUANTIZE])(&a, p.stream);
        }
        if (status != FMM_OK) return failed(status, "fmm_fp8_quantize");
        const int first = forms & 1 ? 0 : 2, count = forms == 3 ? 4 : 2;
        PyObject* r = PyTuple_New(count);
        if (r) for (int i = 0; i < count; ++i) PyTuple_SET_ITEM(r, i, THPVariable_Wrap(std::move(out[first + i])));
        return r;
    } catch (...) { return thrown(called); }
}

// product(which, a, a_scales, b, b_scales, offsets or None, bias or None, dtype, out or None, accumulate): which 1: matmul, 2: grad_input
PyObject* product(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    bool called = false;
    try {
        NOT_USUAL(n != 10);
        const long which = PyLong_AsLong(args[0]);
        const at::Tensor *a = tensor(args[1]), *as = tensor(args[2]), *b = tensor(args[3]), *bs = tensor(args[4]);
        Place p;
        NOT_USUAL((which != MATMUL && which != GRAD_INPUT) || !entry[which] || !place_of(a, p) || a->dim() != 2);
        fmm_fp8_product_t c = {};
        const int accumulate = PyObject_IsTrue(args[9]);
        const int64_t groups = groups_of(args[5], p, c.offsets), M = a->size(0), depth = a->size(1);
        NOT_USUAL(accumulate < 0 || (accumulate && args[8] == Py_None) || groups < 0 || M == 0 || depth == 0 || !matrix(a, p, CODES, M, depth, 16, c.lda) ||
                  !scales_of(as, p, blocks(depth), M, c.lda_scales, c.loose) || !weight(b, p, groups, c.ldb, c.step_b));
        const int64_t N = b->size(-2), K = b->size(-1), cols = which == MATMUL ? N : K;
        NOT_USUAL(depth != (which == MATMUL ? K : N));
        NOT_USUAL(groups ? !dense(bs, p, at::kFloat, {groups, blocks(N), blocks(K)}) : !dense(bs, p, at::kFloat, {blocks(N), blocks(K)}));
        at::Tensor out;
        at::ScalarType type;
        int64_t step;
        NOT_USUAL(!output(args[8], args[7], {M, cols}, p, out, type, c.ldo, step));
        if (args[6] != Py_None) {
            const at::Tensor* bias = tensor(args[6]);
            NOT_USUAL(which != MATMUL || (groups ? !dense(bias, p, type, {groups, N}) : !dense(bias, p, type, {N})));
            c.bias = bias->data_ptr();
        }
        c.type = (fmm_type_t)type_of(type); c.accumulate = accumulate; c.M = M; c.N = N; c.K = K; c.groups = groups;
        c.a = static_cast<const uint8_t*>(a->data_ptr()); c.a_scales = static_cast<const float*>(as->data_ptr());
        c.b = static_cast<const uint8_t*>(b->data_ptr()); c.b_scales = static_cast<const float*>(bs->data_ptr());
        fmm_status_t status;
        {
            const OthersRun others;
            if (!out.defined()) out = empty({M, cols}, type, p);
            c.out = out.data_ptr();
            called = true;
            status = reinterpret_cast<Product>(entry[which])(&c, p.stream);
        }
        if (status != FMM_OK) return failed(status, which == MATMUL ? "fmm_fp8_matmul" : "fmm_fp8_grad_input");
        if (args[8] != Py_None) { Py_INCREF(args[8]); return args[8]; }
        return THPVariable_Wrap(std::move(out));
    } catch (...) { return thrown(called); }
}

// grad_weight(dy, dy_scales, x, x_scales, offsets or None, dtype, out or None, accumulate[, tokens or None])
PyObject* grad_weight(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    bool called = false;
    try {
        NOT_USUAL((n != 8 && n != 9) || !entry[GRAD_WEIGHT]);
        const at::Tensor *dy = tensor(args[0]), *dys = tensor(args[1]), *x = tensor(args[2]), *xs = tensor(args[3]);
        Place p;
        NOT_USUAL(!place_of(dy, p) || dy->dim() != 2 || !x || x->dim() != 2);
        fmm_fp8_product_t c = {};
        const int accumulate = PyObject_IsTrue(args[7]);
        if (n == 9 && args[8] != Py_None) {
            c.tokens = PyLong_AsLongLong(args[8]);
            NOT_USUAL(c.tokens <= 0);                        // (none: the general way; -1 also where it is no number)
        }
        const int64_t groups = groups_of(args[4], p, c.offsets), M = dy->size(0), N = dy->size(1), K = x->size(1);
        NOT_USUAL(accumulate < 0 || (accumulate && args[6] == Py_None) || groups < 0 || M == 0 || M % 128 || N == 0 || K == 0 || !matrix(dy, p, CODES, M, N, 16, c.lda) ||
                  !matrix(x, p, CODES, M, K, 16, c.ldb) || !scales_of(dys, p, M / 128, N, c.lda_scales, c.loose) || !scales_of(xs, p, M / 128, K, c.ldb_scales, c.loose));
        at::Tensor out;
        at::ScalarType type;
        const int64_t dims[3] = {groups, N, K};
        const at::IntArrayRef shape = groups ? at::IntArrayRef(dims, 3) : at::IntArrayRef(dims + 1, 2);
        NOT_USUAL(!output(args[6], args[5], shape, p, out, type, c.ldo, c.step_out));
        c.type = (fmm_type_t)type_of(type); c.accumulate = accumulate; c.M = M; c.N = N; c.K = K; c.groups = groups;
        c.a = static_cast<const uint8_t*>(dy->data_ptr()); c.a_scales = static_cast<const float*>(dys->data_ptr());
        c.b = static_cast<const uint8_t*>(x->data_ptr()); c.b_scales = static_cast<const float*>(xs->data_ptr());
        fmm_status_t status;
        {
            const OthersRun others;
            if (!out.defined()) out = empty(shape, type, p);
            c.out = out.data_ptr();
            called = true;
            status = reinterpret_cast<Product>(entry[GRAD_WEIGHT])(&c, p.stream);
        }
        if (status != FMM_OK) return failed(status, "fmm_fp8_grad_weight");
        if (args[6] != Py_None) { Py_INCREF(args[6]); return args[6]; }
        return THPVariable_Wrap(std::move(out));
    } catch (...) { return thrown(called); }
}

// clip(list of tensors, max_norm, list of outputs or None), and the norm alone with max_norm None; the norm
PyObject* clip(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    bool called = false;
    try {
        NOT_USUAL(n != 3 || !PyList_Check(args[0]) || (args[2] != Py_None && !PyList_Check(args[2])) || !entry[WORKSPACE_BYTES] || !entry[NORM] || !entry[CLIP]);
        const bool only_norm = args[1] == Py_None;
        const Py_ssize_t count = PyList_GET_SIZE(args[0]);
        double max_norm = 0.0;
        if (!only_norm) {
            NOT_USUAL(!PyFloat_Check(args[1]));
            max_norm = PyFloat_AS_DOUBLE(args[1]);
        }
        Place p;
        NOT_USUAL(count == 0 || (args[2] != Py_None && PyList_GET_SIZE(args[2]) != count) || !place_of(tensor(PyList_GET_ITEM(args[0], 0)), p));
        std::vector<void*> x(count), out(args[2] != Py_None ? count : 0);
        std::vector<int64_t> sizes(count);
        std::vector<uint8_t> types(count);
        for (Py_ssize_t i = 0; i < count; ++i) {
            const at::Tensor* t = tensor(PyList_GET_ITEM(args[0], i));
            NOT_USUAL(!t || !here(t, p, t->scalar_type()) || type_of(t->scalar_type()) < 0 || !t->is_contiguous());
            x[i] = t->data_ptr(); sizes[i] = t->numel(); types[i] = (uint8_t)type_of(t->scalar_type());
            if (args[2] != Py_None) {
                const at::Tensor* o = tensor(PyList_GET_ITEM(args[2], i));
                NOT_USUAL(!here(o, p, t->scalar_type()) || o->numel() != sizes[i] || !o->is_contiguous());
                out[i] = o->data_ptr();
            }
        }
        size_t need = 0;
        NOT_USUAL(reinterpret_cast<WorkspaceBytes>(entry[WORKSPACE_BYTES])(count, &need) != FMM_OK);
        const fmm_gradients_t g = {count, x.data(), out.empty() ? nullptr : out.data(), sizes.data(), types.data()};
        at::Tensor norm;
        fmm_status_t status;
        {
            const OthersRun others;
            norm = empty({}, at::kFloat, p);
            const at::Tensor workspace = empty({(int64_t)need}, at::kByte, p);
            float* to = static_cast<float*>(norm.data_ptr());
            called = true;
            status = only_norm ? reinterpret_cast<Norm>(entry[NORM])(&g, to, workspace.data_ptr(), need, p.stream)
                               : reinterpret_cast<Clip>(entry[CLIP])(&g, max_norm, to, workspace.data_ptr(), need, p.stream);
        }
        if (status != FMM_OK) return failed(status, only_norm ? "fmm_gradient_norm" : "fmm_gradient_clip");
        return THPVariable_Wrap(std::move(norm));
    } catch (...) { return thrown(called); }
}

// bind(addresses of the library's entry points, in the order of the list at the top)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (n != COUNT) { PyErr_SetString(PyExc_ValueError, "bind: another number of entry points"); return nullptr; }
    void* found[COUNT];
    for (int i = 0; i < COUNT; ++i) {
        found[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    std::copy(found, found + COUNT, entry);
    Py_RETURN_NONE;
}

#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(quantize), METHOD(product), METHOD(grad_weight), METHOD(clip), METHOD(bind), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
