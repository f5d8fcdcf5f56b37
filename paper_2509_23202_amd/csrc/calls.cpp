// The binding's per-call work for the plain case of the calls that a decoder makes for every token -- quantize, product, the
// one-launch linears -- in compiled code: a launch of theirs takes 3 us on the GPU, and checks, output tensors and argument
// marshalling in Python took as long as the launch itself (one token against one projection: 6.8 us a call, now 4.7; sixteen tokens through a layer, eight launches: 64, now 44).
//
// Every function returns None for what is not the plain case (a Tensor subclass, a caller's own output or workspace, anything
// that Python code under a mode should see, an argument of another type) and for a call that the library refuses before it launches
// anything: the Python path behind it then takes the call from the start, and raises what it always raised.  An error of the device
// is raised here: the launch has reported it and forgotten it, so that a second try would succeed.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/hip/EmptyTensor.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <initializer_list>

#include "fp4mr.h"

namespace {

// the library's entry points, handed over by the binding that has loaded it (so that there is one copy of it)
struct Entry {
    decltype(&fp4_rotate_quantize) rotate_quantize;
    decltype(&fp4_quantize_weights) quantize_weights;
    decltype(&fp4_rotate_quantize_dense) rotate_quantize_dense;
    decltype(&fp4_gemm) gemm;
    decltype(&fp4_fused_linear) fused_linear;
    decltype(&fp4_w4a16_linear) w4a16_linear;
    decltype(&fp4_workspace_bytes) workspace_bytes;
    decltype(&fp4_packed_bytes) packed_bytes;
} entry;
struct Entry8 {     // of the 8-bit linear layers
    decltype(&fp8_rmsnorm_quantize) rmsnorm_quantize8;
    decltype(&fp8_quantize) quantize8;
    decltype(&fp8_quantize_weights) quantize_weights8;
    decltype(&fp8_gemm) gemm8;
    decltype(&fp8_workspace_bytes) workspace_bytes8;
    decltype(&fp8_grouped_gemm) grouped_gemm8;
} entry8;
struct Entry8i {    // of the 8-bit integer layers, and of the router
    decltype(&int8_rmsnorm_quantize) rmsnorm_quantize8i;
    decltype(&int8_quantize) quantize8i;
    decltype(&int8_gemm) gemm8i;
    decltype(&int8_workspace_bytes) workspace_bytes8i;
    decltype(&int8_grouped_gemm) grouped_gemm8i;
    decltype(&moe_route) route;
    decltype(&moe_workspace_bytes) route_workspace_bytes;
    decltype(&moe_combine) combine;
} entry8i;
PyObject* error;   // the binding's exception, called with a status

// an argument that is a plain Python int in range
bool integer(PyObject* o, int64_t& v)
{
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    v = PyLong_AsLongLongAndOverflow(o, &overflow);
    return overflow == 0;
}

// a plain tensor (not a subclass), or with `none` None
bool tensor(PyObject* o, const at::Tensor*& t, bool none = false)
{
    t = nullptr;
    if (none && o == Py_None) return true;
    if (!THPVariable_CheckExact(o)) return false;
    t = &THPVariable_Unpack(o);
    return t->is_cuda();
}

bool bf16_rows(const at::Tensor& x) { return x.scalar_type() == at::kBFloat16 && x.dim() == 2 && x.is_contiguous(); }

void* pointer(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }

// (not through the dispatcher, which takes 0.4 us for it: plain() has seen that nobody listens there, and where new memory is to be filled that is its work)
at::Tensor empty(at::IntArrayRef shape, at::ScalarType type, const at::Tensor& like)
{
    if (!at::globalContext().deterministicAlgorithms()) return at::detail::empty_cuda(shape, type, like.device(), std::nullopt);
    return at::empty(shape, at::TensorOptions().dtype(type).device(like.device()));
}

void* stream() { return c10::hip::getCurrentHIPStream(c10::hip::current_device()).stream(); }

bool plain() { return !at::impl::torch_function_mode_enabled() && !c10::impl::TorchDispatchModeTLS::any_modes_set(); }

// what a call returns whose status is not FP4MR_OK
PyObject* refused(fp4mr_status_t status)
{
    if (status != FP4MR_ERR_DEVICE) Py_RETURN_NONE;
    if (PyObject* const e = PyObject_CallFunction(error, "i", (int)status)) {
        PyErr_SetObject(reinterpret_cast<PyObject*>(Py_TYPE(e)), e);
        Py_DECREF(e);
    }
    return nullptr;
}

// quantize(x, had_block, fmt, flags, kind, rot): kind 0 rotate_quantize, 1 quantize_weights, 2 rotate_quantize_dense
PyObject* quantize(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor *x, *rot;
    int64_t b, fmt, flags, kind;
    if (n != 6 || !plain() || !tensor(args[0], x) || !integer(args[1], b) || !integer(args[2], fmt) || !integer(args[3], flags) || !integer(args[4], kind) ||
        !tensor(args[5], rot, true) || !bf16_rows(*x) || (fmt != FP4MR_MXFP4 && fmt != FP4MR_NVFP4) || b < 0 || b > 4096 || flags < 0 || flags > 0xffffffffll ||
        (flags & (FP4MR_SCALE_FIT_RANGE | FP4MR_INPUT_F32 | FP4MR_STATIC_TENSOR_SCALE)) || (kind == 2) != (rot != nullptr) || (rot && (!bf16_rows(*rot) || rot->size(0) != b || rot->size(1) != b)))
        Py_RETURN_NONE;
    const int64_t rows = x->size(0), K = x->size(1);
    size_t code_bytes = 0, scale_bytes = 0;
    if (entry.packed_bytes(rows, K, (fp4mr_fmt_t)fmt, (uint32_t)flags & FP4MR_LAYOUT_GEMM, &code_bytes, &scale_bytes) != FP4MR_OK) Py_RETURN_NONE;
    const at::Tensor codes = empty({(int64_t)code_bytes}, at::kByte, *x), scales = empty({(int64_t)scale_bytes}, at::kByte, *x);
    at::Tensor tensor_scale, workspace;
    if (fmt == FP4MR_NVFP4) tensor_scale = empty({1}, at::kFloat, *x);
    const size_t need = entry.workspace_bytes(kind == 1 ? FP4MR_OP_QUANTIZE_WEIGHTS : FP4MR_OP_ROTATE_QUANTIZE, rows, 0, K, (fp4mr_fmt_t)fmt, (uint32_t)flags);
    if (need) workspace = empty({(int64_t)need}, at::kByte, *x);
    float* const ts = tensor_scale.defined() ? static_cast<float*>(tensor_scale.data_ptr()) : nullptr;
    void* const ws = need ? workspace.data_ptr() : nullptr;
    const void* const px = x->data_ptr();
    void *const pc = codes.data_ptr(), *const ps = scales.data_ptr(), *const pr = pointer(rot), *const st = stream();
    fp4mr_status_t status;
    Py_BEGIN_ALLOW_THREADS;
    if (kind == 2) status = entry.rotate_quantize_dense(px, rows, K, (int)b, pr, (fp4mr_fmt_t)fmt, pc, ps, ts, ws, need, (uint32_t)flags, st);
    else status = (kind == 1 ? entry.quantize_weights : entry.rotate_quantize)(px, rows, K, (int)b, (fp4mr_fmt_t)fmt, pc, ps, ts, ws, need, (uint32_t)flags, st);
    Py_END_ALLOW_THREADS;
    if (status != FP4MR_OK) return refused(status);
    PyObject* const out = PyTuple_New(3);
    if (!out) return nullptr;
    PyTuple_SET_ITEM(out, 0, THPVariable_Wrap(codes));
    PyTuple_SET_ITEM(out, 1, THPVariable_Wrap(scales));
    PyTuple_SET_ITEM(out, 2, THPVariable_Wrap(tensor_scale));   // (an undefined tensor is None)
    for (int i = 0; i < 3; ++i)
        if (!PyTuple_GET_ITEM(out, i)) {
            Py_DECREF(out);
            return nullptr;
        }
    return out;
    END_HANDLE_TH_ERRORS
}

// gemm(a_codes, a_scales, a_tensor_scale, w_codes, w_scales, w_tensor_scale, M, N, K, fmt, flags)
PyObject* gemm(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor *ac, *as, *at_, *wc, *ws, *wt;
    int64_t M, N, K, fmt, flags;
    if (n != 11 || !plain() || !tensor(args[0], ac) || !tensor(args[1], as) || !tensor(args[2], at_, true) || !tensor(args[3], wc) || !tensor(args[4], ws) ||
        !tensor(args[5], wt, true) || !integer(args[6], M) || !integer(args[7], N) || !integer(args[8], K) || !integer(args[9], fmt) || !integer(args[10], flags) ||
        M <= 0 || N <= 0 || K <= 0 || (fmt != FP4MR_MXFP4 && fmt != FP4MR_NVFP4) || flags < 0 || flags > 0xffffffffll)
        Py_RETURN_NONE;
    const at::Tensor out = empty({M, N}, flags & FP4MR_OUT_F32 ? at::kFloat : at::kBFloat16, *ac);
    at::Tensor workspace;
    const size_t need = entry.workspace_bytes(FP4MR_OP_GEMM_FASTEST, M, N, K, (fp4mr_fmt_t)fmt, (uint32_t)flags);
    if (need) workspace = empty({(int64_t)need}, at::kByte, *ac);
    void *const pac = pointer(ac), *const pas = pointer(as), *const pwc = pointer(wc), *const pws = pointer(ws), *const po = out.data_ptr();
    float *const pat = static_cast<float*>(pointer(at_)), *const pwt = static_cast<float*>(pointer(wt));
    void *const pw = need ? workspace.data_ptr() : nullptr, *const st = stream();
    fp4mr_status_t status;
    Py_BEGIN_ALLOW_THREADS;
    status = entry.gemm(pac, pas, pat, pwc, pws, pwt, M, N, K, (fp4mr_fmt_t)fmt, po, pw, need, (uint32_t)flags, st);
    Py_END_ALLOW_THREADS;
    if (status != FP4MR_OK) return refused(status);
    return THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}

// linear(x, had_block, w_codes, w_scales, N, fmt, flags, weight_only)
PyObject* linear(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor *x, *wc, *ws;
    int64_t b, N, fmt, flags, weight_only;
    if (n != 8 || !plain() || !tensor(args[0], x) || !integer(args[1], b) || !tensor(args[2], wc) || !tensor(args[3], ws) || !integer(args[4], N) || !integer(args[5], fmt) ||
        !integer(args[6], flags) || !integer(args[7], weight_only) || !bf16_rows(*x) || b < 0 || b > 4096 || N <= 0 || x->size(0) <= 0 ||
        (fmt != FP4MR_MXFP4 && fmt != FP4MR_NVFP4) || flags < 0 || flags > 0xffffffffll)
        Py_RETURN_NONE;
    const int64_t M = x->size(0), K = x->size(1);
    const at::Tensor out = empty({M, N}, flags & FP4MR_OUT_F32 ? at::kFloat : at::kBFloat16, *x);
    const void* const px = x->data_ptr();
    void *const pwc = pointer(wc), *const pws = pointer(ws), *const po = out.data_ptr(), *const st = stream();
    fp4mr_status_t status;
    Py_BEGIN_ALLOW_THREADS;
    status = (weight_only ? entry.w4a16_linear : entry.fused_linear)(px, M, K, (int)b, pwc, pws, N, (fp4mr_fmt_t)fmt, po, (uint32_t)flags | FP4MR_W_LAYOUT_GEMM, st);
    Py_END_ALLOW_THREADS;
    if (status != FP4MR_OK) return refused(status);
    return THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}

// ---- 8-bit linear layers
constexpr int64_t kBlock8 = 128;

// bf16 [M, any] whose rows may be apart
bool bf16_strided(const at::Tensor& x) { return x.scalar_type() == at::kBFloat16 && x.dim() == 2 && x.stride(1) == 1; }
int64_t row_stride(const at::Tensor& x) { return x.size(0) > 1 ? x.stride(0) : x.size(1); }
bool bf16_like(const at::Tensor* t, int64_t rows, int64_t K) { return !t || (bf16_rows(*t) && t->size(0) == rows && t->size(1) == K); }

// codes [.., n, K] and their scales, a row of them for `rows` rows of codes
bool operand8(const at::Tensor& codes, const at::Tensor& scales, int64_t dim, int64_t rows)
{
    if (codes.scalar_type() != at::kFloat8_e4m3fn || scales.scalar_type() != at::kFloat || codes.dim() != dim || scales.dim() != dim || !codes.is_contiguous() || !scales.is_contiguous())
        return false;
    return codes.size(dim - 1) == scales.size(dim - 1) * kBlock8 && scales.size(dim - 2) == (codes.size(dim - 2) + rows - 1) / rows && (dim == 2 || codes.size(0) == scales.size(0));
}

PyObject* tuple(std::initializer_list<at::Tensor> tensors)      // (an undefined one is None)
{
    PyObject* const out = PyTuple_New((Py_ssize_t)tensors.size());
    if (!out) return nullptr;
    Py_ssize_t i = 0;
    for (const at::Tensor& t : tensors) {
        PyObject* const o = THPVariable_Wrap(t);
        if (!o) {
            Py_DECREF(out);
            return nullptr;
        }
        PyTuple_SET_ITEM(out, i++, o);
    }
    return out;
}

// rmsnorm_quantize8(x, weight, eps, residual, norm_out): into new tensors, but for norm_out
PyObject* rmsnorm_quantize8(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor *x, *weight, *residual, *norm;
    if (n != 5 || !plain() || !tensor(args[0], x) || !tensor(args[1], weight) || !PyFloat_CheckExact(args[2]) || !tensor(args[3], residual, true) || !tensor(args[4], norm, true) ||
        !bf16_strided(*x))
        Py_RETURN_NONE;
    const int64_t M = x->size(0), K = x->size(1);
    if (M <= 0 || K <= 0 || K % kBlock8 != 0 || weight->scalar_type() != at::kBFloat16 || weight->dim() != 1 || weight->size(0) != K || !weight->is_contiguous() || !bf16_like(residual, M, K) ||
        !bf16_like(norm, M, K))
        Py_RETURN_NONE;
    const at::Tensor codes = empty({M, K}, at::kFloat8_e4m3fn, *x), scales = empty({M, K / kBlock8}, at::kFloat, *x);
    at::Tensor sum;
    if (residual) sum = empty({M, K}, at::kBFloat16, *x);
    const float eps = (float)PyFloat_AS_DOUBLE(args[2]);
    const void *const px = x->data_ptr(), *const pw = weight->data_ptr();
    void *const pr = pointer(residual), *const pn = pointer(norm), *const pc = codes.data_ptr(), *const ps = residual ? sum.data_ptr() : nullptr, *const st = stream();
    float* const psc = static_cast<float*>(scales.data_ptr());
    const int64_t apart = row_stride(*x);
    fp4mr_status_t status;
    Py_BEGIN_ALLOW_THREADS;
    status = entry8.rmsnorm_quantize8(px, apart, pr, pw, M, K, eps, pc, psc, ps, pn, 0, st);
    Py_END_ALLOW_THREADS;
    if (status != FP4MR_OK) return refused(status);
    return tuple({codes, scales, sum});
    END_HANDLE_TH_ERRORS
}

// quantize8(x, flags)
PyObject* quantize8(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor* x;
    int64_t flags;
    if (n != 2 || !plain() || !tensor(args[0], x) || !integer(args[1], flags) || (flags & ~(int64_t)FP4MR_SILU_MUL) || !bf16_strided(*x)) Py_RETURN_NONE;
    const int64_t M = x->size(0), held = x->size(1), K = flags ? held / 2 : held;
    if (M <= 0 || K <= 0 || K % kBlock8 != 0 || (flags && held % 2 != 0)) Py_RETURN_NONE;
    const at::Tensor codes = empty({M, K}, at::kFloat8_e4m3fn, *x), scales = empty({M, K / kBlock8}, at::kFloat, *x);
    const void* const px = x->data_ptr();
    void *const pc = codes.data_ptr(), *const st = stream();
    float* const psc = static_cast<float*>(scales.data_ptr());
    const int64_t apart = row_stride(*x);
    fp4mr_status_t status;
    Py_BEGIN_ALLOW_THREADS;
    status = entry8.quantize8(px, apart, M, K, pc, psc, (uint32_t)flags, st);
    Py_END_ALLOW_THREADS;
    if (status != FP4MR_OK) return refused(status);
    return tuple({codes, scales});
    END_HANDLE_TH_ERRORS
}

// quantize_weights8(w)
PyObject* quantize_weights8(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor* w;
    if (n != 1 || !plain() || !tensor(args[0], w) || w->scalar_type() != at::kBFloat16 || !w->is_contiguous() || (w->dim() != 2 && w->dim() != 3)) Py_RETURN_NONE;
    const int64_t experts = w->dim() == 3 ? w->size(0) : 1, N = w->size(-2), K = w->size(-1), blocks = (N + kBlock8 - 1) / kBlock8;
    if (experts <= 0 || N <= 0 || K <= 0 || K % kBlock8 != 0) Py_RETURN_NONE;
    const at::Tensor codes = empty(w->sizes(), at::kFloat8_e4m3fn, *w);
    const at::Tensor scales = w->dim() == 3 ? empty({experts, blocks, K / kBlock8}, at::kFloat, *w) : empty({blocks, K / kBlock8}, at::kFloat, *w);
    const void* const pw = w->data_ptr();
    void *const pc = codes.data_ptr(), *const st = stream();
    float* const psc = static_cast<float*>(scales.data_ptr());
    fp4mr_status_t status;
    Py_BEGIN_ALLOW_THREADS;
    status = entry8.quantize_weights8(pw, experts, N, K, pc, psc, 0, st);
    Py_END_ALLOW_THREADS;
    if (status != FP4MR_OK) return refused(status);
    return tuple({codes, scales});
    END_HANDLE_TH_ERRORS
}

// gemm8(a_codes, a_scales, w_codes, w_scales, flags), and with two arguments more, offsets and rows (or None), the product by expert
PyObject* gemm8(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor *a, *sa, *w, *sw, *offsets = nullptr, *rows = nullptr;
    int64_t flags;
    const bool grouped = n == 7;
    if ((n != 5 && !grouped) || !plain() || !tensor(args[0], a) || !tensor(args[1], sa) || !tensor(args[2], w) || !tensor(args[3], sw) || !integer(args[4], flags) ||
        (flags & ~(int64_t)FP4MR_OUT_F32) || !operand8(*a, *sa, 2, 1) || !operand8(*w, *sw, grouped ? 3 : 2, kBlock8) || a->size(1) != w->size(-1))
        Py_RETURN_NONE;
    if (grouped && (!tensor(args[5], offsets) || !tensor(args[6], rows, true) || offsets->scalar_type() != at::kInt || !offsets->is_contiguous() || offsets->numel() != w->size(0) + 1 ||
                    (rows && (rows->scalar_type() != at::kInt || rows->dim() != 1 || !rows->is_contiguous()))))
        Py_RETURN_NONE;
    const int64_t a_rows = a->size(0), M = rows ? rows->size(0) : a_rows, N = w->size(-2), K = w->size(-1);
    if (M <= 0 || N <= 0 || K <= 0) Py_RETURN_NONE;
    const at::Tensor out = empty({M, N}, flags ? at::kFloat : at::kBFloat16, *a);
    at::Tensor workspace;
    const size_t need = grouped ? 0 : entry8.workspace_bytes8(M, N, K, (uint32_t)flags);
    if (need) workspace = empty({(int64_t)need}, at::kByte, *a);
    const void *const pa = a->data_ptr(), *const pw = w->data_ptr();
    const float *const psa = static_cast<const float*>(sa->data_ptr()), *const psw = static_cast<const float*>(sw->data_ptr());
    const int32_t *const po = static_cast<const int32_t*>(pointer(offsets)), *const pr = static_cast<const int32_t*>(pointer(rows));
    void *const to = out.data_ptr(), *const pws = need ? workspace.data_ptr() : nullptr, *const st = stream();
    const int64_t experts = grouped ? w->size(0) : 1;
    fp4mr_status_t status;
    Py_BEGIN_ALLOW_THREADS;
    if (grouped) status = entry8.grouped_gemm8(pa, psa, a_rows, pw, psw, po, pr, M, experts, N, K, to, (uint32_t)flags, st);
    else status = entry8.gemm8(pa, psa, pw, psw, M, N, K, to, pws, need, (uint32_t)flags, st);
    Py_END_ALLOW_THREADS;
    if (status != FP4MR_OK) return refused(status);
    return THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}

// ---- the integer form of the 8-bit layers, and the router: on the current device
bool here(const at::Tensor* t) { return !t || t->get_device() == c10::hip::current_device(); }
bool codes8i(const at::Tensor& codes, const at::Tensor& scales, int64_t dim)      // [.., rows, K] and [.., rows]
{
    if (codes.scalar_type() != at::kChar || scales.scalar_type() != at::kFloat || codes.dim() != dim || scales.dim() != dim - 1 || !codes.is_contiguous() || !scales.is_contiguous()) return false;
    return codes.size(dim - 2) == scales.size(dim - 2) && (dim == 2 || codes.size(0) == scales.size(0)) && here(&codes) && here(&scales);
}

// rmsnorm_quantize8i(x, weight, eps, residual, norm_out): into new tensors, but for norm_out
PyObject* rmsnorm_quantize8i(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor *x, *weight, *residual, *norm;
    if (n != 5 || !plain() || !tensor(args[0], x) || !tensor(args[1], weight) || !PyFloat_CheckExact(args[2]) || !tensor(args[3], residual, true) || !tensor(args[4], norm, true) ||
        !bf16_strided(*x))
        Py_RETURN_NONE;
    const int64_t M = x->size(0), K = x->size(1);
    if (M <= 0 || K <= 0 || weight->scalar_type() != at::kBFloat16 || weight->dim() != 1 || weight->size(0) != K || !weight->is_contiguous() || !bf16_like(residual, M, K) ||
        !bf16_like(norm, M, K) || !here(x) || !here(weight) || !here(residual) || !here(norm))
        Py_RETURN_NONE;
    const at::Tensor codes = empty({M, K}, at::kChar, *x), scales = empty({M}, at::kFloat, *x);
    at::Tensor sum;
    if (residual) sum = empty({M, K}, at::kBFloat16, *x);
    const float eps = (float)PyFloat_AS_DOUBLE(args[2]);
    const void *const px = x->data_ptr(), *const pw = weight->data_ptr();
    void *const pr = pointer(residual), *const pn = pointer(norm), *const pc = codes.data_ptr(), *const ps = residual ? sum.data_ptr() : nullptr, *const st = stream();
    float* const psc = static_cast<float*>(scales.data_ptr());
    const int64_t apart = row_stride(*x);
    fp4mr_status_t status;
    Py_BEGIN_ALLOW_THREADS;
    status = entry8i.rmsnorm_quantize8i(px, apart, pr, pw, M, K, eps, pc, psc, ps, pn, 0, st);
    Py_END_ALLOW_THREADS;
    if (status != FP4MR_OK) return refused(status);
    return tuple({codes, scales, sum});
    END_HANDLE_TH_ERRORS
}

// quantize8i(x, flags): rows, or contiguous weights of several experts
PyObject* quantize8i(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor* x;
    int64_t flags;
    if (n != 2 || !plain() || !tensor(args[0], x) || !integer(args[1], flags) || (flags & ~(int64_t)FP4MR_SILU_MUL) || x->scalar_type() != at::kBFloat16 || !here(x) ||
        !(x->dim() == 2 ? x->stride(1) == 1 : x->dim() == 3 && x->is_contiguous()))
        Py_RETURN_NONE;
    const int64_t held = x->size(-1), K = flags ? held / 2 : held, outer = x->dim() == 3 ? x->size(0) : 1, inner = x->size(-2), M = outer * inner;
    if (M <= 0 || K <= 0 || (flags && held % 2 != 0)) Py_RETURN_NONE;
    const at::Tensor codes = x->dim() == 3 ? empty({outer, inner, K}, at::kChar, *x) : empty({M, K}, at::kChar, *x);
    const at::Tensor scales = x->dim() == 3 ? empty({outer, inner}, at::kFloat, *x) : empty({M}, at::kFloat, *x);
    const void* const px = x->data_ptr();
    void *const pc = codes.data_ptr(), *const st = stream();
    float* const psc = static_cast<float*>(scales.data_ptr());
    const int64_t apart = x->dim() == 3 ? held : row_stride(*x);
    fp4mr_status_t status;
    Py_BEGIN_ALLOW_THREADS;
    status = entry8i.quantize8i(px, apart, M, K, pc, psc, (uint32_t)flags, st);
    Py_END_ALLOW_THREADS;
    if (status != FP4MR_OK) return refused(status);
    return tuple({codes, scales});
    END_HANDLE_TH_ERRORS
}

// gemm8i(a_codes, a_scales, w_codes, w_scales, flags), and with two arguments more, offsets and rows (or None), the product by expert
PyObject* gemm8i(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor *a, *sa, *w, *sw, *offsets = nullptr, *rows = nullptr;
    int64_t flags;
    const bool grouped = n == 7;
    if ((n != 5 && !grouped) || !plain() || !tensor(args[0], a) || !tensor(args[1], sa) || !tensor(args[2], w) || !tensor(args[3], sw) || !integer(args[4], flags) ||
        (flags & ~(int64_t)FP4MR_OUT_F32) || !codes8i(*a, *sa, 2) || !codes8i(*w, *sw, grouped ? 3 : 2) || a->size(1) != w->size(-1))
        Py_RETURN_NONE;
    if (grouped && (!tensor(args[5], offsets) || !tensor(args[6], rows, true) || offsets->scalar_type() != at::kInt || offsets->dim() != 1 || !offsets->is_contiguous() ||
                    offsets->numel() != w->size(0) + 1 || !here(offsets) || (rows && (rows->scalar_type() != at::kInt || rows->dim() != 1 || !rows->is_contiguous() || !here(rows)))))
        Py_RETURN_NONE;
    const int64_t a_rows = a->size(0), M = rows ? rows->size(0) : a_rows, N = w->size(-2), K = w->size(-1);
    if (M <= 0 || N <= 0 || K <= 0) Py_RETURN_NONE;
    const at::Tensor out = empty({M, N}, flags ? at::kFloat : at::kBFloat16, *a);
    at::Tensor workspace;
    const size_t need = grouped ? 0 : entry8i.workspace_bytes8i(M, N, K);
    if (need) workspace = empty({(int64_t)need}, at::kByte, *a);
    const void *const pa = a->data_ptr(), *const pw = w->data_ptr();
    const float *const psa = static_cast<const float*>(sa->data_ptr()), *const psw = static_cast<const float*>(sw->data_ptr());
    const int32_t *const po = static_cast<const int32_t*>(pointer(offsets)), *const pr = static_cast<const int32_t*>(pointer(rows));
    void *const to = out.data_ptr(), *const pws = need ? workspace.data_ptr() : nullptr, *const st = stream();
    const int64_t experts = grouped ? w->size(0) : 1;
    fp4mr_status_t status;
    Py_BEGIN_ALLOW_THREADS;
    if (grouped) status = entry8i.grouped_gemm8i(pa, psa, a_rows, pw, psw, po, pr, M, experts, N, K, to, (uint32_t)flags, st);
    else status = entry8i.gemm8i(pa, psa, pw, psw, M, N, K, to, pws, need, (uint32_t)flags, st);
    Py_END_ALLOW_THREADS;
    if (status != FP4MR_OK) return refused(status);
    return THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}

// route(logits, top, bias, groups, top_groups, scale, flags)
PyObject* route(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor *z, *bias;
    int64_t top, groups, top_groups, flags;
    if (n != 7 || !plain() || !tensor(args[0], z) || !integer(args[1], top) || !tensor(args[2], bias, true) || !integer(args[3], groups) || !integer(args[4], top_groups) ||
        !PyFloat_CheckExact(args[5]) || !integer(args[6], flags) || flags < 0 || flags > 0xffffffffll || z->dim() != 2 || !here(z) || !here(bias))
        Py_RETURN_NONE;
    const int64_t T = z->size(0), E = z->size(1);
    const bool f32 = z->scalar_type() == at::kFloat;
    if ((!f32 && (z->scalar_type() != at::kBFloat16 || (flags & FP4MR_INPUT_F32))) || T <= 0 || E <= 0 || z->stride(1) != 1 || top <= 0 || top > E || T > (1ll << 24) ||
        (bias && (bias->scalar_type() != at::kFloat || bias->dim() != 1 || bias->size(0) != E || !bias->is_contiguous())))
        Py_RETURN_NONE;
    const at::Tensor weights = empty({T, top}, at::kFloat, *z), experts = empty({T, top}, at::kInt, *z), rows = empty({T * top}, at::kInt, *z), offsets = empty({E + 1}, at::kInt, *z),
                     places = empty({T, top}, at::kInt, *z);
    at::Tensor workspace;
    const size_t need = entry8i.route_workspace_bytes(T, E, top);
    if (need) workspace = empty({(int64_t)need}, at::kByte, *z);
    const void* const pz = z->data_ptr();
    const float* const pb = static_cast<const float*>(pointer(bias));
    float* const pw = static_cast<float*>(weights.data_ptr());
    int32_t *const pe = static_cast<int32_t*>(experts.data_ptr()), *const pr = static_cast<int32_t*>(rows.data_ptr()), *const po = static_cast<int32_t*>(offsets.data_ptr()),
            *const pp = static_cast<int32_t*>(places.data_ptr());
    void *const ws = need ? workspace.data_ptr() : nullptr, *const st = stream();
    const int64_t apart = T > 1 ? z->stride(0) : E;
    const float scale = (float)PyFloat_AS_DOUBLE(args[5]);
    const uint32_t all = (uint32_t)flags | (f32 ? FP4MR_INPUT_F32 : 0u);
    fp4mr_status_t status;
    Py_BEGIN_ALLOW_THREADS;
    status = entry8i.route(pz, apart, pb, T, E, top, groups, top_groups, scale, pw, pe, pr, po, pp, ws, need, all, st);
    Py_END_ALLOW_THREADS;
    if (status != FP4MR_OK) return refused(status);
    return tuple({weights, experts, rows, offsets, places});
    END_HANDLE_TH_ERRORS
}

// combine(y, places, weights, shared, flags)
PyObject* combine(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor *y, *places, *weights, *shared;
    int64_t flags;
    if (n != 5 || !plain() || !tensor(args[0], y) || !tensor(args[1], places) || !tensor(args[2], weights) || !tensor(args[3], shared, true) || !integer(args[4], flags) ||
        (flags & ~(int64_t)FP4MR_OUT_F32) || y->dim() != 2 || places->dim() != 2 || !y->is_contiguous() || !places->is_contiguous() || !weights->is_contiguous() ||
        places->scalar_type() != at::kInt || weights->scalar_type() != at::kFloat || weights->sizes() != places->sizes() || !here(y) || !here(places) || !here(weights) || !here(shared))
        Py_RETURN_NONE;
    const int64_t rows = y->size(0), H = y->size(1), T = places->size(0), top = places->size(1);
    const bool y_f32 = y->scalar_type() == at::kFloat, s_f32 = shared && shared->scalar_type() == at::kFloat;
    if ((!y_f32 && y->scalar_type() != at::kBFloat16) || T <= 0 || H <= 0 ||
        (shared && ((!s_f32 && shared->scalar_type() != at::kBFloat16) || shared->dim() != 2 || shared->size(0) != T || shared->size(1) != H || !shared->is_contiguous())))
        Py_RETURN_NONE;
    const at::Tensor out = empty({T, H}, flags ? at::kFloat : at::kBFloat16, *y);
    const void *const py = y->data_ptr(), *const psh = pointer(shared);
    const int32_t* const pp = static_cast<const int32_t*>(places->data_ptr());
    const float* const pw = static_cast<const float*>(weights->data_ptr());
    void *const to = out.data_ptr(), *const st = stream();
    const uint32_t all = (uint32_t)flags | (y_f32 ? FP4MR_INPUT_F32 : 0u) | (s_f32 ? FP4MR_SHARED_F32 : 0u);
    fp4mr_status_t status;
    Py_BEGIN_ALLOW_THREADS;
    status = entry8i.combine(py, rows, pp, pw, psh, T, top, H, to, all, st);
    Py_END_ALLOW_THREADS;
    if (status != FP4MR_OK) return refused(status);
    return THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}

// The addresses of the entry points of `to` in its order, from Python integers.
template <typename E>
bool addresses(PyObject* const* args, E& to)
{
    constexpr Py_ssize_t count = sizeof(E) / sizeof(void*);
    void* p[count];
    for (Py_ssize_t i = 0; i < count; ++i) {
        p[i] = PyLong_AsVoidPtr(args[i]);
        if (!p[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "a null entry point");
            return false;
        }
    }
    static_assert(sizeof(p) == sizeof(to), "one address per entry point");
    std::memcpy(&to, p, sizeof(to));
    return true;
}

// bind(addresses of the eight entry points, in the order of Entry, and the exception)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    constexpr Py_ssize_t count = sizeof(Entry) / sizeof(void*);
    if (n != count + 1 || !PyCallable_Check(args[count])) {
        PyErr_SetString(PyExc_TypeError, "bind() takes eight addresses and an exception");
        return nullptr;
    }
    if (!addresses(args, entry)) return nullptr;
    Py_INCREF(args[count]);
    Py_XSETREF(error, args[count]);
    Py_RETURN_NONE;
}

// bind8(addresses of the six entry points, in the order of Entry8), behind bind()
PyObject* bind8(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (n != (Py_ssize_t)(sizeof(Entry8) / sizeof(void*))) {
        PyErr_SetString(PyExc_TypeError, "bind8() takes six addresses");
        return nullptr;
    }
    if (!addresses(args, entry8)) return nullptr;
    Py_RETURN_NONE;
}

// bind8i(addresses of the eight entry points, in the order of Entry8i), behind bind()
PyObject* bind8i(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (n != (Py_ssize_t)(sizeof(Entry8i) / sizeof(void*))) {
        PyErr_SetString(PyExc_TypeError, "bind8i() takes eight addresses");
        return nullptr;
    }
    if (!addresses(args, entry8i)) return nullptr;
    Py_RETURN_NONE;
}

template <typename F>
PyCFunction method(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef methods[] = {{"bind", method(bind), METH_FASTCALL, nullptr},
                         {"bind8", method(bind8), METH_FASTCALL, nullptr},
                         {"quantize", method(quantize), METH_FASTCALL, nullptr},
                         {"gemm", method(gemm), METH_FASTCALL, nullptr},
                         {"linear", method(linear), METH_FASTCALL, nullptr},
                         {"rmsnorm_quantize8", method(rmsnorm_quantize8), METH_FASTCALL, nullptr},
                         {"quantize8", method(quantize8), METH_FASTCALL, nullptr},
                         {"quantize_weights8", method(quantize_weights8), METH_FASTCALL, nullptr},
                         {"gemm8", method(gemm8), METH_FASTCALL, nullptr},
                         {"bind8i", method(bind8i), METH_FASTCALL, nullptr},
                         {"rmsnorm_quantize8i", method(rmsnorm_quantize8i), METH_FASTCALL, nullptr},
                         {"quantize8i", method(quantize8i), METH_FASTCALL, nullptr},
                         {"gemm8i", method(gemm8i), METH_FASTCALL, nullptr},
                         {"route", method(route), METH_FASTCALL, nullptr},
                         {"combine", method(combine), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
