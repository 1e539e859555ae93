// Marshalling of torch tensors for the operators of a transformer's step: a small Python module in C++, because these calls
// take 4 to 40 us on the GPU and the same work in Python took 10 to 45 us on the host.  It checks what it is given,
// allocates results and workspaces with torch on the current stream, calls the C ABI and returns the status; no arithmetic.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/core/LegacyTypeDispatch.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <initializer_list>
#include <stdexcept>
#include <string>
#include <vector>

#include "../../include/daf.h"

namespace {

struct Refusal : std::invalid_argument {
    using std::invalid_argument::invalid_argument;
};
[[noreturn]] void refuse(const char *where, const std::string &what) { throw Refusal(std::string(where) + ": " + what); }

std::string shape_of(const at::Tensor &t)
{
    std::string s = "(";
    for (int64_t n : t.sizes()) s += std::to_string(n) + ", ";
    return s + ")";
}

const at::Tensor &tensor(const char *where, PyObject *o)
{
    if (!THPVariable_Check(o)) refuse(where, "expected a tensor");
    return THPVariable_Unpack(o);
}
// None gives an undefined tensor
at::Tensor maybe(const char *where, PyObject *o) { return o == Py_None ? at::Tensor() : tensor(where, o); }

uint32_t code(const char *where, const at::Tensor &t)
{
    switch (t.scalar_type()) {
    case at::kFloat: return DAF_F32;
    case at::kHalf: return DAF_F16;
    case at::kBFloat16: return DAF_BF16;
    default: refuse(where, std::string("tensors of ") + at::toString(t.scalar_type()) + " are not supported");
    }
}
int device(const char *where, const at::Tensor &t)
{
    if (!t.is_cuda()) refuse(where, "expects CUDA tensors");
    return t.get_device();
}
void same_device(const char *where, int index, const at::Tensor &t)
{
    if (t.defined() && (!t.is_cuda() || t.get_device() != index)) refuse(where, "all tensors belong on one CUDA device");
}
void *ptr(const at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }
bool aligned(const at::Tensor &t, uintptr_t to) { return (reinterpret_cast<uintptr_t>(t.data_ptr()) & (to - 1)) == 0; }
void onto_boundary(at::Tensor &t, uintptr_t to)                     // t is contiguous
{
    if (t.defined() && !aligned(t, to)) t = t.clone();
}
at::Tensor bytes(uint64_t n, const at::Tensor &like) { return at::empty({(int64_t)n}, like.options().dtype(at::kByte)); }
at::Tensor dense(at::IntArrayRef shape, const at::Tensor &like) { return at::empty(shape, like.options()); }

// The caller's tensor is about to be written: autograd may keep it for something else.
void modified(const at::Tensor &t)
{
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

PyObject *wrap(const at::Tensor &t)
{
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}
PyObject *answer(std::initializer_list<at::Tensor> ts, daf_status status)
{
    PyObject *r = PyTuple_New((Py_ssize_t)ts.size() + 1);
    Py_ssize_t i = 0;
    for (const at::Tensor &t : ts) PyTuple_SET_ITEM(r, i++, wrap(t));
    PyTuple_SET_ITEM(r, i, PyLong_FromLong(status));
    return r;
}
bool truth(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Refusal("a truth value was expected");
    return v != 0;
}
double number(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Refusal("a number was expected");
    return v;
}

template <typename F> PyObject *guarded(Py_ssize_t given, Py_ssize_t wanted, F body)
{
    if (given != wanted) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        at::AutoDispatchBelowADInplaceOrView below;                 // nothing here is recorded
        return body();
    } catch (const Refusal &e) {
        PyErr_Clear();
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (...) {                                                 // torch's own, as torch tells them (out of memory among them)
        torch::translate_exception_to_python(std::current_exception());
    }
    return nullptr;
}

// --------------------------------------------------------------------------------------------- attention
// A tensor that the kernels can address: rows contiguous and on 16-byte boundaries, nothing broadcast.
bool addressable(const at::Tensor &t)
{
    const int64_t unit = 16 / t.element_size();
    const at::IntArrayRef n = t.sizes(), s = t.strides();
    if (s[3] != 1 && n[3] > 1) return false;
    for (int i = 0; i < 3; i++)
        if (n[i] > 1 && (s[i] % unit || s[i] < n[3])) return false;
    return aligned(t, 16);
}
at::Tensor readable(const at::Tensor &t)
{
    if (addressable(t)) return t;
    at::Tensor c = t.contiguous();
    return aligned(c, 16) ? c : c.clone();
}
void strides(uint64_t (&to)[3], const at::Tensor &t)
{
    for (int i = 0; i < 3; i++) to[i] = (uint64_t)t.stride(i);
}
void like(const char *where, const char *name, const at::Tensor &t, const at::Tensor &model)
{
    if (t.scalar_type() != model.scalar_type() || t.sizes() != model.sizes())
        refuse(where, std::string(name) + " is " + at::toString(t.scalar_type()) + " " + shape_of(t) + ", expected " + at::toString(model.scalar_type()) + " " + shape_of(model));
    same_device(where, model.get_device(), t);
}
void writable(const char *where, const char *name, const at::Tensor &t)
{
    if (t.numel() && !addressable(t)) refuse(where, std::string(name) + " needs a contiguous last dimension and rows on 16-byte boundaries");
}

struct Attention {
    daf_attention_params p{};
    at::Tensor q, k, v, lengths;
    Attention(const char *where, PyObject *const *a, PyObject *key_lengths, PyObject *causal, PyObject *scale)
    {
        q = tensor(where, a[0]);
        k = tensor(where, a[1]);
        v = tensor(where, a[2]);
        const int index = device(where, q);
        if (q.dim() != 4 || k.dim() != 4 || v.sizes() != k.sizes()) refuse(where, "expects q [B, Sq, H, D], k and v [B, Sk, Hkv, D]");
        if (q.size(0) != k.size(0) || q.size(3) != k.size(3) || k.size(2) == 0 || q.size(2) % k.size(2))
            refuse(where, "q " + shape_of(q) + " and k " + shape_of(k) + " do not belong together");
        if (k.scalar_type() != q.scalar_type() || v.scalar_type() != q.scalar_type()) refuse(where, "q, k and v have one type");
        same_device(where, index, k);
        same_device(where, index, v);
        lengths = maybe(where, key_lengths);
        if (lengths.defined() && (lengths.scalar_type() != at::kInt || lengths.dim() != 1 || lengths.size(0) != q.size(0) || !lengths.is_contiguous()))
            refuse(where, "key_lengths is a contiguous int32 tensor of " + std::to_string(q.size(0)) + " lengths");
        same_device(where, index, lengths);
        for (int64_t n : {q.size(0), q.size(1), k.size(1), q.size(2), q.size(3)})
            if (n > 0x7FFFFFFF) refuse(where, "a dimension is too large");
        p.struct_size = sizeof(p);
        p.dtype = code(where, q);
        p.batch = (uint32_t)q.size(0);
        p.queries = (uint32_t)q.size(1);
        p.keys = (uint32_t)k.size(1);
        p.heads = (uint32_t)q.size(2);
        p.kv_heads = (uint32_t)k.size(2);
        p.head_dim = (uint32_t)q.size(3);
        p.causal = truth(causal) ? 1u : 0u;
        p.scale = scale == Py_None ? (float)(1.0 / std::sqrt((double)q.size(3))) : (float)number(scale);
        q = readable(q);
        k = readable(k);
        v = readable(v);
        strides(p.q_stride, q);
        strides(p.k_stride, k);
        strides(p.v_stride, v);
    }
    void check_lse(const char *where, const at::Tensor &lse) const
    {
        if (lse.scalar_type() != at::kFloat || lse.dim() != 3 || lse.size(0) != q.size(0) || lse.size(1) != q.size(2) || lse.size(2) != q.size(1) || !lse.is_contiguous())
            refuse(where, "lse is a contiguous float32 tensor [B, H, Sq]");
        same_device(where, q.get_device(), lse);
    }
};

// (q, k, v, key_lengths, out, lse, causal, scale, check) -> (out, lse, status)
PyObject *attention(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 9, [&]() {
        const char *const where = "attention";
        Attention t(where, a, a[3], a[6], a[7]);
        const c10::cuda::CUDAGuard on(t.q.device());
        const cudaStream_t stream = c10::cuda::getCurrentCUDAStream().stream();
        at::Tensor out = maybe(where, a[4]), lse = maybe(where, a[5]);
        if (!out.defined()) out = dense(t.q.sizes(), t.q);
        else like(where, "out", out, t.q), writable(where, "out", out), modified(out);
        if (!lse.defined()) lse = at::empty({t.q.size(0), t.q.size(2), t.q.size(1)}, t.q.options().dtype(at::kFloat));
        else t.check_lse(where, lse), modified(lse);
        strides(t.p.out_stride, out);
        const uint64_t size = daf_attention_workspace(&t.p);
        const at::Tensor ws = bytes(size, t.q);
        daf_status st = daf_attention(&t.p, ptr(t.q), ptr(t.k), ptr(t.v), static_cast<const int32_t *>(ptr(t.lengths)), ptr(out),
                                      static_cast<float *>(ptr(lse)), ptr(ws), size, stream);
        if (st == DAF_OK && truth(a[8]) && out.numel()) st = daf_poll_status(ptr(ws), stream);
        return answer({out, lse}, st);
    });
}

// (q, k, v, out, lse, grad_out, key_lengths, grad_q, grad_k, grad_v, causal, scale, check) -> (grad_q, grad_k, grad_v, status)
PyObject *attention_grad(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 13, [&]() {
        const char *const where = "attention_grad";
        Attention t(where, a, a[6], a[10], a[11]);
        const c10::cuda::CUDAGuard on(t.q.device());
        const cudaStream_t stream = c10::cuda::getCurrentCUDAStream().stream();
        at::Tensor out = tensor(where, a[3]), grad_out = tensor(where, a[5]);
        const at::Tensor &lse = tensor(where, a[4]);
        like(where, "out", out, t.q);
        like(where, "grad_out", grad_out, t.q);
        t.check_lse(where, lse);
        out = readable(out);
        grad_out = readable(grad_out);
        at::Tensor g[3];
        const at::Tensor *const model[3] = {&t.q, &t.k, &t.v};
        const char *const name[3] = {"grad_q", "grad_k", "grad_v"};
        for (int i = 0; i < 3; i++) {
            g[i] = maybe(where, a[7 + i]);
            if (!g[i].defined()) g[i] = dense(model[i]->sizes(), *model[i]);
            else like(where, name[i], g[i], *model[i]), writable(where, name[i], g[i]), modified(g[i]);
        }
        strides(t.p.out_stride, out);
        strides(t.p.grad_out_stride, grad_out);
        strides(t.p.grad_q_stride, g[0]);
        strides(t.p.grad_k_stride, g[1]);
        strides(t.p.grad_v_stride, g[2]);
        const uint64_t size = daf_attention_grad_workspace(&t.p);
        const at::Tensor ws = bytes(size, t.q);
        daf_status st = daf_attention_grad(&t.p, ptr(t.q), ptr(t.k), ptr(t.v), static_cast<const int32_t *>(ptr(t.lengths)), ptr(out),
                                           static_cast<const float *>(ptr(lse)), ptr(grad_out), ptr(g[0]), ptr(g[1]), ptr(g[2]), ptr(ws), size, stream);
        if (st == DAF_OK && truth(a[12]) && (g[0].numel() || g[1].numel())) st = daf_poll_status(ptr(ws), stream);
        return answer({g[0], g[1], g[2]}, st);
    });
}

// --------------------------------------------------------------------------------------------- join
struct Join {
    daf_norm_params p{};
    at::Tensor x, y, weight, bias, gate, post_weight, post_bias;
    // a: x (or z), y, weight, bias, gate, post_weight, post_bias, residual_scale, kind, eps
    Join(const char *where, PyObject *const *a)
    {
        x = tensor(where, a[0]);
        const int index = device(where, x);
        y = tensor(where, a[1]);
        weight = tensor(where, a[2]);
        bias = maybe(where, a[3]);
        gate = maybe(where, a[4]);
        post_weight = maybe(where, a[5]);
        post_bias = maybe(where, a[6]);
        if (x.dim() < 1) refuse(where, "expects rows");
        const int64_t width = x.size(-1), kind = (int64_t)number(a[8]);
        if (width > 0x7FFFFFFF) refuse(where, "rows are too wide");
        p.struct_size = sizeof(p);
        p.dtype = code(where, x);
        p.param_dtype = code(where, weight);
        p.kind = (uint32_t)kind;
        p.rows = width ? (uint64_t)(x.numel() / width) : 0u;
        p.width = (uint32_t)width;
        p.residual_scale = (float)number(a[7]);
        p.eps = (float)number(a[9]);
        activation(where, "y", y);
        if (!x.is_contiguous()) refuse(where, "activations are contiguous");
        const at::Tensor *const vectors[4] = {&weight, &bias, &post_weight, &post_bias};
        for (const at::Tensor *v : vectors)
            if (v->defined()) parameter(where, index, *v, v->dim() == 1 && v->size(0) == width);
        if (gate.defined()) {
            const bool one = gate.dim() == 1;
            parameter(where, index, gate, (one && gate.size(0) == width) || (gate.dim() == 2 && gate.size(0) > 0 && gate.size(1) == width));
            p.gates = one ? 1u : (uint32_t)gate.size(0);
        }
        for (at::Tensor *const v : {&x, &y}) onto_boundary(*v, boundary());
        for (at::Tensor *const v : {&weight, &bias, &gate, &post_weight, &post_bias}) onto_boundary(*v, 16);
    }
    uintptr_t boundary() const { return p.dtype == DAF_F32 ? 32 : 16; }
    void result(const char *where, const char *name, const at::Tensor &t) const
    {
        activation(where, name, t);
        if (!aligned(t, boundary())) refuse(where, std::string(name) + " needs a start on a " + std::to_string(boundary()) + "-byte boundary");
        modified(t);
    }
    void activation(const char *where, const char *name, const at::Tensor &t) const
    {
        like(where, name, t, x);
        if (!t.is_contiguous()) refuse(where, "activations are contiguous");
    }
    void parameter(const char *where, int index, const at::Tensor &t, bool shape) const
    {
        same_device(where, index, t);
        if (!shape || t.scalar_type() != weight.scalar_type() || !t.is_contiguous())
            refuse(where, "weights and biases are contiguous vectors of the rows' width and of one type, a gate is [width] or [G, width]");
    }
};

// (x, y, weight, bias, gate, post_weight, post_bias, residual_scale, kind, eps, z, h) -> (z, h, status)
PyObject *residual_norm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 12, [&]() {
        const char *const where = "residual_norm";
        const Join t(where, a);
        const c10::cuda::CUDAGuard on(t.x.device());
        at::Tensor z = maybe(where, a[10]), h = maybe(where, a[11]);
        if (z.defined()) t.result(where, "z", z);
        else z = dense(t.x.sizes(), t.x);
        if (h.defined()) t.result(where, "h", h);
        else h = dense(t.x.sizes(), t.x);
        const daf_status st = daf_residual_norm(&t.p, ptr(t.x), ptr(t.y), ptr(t.weight), ptr(t.bias), ptr(t.gate), ptr(t.post_weight), ptr(t.post_bias),
                                                ptr(z), ptr(h), c10::cuda::getCurrentCUDAStream().stream());
        return answer({z, h}, st);
    });
}

// (z, y, weight, bias, gate, post_weight, post_bias, residual_scale, kind, eps, grad_z, grad_h)
//     -> (x, y, weight, bias, gate, post_weight, post_bias, status)
PyObject *residual_norm_grad(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 12, [&]() {
        const char *const where = "residual_norm_grad";
        const Join t(where, a);
        const c10::cuda::CUDAGuard on(t.x.device());
        at::Tensor grad_z = maybe(where, a[10]), grad_h = tensor(where, a[11]);
        if (grad_z.defined()) t.activation(where, "grad_z", grad_z);
        t.activation(where, "grad_h", grad_h);
        onto_boundary(grad_z, t.boundary());
        onto_boundary(grad_h, t.boundary());
        const auto as = [](const at::Tensor &v) { return v.defined() ? dense(v.sizes(), v) : at::Tensor(); };
        const at::Tensor gx = as(t.x), gy = as(t.x), gw = as(t.weight), gb = as(t.bias), gg = as(t.gate), gpw = as(t.post_weight), gpb = as(t.post_bias);
        const uint64_t size = daf_residual_norm_grad_workspace(&t.p);
        const at::Tensor ws = bytes(size, t.x);
        const daf_status st = daf_residual_norm_grad(&t.p, ptr(t.x), ptr(t.y), ptr(t.weight), ptr(t.gate), ptr(t.post_weight), ptr(t.post_bias), ptr(grad_z),
                                                     ptr(grad_h), ptr(gx), ptr(gy), ptr(gw), ptr(gb), ptr(gg), ptr(gpw), ptr(gpb), ptr(ws), size,
                                                     c10::cuda::getCurrentCUDAStream().stream());
        return answer({gx, gy, gw, gb, gg, gpw, gpb}, st);
    });
}

// --------------------------------------------------------------------------------------------- clipping
// (grads: list, out: list or None, max_norm, eps) -> (norm, status)
PyObject *clip_grad_norm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 4, [&]() {
        const char *const where = "clip_grad_norm";
        if (!PyList_Check(a[0]) || (a[1] != Py_None && !PyList_Check(a[1]))) refuse(where, "expects lists of tensors");
        const size_t count = (size_t)PyList_GET_SIZE(a[0]);
        if (count == 0) refuse(where, "expects at least one tensor");
        if (a[1] != Py_None && (size_t)PyList_GET_SIZE(a[1]) != count) refuse(where, "out holds one tensor for each gradient");
        std::vector<uint32_t> types(count);
        std::vector<uint64_t> numel(count);
        std::vector<const void *> src(count);
        std::vector<void *> dst(count);
        const at::Tensor &first = tensor(where, PyList_GET_ITEM(a[0], 0));
        const int index = device(where, first);
        for (size_t i = 0; i < count; i++) {
            const at::Tensor &g = tensor(where, PyList_GET_ITEM(a[0], (Py_ssize_t)i));
            same_device(where, index, g);
            if (!g.is_non_overlapping_and_dense()) refuse(where, "expects tensors without gaps, in any order");
            types[i] = code(where, g);
            numel[i] = (uint64_t)g.numel();
            src[i] = dst[i] = g.data_ptr();
            if (a[1] == Py_None) {
                modified(g);
                continue;
            }
            const at::Tensor &o = tensor(where, PyList_GET_ITEM(a[1], (Py_ssize_t)i));
            same_device(where, index, o);
            const bool alike = o.is_contiguous() ? g.is_contiguous() : o.sizes() == g.sizes() && o.strides() == g.strides();
            if (o.scalar_type() != g.scalar_type() || o.numel() != g.numel() || !alike)
                refuse(where, "an output differs from its gradient in size, type or order");
            dst[i] = o.data_ptr();
            modified(o);
        }
        const c10::cuda::CUDAGuard on(first.device());
        const at::Tensor norm = at::empty({}, first.options().dtype(at::kFloat));
        const uint64_t size = daf_clip_norm_workspace((uint32_t)count);
        const at::Tensor ws = bytes(size, first);
        const daf_status st = daf_clip_norm_batch((uint32_t)count, types.data(), src.data(), dst.data(), numel.data(), (float)number(a[2]), (float)number(a[3]),
                                                  static_cast<float *>(ptr(norm)), ptr(ws), size, c10::cuda::getCurrentCUDAStream().stream());
        return answer({norm}, st);
    });
}

// (tensor) -> whether it fills its memory without gaps or overlaps, in any order
PyObject *gap_free(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 1, [&]() { return PyBool_FromLong(tensor("gap_free", a[0]).is_non_overlapping_and_dense()); });
}

#define DAF_METHOD(NAME) {#NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(&NAME)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {DAF_METHOD(attention), DAF_METHOD(attention_grad), DAF_METHOD(residual_norm), DAF_METHOD(residual_norm_grad),
                         DAF_METHOD(clip_grad_norm), DAF_METHOD(gap_free), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
