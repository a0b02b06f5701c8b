// The binding's host path in native code: takes the pointers out of torch tensors, allocates what the caller did not
// hand over (output buffers, workspaces) and calls the C ABI of include/nvfp4.h.  Argument marshalling only, with the
// names of the C functions; binding.py holds the Python signatures.
//
// A small call is bound by this work, not by its kernels: through ctypes and torch.empty a quantizer call spent 15.5 us
// on the host (three output buffers and a workspace 6.6, the current stream 2.9, argument objects 2.5, the launch 3.4),
// of which the launch and four allocations at 0.5 us each remain.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/impl/DeviceGuardImplInterface.h>
#include <torch/csrc/Device.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <algorithm>
#include <vector>

#include "../../include/nvfp4.h"

namespace {

PyObject *s_codes, *s_scales, *s_global_scale, *s_rows, *s_K;      // attribute names

struct Fail {};                                                     // a Python error has been set

void fail(PyObject *type, const char *text)
{
    PyErr_SetString(type, text);
    throw Fail();
}
void require(bool ok, const char *text)
{
    if (!ok) fail(PyExc_AssertionError, text);
}

const at::Tensor &tensor(PyObject *o)
{
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, "expected a torch.Tensor");
    return THPVariable_Unpack(o);
}
void *address(PyObject *o) { return o == Py_None ? nullptr : tensor(o).data_ptr(); }

long long number(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Fail();
    return v;
}
void *stream_of(PyObject *o)
{
    void *p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) throw Fail();
    return p;
}

PyObject *attribute(PyObject *o, PyObject *name)                    // (borrowed by the caller for as long as o keeps it)
{
    PyObject *a = PyObject_GetAttr(o, name);
    if (!a) throw Fail();
    return a;
}

// An NVFP4Tensor; holds references, so the buffers live through the call whatever other threads do to the object (what
// stands in the argument list itself is held by the caller)
struct Quantized {
    nvfp4_tensor t{};
    at::Tensor codes, scales, global_scale;
    explicit Quantized(PyObject *o)
    {
        t.codes = static_cast<uint8_t *>(buffer(o, s_codes, codes));
        t.scales = static_cast<uint8_t *>(buffer(o, s_scales, scales));
        t.global_scale = static_cast<float *>(buffer(o, s_global_scale, global_scale));
        t.rows = count(o, s_rows);
        t.K = count(o, s_K);
    }
    nvfp4_tensor *c() { return &t; }

private:
    static void *buffer(PyObject *o, PyObject *name, at::Tensor &keep)
    {
        PyObject *a = attribute(o, name);
        const bool is = THPVariable_Check(a);
        if (is) keep = THPVariable_Unpack(a);
        Py_DECREF(a);
        if (!is) fail(PyExc_TypeError, "expected an NVFP4Tensor");
        return keep.data_ptr();
    }
    static int64_t count(PyObject *o, PyObject *name)
    {
        PyObject *a = attribute(o, name);
        const long long v = PyLong_AsLongLong(a);
        Py_DECREF(a);
        if (v == -1 && PyErr_Occurred()) throw Fail();
        return v;
    }
};

at::Tensor bytes_on(const at::Device &device, int64_t n) { return at::empty({n}, at::TensorOptions().device(device).dtype(at::kByte)); }

// the caller's workspace, or one for this call: from the current stream's pool, and back to it when the call returns,
// behind the launches.  So the stream of a call without a workspace is torch's current one (binding.py sees to it).
struct Workspace {
    at::Tensor t;
    Workspace(PyObject *given, const at::Device &device, int op, int64_t a, int64_t b, int64_t c = 0)
    {
        if (given != Py_None) t = tensor(given);
        else t = bytes_on(device, std::max<int64_t>(16, (int64_t)nvfp4_workspace_bytes(op, a, b, c)));
    }
    void *data() const { return t.data_ptr(); }
    size_t size() const { return (size_t)t.numel(); }
};

// the library may wait for a lock: not under the GIL, which is taken again however the call ends (what torch throws
// while the arguments of the call are put together becomes a Python error)
struct WithoutGil {
    PyThreadState *saved = PyEval_SaveThread();
    ~WithoutGil() { PyEval_RestoreThread(saved); }
};
template <class F>
PyObject *status(F &&call)
{
    int rc;
    {
        WithoutGil released;
        rc = call();
    }
    return PyLong_FromLong(rc);
}

const at::Tensor &matrix(PyObject *o)
{
    const at::Tensor &x = tensor(o);
    require(x.scalar_type() == at::kBFloat16 && x.dim() == 2 && x.stride(1) == 1, "expected a bf16 matrix with unit stride along its rows");
    return x;
}
const at::Tensor &heads(PyObject *o)
{
    const at::Tensor &x = tensor(o);
    require(x.scalar_type() == at::kBFloat16 && x.dim() == 3 && x.is_contiguous(), "expected a contiguous bf16 tensor [T, H, d]");
    return x;
}

// ---- allocation -------------------------------------------------------------------------------------
// buffers(rows, K, device) -> codes [rows, K/2] u8, scales [rows, K/16] u8, global_scale [1] f32
PyObject *buffers(PyObject *const *a)
{
    const int64_t rows = number(a[0]), K = number(a[1]);
    const at::Device device = ((THPDevice *)a[2])->device;
    const auto bytes = at::TensorOptions().device(device).dtype(at::kByte);
    PyObject *r = PyTuple_New(3);
    if (!r) throw Fail();
    try {
        PyTuple_SET_ITEM(r, 0, THPVariable_Wrap(at::empty({rows, K / 2}, bytes)));
        PyTuple_SET_ITEM(r, 1, THPVariable_Wrap(at::empty({rows, K / 16}, bytes)));
        PyTuple_SET_ITEM(r, 2, THPVariable_Wrap(at::empty({1}, bytes.dtype(at::kFloat))));
    } catch (...) {
        Py_DECREF(r);
        throw;
    }
    return r;
}
// output(like, M, N, is_bf16) -> [M, N] beside `like`
PyObject *output(PyObject *const *a)
{
    return THPVariable_Wrap(at::empty({number(a[1]), number(a[2])},
                                      at::TensorOptions().device(tensor(a[0]).device()).dtype(a[3] == Py_True ? at::kBFloat16 : at::kFloat)));
}

// ---- quantizers: (x, ..., out, workspace, stream) -----------------------------------------------------
PyObject *quantize(PyObject *const *a)                              // x, block_axis, scale, out, workspace, stream
{
    const at::Tensor &x = matrix(a[0]);
    const int axis = (int)number(a[1]);
    Quantized out(a[3]);
    Workspace ws(a[4], x.device(), NVFP4_OP_QUANTIZE, x.size(0), x.size(1));
    const float *scale = static_cast<const float *>(address(a[2]));
    void *s = stream_of(a[5]), *p = x.data_ptr();
    return status([&] { return nvfp4_quantize(p, x.size(0), x.size(1), x.stride(0), axis, scale, out.c(), ws.data(), ws.size(), s); });
}
PyObject *quantize_4over6(PyObject *const *a)                       // x, scale, out, workspace, stream
{
    const at::Tensor &x = matrix(a[0]);
    Quantized out(a[2]);
    Workspace ws(a[3], x.device(), NVFP4_OP_QUANTIZE_4OVER6, x.size(0), x.size(1));
    const float *scale = static_cast<const float *>(address(a[1]));
    void *s = stream_of(a[4]), *p = x.data_ptr();
    return status([&] { return nvfp4_quantize_4over6(p, x.size(0), x.size(1), x.stride(0), scale, out.c(), ws.data(), ws.size(), s); });
}
PyObject *quantize_rht(PyObject *const *a)                          // x, sign_mask, scale, out, workspace, stream
{
    const at::Tensor &x = matrix(a[0]);
    const uint32_t mask = (uint32_t)number(a[1]);
    Quantized out(a[3]);
    Workspace ws(a[4], x.device(), NVFP4_OP_QUANTIZE_RHT, x.size(0), x.size(1));
    const float *scale = static_cast<const float *>(address(a[2]));
    void *s = stream_of(a[5]), *p = x.data_ptr();
    return status([&] { return nvfp4_quantize_rht(p, x.size(0), x.size(1), x.stride(0), mask, scale, out.c(), ws.data(), ws.size(), s); });
}
PyObject *quantize_2d(PyObject *const *a)                           // w, scale, out, out_t or None, workspace, stream
{
    const at::Tensor &w = matrix(a[0]);
    Quantized out(a[2]);
    const bool transposed = a[3] != Py_None;
    Quantized out_t(transposed ? a[3] : a[2]);
    Workspace ws(a[4], w.device(), NVFP4_OP_QUANTIZE_2D, w.size(0), w.size(1));
    const float *scale = static_cast<const float *>(address(a[1]));
    void *s = stream_of(a[5]), *p = w.data_ptr();
    return status([&] { return nvfp4_quantize_2d(p, w.size(0), w.size(1), w.stride(0), scale, out.c(), transposed ? out_t.c() : nullptr, ws.data(), ws.size(), s); });
}
PyObject *quantize_for_all_to_all(PyObject *const *a)               // x, P, scale, out, workspace, stream
{
    const at::Tensor &x = heads(a[0]);
    const int64_t P = number(a[1]);
    Quantized out(a[3]);
    Workspace ws(a[4], x.device(), NVFP4_OP_QUANTIZE_A2A, x.size(0), x.size(1), x.size(2));
    const float *scale = static_cast<const float *>(address(a[2]));
    void *s = stream_of(a[5]), *p = x.data_ptr();
    return status([&] { return nvfp4_quantize_for_all_to_all(p, x.size(0), x.size(1), x.size(2), P, scale, out.c(), ws.data(), ws.size(), s); });
}

// ---- KV cache -----------------------------------------------------------------------------------------
template <int OP, class F>
PyObject *kv_write(PyObject *const *a, F f)                         // kv, out, workspace, stream
{
    const at::Tensor &x = heads(a[0]);
    Quantized out(a[1]);
    Workspace ws(a[2], x.device(), OP, x.size(0), x.size(1), x.size(2));
    void *s = stream_of(a[3]), *p = x.data_ptr();
    return status([&] { return f(p, x.size(0), x.size(1), x.size(2), out.c(), ws.data(), ws.size(), s); });
}
PyObject *kv_quant(PyObject *const *a) { return kv_write<NVFP4_OP_KV_QUANT>(a, nvfp4_kv_quant); }
PyObject *kv_quant_4over6(PyObject *const *a) { return kv_write<NVFP4_OP_KV_QUANT_4OVER6>(a, nvfp4_kv_quant_4over6); }
PyObject *kv_quant_noalloc(PyObject *const *a)                      // kv, out, stream
{
    const at::Tensor &x = heads(a[0]);
    Quantized out(a[1]);
    void *s = stream_of(a[2]), *p = x.data_ptr();
    return status([&] { return nvfp4_kv_quant_noalloc(p, x.size(0), x.size(1), x.size(2), out.c(), s); });
}
PyObject *kv_quant_k(PyObject *const *a)                            // k, out, row_mean, workspace, stream
{
    const at::Tensor &x = heads(a[0]);
    Quantized out(a[1]);
    Workspace ws(a[3], x.device(), NVFP4_OP_KV_QUANT_K, x.size(0), x.size(1), x.size(2));
    void *mean = address(a[2]), *s = stream_of(a[4]), *p = x.data_ptr();
    return status([&] { return nvfp4_kv_quant_k(p, x.size(0), x.size(1), x.size(2), out.c(), mean, ws.data(), ws.size(), s); });
}
PyObject *kv_dequant(PyObject *const *a)                            // q, T, H, d, out, stream
{
    Quantized q(a[0]);
    const int64_t T = number(a[1]), H = number(a[2]), d = number(a[3]);
    void *out = address(a[4]), *s = stream_of(a[5]);
    return status([&] { return nvfp4_kv_dequant(q.c(), out, T, H, d, s); });
}
PyObject *kv_dequant_gather(PyObject *const *a)                     // [(q, row_mean or None, T), ...], H, d, out, stream
{
    // tuples of our own: a list may change under the call (attributes are read on the way, and the GIL is released)
    struct Owned {
        PyObject *o;
        explicit Owned(PyObject *sequence) : o(PySequence_Tuple(sequence))
        {
            if (!o) throw Fail();
        }
        Owned(const Owned &) = delete;
        ~Owned() { Py_DECREF(o); }
    } seq(a[0]);
    const Py_ssize_t n = PyTuple_GET_SIZE(seq.o);
    std::vector<nvfp4_kv_chunk> chunks((size_t)std::max<Py_ssize_t>(n, 1));     // (an empty list is refused for its size, not as a null pointer)
    std::vector<Quantized> keep;
    std::vector<at::Tensor> keep_means;
    keep.reserve((size_t)n);
    keep_means.reserve((size_t)n);
    for (Py_ssize_t i = 0; i < n; ++i) {
        const Owned c(PyTuple_GET_ITEM(seq.o, i));
        if (PyTuple_GET_SIZE(c.o) != 3) fail(PyExc_ValueError, "a chunk is (NVFP4Tensor, row_mean or None, T)");
        PyObject *mean = PyTuple_GET_ITEM(c.o, 1);
        keep.emplace_back(PyTuple_GET_ITEM(c.o, 0));
        if (mean != Py_None) keep_means.push_back(tensor(mean));
        chunks[(size_t)i] = {keep.back().t, address(mean), number(PyTuple_GET_ITEM(c.o, 2))};
    }
    const int64_t H = number(a[1]), d = number(a[2]);
    void *out = address(a[3]), *s = stream_of(a[4]);
    return status([&] { return nvfp4_kv_dequant_gather(chunks.data(), (int)n, out, H, d, s); });
}

// ---- GEMMs --------------------------------------------------------------------------------------------
PyObject *gemm(PyObject *const *a)                                  // A, W, out_dtype, Y, stream
{
    Quantized A(a[0]), W(a[1]);
    const int dtype = (int)number(a[2]);
    const at::Tensor &Y = tensor(a[3]);
    void *s = stream_of(a[4]), *p = Y.data_ptr();
    return status([&] { return nvfp4_gemm(A.c(), W.c(), p, Y.stride(0), dtype, s); });
}
PyObject *gemm_scale_out(PyObject *const *a)                        // A, W, Y, scale_out, workspace, stream
{
    Quantized A(a[0]), W(a[1]);
    const at::Tensor &Y = tensor(a[2]);
    Workspace ws(a[4], A.codes.device(), NVFP4_OP_GEMM_SCALE_OUT, A.t.rows, W.t.rows);
    float *scale = static_cast<float *>(address(a[3]));
    void *s = stream_of(a[5]), *p = Y.data_ptr();
    return status([&] { return nvfp4_gemm_scale_out(A.c(), W.c(), p, Y.stride(0), scale, ws.data(), ws.size(), s); });
}
PyObject *lora_down(PyObject *const *a)                             // x, a, t, workspace, stream
{
    const at::Tensor &x = matrix(a[0]), &f = tensor(a[1]);
    require(f.scalar_type() == at::kBFloat16 && f.is_contiguous() && f.dim() == 2 && f.size(0) == NVFP4_LORA_RANK && f.size(1) == x.size(1),
            "expected a contiguous bf16 factor [128, K]");
    Workspace ws(a[3], x.device(), NVFP4_OP_LORA_DOWN, x.size(0), x.size(1));
    void *t = address(a[2]), *s = stream_of(a[4]), *p = x.data_ptr(), *pa = f.data_ptr();
    return status([&] { return nvfp4_lora_down(p, x.size(0), x.size(1), x.stride(0), pa, t, ws.data(), ws.size(), s); });
}
PyObject *gemm_lora(PyObject *const *a)                             // A, W, t, b, lora_scale, out_dtype, Y, stream
{
    Quantized A(a[0]), W(a[1]);
    const at::Tensor &t = tensor(a[2]), &b = tensor(a[3]), &Y = tensor(a[6]);
    require(t.is_contiguous() && b.is_contiguous() && t.dim() == 2 && b.dim() == 2 && t.size(0) == A.t.rows && b.size(0) == W.t.rows &&
                t.size(1) == NVFP4_LORA_RANK && b.size(1) == NVFP4_LORA_RANK,
            "expected contiguous factors t [M, 128] and b [N, 128]");
    const double scale = PyFloat_AsDouble(a[4]);
    if (scale == -1.0 && PyErr_Occurred()) throw Fail();
    const int dtype = (int)number(a[5]);
    void *s = stream_of(a[7]), *pt = t.data_ptr(), *pb = b.data_ptr(), *py = Y.data_ptr();
    return status([&] { return nvfp4_gemm_lora(A.c(), W.c(), pt, pb, (float)scale, py, Y.stride(0), dtype, s); });
}
PyObject *gemm_act_quant(PyObject *const *a)                        // A, W, act, scale, out, h_bf16, workspace, stream
{
    Quantized A(a[0]), W(a[1]), out(a[4]);
    const int act = (int)number(a[2]);
    const float *scale = static_cast<const float *>(address(a[3]));
    void *h = address(a[5]);
    const int flags = (h ? 1 : 0) | ((scale && A.t.K % 64 == 0) ? 2 : 0);
    Workspace ws(a[6], A.codes.device(), NVFP4_OP_GEMM_ACT_QUANT, A.t.rows, W.t.rows, flags);
    void *s = stream_of(a[7]);
    return status([&] { return nvfp4_gemm_act_quant(A.c(), W.c(), act, scale, out.c(), h, ws.data(), ws.size(), s); });
}

// ---- norm and rotation, paged cache, attention ----------------------------------------------------------
// Everything these calls take lies on the current GPU: a tensor elsewhere would be an address that the kernels cannot read.
struct OnDevice {
    at::Device device = c10::impl::getDeviceGuardImpl(at::kCUDA)->getDevice();
    const at::Tensor &operator()(const at::Tensor &t) const
    {
        require(t.device() == device, "expected tensors on the current GPU");
        return t;
    }
};
// [T, H, d] with whole rows: heads one behind the other, any distance from token to token
const at::Tensor &rows(const at::Tensor &x)
{
    require(x.scalar_type() == at::kBFloat16 && x.dim() == 3 && x.stride(2) == 1 && x.stride(1) == x.size(2), "expected a bf16 tensor [T, H, d] with contiguous [H, d]");
    return x;
}
const at::Tensor &rows(const OnDevice &on, PyObject *o) { return rows(on(tensor(o))); }
int64_t token_stride(const at::Tensor &x) { return x.size(0) > 1 ? x.stride(0) : x.size(1) * x.size(2); }
const at::Tensor &vector_of(const OnDevice &on, PyObject *o, at::ScalarType type, int dims, const char *text)
{
    const at::Tensor &x = on(tensor(o));
    require(x.scalar_type() == type && x.dim() == dims && x.is_contiguous(), text);
    return x;
}
const at::Tensor &workspace_of(const OnDevice &on, PyObject *o)
{
    const at::Tensor &x = on(tensor(o));
    require(x.is_contiguous(), "expected a contiguous workspace");               // (an expanded one has fewer bytes than it says)
    return x;
}
// An output: the caller's tensor, or a new one (an allocation here costs 0.7 us, one through torch.empty 2.3), handed back with the status.
// A new one holds nothing: calls that leave rows out are told so, and set them to zero.
struct Output {
    PyObject *given = Py_None;
    at::Tensor t;
    Output() = default;                                               // none
    Output(const OnDevice &on, PyObject *o, at::IntArrayRef sizes, at::ScalarType type) : given(o)
    {
        t = o == Py_None ? at::empty(sizes, at::TensorOptions().device(on.device).dtype(type)) : on(tensor(o));
    }
    bool fresh() const { return given == Py_None && t.defined(); }
    PyObject *handed_back() const
    {
        if (fresh()) return THPVariable_Wrap(t);
        Py_INCREF(given);
        return given;
    }
};
// (status, output, ...) of a call
template <class F>
PyObject *status_and(std::initializer_list<const Output *> outputs, F &&call)
{
    PyObject *rc = status(call), *r = rc ? PyTuple_New(1 + (Py_ssize_t)outputs.size()) : nullptr;
    if (!r) {
        Py_XDECREF(rc);
        throw Fail();
    }
    PyTuple_SET_ITEM(r, 0, rc);
    try {
        Py_ssize_t i = 1;
        for (const Output *o : outputs) {
            PyObject *t = o->handed_back();
            if (!t) throw Fail();
            PyTuple_SET_ITEM(r, i++, t);
        }
    } catch (...) {
        Py_DECREF(r);
        throw;
    }
    return r;
}
double real(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Fail();
    return v;
}
// (positions, freqs, axis_pairs, interleaved) or None
struct Rope {
    nvfp4_rope r{};
    at::Tensor positions, freqs;
    nvfp4_rope *c = nullptr;
    Rope(const OnDevice &on, PyObject *o, int64_t T)
    {
        if (o == Py_None) return;
        if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4 || !PyTuple_Check(PyTuple_GET_ITEM(o, 2))) fail(PyExc_TypeError, "expected an NVFP4Rope");
        PyObject *pairs = PyTuple_GET_ITEM(o, 2);
        r.axes = PyTuple_GET_SIZE(pairs);
        require(r.axes <= NVFP4_ROPE_MAX_AXES, "at most 4 position axes");
        int64_t P = 0;
        for (int64_t i = 0; i < r.axes; ++i) P += r.axis_pairs[i] = number(PyTuple_GET_ITEM(pairs, i));
        r.interleaved = PyTuple_GET_ITEM(o, 3) == Py_True;
        positions = vector_of(on, PyTuple_GET_ITEM(o, 0), at::kInt, 2, "expected contiguous int32 positions [T, axes]");
        freqs = vector_of(on, PyTuple_GET_ITEM(o, 1), at::kFloat, 1, "expected contiguous fp32 frequencies [pairs]");
        require(positions.size(0) == T && positions.size(1) == r.axes, "expected positions of T tokens and as many axes as axis_pairs");
        require(freqs.size(0) == P, "expected a frequency for each pair");
        r.positions = static_cast<const int32_t *>(positions.data_ptr());
        r.freqs = static_cast<const float *>(freqs.data_ptr());
        c = &r;
    }
};
const at::Tensor &weight_of(const OnDevice &on, PyObject *o, int64_t d)
{
    const at::Tensor &w = vector_of(on, o, at::kBFloat16, 1, "expected a contiguous bf16 weight [d]");
    require(w.size(0) == d, "expected a weight of d elements");
    return w;
}
PyObject *qk_norm_rope(PyObject *const *a)                          // q, k, q_weight, k_weight, rope, eps, q_out, k_out, stream
{
    const OnDevice on;
    nvfp4_heads h[2]{}, *given[2] = {nullptr, nullptr};
    Output out[2];
    int64_t T = -1, d = -1;
    for (int i = 0; i < 2; ++i) {
        if (a[i] == Py_None) continue;
        const at::Tensor &x = rows(on, a[i]);
        out[i] = Output(on, a[6 + i], x.sizes(), at::kBFloat16);
        const at::Tensor &y = rows(out[i].t);
        require((T < 0 || T == x.size(0)) && (d < 0 || d == x.size(2)), "queries and keys of the same tokens and head size");
        require(y.sizes() == x.sizes(), "an output has its input's shape");
        T = x.size(0);
        d = x.size(2);
        h[i] = {x.data_ptr(), token_stride(x), a[2 + i] == Py_None ? nullptr : weight_of(on, a[2 + i], d).data_ptr(), y.data_ptr(), token_stride(y), x.size(1)};
        given[i] = &h[i];
    }
    const Rope rope(on, a[4], T);
    const float eps = (float)real(a[5]);
    void *s = stream_of(a[8]);
    return status_and({&out[0], &out[1]}, [&] { return nvfp4_qk_norm_rope(given[0], given[1], T, d, eps, rope.c, s); });
}
// dq, dk, q, k, q_weight, k_weight, rope, eps, dq_in, dk_in, dq_weight, dk_weight, weight_grads, workspace, stream
PyObject *qk_norm_rope_backward(PyObject *const *a)
{
    const OnDevice on;
    nvfp4_heads_grad h[2]{}, *given[2] = {nullptr, nullptr};
    Output out[2], dweight[2];
    int64_t T = -1, d = -1;
    bool weights = false;
    for (int i = 0; i < 2; ++i) {
        if (a[i] == Py_None) continue;
        const at::Tensor &dy = rows(on, a[i]);
        out[i] = Output(on, a[8 + i], dy.sizes(), at::kBFloat16);
        const at::Tensor &dx = rows(out[i].t);
        require((T < 0 || T == dy.size(0)) && (d < 0 || d == dy.size(2)), "queries and keys of the same tokens and head size");
        require(dx.sizes() == dy.sizes(), "a gradient has its input's shape");
        T = dy.size(0);
        d = dy.size(2);
        h[i].dy = dy.data_ptr();
        h[i].ld_dy = token_stride(dy);
        h[i].dx = dx.data_ptr();
        h[i].ld_dx = token_stride(dx);
        h[i].H = dy.size(1);
        if (a[4 + i] != Py_None) {
            const at::Tensor &x = rows(on, a[2 + i]);
            require(x.sizes() == dy.sizes(), "a gradient has its input's shape");
            h[i].x = x.data_ptr();
            h[i].ld_x = token_stride(x);
            h[i].weight = weight_of(on, a[4 + i], d).data_ptr();
            if (a[10 + i] != Py_None || number(a[12])) {
                dweight[i] = Output(on, a[10 + i], {d}, at::kFloat);
                const at::Tensor &dw = dweight[i].t;
                require(dw.scalar_type() == at::kFloat && dw.dim() == 1 && dw.is_contiguous() && dw.size(0) == d, "expected a contiguous fp32 weight gradient [d]");
                h[i].dweight = static_cast<float *>(dw.data_ptr());
                weights = true;
            }
        }
        else dweight[i].given = a[10 + i];
        given[i] = &h[i];
    }
    const Rope rope(on, a[6], T);
    const float eps = (float)real(a[7]);
    at::Tensor ws;
    if (a[13] != Py_None) ws = workspace_of(on, a[13]);
    else if (weights) ws = bytes_on(on.device, std::max<int64_t>(16, (int64_t)nvfp4_workspace_bytes(NVFP4_OP_QK_NORM_ROPE_BACKWARD, T, d, 0)));
    void *s = stream_of(a[14]), *w = ws.defined() ? ws.data_ptr() : nullptr;
    const size_t n = ws.defined() ? (size_t)ws.nbytes() : 0;
    return status_and({&out[0], &out[1], &dweight[0], &dweight[1]}, [&] { return nvfp4_qk_norm_rope_backward(given[0], given[1], T, d, eps, rope.c, w, n, s); });
}

// the tuple that an NVFP4KvCache keeps: k_codes, k_scales, k_global, k_mean or None, v_codes, v_scales, v_global
struct Pages {
    nvfp4_kv_cache c{};
    at::Tensor keep[7];
    Pages(const OnDevice &on, PyObject *o)
    {
        if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 7) fail(PyExc_TypeError, "expected an NVFP4KvCache");
        void *p[7] = {};
        for (int i = 0; i < 7; ++i) {
            if (i == 3 && PyTuple_GET_ITEM(o, i) == Py_None) continue;
            keep[i] = on(tensor(PyTuple_GET_ITEM(o, i)));
            p[i] = keep[i].data_ptr();
        }
        c.k_codes = static_cast<uint8_t *>(p[0]);
        c.k_scales = static_cast<uint8_t *>(p[1]);
        c.k_global = static_cast<float *>(p[2]);
        c.k_mean = p[3];
        c.v_codes = static_cast<uint8_t *>(p[4]);
        c.v_scales = static_cast<uint8_t *>(p[5]);
        c.v_global = static_cast<float *>(p[6]);
        c.n_pages = keep[0].size(0);                                 // (shapes and strides: checked once, by the NVFP4KvCache)
        c.page_tokens = keep[0].size(1);
        c.H = keep[0].size(2);
        c.d = 2 * keep[0].size(3);
    }
};
PyObject *kv_cache_write(PyObject *const *a)                        // cache, k, v, slots, scale_search, stream
{
    const OnDevice on;
    const Pages pages(on, a[0]);
    const at::Tensor &slots = vector_of(on, a[3], at::kLong, 1, "expected contiguous int64 slots [T]");
    void *p[2] = {};
    int64_t ld[2] = {};
    for (int i = 0; i < 2; ++i) {
        if (a[1 + i] == Py_None) continue;
        const at::Tensor &x = rows(on, a[1 + i]);
        require(x.size(0) == slots.size(0) && x.size(1) == pages.c.H && x.size(2) == pages.c.d, "expected a token of the cache's heads for each slot");
        p[i] = x.data_ptr();
        ld[i] = token_stride(x);
    }
    const int search = (int)number(a[4]);
    void *s = stream_of(a[5]);
    return status([&] { return nvfp4_kv_cache_write(&pages.c, p[0], ld[0], p[1], ld[1], static_cast<const int64_t *>(slots.data_ptr()), slots.size(0), search, s); });
}
PyObject *kv_cache_read(PyObject *const *a)                         // cache, slots, k_out, v_out, stream
{
    const OnDevice on;
    const Pages pages(on, a[0]);
    const at::Tensor &slots = vector_of(on, a[1], at::kLong, 1, "expected contiguous int64 slots [T]");
    void *p[2] = {};
    Output out[2];
    for (int i = 0; i < 2; ++i) {
        if (a[2 + i] == Py_None && a[3 - i] != Py_None) continue;           // (one of them alone)
        out[i] = Output(on, a[2 + i], {slots.size(0), pages.c.H, pages.c.d}, at::kBFloat16);
        const at::Tensor &x = out[i].t;
        require(x.scalar_type() == at::kBFloat16 && x.dim() == 3 && x.is_contiguous(), "expected a contiguous bf16 tensor [T, H, d]");
        require(x.size(0) == slots.size(0) && x.size(1) == pages.c.H && x.size(2) == pages.c.d, "expected room for a token of the cache's heads for each slot");
        p[i] = x.data_ptr();
    }
    void *s = stream_of(a[4]);
    const auto read = out[0].fresh() || out[1].fresh() ? nvfp4_kv_cache_read_new : nvfp4_kv_cache_read;         // (both are new, or none)
    return status_and({&out[0], &out[1]}, [&] { return read(&pages.c, static_cast<const int64_t *>(slots.data_ptr()), slots.size(0), p[0], p[1], s); });
}
// q, cache, page_table, kv_lens, q_starts, max_q, softmax_scale, causal, window, sink, out_dtype, out, lse, workspace, stream
PyObject *kv_attention(PyObject *const *a)
{
    const OnDevice on;
    const at::Tensor &q = rows(on, a[0]);
    const Pages pages(on, a[1]);
    const nvfp4_kv_cache &c = pages.c;
    const at::Tensor &table = vector_of(on, a[2], at::kInt, 2, "expected a contiguous int32 page table [B, max_pages]");
    const at::Tensor &lens = vector_of(on, a[3], at::kInt, 1, "expected contiguous int32 lengths [B]");
    const at::Tensor &starts = vector_of(on, a[4], at::kInt, 1, "expected contiguous int32 query offsets [B + 1]");
    const int64_t B = table.size(0), total_q = q.size(0), Hq = q.size(1), max_q = number(a[5]), window = number(a[8]), sink = number(a[9]);
    require(lens.size(0) == B && starts.size(0) == B + 1, "expected B lengths and B + 1 query offsets");
    require(q.size(2) == c.d, "expected queries of the cache's head size");
    const float scale = (float)real(a[6]);
    const int causal = (int)number(a[7]), dtype = (int)number(a[10]);
    const Output o(on, a[11], q.sizes(), dtype == NVFP4_OUT_F32 ? at::kFloat : at::kBFloat16), log_sum(on, a[12], {total_q, Hq}, at::kFloat);
    const at::Tensor &out = o.t, &l = log_sum.t;
    require(out.scalar_type() == (dtype == NVFP4_OUT_F32 ? at::kFloat : at::kBFloat16) && out.sizes() == q.sizes() && out.stride(2) == 1 && out.stride(1) == c.d,
            "expected an output of the queries' shape and the chosen type with contiguous [H, d]");
    require(l.scalar_type() == at::kFloat && l.dim() == 2 && l.is_contiguous() && l.size(0) == total_q && l.size(1) == Hq, "expected a contiguous fp32 lse [total_q, H]");
    float *const lse = static_cast<float *>(l.data_ptr());
    const int fresh = (o.fresh() ? NVFP4_OUT_NEW : 0) | (log_sum.fresh() ? NVFP4_LSE_NEW : 0);
    at::Tensor ws;
    if (a[13] != Py_None) ws = workspace_of(on, a[13]);
    else if (const size_t n = nvfp4_kv_attention_workspace_bytes(total_q, Hq, c.H, c.d, table.size(1) * c.page_tokens, B, max_q, window, sink)) ws = bytes_on(on.device, (int64_t)n);
    void *s = stream_of(a[14]), *w = ws.defined() ? ws.data_ptr() : nullptr, *pq = q.data_ptr(), *po = out.data_ptr();
    const size_t n = ws.defined() ? (size_t)ws.nbytes() : 0;
    const int32_t *pt = static_cast<const int32_t *>(table.data_ptr()), *pl = static_cast<const int32_t *>(lens.data_ptr()), *ps = static_cast<const int32_t *>(starts.data_ptr());
    return status_and({&o, &log_sum}, [&] {
        return nvfp4_kv_attention(pq, token_stride(q), total_q, Hq, &c, pt, table.size(1), pl, ps, B, max_q, scale, causal, window, sink, po, token_stride(out), dtype | fresh, lse, w, n, s);
    });
}

// one Python function: fixed number of positional arguments, C++ and torch exceptions turned into Python's
template <PyObject *(*F)(PyObject *const *), int N>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "%d arguments expected, %zd given", N, n);
        return nullptr;
    }
    try {
        return F(args);
    } catch (const Fail &) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}
template <PyObject *(*F)(PyObject *const *), int N>
constexpr PyMethodDef method(const char *name)
{
    return {name, (PyCFunction)(void (*)(void))entry<F, N>, METH_FASTCALL, nullptr};
}

}  // namespace

extern "C" PyObject *PyInit__host(void)
{
    static PyMethodDef methods[] = {
        method<buffers, 3>("buffers"), method<output, 4>("output"), method<quantize, 6>("quantize"),
        method<quantize_4over6, 5>("quantize_4over6"), method<quantize_rht, 6>("quantize_rht"), method<quantize_2d, 6>("quantize_2d"),
        method<quantize_for_all_to_all, 6>("quantize_for_all_to_all"), method<kv_quant, 4>("kv_quant"),
        method<kv_quant_4over6, 4>("kv_quant_4over6"), method<kv_quant_noalloc, 3>("kv_quant_noalloc"), method<kv_quant_k, 5>("kv_quant_k"),
        method<kv_dequant, 6>("kv_dequant"), method<kv_dequant_gather, 5>("kv_dequant_gather"), method<gemm, 5>("gemm"),
        method<gemm_scale_out, 6>("gemm_scale_out"), method<lora_down, 5>("lora_down"), method<gemm_lora, 8>("gemm_lora"),
        method<gemm_act_quant, 8>("gemm_act_quant"), method<qk_norm_rope, 9>("qk_norm_rope"),
        method<qk_norm_rope_backward, 15>("qk_norm_rope_backward"), method<kv_cache_write, 6>("kv_cache_write"),
        method<kv_cache_read, 5>("kv_cache_read"), method<kv_attention, 15>("kv_attention"), {nullptr, nullptr, 0, nullptr}};
    static PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};
    s_codes = PyUnicode_InternFromString("codes");
    s_scales = PyUnicode_InternFromString("scales");
    s_global_scale = PyUnicode_InternFromString("global_scale");
    s_rows = PyUnicode_InternFromString("rows");
    s_K = PyUnicode_InternFromString("K");
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", TORCH_VERSION) != 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
