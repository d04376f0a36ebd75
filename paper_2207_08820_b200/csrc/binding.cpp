// Native argument marshalling of the hot entry points (api.py): tensors in, output allocation, one C ABI call (without the GIL).  The
// same work through ctypes costs 10-20 us a call, more than a small layer takes on the GPU.  No arithmetic of the method and no decision
// about it is made here.
#include <ATen/core/grad_mode.h>
#include <ATen/cuda/EmptyTensor.h>
#include <Python.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "bitserial.h"

namespace {

struct Fail {};      // a Python error is set

const at::Tensor& tensor(PyObject* o)
{
    if (!THPVariable_Check(o)) { PyErr_SetString(PyExc_TypeError, "expected a tensor"); throw Fail(); }
    return THPVariable_Unpack(o);
}
void* pointer(const at::Tensor& t)
{
    if (!t.is_cuda() || !t.is_contiguous()) { PyErr_SetString(PyExc_ValueError, "expected a contiguous CUDA tensor"); throw Fail(); }
    return t.data_ptr();
}
// The library call runs without the GIL: a launch can wait for room in the stream's queue.
struct NoGil {
    PyThreadState* state = PyEval_SaveThread();
    ~NoGil() { PyEval_RestoreThread(state); }
};
void* pointer_or_null(PyObject* o) { return o == Py_None ? nullptr : pointer(tensor(o)); }
int integer(PyObject* o)
{
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw Fail();
    if (v > 0x7fffffffL || v < -0x7fffffffL - 1) { PyErr_SetString(PyExc_OverflowError, "integer argument out of range"); throw Fail(); }
    return static_cast<int>(v);
}
float real(PyObject* o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Fail();
    return static_cast<float>(v);
}
// `stream` argument: None (the current stream) or a torch stream.
void* stream_of(PyObject* o)
{
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
    PyObject* s = PyObject_GetAttrString(o, "cuda_stream");
    if (!s) throw Fail();
    void* p = reinterpret_cast<void*>(PyLong_AsUnsignedLongLong(s));
    Py_DECREF(s);
    if (PyErr_Occurred()) throw Fail();
    return p;
}
at::Tensor words(at::IntArrayRef shape, const at::Tensor& like)
{
    return at::detail::empty_cuda(shape, at::kInt, like.device(), std::nullopt);
}
PyObject* give(const at::Tensor& t) { return t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None); }

PyObject* result(int status, const at::Tensor& a, const at::Tensor& b)
{
    return Py_BuildValue("(iNN)", status, give(a), give(b));
}

void need(Py_ssize_t got, Py_ssize_t want)
{
    if (got != want) { PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", want, got); throw Fail(); }
}

template <typename F>
PyObject* guarded(F f)
{
    try {
        return f();
    } catch (const Fail&) {
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// Prepared filters of three bits for narrow activations hold both forms, int8 and nibbles (tc_prepare_weights in api.py): the nibbles where they are
// wanted, with the sign that says so.
const int8_t* prepared(const at::Tensor& t, int O, int C, int R, int S, int w_bits, int a_bits, int& w_sign)
{
    const int8_t* p = static_cast<const int8_t*>(pointer(t));
    if (w_bits != 3 || a_bits > 2 || w_sign != BS_SIGNED) return p;
    const size_t bytes = bs_tc_weights_bytes(O, C, R, S);
    if (bytes == 0 || t.nbytes() != 2 * bytes) return p;
    w_sign = BS_SIGNED_NIBBLES;
    return p + bytes;
}

void mismatch(const char* what) { PyErr_SetString(PyExc_ValueError, what); throw Fail(); }

// act, wgt, C, stride, pad, a_sign, w_sign, scale, bias, relu, out_bits, out_sign, residual, res_scale, res_bits, res_sign, res_c_offset,
// res_c_total, out_i32, want_i32, i32_layout, out_packed, out_c_offset, out_c_total, workspace, wgt_tc, chained, stream
PyObject* conv2d(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&] {
        need(n, 28);
        const at::Tensor &act = tensor(a[0]), &wgt = tensor(a[1]);
        if (act.dim() != 5 || wgt.dim() != 5) mismatch("packed tensors of five dimensions expected");
        bs_conv_params p{};
        p.C = integer(a[2]);
        if (act.size(3) != wgt.size(3) || act.size(3) != (p.C + 31) / 32) mismatch("channel words of activations and weights disagree");
        p.N = static_cast<int>(act.size(0)); p.H = static_cast<int>(act.size(1)); p.W = static_cast<int>(act.size(2));
        p.a_bits = static_cast<int>(act.size(4));
        p.O = static_cast<int>(wgt.size(0)); p.R = static_cast<int>(wgt.size(1)); p.S = static_cast<int>(wgt.size(2));
        p.w_bits = static_cast<int>(wgt.size(4));
        p.stride = integer(a[3]); p.pad = integer(a[4]); p.a_sign = integer(a[5]); p.w_sign = integer(a[6]);
        if (p.stride == 0) mismatch("stride is zero");
        p.scale = static_cast<const float*>(pointer_or_null(a[7])); p.bias = static_cast<const float*>(pointer_or_null(a[8]));
        p.relu = PyObject_IsTrue(a[9]);
        p.out_bits = integer(a[10]); p.out_sign = integer(a[11]);
        p.residual = static_cast<const uint32_t*>(pointer_or_null(a[12]));
        p.res_scale = real(a[13]); p.res_bits = integer(a[14]); p.res_sign = integer(a[15]); p.res_c_offset = integer(a[16]);
        p.res_c_total = integer(a[17]);
        if (p.res_c_total == 0) p.res_c_total = p.res_c_offset + p.O;
        p.i32_layout = integer(a[20]);
        p.out_c_offset = integer(a[22]); p.out_c_total = integer(a[23]);
        auto fdiv = [](int x, int y) { return x / y - (x % y != 0 && (x < 0) != (y < 0)); };
        const int64_t P = fdiv(p.H + 2 * p.pad - p.R, p.stride) + 1, Q = fdiv(p.W + 2 * p.pad - p.S, p.stride) + 1;
        const uint32_t* ap = static_cast<const uint32_t*>(pointer(act));
        const int8_t* tc = a[25] == Py_None ? nullptr : prepared(tensor(a[25]), p.O, p.C, p.R, p.S, p.w_bits, p.a_bits, p.w_sign);
        const uint32_t* wp = tc ? nullptr : static_cast<const uint32_t*>(pointer(wgt));
        at::Tensor i32, packed;
        if (a[18] != Py_None) i32 = tensor(a[18]);
        else if (PyObject_IsTrue(a[19])) i32 = p.i32_layout == BS_NCHW ? words({p.N, p.O, P, Q}, act) : words({p.N, P, Q, p.O}, act);
        if (p.out_bits > 0) {
            if (p.out_c_total == 0) p.out_c_total = p.out_c_offset + p.O;
            if (a[21] != Py_None) {
                packed = tensor(a[21]);
            } else {
                const int64_t ow = (p.out_c_total + 31) / 32;
                packed = words({p.N, P, Q, ow, p.out_bits}, act);
                // the layer overwrites its own channel words in full; words of other channels of a wider tensor start at zero
                if (ow != (p.O + 31) / 32) packed.zero_();
            }
        }
        void* st = stream_of(a[27]);
        int32_t* ip = i32.defined() ? static_cast<int32_t*>(pointer(i32)) : nullptr;
        uint32_t* op = packed.defined() ? static_cast<uint32_t*>(pointer(packed)) : nullptr;
        void* ws = tc || a[24] == Py_None ? nullptr : pointer(tensor(a[24]));
        const size_t ws_bytes = ws ? tensor(a[24]).nbytes() : 0;
        const bool use_ws = !tc && a[24] != Py_None, chained = PyObject_IsTrue(a[26]);
        int rc;
        {
            NoGil free;
            rc = tc ? (chained ? bitserial_conv2d_tc_chained(ap, tc, &p, ip, op, st) : bitserial_conv2d_tc(ap, tc, &p, ip, op, st))
                 : use_ws ? bitserial_conv2d_ws(ap, wp, &p, ip, op, ws, ws_bytes, st)
                          : bitserial_conv2d(ap, wp, &p, ip, op, st);
        }
        return result(rc, i32, packed);
    });
}

// a, w (packed rows) or w_tc, N, w_bits (both -1 with packed rows), K, a_sign, w_sign, scale, bias, relu, out_bits, out_sign, out_i32, want_i32,
// out_packed, workspace, stream
PyObject* gemm(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&] {
        need(n, 17);
        const at::Tensor &x = tensor(a[0]), &w = tensor(a[1]);
        if (x.dim() != 3) mismatch("packed rows of three dimensions expected");
        const int M = static_cast<int>(x.size(0)), a_bits = static_cast<int>(x.size(2)), K = integer(a[4]);
        int N = integer(a[2]), w_bits = integer(a[3]);
        const bool tc = N >= 0;
        if (!tc) {
            if (w.dim() != 3) mismatch("packed rows of three dimensions expected");
            if (x.size(1) != w.size(1) || x.size(1) != (static_cast<int64_t>(K) + 31) / 32) mismatch("reduction words of the operands disagree");
            N = static_cast<int>(w.size(0)); w_bits = static_cast<int>(w.size(2));
        }
        const int a_sign = integer(a[5]);
        int w_sign = integer(a[6]);
        const float *scale = static_cast<const float*>(pointer_or_null(a[7])), *bias = static_cast<const float*>(pointer_or_null(a[8]));
        const int relu = PyObject_IsTrue(a[9]), out_bits = integer(a[10]), out_sign = integer(a[11]);
        const uint32_t* xp = static_cast<const uint32_t*>(pointer(x));
        const void* wp = tc ? prepared(w, N, K, 1, 1, w_bits, a_bits, w_sign) : pointer(w);
        at::Tensor i32, packed;
        if (a[12] != Py_None) i32 = tensor(a[12]);
        else if (PyObject_IsTrue(a[13])) i32 = words({M, N}, x);
        if (out_bits > 0) packed = a[14] != Py_None ? tensor(a[14]) : words({M, (static_cast<int64_t>(N) + 31) / 32, out_bits}, x);
        void* st = stream_of(a[16]);
        int32_t* ip = i32.defined() ? static_cast<int32_t*>(pointer(i32)) : nullptr;
        uint32_t* op = packed.defined() ? static_cast<uint32_t*>(pointer(packed)) : nullptr;
        const bs_sign_t as = static_cast<bs_sign_t>(a_sign), wsn = static_cast<bs_sign_t>(w_sign), os = static_cast<bs_sign_t>(out_sign);
        const bool use_ws = !tc && a[15] != Py_None;
        void* ws = use_ws ? pointer(tensor(a[15])) : nullptr;
        const size_t ws_bytes = use_ws ? tensor(a[15]).nbytes() : 0;
        const int8_t* w8 = static_cast<const int8_t*>(wp);
        const uint32_t* w32 = static_cast<const uint32_t*>(wp);
        int rc;
        {
            NoGil free;
            rc = tc ? bitserial_gemm_tc(xp, w8, M, N, K, a_bits, as, w_bits, wsn, scale, bias, relu, out_bits, os, ip, op, st)
                 : use_ws ? bitserial_gemm_ws(xp, w32, M, N, K, a_bits, as, w_bits, wsn, scale, bias, relu, out_bits, os, ip, op, ws, ws_bytes, st)
                          : bitserial_gemm(xp, w32, M, N, K, a_bits, as, w_bits, wsn, scale, bias, relu, out_bits, os, ip, op, st);
        }
        return result(rc, i32, packed);
    });
}

// x, act_scale, a_bits, a_sign, layout, out, stream
PyObject* bitpack(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&] {
        need(n, 7);
        const at::Tensor& x = tensor(a[0]);
        if (x.scalar_type() != at::kFloat && x.scalar_type() != at::kChar) mismatch("x must be float32 or int8");
        if (x.dim() != 4) mismatch("x must have four dimensions");
        const int bits = integer(a[2]), sign = integer(a[3]), layout = integer(a[4]);
        const bool nchw = layout == BS_NCHW;
        const int64_t N = x.size(0), C = x.size(nchw ? 1 : 3), H = x.size(nchw ? 2 : 1), W = x.size(nchw ? 3 : 2), Cw = (C + 31) / 32;
        const float scale = real(a[1]);
        const void* xp = pointer(x);
        const at::Tensor out = a[5] != Py_None ? tensor(a[5]) : words({N, H, W, Cw, bits > 0 ? bits : 1}, x);
        uint32_t* op = static_cast<uint32_t*>(pointer(out));
        void* st = stream_of(a[6]);
        const bool f32 = x.scalar_type() == at::kFloat;
        int rc;
        {
            NoGil free;
            rc = bitpack_activations(xp, f32, static_cast<bs_layout_t>(layout), static_cast<int>(N), static_cast<int>(C), static_cast<int>(H),
                                     static_cast<int>(W), scale, bits, static_cast<bs_sign_t>(sign), op, st);
        }
        at::Tensor view = out;
        if (rc == BS_OK && a[5] != Py_None) view = out.view({N, H, W, Cw, bits});
        return result(rc, view, at::Tensor());
    });
}

// x, act_scale, a_bits, out, operands (of a sequence), stream
PyObject* bitpack_operands(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&] {
        need(n, 6);
        const at::Tensor &x = tensor(a[0]), &out = tensor(a[3]);
        if (x.scalar_type() != at::kFloat) mismatch("x must be float32");
        if (x.dim() != 4) mismatch("x must have four dimensions");
        const float scale = real(a[1]);
        const int bits = integer(a[2]);
        const float* xp = static_cast<const float*>(pointer(x));
        uint32_t* op = static_cast<uint32_t*>(pointer(out));
        const bs_operand_tensor* to = reinterpret_cast<const bs_operand_tensor*>(PyLong_AsUnsignedLongLong(a[4]));
        if (PyErr_Occurred()) throw Fail();
        void* st = stream_of(a[5]);
        int rc;
        {
            NoGil free;
            rc = bitpack_activations_operands(xp, static_cast<int>(x.size(0)), static_cast<int>(x.size(1)), static_cast<int>(x.size(2)),
                                              static_cast<int>(x.size(3)), scale, bits, op, to, st);
        }
        return result(rc, at::Tensor(), at::Tensor());
    });
}

// sequence, stream, ready (an operand tensor of it, or None)
PyObject* sequence_run(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&] {
        need(n, 3);
        bs_sequence* s = reinterpret_cast<bs_sequence*>(PyLong_AsUnsignedLongLong(a[0]));
        if (PyErr_Occurred()) throw Fail();
        void* st = stream_of(a[1]);
        const bs_operand_tensor* ready = a[2] == Py_None ? nullptr : reinterpret_cast<const bs_operand_tensor*>(PyLong_AsUnsignedLongLong(a[2]));
        if (PyErr_Occurred()) throw Fail();
        int rc;
        {
            NoGil free;
            rc = bs_sequence_run_ready(s, ready, st);
        }
        return PyLong_FromLong(rc);
    });
}

// dicts, values, addresses (three tuples): whether the dicts, one after the other, still hold these very objects, the tensors among them
// (address not None) at these addresses.  A pass asks this of a few hundred entries (362: 2.8 us,
// while its first kernel runs).
PyObject* unchanged(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&] {
        need(n, 3);
        if (!PyTuple_Check(a[0]) || !PyTuple_Check(a[1]) || !PyTuple_Check(a[2]) || PyTuple_GET_SIZE(a[1]) != PyTuple_GET_SIZE(a[2])) mismatch("three tuples expected, two of one length");
        const Py_ssize_t count = PyTuple_GET_SIZE(a[1]);
        Py_ssize_t at = 0;
        for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(a[0]); ++i) {
            PyObject *d = PyTuple_GET_ITEM(a[0], i), *key, *value;
            if (!PyDict_Check(d)) mismatch("dict expected");
            Py_ssize_t pos = 0;
            while (PyDict_Next(d, &pos, &key, &value)) {
                if (at == count || value != PyTuple_GET_ITEM(a[1], at)) Py_RETURN_FALSE;
                PyObject* address = PyTuple_GET_ITEM(a[2], at++);
                if (address == Py_None) continue;
                const at::Tensor& t = THPVariable_CheckExact(value) ? THPVariable_Unpack(value) : tensor(value);
                if (t.const_data_ptr() != PyLong_AsVoidPtr(address)) Py_RETURN_FALSE;
            }
        }
        return PyBool_FromLong(at == count);
    });
}

// ---- 4-bit weights with a scale per group

// The device of a call's tensors and its stream are the current ones while its memory is taken and its work enqueued: what the call allocates belongs
// to the stream that it runs on, and what the caller gives it is not taken for something else before that stream is done with it, though the caller lets
// go of it at once.  `stream` argument: None (the device's current stream) or a torch stream of that device.
struct OnStream {
    c10::cuda::OptionalCUDAGuard device;
    c10::cuda::OptionalCUDAStreamGuard guard;
    std::optional<c10::cuda::CUDAStream> given;
    void* stream;
    OnStream(const at::Tensor& x, PyObject* o)
    {
        if (!x.is_cuda()) mismatch("expected a contiguous CUDA tensor");
        const c10::DeviceIndex at = x.get_device();
        if (at != c10::cuda::current_device()) device.set_index(at);
        if (o == Py_None) {
            stream = c10::cuda::getCurrentCUDAStream(at).stream();
            return;
        }
        const int64_t id = attribute(o, "stream_id"), index = attribute(o, "device_index"), type = attribute(o, "device_type");
        if (index != at) mismatch("the stream belongs to another device than the tensors");
        const c10::cuda::CUDAStream s = c10::cuda::CUDAStream::unpack3(id, static_cast<c10::DeviceIndex>(index), static_cast<c10::DeviceType>(type));
        guard.reset_stream(s);
        given = s;
        stream = s.stream();
    }
    void keep(std::initializer_list<PyObject*> objects) const
    {
        for (PyObject* o : objects)
            if (given && o != Py_None) c10::cuda::CUDACachingAllocator::recordStream(tensor(o).storage().data_ptr(), *given);
    }
    static int64_t attribute(PyObject* o, const char* name)
    {
        PyObject* v = PyObject_GetAttrString(o, name);
        if (!v) throw Fail();
        const int64_t r = PyLong_AsLongLong(v);
        Py_DECREF(v);
        if (r == -1 && PyErr_Occurred()) throw Fail();
        return r;
    }
};
at::Tensor fresh(at::IntArrayRef shape, at::ScalarType t, const at::Tensor& like) { return at::detail::empty_cuda(shape, t, like.device(), std::nullopt); }
void same_device(const at::Tensor& t, const at::Tensor& x) { if (t.device() != x.device()) mismatch("tensors on different devices"); }
bs_float_t float_type(const at::Tensor& t)
{
    const at::ScalarType k = t.scalar_type();
    if (k != at::kFloat && k != at::kHalf && k != at::kBFloat16) mismatch("float32, float16 or bfloat16 expected");
    return k == at::kFloat ? BS_F32 : k == at::kHalf ? BS_F16 : BS_BF16;
}
// Rows of K values: a contiguous tensor, or a matrix whose rows are.  Returns how far apart they are.
int64_t row_pitch(const at::Tensor& t, int64_t K)
{
    if (t.is_contiguous()) return K;
    if (t.dim() != 2 || t.stride(1) != 1) mismatch("expected a contiguous tensor or a matrix with contiguous rows");
    return t.size(0) == 1 ? K : t.stride(0);
}
int small(int64_t v) { if (v > 0x7fffffff) mismatch("tensor too large"); return static_cast<int>(v); }
// Whether the rows of two tensors share memory.  Rows as far apart as the others may lie between them; what else reaches into the other's range is taken to overlap.
bool overlap(const at::Tensor& a, int64_t a_pitch, const at::Tensor& b, int64_t b_pitch)
{
    const int64_t a_wide = a.size(-1) * a.element_size(), b_wide = b.size(-1) * b.element_size(), a_step = a_pitch * a.element_size(), b_step = b_pitch * b.element_size();
    const int64_t from = static_cast<const char*>(b.const_data_ptr()) - static_cast<const char*>(a.const_data_ptr());       // b's first row from a's
    auto length = [](const at::Tensor& t, int64_t step, int64_t wide) { return (t.numel() / t.size(-1) - 1) * step + wide; };
    if (from >= length(a, a_step, a_wide) || -from >= length(b, b_step, b_wide)) return false;
    if (a_step != b_step || a_step <= 0) return true;
    const int64_t in = (from % a_step + a_step) % a_step;       // where b's rows begin, from the rows of a before them
    return in < a_wide || in + b_wide > a_step;
}
const void* prepared_w4(const at::Tensor& t, const at::Tensor& x, int64_t matrices, int O, int K, int group, int zeros)
{
    const size_t bytes = bs_w4_bytes(O, K, group, zeros);
    if (bytes == 0 || t.nbytes() != bytes * matrices) mismatch("prepared weights of another size");
    same_device(t, x);
    return pointer(t);
}

// The products have no backward pass: a result without a gradient must not stand where one is recorded.
void no_gradient(const at::Tensor& t)
{
    if (t.requires_grad() && at::GradMode::is_enabled()) mismatch("there is no gradient through 4-bit weights: a tensor that requires one is taken under torch.no_grad() only");
}

// w, group, zeros, type (bs_float_t of the scales), stream
PyObject* w4_quantise(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&] {
        need(n, 5);
        const at::Tensor& w = tensor(a[0]);
        if (w.dim() < 2 || w.numel() == 0) mismatch("weights of two or more dimensions, none of them zero, expected");
        const int group = integer(a[1]), zeros = PyObject_IsTrue(a[2]);
        const bs_float_t type = static_cast<bs_float_t>(integer(a[3])), from = float_type(w);
        if (group <= 0 || (type != BS_F16 && type != BS_BF16)) mismatch("a positive group and scales of float16 or bfloat16 expected");
        const OnStream on(w, a[4]);
        const int K = small(w.size(-1));
        const int64_t ld = row_pitch(w, K), rows = w.numel() / K;
        // a stack of matrices is one of all their rows, as many of them in a call as it takes (a multiple of 16: parts begin on 16-byte boundaries)
        const int64_t most = w.size(-2) <= 1 << 20 ? 1 << 20 : small(rows);
        std::vector<int64_t> shape(w.sizes().begin(), w.sizes().end());
        const at::Tensor codes = fresh(shape, at::kChar, w);
        shape.back() = (K + static_cast<int64_t>(group) - 1) / group;
        const at::Tensor scales = fresh(shape, type == BS_F16 ? at::kHalf : at::kBFloat16, w);
        at::Tensor z;
        if (zeros) z = fresh(shape, at::kChar, w);
        const char* wp = static_cast<const char*>(w.const_data_ptr());
        char *cp = static_cast<char*>(codes.data_ptr()), *sp = static_cast<char*>(scales.data_ptr()), *zp = zeros ? static_cast<char*>(z.data_ptr()) : nullptr;
        const int64_t G = shape.back(), w_size = w.element_size(), s_size = scales.element_size();
        int rc = BS_OK;
        on.keep({a[0]});
        {
            NoGil free;
            for (int64_t o = 0; o < rows && rc == BS_OK; o += most)
                rc = bs_w4_quantise(wp + o * ld * w_size, from, static_cast<int>(rows - o < most ? rows - o : most), K, ld, group, type, reinterpret_cast<int8_t*>(cp + o * K),
                                    sp + o * G * s_size, zp ? reinterpret_cast<int8_t*>(zp + o * G) : nullptr, on.stream);
        }
        return Py_BuildValue("(iNNN)", rc, give(codes), give(scales), give(z));
    });
}

// codes [O, K] or [E, O, K], scales, zeros or None, group, stream
PyObject* w4_prepare(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&] {
        need(n, 5);
        const at::Tensor &codes = tensor(a[0]), &scales = tensor(a[1]);
        if (codes.scalar_type() != at::kChar || (codes.dim() != 2 && codes.dim() != 3) || codes.numel() == 0) mismatch("int8 codes [O, K] or [E, O, K] expected");
        const int group = integer(a[3]);
        if (group <= 0) mismatch("a positive group expected");
        const int K = small(codes.size(-1)), O = small(codes.size(-2)), E = codes.dim() == 3 ? small(codes.size(0)) : 1;
        const int64_t G = (K + static_cast<int64_t>(group) - 1) / group;
        auto fits = [&](const at::Tensor& t) {
            if (t.dim() != codes.dim() || t.size(-1) != G || t.size(-2) != O || (E > 1 && t.size(0) != E) || t.numel() != static_cast<int64_t>(E) * O * G)
                mismatch("one scale (and zero point) per group of a row expected");
            same_device(t, codes);
        };
        fits(scales);
        if (float_type(scales) == BS_F32) mismatch("scales of float16 or bfloat16 expected");
        const int8_t* z = nullptr;
        if (a[2] != Py_None) {
            const at::Tensor& t = tensor(a[2]);
            if (t.scalar_type() != at::kChar) mismatch("int8 zero points expected");
            fits(t);
            z = static_cast<const int8_t*>(pointer(t));
        }
        const OnStream on(codes, a[4]);
        const size_t bytes = bs_w4_bytes(O, K, group, z != nullptr);
        if (bytes == 0) return Py_BuildValue("(iN)", static_cast<int>(BS_ERR_UNSUPPORTED), Py_NewRef(Py_None));
        const void *cp = pointer(codes), *sp = pointer(scales);
        const at::Tensor out = fresh({static_cast<int64_t>(bytes * E)}, at::kByte, codes);
        int rc;
        on.keep({a[0], a[1], a[2]});
        {
            NoGil free;
            rc = bs_w4_prepare(static_cast<const int8_t*>(cp), sp, z, E, O, K, group, out.data_ptr(), on.stream);
        }
        return Py_BuildValue("(iN)", rc, give(out));
    });
}

// x, prepared, O, K, group, zeros, type, bias or None, out or None, stream
PyObject* w4_gemm(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&] {
        need(n, 10);
        const at::Tensor &x = tensor(a[0]), &w = tensor(a[1]);
        const int O = integer(a[2]), K = integer(a[3]), group = integer(a[4]), zeros = integer(a[5]), type = integer(a[6]);
        for (int i : {0, 7, 8})
            if (a[i] != Py_None) no_gradient(tensor(a[i]));
        if (x.dim() < 1 || x.size(-1) != K) mismatch("the last dimension of x is not the weights' number of columns");
        if (float_type(x) != type) mismatch("x is not of the scales' type");
        const OnStream on(x, a[9]);
        const void* wp = prepared_w4(w, x, 1, O, K, group, zeros);
        const int M = small(x.numel() / K);
        const int64_t ldx = row_pitch(x, K);
        const void* bias = nullptr;
        if (a[7] != Py_None) {
            const at::Tensor& b = tensor(a[7]);
            if (b.scalar_type() != x.scalar_type() || b.dim() != 1 || b.size(0) != O) mismatch("a bias of x's type, one value per row of the weights, expected");
            same_device(b, x);
            bias = pointer(b);
        }
        std::vector<int64_t> shape(x.sizes().begin(), x.sizes().end());
        shape.back() = O;
        at::Tensor y;
        int64_t ldy = O;
        if (a[8] != Py_None) {
            y = tensor(a[8]);
            if (!y.is_cuda() || y.scalar_type() != x.scalar_type() || y.sizes() != at::IntArrayRef(shape)) mismatch("an output of x's type and the product's shape expected");
            same_device(y, x);
            ldy = row_pitch(y, O);
            if (M > 0 && (overlap(y, ldy, x, ldx) || overlap(y, ldy, w, w.numel()) || (bias && overlap(y, ldy, tensor(a[7]), O)))) mismatch("the output overlaps an input");
        } else {
            y = fresh(shape, x.scalar_type(), x);
        }
        if (M == 0) return Py_BuildValue("(iN)", static_cast<int>(BS_OK), give(y));
        const size_t need_ws = bs_w4_gemm_workspace_bytes(M, O, K, group, ldx);
        at::Tensor ws;
        if (need_ws) ws = fresh({static_cast<int64_t>(need_ws)}, at::kByte, x);
        void* yp = y.data_ptr();
        int rc;
        on.keep({a[0], a[1], a[7], a[8]});
        {
            NoGil free;
            rc = bs_w4_gemm(x.const_data_ptr(), ldx, M, wp, O, K, group, zeros, static_cast<bs_float_t>(type), bias, yp, ldy, need_ws ? ws.data_ptr() : nullptr, need_ws,
                            on.stream);
        }
        return Py_BuildValue("(iN)", rc, give(y));
    });
}

// x, router, gate, up, down, I, group_up, zeros_up, group_down, zeros_down, type, top_k, renormalise, out or None, stream
PyObject* w4_moe(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&] {
        need(n, 15);
        const at::Tensor &x = tensor(a[0]), &router = tensor(a[1]);
        const int I = integer(a[5]), gu = integer(a[6]), zu = integer(a[7]), gd = integer(a[8]), zd = integer(a[9]), type = integer(a[10]), top_k = integer(a[11]),
                  renormalise = PyObject_IsTrue(a[12]);
        for (int i : {0, 1, 13})
            if (a[i] != Py_None) no_gradient(tensor(a[i]));
        if (router.dim() != 2 || router.numel() == 0) mismatch("a router [E, H] expected");
        const int E = small(router.size(0)), H = small(router.size(1));
        if (x.dim() < 1 || x.size(-1) != H) mismatch("the last dimension of x is not the router's number of columns");
        if (float_type(x) != type || router.scalar_type() != x.scalar_type()) mismatch("x and the router are not of the scales' type");
        if (top_k < 1 || top_k > E) mismatch("top_k is not between one and the number of experts");
        const OnStream on(x, a[14]);
        same_device(router, x);
        const void* rp = pointer(router);
        const void *gate = prepared_w4(tensor(a[2]), x, E, I, H, gu, zu), *up = prepared_w4(tensor(a[3]), x, E, I, H, gu, zu),
                   *down = prepared_w4(tensor(a[4]), x, E, H, I, gd, zd);
        const int T = small(x.numel() / H);
        const int64_t ldx = row_pitch(x, H);
        at::Tensor y;
        if (a[13] != Py_None) {
            y = tensor(a[13]);
            if (y.scalar_type() != x.scalar_type() || y.sizes() != x.sizes()) mismatch("an output of x's type and shape expected");
            same_device(y, x);
            pointer(y);
            if (T > 0 && (overlap(y, H, x, ldx) || overlap(y, H, router, H))) mismatch("the output overlaps an input");
            for (int i = 2; i < 5 && T > 0; ++i)
                if (overlap(y, H, tensor(a[i]), tensor(a[i]).numel())) mismatch("the output overlaps an input");
        } else {
            y = fresh(x.sizes(), x.scalar_type(), x);
        }
        std::vector<int64_t> shape(x.sizes().begin(), x.sizes().end());
        shape.back() = top_k;
        const at::Tensor experts = fresh(shape, at::kInt, x), weights = fresh(shape, at::kFloat, x);
        if (T == 0) return Py_BuildValue("(iNNN)", static_cast<int>(BS_OK), give(y), give(experts), give(weights));
        const size_t bytes = bs_w4_moe_workspace_bytes(T, top_k, H, I, ldx);
        const at::Tensor ws = fresh({static_cast<int64_t>(bytes)}, at::kByte, x);
        void *yp = y.data_ptr(), *wsp = ws.data_ptr();
        int rc;
        on.keep({a[0], a[1], a[2], a[3], a[4], a[13]});
        {
            NoGil free;
            rc = bs_w4_moe(x.const_data_ptr(), ldx, T, rp, E, H, I, gate, up, gu, zu, down, gd, zd, static_cast<bs_float_t>(type), top_k, renormalise, yp,
                           static_cast<int32_t*>(experts.data_ptr()), static_cast<float*>(weights.data_ptr()), wsp, bytes, on.stream);
        }
        return Py_BuildValue("(iNNN)", rc, give(y), give(experts), give(weights));
    });
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(conv2d), FAST(gemm), FAST(bitpack), FAST(bitpack_operands), FAST(sequence_run), FAST(unchanged),
                         FAST(w4_quantise), FAST(w4_prepare), FAST(w4_gemm), FAST(w4_moe), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&module); }
