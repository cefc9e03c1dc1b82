// The online calls' marshalling in native code: argument checks, output and scratch tensors, the C entry point.  In Python (torch.empty
// twice, a ctypes call of twenty arguments) it took 4.7 us of the 12.9 that a linear costs the host, more than the GPU needs for
// the smallest shapes (two launches of 2.2 us each are the rest).  Calls with an explicit stream keep the Python path, which
// places memory in that stream's pool.  The functions return the entry point's status beside the tensors; the entry points' addresses come
// from the ctypes library, so that there is one copy of it.
#include <Python.h>

#include <stdint.h>

#include <algorithm>
#include <initializer_list>
#include <string>
#include <vector>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/utils/pybind.h>

#include "../../include/qarvd.h"

namespace py = pybind11;
using OptTensor = std::optional<at::Tensor>;

namespace {

decltype(&qarvd_linear) linear_fn = nullptr;
decltype(&qarvd_linear_workspace) linear_workspace_fn = nullptr;
decltype(&qarvd_packed_ld) packed_ld_fn = nullptr;
decltype(&qarvd_quant_act) quant_act_fn = nullptr;
decltype(&qarvd_quant_act_static) quant_act_static_fn = nullptr;
decltype(&qarvd_w8a8_dual_gemm_variant) gemm_fn = nullptr;
decltype(&qarvd_w4a8_dual_gemm) gemm_w4_fn = nullptr;
decltype(&qarvd_w8a8_dual_gemm_q8) gemm_q8_fn = nullptr;

decltype(&qarvd_dual_gemm_fused) gemm_fused_fn = nullptr;
decltype(&qarvd_linear_fused) linear_fused_fn = nullptr;
decltype(&qarvd_qk_norm_rope) heads_fn = nullptr;
decltype(&qarvd_linear_qkv) linear_qkv_fn = nullptr;

void init(const std::vector<uintptr_t> &a)
{
    linear_fn = reinterpret_cast<decltype(linear_fn)>(a.at(0));
    linear_workspace_fn = reinterpret_cast<decltype(linear_workspace_fn)>(a.at(1));
    packed_ld_fn = reinterpret_cast<decltype(packed_ld_fn)>(a.at(2));
    quant_act_fn = reinterpret_cast<decltype(quant_act_fn)>(a.at(3));
    quant_act_static_fn = reinterpret_cast<decltype(quant_act_static_fn)>(a.at(4));
    gemm_fn = reinterpret_cast<decltype(gemm_fn)>(a.at(5));
    gemm_w4_fn = reinterpret_cast<decltype(gemm_w4_fn)>(a.at(6));
    gemm_q8_fn = reinterpret_cast<decltype(gemm_q8_fn)>(a.at(7));
}

void init_block(const std::vector<uintptr_t> &a)
{
    gemm_fused_fn = reinterpret_cast<decltype(gemm_fused_fn)>(a.at(0));
    linear_fused_fn = reinterpret_cast<decltype(linear_fused_fn)>(a.at(1));
    heads_fn = reinterpret_cast<decltype(heads_fn)>(a.at(2));
    linear_qkv_fn = reinterpret_cast<decltype(linear_qkv_fn)>(a.at(3));
}

void *ptr(const OptTensor &t) { return t ? t->data_ptr() : nullptr; }

void check_2d(const at::Tensor &t, const char *what)
{
    if (!t.is_cuda() || t.dim() != 2 || t.stride(1) != 1)
        throw py::value_error(std::string(what) + " must be a 2-D device tensor with unit inner stride");
}

qarvd_dtype dtype_of(at::ScalarType s)
{
    if (s == at::kFloat) return QARVD_F32;
    if (s == at::kBFloat16) return QARVD_BF16;
    throw py::type_error("expected float32 or bfloat16, got " + std::string(py::str(py::cast(s))));
}

at::Tensor fresh(at::IntArrayRef size, at::ScalarType dtype, const at::Tensor &like)
{
    return at::empty(size, at::TensorOptions().dtype(dtype).device(like.device()));
}

// Runs a C entry point without the interpreter lock (a launch waits when the queue is full).
template <typename F> int run(F f)
{
    py::gil_scoped_release release;
    return (int)f();
}

py::tuple linear(const at::Tensor &X, const OptTensor &perm, int bits, const at::Tensor &Wq, const at::Tensor &sn, const at::Tensor &so,
                 const OptTensor &bias, int64_t N, int64_t K, int64_t K_o, std::optional<at::ScalarType> out_dtype, uintptr_t stream)
{
    check_2d(X, "X");
    const at::ScalarType out = c10::dtype_or_default(out_dtype);
    const int64_t M = X.size(0);
    if (X.size(1) != K)
        throw py::value_error("X has " + std::to_string(X.size(1)) + " channels, the layer " + std::to_string(K));
    const size_t need = linear_workspace_fn((int32_t)M, (int32_t)K, (int32_t)K_o);
    const at::Tensor ws = fresh({(int64_t)need}, at::kByte, X);
    at::Tensor Y = fresh({M, N}, out, X);
    const qarvd_dtype xdt = dtype_of(X.scalar_type()), ydt = dtype_of(out);
    const int st = run([&] {
        return linear_fn(X.data_ptr(), xdt, X.stride(0), (const int32_t *)ptr(perm), bits, Wq.data_ptr(), Wq.stride(0), (const float *)sn.data_ptr(),
                         (const float *)so.data_ptr(), (const float *)ptr(bias), (int32_t)M, (int32_t)N, (int32_t)K, (int32_t)K_o, Y.data_ptr(),
                         ydt, N, ws.data_ptr(), need, (void *)stream);
    });
    return py::make_tuple(st, std::move(Y));
}

py::tuple quant_act(const at::Tensor &X, const OptTensor &perm, int64_t K_o, OptTensor Xq, OptTensor s_x, uintptr_t stream)
{
    check_2d(X, "X");
    const int64_t M = X.size(0), K = X.size(1);
    if (!Xq) Xq = fresh({M, (int64_t)packed_ld_fn((int32_t)K, (int32_t)K_o)}, at::kChar, X);
    if (!s_x) s_x = fresh({M}, at::kFloat, X);
    const qarvd_dtype xdt = dtype_of(X.scalar_type());
    const int st = run([&] {
        return quant_act_fn(X.data_ptr(), xdt, (int32_t)M, (int32_t)K, X.stride(0), (const int32_t *)ptr(perm), (int32_t)K_o,
                            (int8_t *)Xq->data_ptr(), Xq->stride(0), (float *)s_x->data_ptr(), (void *)stream);
    });
    return py::make_tuple(st, std::move(Xq), std::move(s_x));
}

// The scale is required (None is a TypeError): a call without one must not become the per-token quantizer.
py::tuple quant_act_static(const at::Tensor &X, const OptTensor &perm, int64_t K_o, double scale, OptTensor Xq, uintptr_t stream)
{
    check_2d(X, "X");
    const int64_t M = X.size(0), K = X.size(1);
    if (!Xq) Xq = fresh({M, (int64_t)packed_ld_fn((int32_t)K, (int32_t)K_o)}, at::kChar, X);
    const qarvd_dtype xdt = dtype_of(X.scalar_type());
    const int st = run([&] {
        return quant_act_static_fn(X.data_ptr(), xdt, (int32_t)M, (int32_t)K, X.stride(0), (const int32_t *)ptr(perm), (int32_t)K_o, (float)scale,
                                   (int8_t *)Xq->data_ptr(), Xq->stride(0), (void *)stream);
    });
    return py::make_tuple(st, std::move(Xq));
}

// A vector that is missing (None) is refused by the entry point, with its status.
py::tuple gemm(const at::Tensor &Xq, const OptTensor &s_x, int bits, const at::Tensor &Wq, const OptTensor &sn, const OptTensor &so,
               const OptTensor &bias, int64_t M, int64_t N, int64_t K, int64_t K_o, std::optional<at::ScalarType> out_dtype, OptTensor Y,
               int variant, uintptr_t stream)
{
    if (!Y) Y = fresh({M, N}, c10::dtype_or_default(out_dtype), Xq);
    const qarvd_dtype ydt = dtype_of(Y->scalar_type());
    const int st = run([&] {
        if (bits == 4)
            return gemm_w4_fn((const int8_t *)Xq.data_ptr(), Xq.stride(0), (const float *)ptr(s_x), (const uint8_t *)Wq.data_ptr(), Wq.stride(0),
                              (const float *)ptr(sn), (const float *)ptr(so), (const float *)ptr(bias), (int32_t)M, (int32_t)N, (int32_t)K,
                              (int32_t)K_o, Y->data_ptr(), ydt, Y->stride(0), nullptr, nullptr, variant, (void *)stream);
        return gemm_fn(variant, (const int8_t *)Xq.data_ptr(), Xq.stride(0), (const float *)ptr(s_x), (const int8_t *)Wq.data_ptr(), Wq.stride(0),
                       (const float *)ptr(sn), (const float *)ptr(so), (const float *)ptr(bias), (int32_t)M, (int32_t)N, (int32_t)K,
                       (int32_t)K_o, Y->data_ptr(), ydt, Y->stride(0), nullptr, nullptr, (void *)stream);
    });
    return py::make_tuple(st, std::move(Y));
}

py::tuple gemm_q8(const at::Tensor &Xq, const OptTensor &s_x, const at::Tensor &Wq, const OptTensor &sn, const OptTensor &so, const OptTensor &bias,
                  int64_t M, int64_t N, int64_t K, int64_t K_o, double scale, int act, OptTensor Y8, int variant, uintptr_t stream)
{
    if (!Y8) Y8 = fresh({M, N}, at::kChar, Xq);
    const int st = run([&] {
        return gemm_q8_fn((const int8_t *)Xq.data_ptr(), Xq.stride(0), (const float *)ptr(s_x), (const int8_t *)Wq.data_ptr(), Wq.stride(0),
                          (const float *)ptr(sn), (const float *)ptr(so), (const float *)ptr(bias), (int32_t)M, (int32_t)N, (int32_t)K,
                          (int32_t)K_o, (qarvd_act)act, (float)scale, (int8_t *)Y8->data_ptr(), Y8->stride(0), variant, (void *)stream);
    });
    return py::make_tuple(st, std::move(Y8));
}

// ---- fused endings, head norms and rotation: the checks of binding.py's _layer, _array, _ending, _out, _rope, _norm_weight and _check_heads -----------------

// The tensors are on the device that the call runs on.
void on_device(int64_t device, std::initializer_list<const at::Tensor *> tensors)
{
    for (const at::Tensor *t : tensors)
        if (t && t->get_device() != device)
            throw py::value_error("a tensor is on " + t->device().str() + ", the call on device " + std::to_string(device));
}
const at::Tensor *opt(const OptTensor &t) { return t ? &*t : nullptr; }

// Row stride; a single row's says nothing.
int64_t ld_of(const at::Tensor &t) { return t.size(0) > 1 ? t.stride(0) : std::max(t.stride(0), t.size(1)); }

void check_out(const at::Tensor &t, int64_t M, int64_t N, const char *what)
{
    if (t.dim() != 2 || t.size(0) != M || t.size(1) != N || (N > 1 && t.stride(1) != 1))
        throw py::value_error(std::string(what) + " must be [M, N] with unit inner stride");
}

void check_vector(const OptTensor &t, int64_t n, const char *what)
{
    if (!t) return;
    if (t->scalar_type() != at::kFloat) throw py::type_error(std::string(what) + " must be float32");
    if (t->dim() != 1 || t->size(0) != n || (n > 1 && t->stride(0) != 1))
        throw py::value_error(std::string(what) + " must be a contiguous vector of " + std::to_string(n));
}

void check_array(const at::Tensor *t, int64_t n, at::ScalarType dtype, const char *what)
{
    if (t && t->scalar_type() != dtype) throw py::type_error(std::string(what) + " must be " + (dtype == at::kInt ? "int32" : "float32"));
    if (t && (!t->is_contiguous() || t->numel() < n)) throw py::value_error(std::string(what) + " must be contiguous and hold " + std::to_string(n));
}

void check_layer(const at::Tensor &Wq, const at::Tensor *sn, const at::Tensor *so, const at::Tensor *perm, int64_t N, int64_t K)
{
    if (Wq.dim() != 2 || Wq.size(0) < N || (Wq.size(1) > 1 && Wq.stride(1) != 1))
        throw py::value_error("the layer's Wq must have " + std::to_string(N) + " rows with unit inner stride");
    check_array(sn, N, at::kFloat, "s_normal");
    check_array(so, N, at::kFloat, "s_outlier");
    check_array(perm, K, at::kInt, "perm");
}

qarvd_ending make_ending(int64_t M, int64_t N, int act, const OptTensor &gate, std::optional<int64_t> gate_rows, const OptTensor &residual,
                         at::ScalarType dtype)
{
    qarvd_ending e = {(qarvd_act)act, (int32_t)M, nullptr, N, nullptr, N};
    if (gate) {
        if (gate->scalar_type() != at::kFloat) throw py::type_error("gate must be float32");
        const int64_t dim = gate->dim();
        if ((dim != 1 && dim != 2) || gate->size(-1) != N || (N > 1 && gate->stride(-1) != 1))
            throw py::value_error("gate must be [N] or [groups, N] with unit inner stride");
        const int64_t groups = dim == 2 ? gate->size(0) : 1;
        if (!gate_rows) {
            if (groups == 0 || M % groups) throw py::value_error(std::to_string(M) + " tokens in " + std::to_string(groups) + " groups: give gate_rows");
            gate_rows = M / groups;
        }
        if (*gate_rows < 1 || (*gate_rows < M && groups * *gate_rows < M) || groups < 1)
            throw py::value_error(std::to_string(groups) + " groups of " + std::to_string(*gate_rows) + " tokens do not cover " + std::to_string(M));
        e.gate = (const float *)gate->data_ptr();
        e.gate_rows = (int32_t)std::min(*gate_rows, M);
        e.ldg = dim == 2 ? gate->stride(0) : N;
    } else if (gate_rows) {
        throw py::value_error("gate_rows without a gate");
    }
    if (residual) {
        if (residual->scalar_type() != dtype) throw py::type_error("the residual's type is not the output's");
        check_out(*residual, M, N, "residual");
        e.residual = residual->data_ptr();
        e.ldr = ld_of(*residual);
    }
    return e;
}

py::tuple gemm_fused(const at::Tensor &Xq, const OptTensor &s_x, int bits, const at::Tensor &Wq, const OptTensor &sn, const OptTensor &so,
                     const OptTensor &bias, int64_t M, int64_t N, int64_t K, int64_t K_o, int act, const OptTensor &gate, const OptTensor &residual,
                     std::optional<int64_t> gate_rows, std::optional<at::ScalarType> out_dtype, OptTensor Y, int variant, uintptr_t stream,
                     int64_t device)
{
    const at::ScalarType out = Y ? Y->scalar_type() : c10::dtype_or_default(out_dtype);
    check_layer(Wq, opt(sn), opt(so), nullptr, N, K);
    check_vector(bias, N, "bias");
    const qarvd_ending e = make_ending(M, N, act, gate, gate_rows, residual, out);
    const qarvd_dtype ydt = dtype_of(out);
    on_device(device, {&Xq, opt(s_x), &Wq, opt(sn), opt(so), opt(bias), opt(gate), opt(residual), opt(Y)});
    if (Xq.dim() != 2 || Xq.size(0) < M || (Xq.size(1) > 1 && Xq.stride(1) != 1)) throw py::value_error("Xq must have M rows with unit inner stride");
    check_array(opt(s_x), M, at::kFloat, "s_x");
    if (Y) check_out(*Y, M, N, "Y");
    else Y = fresh({M, N}, out, Xq);
    const int st = run([&] {
        return gemm_fused_fn((const int8_t *)Xq.data_ptr(), Xq.stride(0), (const float *)ptr(s_x), bits, Wq.data_ptr(), Wq.stride(0),
                             (const float *)ptr(sn), (const float *)ptr(so), (const float *)ptr(bias), &e, (int32_t)M, (int32_t)N, (int32_t)K,
                             (int32_t)K_o, Y->data_ptr(), ydt, ld_of(*Y), variant, (void *)stream);
    });
    return py::make_tuple(st, std::move(Y));
}

py::tuple linear_fused(const at::Tensor &X, const OptTensor &perm, int bits, const at::Tensor &Wq, const at::Tensor &sn, const at::Tensor &so,
                       const OptTensor &bias, int64_t N, int64_t K, int64_t K_o, int act, const OptTensor &gate, const OptTensor &residual,
                       std::optional<int64_t> gate_rows, std::optional<at::ScalarType> out_dtype, OptTensor Y, uintptr_t stream, int64_t device)
{
    check_2d(X, "X");
    const int64_t M = X.size(0);
    if (X.size(1) != K) throw py::value_error("X has " + std::to_string(X.size(1)) + " channels, the layer " + std::to_string(K));
    const at::ScalarType out = Y ? Y->scalar_type() : c10::dtype_or_default(out_dtype);
    const at::Tensor *const order = K_o > 0 ? opt(perm) : nullptr;
    check_layer(Wq, &sn, &so, order, N, K);
    check_vector(bias, N, "bias");
    const qarvd_ending e = make_ending(M, N, act, gate, gate_rows, residual, out);
    const qarvd_dtype xdt = dtype_of(X.scalar_type()), ydt = dtype_of(out);
    on_device(device, {&X, &Wq, &sn, &so, order, opt(bias), opt(gate), opt(residual), opt(Y)});
    if (Y) check_out(*Y, M, N, "Y");
    const size_t need = linear_workspace_fn((int32_t)M, (int32_t)K, (int32_t)K_o);
    const at::Tensor ws = fresh({(int64_t)need}, at::kByte, X);
    if (!Y) Y = fresh({M, N}, out, X);
    const int st = run([&] {
        return linear_fused_fn(X.data_ptr(), xdt, ld_of(X), (const int32_t *)ptr(perm), bits, Wq.data_ptr(), Wq.stride(0), (const float *)sn.data_ptr(),
                               (const float *)so.data_ptr(), (const float *)ptr(bias), &e, (int32_t)M, (int32_t)N, (int32_t)K, (int32_t)K_o,
                               Y->data_ptr(), ydt, ld_of(*Y), ws.data_ptr(), need, (void *)stream);
    });
    return py::make_tuple(st, std::move(Y));
}

// False without a rotation.
bool make_rope(const std::optional<std::vector<int64_t>> &axes, const OptTensor &freq, bool interleaved, const OptTensor &pos, int64_t M, qarvd_rope *r)
{
    if (!axes) {
        if (pos) throw py::value_error("positions without a rope");
        return false;
    }
    const int64_t n = (int64_t)axes->size();
    if (n < 1 || n > 3) throw py::value_error("one to three axes, not " + std::to_string(n));
    if (!pos || pos->scalar_type() != at::kInt) throw py::type_error("pos must be int32");
    const bool flat = pos->dim() == 1 && n == 1;
    if (flat ? pos->size(0) != M : (pos->dim() != 2 || pos->size(0) != M || pos->size(1) != n || (n > 1 && pos->stride(1) != 1)))
        throw py::value_error("pos must be [M, " + std::to_string(n) + "] with unit inner stride");
    int64_t half = 0;
    *r = qarvd_rope{(const int32_t *)pos->data_ptr(), pos->stride(0), nullptr, (int32_t)n, {0, 0, 0}, interleaved ? 1 : 0};
    for (int64_t i = 0; i < n; ++i) {
        half += (*axes)[i];
        r->axis_dims[i] = (int32_t)(*axes)[i];
    }
    half /= 2;
    if (!freq || freq->scalar_type() != at::kDouble) throw py::type_error("rope.freq must be float64");
    if (freq->dim() != 1 || freq->size(0) != half || (half > 1 && freq->stride(0) != 1))
        throw py::value_error("rope.freq must be a contiguous vector of " + std::to_string(half));
    r->freq = (const double *)freq->data_ptr();
    return true;
}

void check_norm_weight(const OptTensor &w, int norm, int64_t heads, int64_t D, const char *what)
{
    if (w && norm == QARVD_NORM_NONE) throw py::value_error(std::string(what) + " without a norm");
    check_vector(w, norm == QARVD_NORM_ROW ? heads * D : D, what);
}

void check_heads(const at::Tensor &x, const char *what, const at::Tensor *like = nullptr)
{
    if (!x.is_cuda() || x.dim() != 3 || (x.size(2) > 1 && x.stride(2) != 1))
        throw py::value_error(std::string(what) + " must be a [tokens, heads, channels] device tensor with unit inner stride");
    if (like && (x.sizes() != like->sizes() || x.scalar_type() != like->scalar_type()))
        throw py::value_error(std::string(what) + " must have the shape and type of what it is the output of");
}

qarvd_heads heads_of(const at::Tensor &x, const at::Tensor &out, const OptTensor &w)
{
    return qarvd_heads{x.data_ptr(), x.stride(0), x.stride(1), out.data_ptr(), out.stride(0), out.stride(1), (const float *)ptr(w), (int32_t)x.size(1)};
}

py::tuple heads(const at::Tensor &Q, const OptTensor &K, int norm, const OptTensor &wq, const OptTensor &wk, double eps, const OptTensor &pos,
                const std::optional<std::vector<int64_t>> &axes, const OptTensor &freq, bool interleaved, OptTensor out_q, OptTensor out_k,
                uintptr_t stream, int64_t device)
{
    check_heads(Q, "Q");
    const int64_t M = Q.size(0), D = Q.size(2);
    if (M > INT32_MAX) throw py::value_error("more than 2^31 - 1 tokens");
    check_norm_weight(wq, norm, Q.size(1), D, "weight_q");
    qarvd_rope r;
    const bool turn = make_rope(axes, freq, interleaved, pos, M, &r);
    if (!K) {
        if (wk || out_k) throw py::value_error("weight_k or out_k without K");
    } else {
        check_heads(*K, "K");
        if (K->size(0) != M || K->size(2) != D || K->scalar_type() != Q.scalar_type())
            throw py::value_error("Q and K must have the same tokens, channels and type");
        check_norm_weight(wk, norm, K->size(1), D, "weight_k");
    }
    if (out_q) check_heads(*out_q, "out_q", &Q);
    if (out_k) check_heads(*out_k, "out_k", &*K);
    const qarvd_dtype dt = dtype_of(Q.scalar_type());
    on_device(device, {&Q, opt(K), opt(wq), opt(wk), opt(pos), axes ? opt(freq) : nullptr, opt(out_q), opt(out_k)});
    if (!out_q) out_q = fresh(Q.sizes(), Q.scalar_type(), Q);
    if (K && !out_k) out_k = fresh(K->sizes(), K->scalar_type(), *K);
    const qarvd_heads q = heads_of(Q, *out_q, wq);
    qarvd_heads k = {};
    if (K) k = heads_of(*K, *out_k, wk);
    const int st = run([&] {
        return heads_fn(&q, K ? &k : nullptr, dt, (int32_t)M, (int32_t)D, (qarvd_norm)norm, (float)eps, turn ? &r : nullptr, (void *)stream);
    });
    return py::make_tuple(st, std::move(out_q), std::move(out_k));
}

py::tuple linear_qkv(const at::Tensor &X, const OptTensor &perm, int bits, const at::Tensor &Wq, const at::Tensor &sn, const at::Tensor &so,
                     const OptTensor &bias, int64_t N, int64_t K, int64_t K_o, int64_t heads_q, int64_t heads_k, int64_t D, int norm,
                     const OptTensor &wq, const OptTensor &wk, double eps, const OptTensor &pos, const std::optional<std::vector<int64_t>> &axes,
                     const OptTensor &freq, bool interleaved, std::optional<at::ScalarType> out_dtype, uintptr_t stream, int64_t device)
{
    check_2d(X, "X");
    const int64_t M = X.size(0);
    if (X.size(1) != K) throw py::value_error("X has " + std::to_string(X.size(1)) + " channels, the layer " + std::to_string(K));
    const at::Tensor *const order = K_o > 0 ? opt(perm) : nullptr;
    check_layer(Wq, &sn, &so, order, N, K);
    check_vector(bias, N, "bias");
    check_norm_weight(wq, norm, heads_q, D, "weight_q");
    check_norm_weight(wk, norm, heads_k, D, "weight_k");
    qarvd_rope r;
    const bool turn = make_rope(axes, freq, interleaved, pos, M, &r);
    const at::ScalarType out = c10::dtype_or_default(out_dtype);
    const qarvd_dtype xdt = dtype_of(X.scalar_type()), ydt = dtype_of(out);
    on_device(device, {&X, &Wq, &sn, &so, order, opt(bias), opt(wq), opt(wk), opt(pos), axes ? opt(freq) : nullptr});
    const size_t need = linear_workspace_fn((int32_t)M, (int32_t)K, (int32_t)K_o);
    const at::Tensor ws = fresh({(int64_t)need}, at::kByte, X);
    at::Tensor Y = fresh({M, N}, out, X);
    const int st = run([&] {
        return linear_qkv_fn(X.data_ptr(), xdt, ld_of(X), (const int32_t *)ptr(perm), bits, Wq.data_ptr(), Wq.stride(0), (const float *)sn.data_ptr(),
                             (const float *)so.data_ptr(), (const float *)ptr(bias), (int32_t)M, (int32_t)N, (int32_t)K, (int32_t)K_o,
                             (int32_t)heads_q, (int32_t)heads_k, (int32_t)D, (qarvd_norm)norm, (const float *)ptr(wq), (const float *)ptr(wk),
                             (float)eps, turn ? &r : nullptr, Y.data_ptr(), ydt, N, ws.data_ptr(), need, (void *)stream);
    });
    return py::make_tuple(st, std::move(Y));
}

}  // namespace

PYBIND11_MODULE(_host, m)
{
    m.attr("torch_version") = QARVD_TORCH_VERSION;      // whose headers this was compiled against
    m.def("init", &init);
    m.def("linear", &linear);
    m.def("quant_act", &quant_act);
    m.def("quant_act_static", &quant_act_static);
    m.def("gemm", &gemm);
    m.def("gemm_q8", &gemm_q8);
    m.def("init_block", &init_block);
    m.def("gemm_fused", &gemm_fused);
    m.def("linear_fused", &linear_fused);
    m.def("heads", &heads);
    m.def("linear_qkv", &linear_qkv);
}
