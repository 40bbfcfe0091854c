// Argument checks of the operators around the GEMMs, as part of the _native extension: a norm of
// one token is a launch of a few microseconds, and an optimizer step looks at five
// tensors per weight.  Nothing is kept between calls.
#include <c10/hip/HIPFunctions.h>

#include <algorithm>
#include <vector>

#include "native_checks.h"

namespace {

int operand_code(at::ScalarType t) { return t == at::kFloat8_e4m3fn ? CLEAVE_E4M3 : dtype_code(t); }

// A matrix of `rows` x `cols` elements of one type on the current device; nothing where None is allowed.
struct Operand {
  void* ptr = nullptr;
  int64_t ld = 0, rows = 0, cols = 0;
  at::ScalarType type = at::kFloat;
};

void on_current_device(const at::Tensor& t, const char* what) {
  if (t.is_cuda() && t.get_device() == c10::hip::current_device()) return;
  PyErr_Format(PyExc_ValueError, "%s must be on the current device", what);
  throw Raised{};
}

Operand operand(PyObject* o, const char* what) {
  const Matrix m = matrix(o, what);
  on_current_device(THPVariable_Unpack(o), what);
  // (torch gives a matrix of one row, or of none, any stride)
  return Operand{m.ptr, m.rows > 1 ? m.ld : std::max(m.ld, m.cols), m.rows, m.cols, m.type};
}

Operand like(PyObject* o, const char* what, int64_t rows, int64_t cols, at::ScalarType type, bool optional = false) {
  if (optional && o == Py_None) return Operand{};
  const Operand m = operand(o, what);
  if (m.rows != rows || m.cols != cols || m.type != type) {
    PyErr_Format(PyExc_ValueError, "%s must be %lld x %lld torch.%s", what, static_cast<long long>(rows),
                 static_cast<long long>(cols), c10::toString(type));
    throw Raised{};
  }
  return m;
}

// `n` contiguous floats (at least, for workspaces).
float* floats(PyObject* o, const char* what, int64_t n, bool optional = false, bool at_least = false) {
  if (optional && o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, what);
  on_current_device(t, what);
  if (t.scalar_type() != at::kFloat || !t.is_contiguous() || (at_least ? t.numel() < n : t.numel() != n)) {
    PyErr_Format(PyExc_ValueError, "%s must be a contiguous fp32 device tensor of %s%lld elements", what,
                 at_least ? "at least " : "", static_cast<long long>(n));
    throw Raised{};
  }
  return static_cast<float*>(t.data_ptr());
}

double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised{};
  return v;
}

// rms_norm(x, weight, y, residual, sum_out, inv_rms, scales, eps, stream)
PyObject* py_rms_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expect_args(n, 9);
    const Operand x = operand(a[0], "x");
    const int dt = dtype_code(x.type);
    const float* w = floats(a[1], "weight", x.cols);
    const Operand y = operand(a[2], "y");
    const int ydt = operand_code(y.type);
    if (y.rows != x.rows || y.cols != x.cols || (ydt != dt && ydt != CLEAVE_E4M3))
      raise(PyExc_ValueError, "y must have x's shape, and x's dtype or float8_e4m3fn");
    const Operand r = like(a[3], "residual", x.rows, x.cols, x.type, true);
    const Operand s = like(a[4], "sum_out", x.rows, x.cols, x.type, true);
    float* inv = floats(a[5], "inv_rms", x.rows, true);
    float* scales = floats(a[6], "scales", x.rows, true);
    if ((ydt == CLEAVE_E4M3) != (a[6] != Py_None)) raise(PyExc_ValueError, "scales belong to y in float8_e4m3fn, and only to that");
    const float eps = static_cast<float>(real(a[7]));
    void* stream = stream_of(a[8]);
    if (x.rows == 0) return PyLong_FromLong(CLEAVE_OK);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = cleave_rms_norm(x.rows, x.cols, x.ptr, x.ld, r.ptr, r.ld, dt, w, eps, y.ptr, y.ld, ydt, scales, s.ptr, s.ld, inv, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  });
}

// rms_norm_backward(dy, h, weight, inv_rms, dx, dweight, workspace, dsum, stream)
PyObject* py_rms_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expect_args(n, 9);
    const Operand dy = operand(a[0], "dy");
    const int dt = dtype_code(dy.type);
    const Operand h = like(a[1], "h", dy.rows, dy.cols, dy.type);
    const float* w = floats(a[2], "weight", dy.cols);
    const float* inv = floats(a[3], "inv_rms", dy.rows);
    const Operand dx = like(a[4], "dx", dy.rows, dy.cols, dy.type);
    float* dw = floats(a[5], "dweight", dy.cols);
    float* ws = floats(a[6], "workspace", cleave_rms_norm_workspace(dy.rows, dy.cols), false, true);
    const Operand ds = like(a[7], "dsum", dy.rows, dy.cols, dy.type, true);
    void* stream = stream_of(a[8]);
    // (tensors without elements have no address: any stands for them)
    const auto some = [&](const void* p) { return dy.rows ? p : ws; };
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = cleave_rms_norm_backward(dy.rows, dy.cols, some(dy.ptr), dy.ld, some(h.ptr), h.ld, dy.rows ? ds.ptr : nullptr, ds.ld, dt,
                                  w, static_cast<const float*>(some(inv)), const_cast<void*>(some(dx.ptr)), dx.ld, dw, ws, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  });
}

// layer_norm(x, weight, y, bias, residual, sum_out, mean, inv_std, scales, eps, stream)
PyObject* py_layer_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expect_args(n, 11);
    const Operand x = operand(a[0], "x");
    const int dt = dtype_code(x.type);
    const float* w = floats(a[1], "weight", x.cols);
    const Operand y = operand(a[2], "y");
    const int ydt = operand_code(y.type);
    if (y.rows != x.rows || y.cols != x.cols || (ydt != dt && ydt != CLEAVE_E4M3))
      raise(PyExc_ValueError, "y must have x's shape, and x's dtype or float8_e4m3fn");
    const float* b = floats(a[3], "bias", x.cols, true);
    const Operand r = like(a[4], "residual", x.rows, x.cols, x.type, true);
    const Operand s = like(a[5], "sum_out", x.rows, x.cols, x.type, true);
    float* mean = floats(a[6], "mean", x.rows, true);
    float* inv = floats(a[7], "inv_std", x.rows, true);
    float* scales = floats(a[8], "scales", x.rows, true);
    if ((ydt == CLEAVE_E4M3) != (a[8] != Py_None)) raise(PyExc_ValueError, "scales belong to y in float8_e4m3fn, and only to that");
    const float eps = static_cast<float>(real(a[9]));
    void* stream = stream_of(a[10]);
    if (x.rows == 0) return PyLong_FromLong(CLEAVE_OK);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = cleave_layer_norm(x.rows, x.cols, x.ptr, x.ld, r.ptr, r.ld, dt, w, b, eps, y.ptr, y.ld, ydt, scales, s.ptr, s.ld, mean,
                           inv, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  });
}

// layer_norm_backward(dy, h, weight, mean, inv_std, dx, dweight, workspace, dbias, dsum, stream)
PyObject* py_layer_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expect_args(n, 11);
    const Operand dy = operand(a[0], "dy");
    const int dt = dtype_code(dy.type);
    const Operand h = like(a[1], "h", dy.rows, dy.cols, dy.type);
    const float* w = floats(a[2], "weight", dy.cols);
    const float* mean = floats(a[3], "mean", dy.rows);
    const float* inv = floats(a[4], "inv_std", dy.rows);
    const Operand dx = like(a[5], "dx", dy.rows, dy.cols, dy.type);
    float* dw = floats(a[6], "dweight", dy.cols);
    float* ws = floats(a[7], "workspace", cleave_layer_norm_workspace(dy.rows, dy.cols), false, true);
    float* db = floats(a[8], "dbias", dy.cols, true);
    const Operand ds = like(a[9], "dsum", dy.rows, dy.cols, dy.type, true);
    void* stream = stream_of(a[10]);
    // (tensors without elements have no address: any stands for them)
    const auto some = [&](const void* p) { return dy.rows ? p : ws; };
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = cleave_layer_norm_backward(dy.rows, dy.cols, some(dy.ptr), dy.ld, some(h.ptr), h.ld, dy.rows ? ds.ptr : nullptr, ds.ld,
                                    dt, w, static_cast<const float*>(some(mean)), static_cast<const float*>(some(inv)),
                                    const_cast<void*>(some(dx.ptr)), dx.ld, dw, db, ws, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  });
}

// bias_grad(dy, dbias, workspace, stream)
PyObject* py_bias_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expect_args(n, 4);
    const Operand dy = operand(a[0], "dy");
    const int dt = dtype_code(dy.type);
    float* db = floats(a[1], "dbias", dy.cols);
    float* ws = floats(a[2], "workspace", cleave_bias_grad_workspace(dy.rows, dy.cols), false, true);
    void* stream = stream_of(a[3]);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = cleave_bias_grad(dy.rows, dy.cols, dy.rows ? dy.ptr : ws, dy.ld, dt, db, ws, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  });
}

// A list or tuple of tensors (not a tensor, which is a sequence of its rows); none where None is given.
struct Tensors {
  PyObject* seq = nullptr;   // borrowed
  const char* what;
  Tensors(PyObject* o, const char* name, Py_ssize_t want) : what(name) {
    if (o == Py_None) return;
    if (!PyList_Check(o) && !PyTuple_Check(o)) {
      PyErr_Format(PyExc_TypeError, "%s must be a list of tensors", what);
      throw Raised{};
    }
    seq = o;
    if (want >= 0 && PySequence_Fast_GET_SIZE(seq) != want) {
      PyErr_Format(PyExc_ValueError, "%s must have one tensor for each of w", what);
      throw Raised{};
    }
  }
  Py_ssize_t size() const { return seq ? PySequence_Fast_GET_SIZE(seq) : 0; }
  const at::Tensor& operator[](Py_ssize_t k) const { return tensor(PySequence_Fast_GET_ITEM(seq, k), what); }
  void* at_k(Py_ssize_t k, int64_t n, at::ScalarType type) const {
    const at::Tensor& t = (*this)[k];
    on_current_device(t, what);
    if (t.scalar_type() != type || t.numel() != n || !t.is_contiguous()) {
      PyErr_Format(PyExc_ValueError, "%s[%zd] must be a contiguous torch.%s device tensor of %lld elements", what, k,
                   c10::toString(type), static_cast<long long>(n));
      throw Raised{};
    }
    return t.data_ptr();
  }
};

// adamw(w, g, m, v, m_scales, v_scales, copies, grad_scale, lr, beta1, beta2, eps, weight_decay, step, stream)
PyObject* py_adamw(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expect_args(n, 15);
    if (a[0] == Py_None) raise(PyExc_TypeError, "w must be a list of tensors");
    const Tensors w(a[0], "w", -1);
    const Py_ssize_t count = w.size();
    const Tensors g(a[1], "grads", count), m(a[2], "m", count), v(a[3], "v", count);
    const Tensors ms(a[4], "m_scales", count), vs(a[5], "v_scales", count), copies(a[6], "copies", count);
    if (!g.seq || !m.seq || !v.seq) raise(PyExc_TypeError, "grads, m and v must be lists of tensors");
    if (!ms.seq != !vs.seq) raise(PyExc_ValueError, "m_scales and v_scales come together");
    const at::ScalarType state = ms.seq ? at::kFloat8_e4m3fn : at::kFloat;
    const at::ScalarType grad = count ? g[0].scalar_type() : at::kFloat;
    const int gdt = dtype_code(grad);
    std::vector<int64_t> sizes(count);
    std::vector<void*> p[7];
    for (auto& list : p) list.resize(count);
    for (Py_ssize_t k = 0; k < count; ++k) {
      const int64_t size = sizes[k] = w[k].numel();
      const int64_t blocks = (size + 255) / 256;
      p[0][k] = w.at_k(k, size, at::kFloat);
      p[1][k] = g.at_k(k, size, grad);
      p[2][k] = m.at_k(k, size, state);
      p[3][k] = v.at_k(k, size, state);
      if (ms.seq) {
        p[4][k] = ms.at_k(k, blocks, at::kFloat);
        p[5][k] = vs.at_k(k, blocks, at::kFloat);
      }
      if (copies.seq) p[6][k] = copies.at_k(k, size, at::kBFloat16);
    }
    const float* clip = floats(a[7], "grad_scale", 1, true);
    const double lr = real(a[8]), beta1 = real(a[9]), beta2 = real(a[10]), eps = real(a[11]), decay = real(a[12]);
    const int64_t step = integer(a[13]);
    void* stream = stream_of(a[14]);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = cleave_adamw(count, sizes.data(), reinterpret_cast<float* const*>(p[0].data()), p[1].data(), gdt, p[2].data(),
                      p[3].data(), ms.seq ? reinterpret_cast<float* const*>(p[4].data()) : nullptr,
                      vs.seq ? reinterpret_cast<float* const*>(p[5].data()) : nullptr, copies.seq ? p[6].data() : nullptr, clip,
                      lr, beta1, beta2, eps, decay, step, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  });
}

// linear(plan address, M, N, K, workspace, A, B, C, transA, transB, bias, act, act_grad, residual, preact, scale_a,
//        scale_b, partials, stream)
PyObject* py_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expect_args(n, 19);
    const int64_t M = integer(a[1]), N = integer(a[2]), K = integer(a[3]), elems = integer(a[4]);
    const Operand A = operand(a[5], "A"), B = operand(a[6], "B"), C = operand(a[7], "C");
    cleave_linear_args args{};
    args.transA = static_cast<int32_t>(integer(a[8]));
    args.transB = static_cast<int32_t>(integer(a[9]));
    if (A.type != B.type) raise(PyExc_TypeError, "A and B must have the same dtype");
    args.dtype = operand_code(A.type);
    args.out_dtype = dtype_code(C.type);
    const bool ta = args.transA != 0, tb = args.transB != 0;
    if (A.rows != (ta ? K : M) || A.cols != (ta ? M : K) || B.rows != (tb ? N : K) || B.cols != (tb ? K : N) || C.rows != M ||
        C.cols != N) {
      PyErr_Format(PyExc_ValueError, "shapes (%lld, %lld), (%lld, %lld), (%lld, %lld) do not match the plan",
                   static_cast<long long>(A.rows), static_cast<long long>(A.cols), static_cast<long long>(B.rows),
                   static_cast<long long>(B.cols), static_cast<long long>(C.rows), static_cast<long long>(C.cols));
      throw Raised{};
    }
    const Operand residual = like(a[13], "residual", M, N, C.type, true);
    const Operand preact = like(a[14], "preact", M, N, C.type, true);
    args.A = A.ptr;
    args.lda = A.ld;
    args.B = B.ptr;
    args.ldb = B.ld;
    args.C = C.ptr;
    args.ldc = C.ld;
    args.bias = floats(a[10], "bias", N, true);
    args.act = static_cast<int32_t>(integer(a[11]));
    args.act_grad = static_cast<int32_t>(integer(a[12]));
    args.residual = residual.ptr;
    args.ldr = residual.ld;
    args.preact = preact.ptr;
    args.ldz = preact.ld;
    args.scale_a = floats(a[15], "scale_a", M, true);
    args.scale_b = floats(a[16], "scale_b", N, true);
    if (args.dtype != CLEAVE_E4M3 && (args.scale_a || args.scale_b)) raise(PyExc_ValueError, "scales belong to operands in float8_e4m3fn");
    if (args.dtype == CLEAVE_E4M3 && (!args.scale_a || !args.scale_b)) raise(PyExc_ValueError, "operands in float8_e4m3fn need scale_a and scale_b");
    if (elems > 0) args.partials = floats(a[17], "partials", elems, false, true);
    cleave_plan* plan = static_cast<cleave_plan*>(address(a[0]));
    void* stream = stream_of(a[18]);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = cleave_linear(plan, &args, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  });
}

// The shape of a stored operand B.
void expect_b(const Operand& b, bool transposed, int64_t N, int64_t K, const char* what) {
  if (b.rows == (transposed ? N : K) && b.cols == (transposed ? K : N)) return;
  PyErr_Format(PyExc_ValueError, "%s of shape (%lld, %lld) does not match the plan", what, static_cast<long long>(b.rows),
               static_cast<long long>(b.cols));
  throw Raised{};
}

// linear_gated(plan address, M, N, K, A, B_gate, B_up, C, transB, act, bias_gate, bias_up, gate, up, scale_a, scale_gate, scale_up,
//              partials, stream)
PyObject* py_linear_gated(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expect_args(n, 19);
    const int64_t M = integer(a[1]), N = integer(a[2]), K = integer(a[3]);
    const Operand C = operand(a[7], "C");
    const Operand A = like(a[4], "A", M, K, operand(a[4], "A").type), Bg = operand(a[5], "B_gate"), Bu = operand(a[6], "B_up");
    cleave_gated_args args{};
    args.transB = static_cast<int32_t>(integer(a[8]));
    args.dtype = operand_code(A.type);
    args.out_dtype = dtype_code(C.type);
    if (A.type != Bg.type || A.type != Bu.type) raise(PyExc_TypeError, "A, B_gate and B_up must have the same dtype");
    expect_b(Bg, args.transB != 0, N, K, "B_gate");
    expect_b(Bu, args.transB != 0, N, K, "B_up");
    if (Bg.rows > 1 && Bg.ld != Bu.ld) raise(PyExc_ValueError, "B_gate and B_up must have the same row stride");
    if (C.rows != M || C.cols != N) raise(PyExc_ValueError, "C must be M x N");
    const Operand gate = like(a[12], "gate", M, N, C.type, true), up = like(a[13], "up", M, N, C.type, true);
    args.A = A.ptr;
    args.lda = A.ld;
    args.B_gate = Bg.ptr;
    args.B_up = Bu.ptr;
    args.ldb = Bg.ld;
    args.C = C.ptr;
    args.ldc = C.ld;
    args.act = static_cast<int32_t>(integer(a[9]));
    args.bias_gate = floats(a[10], "bias_gate", N, true);
    args.bias_up = floats(a[11], "bias_up", N, true);
    args.gate = gate.ptr;
    args.ld_gate = gate.ld;
    args.up = up.ptr;
    args.ld_up = up.ld;
    args.scale_a = floats(a[14], "scale_a", M, true);
    args.scale_gate = floats(a[15], "scale_gate", N, true);
    args.scale_up = floats(a[16], "scale_up", N, true);
    const bool scaled = args.scale_a && args.scale_gate && args.scale_up;
    if (args.dtype != CLEAVE_E4M3 && (args.scale_a || args.scale_gate || args.scale_up))
      raise(PyExc_ValueError, "scales belong to operands in float8_e4m3fn");
    if (args.dtype == CLEAVE_E4M3 && !scaled)
      raise(PyExc_ValueError, "operands in float8_e4m3fn need scale_a, scale_gate and scale_up");
    cleave_plan* plan = static_cast<cleave_plan*>(address(a[0]));
    // (a workspace shorter than this call's is as good as none: the call says whether it needs one)
    const int64_t least = cleave_gated_workspace(plan, 0);
    if (a[17] != Py_None && least > 0 && tensor(a[17], "partials").numel() > 0 &&
        (cleave_gated_workspace(plan, 1) > 0 || tensor(a[17], "partials").numel() >= least))
      args.partials = floats(a[17], "partials", least, false, true);
    void* stream = stream_of(a[18]);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = cleave_linear_gated(plan, &args, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  });
}

// linear_gated_grad(plan address, M, N, K, A, B, gate, up, dgate, dup, transB, act, partials, stream)
PyObject* py_linear_gated_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expect_args(n, 14);
    const int64_t M = integer(a[1]), N = integer(a[2]), K = integer(a[3]);
    const Operand A = like(a[4], "A", M, K, operand(a[4], "A").type), B = operand(a[5], "B");
    if (A.type != B.type) raise(PyExc_TypeError, "A and B must have the same dtype");
    cleave_gated_grad_args args{};
    args.transB = static_cast<int32_t>(integer(a[10]));
    args.dtype = dtype_code(A.type);
    expect_b(B, args.transB != 0, N, K, "B");
    const Operand gate = like(a[6], "gate", M, N, operand(a[6], "gate").type), up = like(a[7], "up", M, N, gate.type);
    const Operand dgate = like(a[8], "dgate", M, N, gate.type), dup = like(a[9], "dup", M, N, gate.type);
    args.out_dtype = dtype_code(gate.type);
    args.A = A.ptr;
    args.lda = A.ld;
    args.B = B.ptr;
    args.ldb = B.ld;
    args.gate = gate.ptr;
    args.ld_gate = gate.ld;
    args.up = up.ptr;
    args.ld_up = up.ld;
    args.dgate = dgate.ptr;
    args.ld_dgate = dgate.ld;
    args.dup = dup.ptr;
    args.ld_dup = dup.ld;
    args.act = static_cast<int32_t>(integer(a[11]));
    cleave_plan* plan = static_cast<cleave_plan*>(address(a[0]));
    const int64_t least = cleave_gated_grad_workspace(plan, 0);
    if (a[12] != Py_None && least > 0 && tensor(a[12], "partials").numel() > 0 &&
        (cleave_gated_grad_workspace(plan, 1) > 0 || tensor(a[12], "partials").numel() >= least))
      args.partials = floats(a[12], "partials", least, false, true);
    void* stream = stream_of(a[13]);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = cleave_linear_gated_grad(plan, &args, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  });
}

// Contiguous int64 elements: one for each row, or rows x cols.
int64_t* tokens(PyObject* o, const char* what, int64_t rows, int64_t cols, bool optional = false) {
  if (optional && o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, what);
  on_current_device(t, what);
  const bool shaped = cols < 0 ? t.dim() == 1 && t.size(0) == rows : t.dim() == 2 && t.size(0) == rows && t.size(1) == cols;
  if (t.scalar_type() != at::kLong || !shaped || !t.is_contiguous()) {
    PyErr_Format(PyExc_ValueError, "%s must be a contiguous int64 device tensor, one %s each of the %lld rows", what,
                 cols < 0 ? "element for" : "row for", static_cast<long long>(rows));
    throw Raised{};
  }
  return static_cast<int64_t*>(t.data_ptr());
}

// log_probs(logits, ids, logp, lse, entropy, top_ids, top_logp, scale, workspace, stream)
PyObject* py_log_probs(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expect_args(n, 10);
    const Operand l = operand(a[0], "logits");
    const int dt = dtype_code(l.type);
    const int64_t* ids = tokens(a[1], "ids", l.rows, -1, true);
    float* logp = floats(a[2], "logp", l.rows, true);
    if ((a[1] == Py_None) != (a[2] == Py_None)) raise(PyExc_ValueError, "ids and logp come together");
    float* lse = floats(a[3], "lse", l.rows, true);
    float* entropy = floats(a[4], "entropy", l.rows, true);
    int64_t top = 0;
    if ((a[5] == Py_None) != (a[6] == Py_None)) raise(PyExc_ValueError, "top_ids and top_logp come together");
    if (a[5] != Py_None) {
      const at::Tensor& t = tensor(a[5], "top_ids");
      if (t.dim() != 2) raise(PyExc_ValueError, "top_ids must be rows x n_top");
      top = t.size(1);
    }
    int64_t* top_ids = tokens(a[5], "top_ids", l.rows, top, true);
    float* top_logp = floats(a[6], "top_logp", l.rows * top, true);
    const float scale = static_cast<float>(real(a[7]));
    const int64_t elems = cleave_log_probs_workspace(l.rows, l.cols, top);
    float* ws = elems > 0 ? floats(a[8], "workspace", elems, false, true) : nullptr;
    void* stream = stream_of(a[9]);
    if (l.rows == 0) return PyLong_FromLong(CLEAVE_OK);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = cleave_log_probs(l.rows, l.cols, l.ptr, l.ld, dt, scale, ids, logp, lse, entropy, top, top ? top_ids : nullptr,
                          top ? top_logp : nullptr, ws, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  });
}

// log_probs_backward(logits, lse, dlogits, ids, dlogp, entropy, dentropy, scale, stream)
PyObject* py_log_probs_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expect_args(n, 9);
    const Operand l = operand(a[0], "logits");
    const int dt = dtype_code(l.type);
    const float* lse = floats(a[1], "lse", l.rows);
    const Operand d = like(a[2], "dlogits", l.rows, l.cols, l.type);
    const int64_t* ids = tokens(a[3], "ids", l.rows, -1, true);
    const float* dlogp = floats(a[4], "dlogp", l.rows, true);
    const float* entropy = floats(a[5], "entropy", l.rows, true);
    const float* dentropy = floats(a[6], "dentropy", l.rows, true);
    if ((a[3] == Py_None) != (a[4] == Py_None)) raise(PyExc_ValueError, "ids and dlogp come together");
    if ((a[5] == Py_None) != (a[6] == Py_None)) raise(PyExc_ValueError, "entropy and dentropy come together");
    if (a[3] == Py_None && a[5] == Py_None) raise(PyExc_ValueError, "a gradient of logp or of the entropy is needed");
    const float scale = static_cast<float>(real(a[7]));
    void* stream = stream_of(a[8]);
    if (l.rows == 0) return PyLong_FromLong(CLEAVE_OK);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = cleave_log_probs_backward(l.rows, l.cols, l.ptr, l.ld, dt, scale, ids, lse, dlogp, entropy, dentropy, d.ptr, d.ld, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  });
}

PyMethodDef kOperatorMethods[] = {{"linear", as_function(py_linear), METH_FASTCALL, nullptr},
                                  {"linear_gated", as_function(py_linear_gated), METH_FASTCALL, nullptr},
                                  {"linear_gated_grad", as_function(py_linear_gated_grad), METH_FASTCALL, nullptr},
                                  {"rms_norm", as_function(py_rms_norm), METH_FASTCALL, nullptr},
                                  {"rms_norm_backward", as_function(py_rms_norm_backward), METH_FASTCALL, nullptr},
                                  {"layer_norm", as_function(py_layer_norm), METH_FASTCALL, nullptr},
                                  {"layer_norm_backward", as_function(py_layer_norm_backward), METH_FASTCALL, nullptr},
                                  {"log_probs", as_function(py_log_probs), METH_FASTCALL, nullptr},
                                  {"log_probs_backward", as_function(py_log_probs_backward), METH_FASTCALL, nullptr},
                                  {"bias_grad", as_function(py_bias_grad), METH_FASTCALL, nullptr},
                                  {"adamw", as_function(py_adamw), METH_FASTCALL, nullptr},
                                  {nullptr, nullptr, 0, nullptr}};

}  // namespace

PyMethodDef* operator_methods() { return kOperatorMethods; }
