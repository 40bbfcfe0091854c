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

PyMethodDef kOperatorMethods[] = {{"linear", as_function(py_linear), METH_FASTCALL, nullptr},
{"rms_norm", as_function(py_rms_norm), METH_FASTCALL, nullptr},
                                  {"rms_norm_backward", as_function(py_rms_norm_backward), METH_FASTCALL, nullptr},
                                  {"bias_grad", as_function(py_bias_grad), METH_FASTCALL, nullptr},
                                  {"adamw", as_function(py_adamw), METH_FASTCALL, nullptr},
                                  {nullptr, nullptr, 0, nullptr}};

}  // namespace

PyMethodDef* operator_methods() { return kOperatorMethods; }
