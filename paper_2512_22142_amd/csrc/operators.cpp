// C-ABI entry points of the operators around the GEMMs: checks, and the launches.
// Nothing is allocated, copied or kept between calls.
#include "operators.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <limits>

#include "kernels.h"

namespace {

#define CLEAVE_HIP(expr)                                         \
  do {                                                           \
    const hipError_t e__ = (expr);                               \
    if (e__ != hipSuccess) return cleave::record_hip_error(e__); \
  } while (0)

bool aligned(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

int element_bytes(int dtype) { return dtype == CLEAVE_F32 ? 4 : dtype == CLEAVE_BF16 ? 2 : dtype == CLEAVE_E4M3 ? 1 : 0; }

constexpr int64_t kMost = std::numeric_limits<int32_t>::max();

// Checks of the matrices of rows x cols that one kernel walks.
struct Matrices {
  int64_t cols;
  bool ok;
  Matrices(int64_t r, int64_t c) : cols(c), ok(r >= 0 && c >= 1 && r <= kMost && c <= kMost) {}
  void add(const void* p, int64_t ld, int dtype, bool optional = false) {
    ok = ok && (p ? ld >= cols && aligned(p, element_bytes(dtype)) : optional);
  }
  void add_vector(const float* p, bool optional = false) { ok = ok && (p ? aligned(p, 4) : optional); }
};

// Whether an output may take an input's place: the same elements at the same places, each read and written by one
// thread.  (Rows of another pitch or type would lie over rows that others have yet to read.)
bool in_place(const void* out, int64_t ldo, int out_dtype, const void* in, int64_t ldi, int dtype, int64_t rows) {
  return !out || out != in || rows == 0 || (out_dtype == dtype && (ldo == ldi || rows == 1));
}

bool float_dtype(int dtype) { return dtype == CLEAVE_F32 || dtype == CLEAVE_BF16; }

}  // namespace

extern "C" int cleave_rms_norm(int64_t rows, int64_t cols, const void* x, int64_t ldx, const void* residual, int64_t ldr,
                               int dtype, const float* weight, float eps, void* y, int64_t ldy, int y_dtype, float* scales,
                               void* sum_out, int64_t lds, float* inv_rms, void* hip_stream) {
  if (!float_dtype(dtype) || (y_dtype != dtype && y_dtype != CLEAVE_E4M3)) return CLEAVE_EINVAL;
  if ((y_dtype == CLEAVE_E4M3) != (scales != nullptr)) return CLEAVE_EINVAL;
  if (!(eps >= 0.0f) || std::isinf(eps)) return CLEAVE_EINVAL;
  Matrices m(rows, cols);
  m.add(x, ldx, dtype);
  m.add(residual, ldr, dtype, true);
  m.add(y, ldy, y_dtype);
  m.add(sum_out, lds, dtype, true);
  m.add_vector(weight);
  m.add_vector(scales, true);
  m.add_vector(inv_rms, true);
  if (!m.ok) return CLEAVE_EINVAL;
  if (!in_place(y, ldy, y_dtype, x, ldx, dtype, rows) || !in_place(y, ldy, y_dtype, residual, ldr, dtype, rows) ||
      !in_place(sum_out, lds, dtype, x, ldx, dtype, rows) || !in_place(sum_out, lds, dtype, residual, ldr, dtype, rows) ||
      (rows > 0 && y == sum_out))
    return CLEAVE_EINVAL;
  if (rows == 0) return CLEAVE_OK;
  const cleave::NormArgs args{x, residual, weight, y, scales, sum_out, inv_rms, rows, cols, ldx, ldr, ldy, lds, eps};
  CLEAVE_HIP(cleave::launch_rms_norm(args, dtype, static_cast<hipStream_t>(hip_stream)));
  return CLEAVE_OK;
}

extern "C" int64_t cleave_rms_norm_workspace(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 1 || rows > kMost || cols > kMost) return CLEAVE_EINVAL;
  return cols * std::max(1, cleave::rms_norm_partial_rows(rows, cols));
}

extern "C" int cleave_rms_norm_backward(int64_t rows, int64_t cols, const void* dy, int64_t lddy, const void* h, int64_t ldh,
                                        const void* dsum, int64_t ldds, int dtype, const float* weight, const float* inv_rms,
                                        void* dx, int64_t lddx, float* dweight, float* workspace, void* hip_stream) {
  if (!float_dtype(dtype)) return CLEAVE_EINVAL;
  Matrices m(rows, cols);
  m.add(dy, lddy, dtype);
  m.add(h, ldh, dtype);
  m.add(dsum, ldds, dtype, true);
  m.add(dx, lddx, dtype);
  m.add_vector(weight);
  m.add_vector(inv_rms);
  m.add_vector(dweight);
  m.add_vector(workspace);
  if (!m.ok) return CLEAVE_EINVAL;
  if (!in_place(dx, lddx, dtype, dy, lddy, dtype, rows) || !in_place(dx, lddx, dtype, h, ldh, dtype, rows) ||
      !in_place(dx, lddx, dtype, dsum, ldds, dtype, rows))
    return CLEAVE_EINVAL;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const int partial_rows = cleave::rms_norm_partial_rows(rows, cols);
  if (rows > 0) {
    const cleave::NormBackwardArgs args{dy, h, dsum, weight, inv_rms, dx, workspace, rows, cols, lddy, ldh, ldds, lddx};
    CLEAVE_HIP(cleave::launch_rms_norm_backward(args, dtype, partial_rows, stream));
  }
  CLEAVE_HIP(cleave::launch_join_rows(workspace, partial_rows, cols, dweight, stream));   // no rows: zeros
  return CLEAVE_OK;
}

extern "C" int64_t cleave_bias_grad_workspace(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 1 || rows > kMost || cols > kMost) return CLEAVE_EINVAL;
  return cols * cleave::column_sum_chunks(rows, cols);
}

extern "C" int cleave_bias_grad(int64_t rows, int64_t cols, const void* dy, int64_t lddy, int dtype, float* dbias,
                                float* workspace, void* hip_stream) {
  if (!float_dtype(dtype)) return CLEAVE_EINVAL;
  Matrices m(rows, cols);
  m.add(dy, lddy, dtype);
  m.add_vector(dbias);
  m.add_vector(workspace);
  if (!m.ok) return CLEAVE_EINVAL;
  const cleave::ColumnSumArgs args{dy, lddy, rows, cols, dbias, workspace, cleave::column_sum_chunks(rows, cols)};
  CLEAVE_HIP(cleave::launch_column_sum(args, dtype, static_cast<hipStream_t>(hip_stream)));
  return CLEAVE_OK;
}

extern "C" int cleave_adamw(int64_t n_tensors, const int64_t* sizes, float* const* w, const void* const* g, int g_dtype,
                            void* const* m, void* const* v, float* const* m_scale, float* const* v_scale,
                            void* const* w_bf16, const float* grad_scale, double lr, double beta1, double beta2, double eps,
                            double weight_decay, int64_t step, void* hip_stream) {
  if (n_tensors < 0 || !float_dtype(g_dtype)) return CLEAVE_EINVAL;
  if (n_tensors > 0 && (!sizes || !w || !g || !m || !v)) return CLEAVE_EINVAL;
  const bool states_8bit = m_scale != nullptr;
  if (states_8bit != (v_scale != nullptr)) return CLEAVE_EINVAL;
  if (step < 1 || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0) || !(lr == lr) ||
      !(weight_decay == weight_decay) || !aligned(grad_scale, 4))
    return CLEAVE_EINVAL;
  const int gb = element_bytes(g_dtype);
  const uintptr_t sb = states_8bit ? 1 : 4;
  for (int64_t k = 0; k < n_tensors; ++k) {
    if (sizes[k] < 0 || sizes[k] >= int64_t{1} << 40) return CLEAVE_EINVAL;
    if (sizes[k] == 0) continue;
    if (!w[k] || !g[k] || !m[k] || !v[k] || (states_8bit && (!m_scale[k] || !v_scale[k])) || (w_bf16 && !w_bf16[k]))
      return CLEAVE_EINVAL;
    if (!aligned(w[k], 4) || !aligned(g[k], gb) || !aligned(m[k], sb) || !aligned(v[k], sb) ||
        (states_8bit && (!aligned(m_scale[k], 4) || !aligned(v_scale[k], 4))) || (w_bf16 && !aligned(w_bf16[k], 2)))
      return CLEAVE_EINVAL;
  }
  cleave::AdamWArgs args{};
  args.grad_scale = grad_scale;
  args.lr = static_cast<float>(lr);
  args.beta1 = static_cast<float>(beta1);
  args.one_minus_beta1 = static_cast<float>(1.0 - beta1);
  args.beta2 = static_cast<float>(beta2);
  args.one_minus_beta2 = static_cast<float>(1.0 - beta2);
  args.eps = static_cast<float>(eps);
  args.weight_decay = static_cast<float>(weight_decay);
  args.inv_bias1 = static_cast<float>(1.0 / (1.0 - std::pow(beta1, static_cast<double>(step))));
  args.inv_bias2 = static_cast<float>(1.0 / (1.0 - std::pow(beta2, static_cast<double>(step))));
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  int64_t chunks = 0;
  const auto launch = [&]() -> hipError_t {
    const hipError_t e =
        chunks > 0 ? cleave::launch_adamw(args, static_cast<uint32_t>(chunks), g_dtype, states_8bit, stream) : hipSuccess;
    args.n_tensors = 0;
    chunks = 0;
    return e;
  };
  // (a launch has fewer than 2^32 threads: a tensor of more chunks goes in pieces)
  constexpr int64_t kChunks = int64_t{1} << 23, kPiece = kChunks * cleave::kAdamChunk;
  const auto add = [&](int64_t k, int64_t from) -> hipError_t {
    const int64_t n = std::min(sizes[k] - from, kPiece);
    const int64_t more = (n + cleave::kAdamChunk - 1) / cleave::kAdamChunk;
    if (args.n_tensors == cleave::kAdamTensors || chunks + more > kChunks) {
      const hipError_t e = launch();
      if (e != hipSuccess) return e;
    }
    cleave::AdamTensor& t = args.tensors[args.n_tensors];
    t.w = w[k] + from;
    t.g = static_cast<const unsigned char*>(g[k]) + from * gb;
    t.m = static_cast<unsigned char*>(m[k]) + from * static_cast<int64_t>(sb);
    t.v = static_cast<unsigned char*>(v[k]) + from * static_cast<int64_t>(sb);
    t.m_scale = states_8bit ? m_scale[k] + from / 256 : nullptr;
    t.v_scale = states_8bit ? v_scale[k] + from / 256 : nullptr;
    t.copy = w_bf16 ? static_cast<uint16_t*>(w_bf16[k]) + from : nullptr;
    t.n = static_cast<uint64_t>(n);
    chunks += more;
    args.chunk_end[args.n_tensors++] = static_cast<uint32_t>(chunks);
    return hipSuccess;
  };
  for (int64_t k = 0; k < n_tensors; ++k)
    for (int64_t from = 0; from < sizes[k]; from += kPiece) CLEAVE_HIP(add(k, from));
  CLEAVE_HIP(launch());
  return CLEAVE_OK;
}
