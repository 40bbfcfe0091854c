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

using cleave::apart;

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
      (rows > 0 && !(apart({y, sum_out, scales, inv_rms}, {weight}) && apart({scales, inv_rms}, {x, residual}))))
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
  if (!m.ok || dweight == workspace) return CLEAVE_EINVAL;
  if (!in_place(dx, lddx, dtype, dy, lddy, dtype, rows) || !in_place(dx, lddx, dtype, h, ldh, dtype, rows) ||
      !in_place(dx, lddx, dtype, dsum, ldds, dtype, rows) ||
      (rows > 0 && !(apart({dx, dweight}, {}) && apart({dx, workspace}, {weight, inv_rms}) && apart({workspace}, {dy, h, dsum}))))
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

extern "C" int cleave_layer_norm(int64_t rows, int64_t cols, const void* x, int64_t ldx, const void* residual, int64_t ldr,
                                 int dtype, const float* weight, const float* bias, float eps, void* y, int64_t ldy, int y_dtype,
                                 float* scales, void* sum_out, int64_t lds, float* mean, float* inv_std, void* hip_stream) {
  if (!float_dtype(dtype) || (y_dtype != dtype && y_dtype != CLEAVE_E4M3)) return CLEAVE_EINVAL;
  if ((y_dtype == CLEAVE_E4M3) != (scales != nullptr)) return CLEAVE_EINVAL;
  if (!(eps >= 0.0f) || std::isinf(eps)) return CLEAVE_EINVAL;
  Matrices m(rows, cols);
  m.add(x, ldx, dtype);
  m.add(residual, ldr, dtype, true);
  m.add(y, ldy, y_dtype);
  m.add(sum_out, lds, dtype, true);
  m.add_vector(weight);
  m.add_vector(bias, true);
  m.add_vector(scales, true);
  m.add_vector(mean, true);
  m.add_vector(inv_std, true);
  if (!m.ok) return CLEAVE_EINVAL;
  if (!in_place(y, ldy, y_dtype, x, ldx, dtype, rows) || !in_place(y, ldy, y_dtype, residual, ldr, dtype, rows) ||
      !in_place(sum_out, lds, dtype, x, ldx, dtype, rows) || !in_place(sum_out, lds, dtype, residual, ldr, dtype, rows) ||
      (rows > 0 && !(apart({y, sum_out, scales, mean, inv_std}, {weight, bias}) && apart({scales, mean, inv_std}, {x, residual}))))
    return CLEAVE_EINVAL;
  if (rows == 0) return CLEAVE_OK;
  const cleave::LayerNormArgs args{x,   residual, weight, bias, y,   scales, sum_out, mean,
                                   inv_std, rows, cols, ldx, ldr, ldy, lds, eps};
  CLEAVE_HIP(cleave::launch_layer_norm(args, dtype, static_cast<hipStream_t>(hip_stream)));
  return CLEAVE_OK;
}

extern "C" int64_t cleave_layer_norm_workspace(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 1 || rows > kMost || cols > kMost) return CLEAVE_EINVAL;
  return (cols + 3) / 4 * 8 * std::max(1, cleave::layer_norm_partial_rows(rows, cols));
}

extern "C" int cleave_layer_norm_backward(int64_t rows, int64_t cols, const void* dy, int64_t lddy, const void* h, int64_t ldh,
                                          const void* dsum, int64_t ldds, int dtype, const float* weight, const float* mean,
                                          const float* inv_std, void* dx, int64_t lddx, float* dweight, float* dbias,
                                          float* workspace, void* hip_stream) {
  if (!float_dtype(dtype)) return CLEAVE_EINVAL;
  Matrices m(rows, cols);
  m.add(dy, lddy, dtype);
  m.add(h, ldh, dtype);
  m.add(dsum, ldds, dtype, true);
  m.add(dx, lddx, dtype);
  m.add_vector(weight);
  m.add_vector(mean);
  m.add_vector(inv_std);
  m.add_vector(dweight);
  m.add_vector(dbias, true);
  m.add_vector(workspace);
  if (!m.ok || !apart({dweight, dbias, workspace}, {})) return CLEAVE_EINVAL;
  if (!in_place(dx, lddx, dtype, dy, lddy, dtype, rows) || !in_place(dx, lddx, dtype, h, ldh, dtype, rows) ||
      !in_place(dx, lddx, dtype, dsum, ldds, dtype, rows) ||
      (rows > 0 && !(apart({dx, dweight, dbias}, {}) && apart({dx, workspace}, {weight, mean, inv_std}) && apart({workspace}, {dy, h, dsum}))))
    return CLEAVE_EINVAL;
  const cleave::LayerNormBackwardArgs args{dy, h,       dsum,  weight, mean, inv_std, dx,   workspace,
                                           dweight, dbias, rows,   cols, lddy,    ldh, ldds, lddx};
  CLEAVE_HIP(cleave::launch_layer_norm_backward(args, dtype, static_cast<hipStream_t>(hip_stream)));
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
  // (one chunk of fp32 leaves a column's sum after its last read, and uses no workspace)
  const bool joined = args.chunks > 1;
  if ((joined && !apart({dbias, workspace}, {rows > 0 ? dy : nullptr})) || (rows > 0 && dy == dbias && dtype == CLEAVE_BF16))
    return CLEAVE_EINVAL;
  CLEAVE_HIP(cleave::launch_column_sum(args, dtype, static_cast<hipStream_t>(hip_stream)));
  return CLEAVE_OK;
}

namespace {

// (columns are counted in 32 bits beyond a row's end)
constexpr int64_t kMostTokens = int64_t{1} << 30;
// (exponents are taken of scale / log 2 times a distance, which may be zero)
constexpr float kMostScale = 0x1p127f;

// Columns of a part of a row: whole lines of sixteen bytes for every group of threads.
int64_t log_probs_chunk(int64_t cols, int parts) { return ((cols + parts - 1) / parts + 511) / 512 * 512; }

}  // namespace

extern "C" int64_t cleave_log_probs_workspace(int64_t rows, int64_t cols, int64_t n_top) {
  if (rows < 0 || cols < 1 || rows > kMost || cols > kMostTokens || n_top < 0 || n_top > cols) return CLEAVE_EINVAL;
  if (n_top > cleave::kMostTop) return CLEAVE_ELIMIT;
  const int64_t parts = cleave::log_probs_parts(rows, cols, n_top);
  return parts == 1 ? 0 : rows * parts * (4 + 2 * n_top);
}

extern "C" int cleave_log_probs(int64_t rows, int64_t cols, const void* logits, int64_t ld, int dtype, float scale,
                                const int64_t* ids, float* logp, float* lse, float* entropy, int64_t n_top, int64_t* top_ids,
                                float* top_logp, float* workspace, void* hip_stream) {
  if (!float_dtype(dtype) || !(scale > 0.0f && scale <= kMostScale)) return CLEAVE_EINVAL;
  Matrices m(rows, cols);
  m.add(logits, ld, dtype);
  m.add_vector(logp, true);
  m.add_vector(lse, true);
  m.add_vector(entropy, true);
  m.add_vector(top_logp, true);
  m.add_vector(workspace, true);
  if (!m.ok || cols > kMostTokens || !aligned(ids, 8) || !aligned(top_ids, 8)) return CLEAVE_EINVAL;
  if ((ids != nullptr) != (logp != nullptr) || n_top < 0 || n_top > cols) return CLEAVE_EINVAL;
  if (n_top > cleave::kMostTop) return CLEAVE_ELIMIT;
  if ((n_top > 0) != (top_ids != nullptr) || (n_top > 0) != (top_logp != nullptr)) return CLEAVE_EINVAL;
  if (!apart({logp, lse, entropy, top_ids, top_logp}, {ids, rows > 0 ? logits : nullptr})) return CLEAVE_EINVAL;
  if (rows == 0) return CLEAVE_OK;
  int parts = cleave::log_probs_parts(rows, cols, n_top);
  if (parts > 1 && (!workspace || !apart({workspace}, {logits, ids, logp, lse, entropy, top_ids, top_logp}))) return CLEAVE_EINVAL;
  const int64_t chunk = log_probs_chunk(cols, parts);
  parts = static_cast<int>((cols + chunk - 1) / chunk);   // (rounding may leave the last ones empty)
  const cleave::LogProbArgs args{logits, ids, logp, lse, entropy, top_ids, top_logp, workspace, rows, cols, ld, scale,
                                 static_cast<int>(n_top), parts, static_cast<int>(std::min(chunk, cols))};
  CLEAVE_HIP(cleave::launch_log_probs(args, dtype, static_cast<hipStream_t>(hip_stream)));
  return CLEAVE_OK;
}

extern "C" int cleave_log_probs_backward(int64_t rows, int64_t cols, const void* logits, int64_t ld, int dtype, float scale,
                                         const int64_t* ids, const float* lse, const float* dlogp, const float* entropy,
                                         const float* dentropy, void* dlogits, int64_t ldd, void* hip_stream) {
  if (!float_dtype(dtype) || !(scale > 0.0f && scale <= kMostScale)) return CLEAVE_EINVAL;
  Matrices m(rows, cols);
  m.add(logits, ld, dtype);
  m.add(dlogits, ldd, dtype);
  m.add_vector(lse);
  m.add_vector(dlogp, true);
  m.add_vector(entropy, true);
  m.add_vector(dentropy, true);
  if (!m.ok || cols > kMostTokens || !aligned(ids, 8)) return CLEAVE_EINVAL;
  if ((ids != nullptr) != (dlogp != nullptr) || (entropy != nullptr) != (dentropy != nullptr) || (!ids && !entropy))
    return CLEAVE_EINVAL;
  if (!in_place(dlogits, ldd, dtype, logits, ld, dtype, rows) ||
      (rows > 0 && !apart({dlogits}, {ids, lse, dlogp, entropy, dentropy})))
    return CLEAVE_EINVAL;
  if (rows == 0) return CLEAVE_OK;
  const cleave::LogProbBackwardArgs args{logits, ids, lse, dlogp, entropy, dentropy, dlogits, rows, cols, ld, ldd, scale, 0, 0.0f};
  CLEAVE_HIP(cleave::launch_log_probs_backward(args, dtype, static_cast<hipStream_t>(hip_stream)));
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
