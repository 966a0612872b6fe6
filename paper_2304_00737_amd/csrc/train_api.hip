// C ABI of libspardl_train.so (declared in include/spardl_train.h): argument
// checks and dispatch.  Nothing here allocates, synchronises or copies
// between host and device.

#include <cmath>

#include "train.hpp"

using namespace spardl_train;

namespace {

bool known(int32_t dtype) { return dtype == SPARDL_BF16 || dtype == SPARDL_FP16 || dtype == SPARDL_FP32; }
int32_t size_of(int32_t dtype) { return dtype == SPARDL_FP32 ? 4 : 2; }
bool element_aligned(const void* p, int32_t size) { return (uintptr_t)p % size == 0; }
constexpr int64_t kMaxRows = (int64_t)1 << 40, kMaxElements = (int64_t)1 << 60;   // of a matrix, its pitch included
int workspace_check(const void* ws, size_t have, size_t need) {
  if (!ws || ((uintptr_t)ws & 255)) return SPARDL_EINVAL;
  return have < need ? SPARDL_ECAPACITY : SPARDL_OK;
}
int status(hipError_t e) { return e == hipSuccess ? SPARDL_OK : SPARDL_EDEVICE; }

bool norm_sizes(int64_t rows, int32_t dim, int32_t dtype) {
  return rows >= 0 && rows <= kMaxRows && dim >= 1 && dim <= SPARDL_NORM_MAX_DIM && known(dtype);
}

// A matrix argument: present unless it has no rows, element aligned, rows of cols elements.
bool matrix(const void* p, int64_t ld, int64_t rows, int64_t cols, int32_t size) {
  return (p || rows == 0) && element_aligned(p, size) && ld >= cols && ld <= kMaxElements / (rows > 1 ? rows : 1);
}
bool vector(const void* p, int64_t n, int32_t size) { return (p || n == 0) && element_aligned(p, size); }

}  // namespace

extern "C" {

int spardl_rms_norm(const void* x, int64_t ld_x, const void* res, int64_t ld_res, const void* weight, void* sum,
                    int64_t ld_sum, void* y, int64_t ld_y, float* rstd, int64_t rows, int32_t dim, float eps,
                    int32_t dtype, hipStream_t stream) {
  if (!norm_sizes(rows, dim, dtype) || !(eps >= 0.f) || std::isinf(eps)) return SPARDL_EINVAL;
  const int32_t z = size_of(dtype);
  if (!matrix(x, ld_x, rows, dim, z) || !matrix(y, ld_y, rows, dim, z) || !vector(weight, dim, z))
    return SPARDL_EINVAL;
  if ((res && !matrix(res, ld_res, rows, dim, z)) || (sum && !matrix(sum, ld_sum, rows, dim, z)) || !element_aligned(rstd, 4))
    return SPARDL_EINVAL;
  return status(launch_rms_norm(x, ld_x, res, ld_res, weight, sum, ld_sum, y, ld_y, rstd, rows, dim, eps, dtype, stream));
}

size_t spardl_rms_norm_workspace_bytes(int64_t rows, int32_t dim) {
  return norm_sizes(rows, dim, SPARDL_FP32) ? rms_norm_ws(rows, dim) : 0;
}

int spardl_rms_norm_backward(const void* dy, int64_t ld_dy, const void* sum, int64_t ld_sum, const void* weight,
                             const float* rstd, const void* dsum, int64_t ld_dsum, void* dx, int64_t ld_dx,
                             float* dweight, int64_t rows, int32_t dim, int32_t dtype, void* ws, size_t ws_bytes,
                             hipStream_t stream) {
  if (!norm_sizes(rows, dim, dtype)) return SPARDL_EINVAL;
  const int32_t z = size_of(dtype);
  if (!matrix(dy, ld_dy, rows, dim, z) || !matrix(sum, ld_sum, rows, dim, z) || !matrix(dx, ld_dx, rows, dim, z) || !vector(weight, dim, z) ||
      !vector(rstd, rows, 4) || !vector(dweight, dim, 4))
    return SPARDL_EINVAL;
  if (dsum && !matrix(dsum, ld_dsum, rows, dim, z)) return SPARDL_EINVAL;
  if (int e = workspace_check(ws, ws_bytes, rms_norm_ws(rows, dim))) return e;
  return status(launch_rms_norm_backward(dy, ld_dy, sum, ld_sum, weight, rstd, dsum, ld_dsum, dx, ld_dx, dweight, rows,
                                         dim, dtype, ws, stream));
}

size_t spardl_distill_workspace_bytes(int64_t rows, int32_t vocab) {
  return rows >= 0 && rows <= kMaxRows && vocab >= 1 ? distill_ws(rows, vocab) : 0;
}

}  // extern "C"

namespace {

int distill_check(const Distill& d) {
  if (d.rows < 0 || d.rows > kMaxRows || d.vocab < 1 || d.top < 1 || d.top > SPARDL_DISTILL_MAX_TOP || !known(d.dtype))
    return SPARDL_EINVAL;
  if (!std::isnormal(d.temperature) || d.temperature < 0.f) return SPARDL_EINVAL;     // log2(e) / it is finite
  if (!matrix(d.logits, d.ld, d.rows, d.vocab, size_of(d.dtype)) || !matrix(d.top_idx, d.ld_top, d.rows, d.top, 4) ||
      !matrix(d.top_val, d.ld_top, d.rows, d.top, 4))
    return SPARDL_EINVAL;
  if (!vector(d.stats, d.rows, 4)) return SPARDL_EINVAL;
  return SPARDL_OK;
}
bool gradient_ok(const Distill& d) {
  return vector(d.dloss, d.rows, 4) && matrix(d.dlogits, d.ld_d, d.rows, d.vocab, size_of(d.dtype));
}

// Sizes whose tiles and launches fit their counters.
bool ffn_sizes(int64_t tokens, int64_t dim, int64_t hidden) {
  const int64_t most = (int64_t)1 << 36;
  return tokens >= 0 && tokens <= INT32_MAX && dim >= 1 && hidden >= 1 && dim <= (1 << 20) && hidden <= (1 << 20) &&
         tokens * dim <= most && tokens * hidden <= most && dim * hidden <= most;
}

int ffn_check(const Ffn& f) {
  if (!ffn_sizes(f.tokens, f.dim, f.hidden)) return SPARDL_EINVAL;
  if (f.dtype != SPARDL_BF16 && f.dtype != SPARDL_FP16) return SPARDL_EINVAL;
  if (f.act != SPARDL_ACT_SILU && f.act != SPARDL_ACT_GELU) return SPARDL_EINVAL;
  if (!matrix(f.x, f.ld_x, f.tokens, f.dim, 2) || !matrix(f.w_gate, f.ld_gate, f.hidden, f.dim, 2) || !matrix(f.w_up, f.ld_up, f.hidden, f.dim, 2) ||
      !matrix(f.w_down, f.ld_down, f.dim, f.hidden, 2))
    return SPARDL_EINVAL;
  if (!f.gate != !f.up || (f.gate && (!matrix(f.gate, f.ld_hidden, f.tokens, f.hidden, 2) || !element_aligned(f.up, 2))))
    return SPARDL_EINVAL;
  return SPARDL_OK;
}

int ffn_workspace(const Ffn& f, bool backward, const void* ws, size_t ws_bytes) {
  // Widths that are no multiple of 8 have gated_ffn_ws ask for copies by themselves, where copies are made.
  auto view = [](const void* p, int64_t ld, int32_t cols) { return cols % 8 == 0 && !rows_aligned(p, ld); };
  const bool views = view(f.x, f.ld_x, f.dim) || view(f.w_gate, f.ld_gate, f.dim) || view(f.w_up, f.ld_up, f.dim) ||
                     view(f.w_down, f.ld_down, f.hidden) || (backward && view(f.dy, f.ld_dy, f.dim));
  return workspace_check(ws, ws_bytes, gated_ffn_ws(f.tokens, f.dim, f.hidden, backward, views));
}

}  // namespace

extern "C" {

int spardl_distill_loss(const void* logits, int64_t ld, const int32_t* top_idx, const float* top_val, int64_t ld_top,
                        int64_t rows, int32_t vocab, int32_t top, float temperature, float* loss, float* stats,
                        int32_t dtype, void* ws, size_t ws_bytes, hipStream_t stream) {
  const Distill d = {logits, ld, top_idx, top_val, ld_top, rows, vocab, top, temperature, loss, stats, nullptr,
                     nullptr, 0, dtype};
  if (int e = distill_check(d)) return e;
  if (!vector(loss, rows, 4)) return SPARDL_EINVAL;
  if (int e = workspace_check(ws, ws_bytes, distill_ws(rows, vocab))) return e;
  return status(launch_distill(d, ws, stream));
}

int spardl_distill_backward(const void* logits, int64_t ld, const int32_t* top_idx, const float* top_val,
                            int64_t ld_top, const float* stats, const float* dloss, int64_t rows, int32_t vocab,
                            int32_t top, float temperature, void* dlogits, int64_t ld_d, int32_t dtype,
                            hipStream_t stream) {
  const Distill d = {logits, ld, top_idx, top_val, ld_top, rows, vocab, top, temperature, nullptr,
                     const_cast<float*>(stats), dloss, dlogits, ld_d, dtype};
  if (int e = distill_check(d)) return e;
  if (!gradient_ok(d)) return SPARDL_EINVAL;
  return status(launch_distill(d, nullptr, stream));
}

int spardl_distill_loss_backward(const void* logits, int64_t ld, const int32_t* top_idx, const float* top_val,
                                 int64_t ld_top, const float* dloss, int64_t rows, int32_t vocab, int32_t top,
                                 float temperature, float* loss, float* stats, void* dlogits, int64_t ld_d,
                                 int32_t dtype, void* ws, size_t ws_bytes, hipStream_t stream) {
  const Distill d = {logits, ld, top_idx, top_val, ld_top, rows, vocab, top, temperature, loss, stats, dloss,
                     dlogits, ld_d, dtype};
  if (int e = distill_check(d)) return e;
  if (!vector(loss, rows, 4) || !gradient_ok(d)) return SPARDL_EINVAL;
  if (int e = workspace_check(ws, ws_bytes, distill_ws(rows, vocab))) return e;
  return status(launch_distill(d, ws, stream));
}

size_t spardl_gated_ffn_workspace_bytes(int64_t tokens, int32_t dim, int32_t hidden, int32_t backward,
                                        int32_t unaligned) {
  if (!ffn_sizes(tokens, dim, hidden)) return 0;
  return gated_ffn_ws(tokens, dim, hidden, backward != 0, unaligned != 0);
}

int spardl_gated_ffn(const void* x, int64_t ld_x, const void* w_gate, int64_t ld_gate, const void* w_up,
                     int64_t ld_up, const void* w_down, int64_t ld_down, void* y, int64_t ld_y, void* gate, void* up,
                     int64_t ld_hidden, int64_t tokens, int32_t dim, int32_t hidden, int32_t act, int32_t dtype,
                     void* ws, size_t ws_bytes, hipStream_t stream) {
  Ffn f = {};
  f.x = x, f.w_gate = w_gate, f.w_up = w_up, f.w_down = w_down, f.y = y, f.gate = gate, f.up = up;
  f.ld_x = ld_x, f.ld_gate = ld_gate, f.ld_up = ld_up, f.ld_down = ld_down, f.ld_y = ld_y, f.ld_hidden = ld_hidden;
  f.tokens = tokens, f.dim = dim, f.hidden = hidden, f.act = act, f.dtype = dtype;
  if (int e = ffn_check(f)) return e;
  if (!matrix(y, ld_y, tokens, dim, 2)) return SPARDL_EINVAL;
  if (int e = ffn_workspace(f, false, ws, ws_bytes)) return e;
  return status(dtype == SPARDL_BF16 ? ffn_forward_bf16(f, ws, stream) : ffn_forward_fp16(f, ws, stream));
}

int spardl_gated_ffn_backward(const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, const void* gate,
                              const void* up, int64_t ld_hidden, const void* w_gate, int64_t ld_gate,
                              const void* w_up, int64_t ld_up, const void* w_down, int64_t ld_down, void* dx,
                              int64_t ld_dx, void* dw_gate, int64_t ld_dgate, void* dw_up, int64_t ld_dup,
                              void* dw_down, int64_t ld_ddown, int32_t dw_dtype, int32_t accumulate, int64_t tokens,
                              int32_t dim, int32_t hidden, int32_t act, int32_t dtype, void* ws, size_t ws_bytes,
                              hipStream_t stream) {
  Ffn f = {};
  f.x = x, f.w_gate = w_gate, f.w_up = w_up, f.w_down = w_down, f.dy = dy;
  f.gate = const_cast<void*>(gate), f.up = const_cast<void*>(up);
  f.dx = dx, f.dw_gate = dw_gate, f.dw_up = dw_up, f.dw_down = dw_down;
  f.ld_x = ld_x, f.ld_gate = ld_gate, f.ld_up = ld_up, f.ld_down = ld_down, f.ld_dy = ld_dy, f.ld_hidden = ld_hidden;
  f.ld_dx = ld_dx, f.ld_dgate = ld_dgate, f.ld_dup = ld_dup, f.ld_ddown = ld_ddown;
  f.tokens = tokens, f.dim = dim, f.hidden = hidden, f.act = act, f.dtype = dtype;
  f.dw_dtype = dw_dtype, f.accumulate = accumulate != 0;
  if (int e = ffn_check(f)) return e;
  if (dw_dtype != dtype && dw_dtype != SPARDL_FP32) return SPARDL_EINVAL;
  const int32_t z = size_of(dw_dtype);
  if ((!gate && tokens > 0) || !matrix(dy, ld_dy, tokens, dim, 2) || (dx && !matrix(dx, ld_dx, tokens, dim, 2)) ||
      !matrix(dw_gate, ld_dgate, hidden, dim, z) || !matrix(dw_up, ld_dup, hidden, dim, z) ||
      !matrix(dw_down, ld_ddown, dim, hidden, z))
    return SPARDL_EINVAL;
  if (int e = ffn_workspace(f, true, ws, ws_bytes)) return e;
  return status(dtype == SPARDL_BF16 ? ffn_backward_bf16(f, ws, stream) : ffn_backward_fp16(f, ws, stream));
}

}  // extern "C"
