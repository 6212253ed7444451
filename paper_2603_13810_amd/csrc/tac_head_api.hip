// Host side of the dense operators' C ABI: argument checks and launch parameters.  Nothing is launched before all of them hold.
#include <cmath>

#include "tac_head_common.h"
#include "tac_quantize_plan.h"

namespace {

constexpr int64_t kMost = (1ll << 31) - 1;

bool float_type(int32_t dtype) { return dtype == TAC_FP32 || dtype == TAC_BF16; }
size_t bytes_of(int32_t dtype) { return dtype == TAC_BF16 ? 2 : 4; }
bool misaligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) != 0; }

int finish(hipError_t e, const char* where) { return e == hipSuccess ? TAC_OK : tac::hip_fail(e, where); }

// rows of `stride` elements, `rows` of them, stay within 2^62 bytes
bool in_reach(int64_t rows, int64_t stride) { return stride >= 0 && stride <= (1ll << 60) / rows; }

int check_norm(const tac_norm_desc_t* d) {
  if (!d) return TAC_ERR_NULL;
  if (d->rows < 1 || d->rows > kMost || d->cols < 1) return TAC_ERR_BAD_SHAPE;
  if (!float_type(d->dtype)) return TAC_ERR_BAD_PARAM;
  if (!(d->eps > 0.0f) || !std::isfinite(d->eps)) return TAC_ERR_BAD_PARAM;
  if (d->cols > TAC_NORM_MAX_COLS) return TAC_ERR_UNSUPPORTED;
  return TAC_OK;
}

bool bad_stride(const void* p, int64_t stride, int64_t rows, int64_t cols) {
  return p && (stride < cols || !in_reach(rows, stride));
}

int check_scan(const tac_scan_desc_t* d) {
  if (!d) return TAC_ERR_NULL;
  if (d->T < 1 || d->T > kMost || d->B < 1 || d->B > 65535 || d->D < 1) return TAC_ERR_BAD_SHAPE;
  if ((int64_t)d->B * d->D > kMost) return TAC_ERR_BAD_SHAPE;
  if (!float_type(d->dtype)) return TAC_ERR_BAD_PARAM;
  return TAC_OK;
}

// steps and sequences may lie in any order, but not on top of each other's channels
bool bad_layout(const tac_scan_desc_t* d, int64_t stride_t, int64_t stride_b) {
  return (d->T > 1 && (stride_t < d->D || !in_reach(d->T, stride_t))) || (d->B > 1 && (stride_b < d->D || !in_reach(d->B, stride_b)));
}

}  // namespace

extern "C" {

size_t tac_code_bytes(int64_t rows, int64_t cols) {
  return rows < 1 || cols < 1 || rows > kMost || cols > kMost ? 0 : (size_t)rows * (size_t)tac::code_pitch(cols);
}

size_t tac_scale_bytes(int64_t rows, int64_t cols) {
  return rows < 1 || cols < 1 || rows > kMost || cols > kMost ? 0 : (size_t)rows * (size_t)tac::scale_pitch(cols);
}

int tac_quantize(const tac_quantize_desc_t* d, const void* src, const uint8_t* src_scales, uint8_t* codes, uint8_t* scales,
                 uint8_t* codes_t, uint8_t* scales_t, void* stream) {
  if (!d || !src || (!codes && !codes_t) || !codes != !scales || !codes_t != !scales_t) return TAC_ERR_NULL;
  if (d->rows < 1 || d->cols < 1 || d->rows > kMost || d->cols > kMost) return TAC_ERR_BAD_SHAPE;
  if (!float_type(d->dtype) && d->dtype != TAC_SCALED) return TAC_ERR_BAD_PARAM;
  if (d->block != TAC_BLOCK_ROW && d->block != TAC_BLOCK_TILE) return TAC_ERR_BAD_PARAM;
  const bool scaled = d->dtype == TAC_SCALED;
  if (scaled && !src_scales) return TAC_ERR_NULL;
  if (!scaled && bad_stride(src, d->src_stride, d->rows, d->cols)) return TAC_ERR_BAD_SHAPE;
  const int64_t tiles = ((d->rows + 127) / 128) * ((d->cols + 127) / 128);
  if (tiles >= tac::kMostTiles) return TAC_ERR_BAD_SHAPE;
  if (misaligned(src, scaled ? 16 : bytes_of(d->dtype)) || (scaled && misaligned(src_scales, 4)) || misaligned(codes, 16) ||
      misaligned(codes_t, 16) || misaligned(scales, 4) || misaligned(scales_t, 4))
    return TAC_ERR_ALIGN;
  const tac::QuantizeParams p = {src, src_scales, codes, scales, codes_t, scales_t, d->rows, d->cols, d->src_stride, d->dtype,
                                 d->block == TAC_BLOCK_TILE};
  return finish(tac::quantize_launch(p, (hipStream_t)stream), "tac_quantize");
}

int tac_dequantize(int64_t rows, int64_t cols, const uint8_t* codes, const uint8_t* scales, int32_t dtype, void* dst,
                   int64_t dst_stride, void* stream) {
  if (!codes || !scales || !dst) return TAC_ERR_NULL;
  if (rows < 1 || cols < 1 || rows > kMost || cols > kMost || bad_stride(dst, dst_stride, rows, cols)) return TAC_ERR_BAD_SHAPE;
  if (!float_type(dtype)) return TAC_ERR_BAD_PARAM;
  if (misaligned(codes, 16) || misaligned(scales, 4) || misaligned(dst, bytes_of(dtype))) return TAC_ERR_ALIGN;
  return finish(tac::dequantize_launch(codes, scales, dst, rows, cols, dst_stride, dtype == TAC_BF16, (hipStream_t)stream),
                "tac_dequantize");
}

int tac_residual_norm(const tac_norm_desc_t* d, const void* x, const void* residual, const float* gain, void* h, void* y,
                      uint8_t* codes, uint8_t* scales, float* rstd, void* stream) {
  const int rc = check_norm(d);
  if (rc) return rc;
  if (!x || (!h && !y && !codes && !rstd) || !codes != !scales) return TAC_ERR_NULL;
  if (bad_stride(x, d->x_stride, d->rows, d->cols) || bad_stride(residual, d->residual_stride, d->rows, d->cols) ||
      bad_stride(h, d->h_stride, d->rows, d->cols) || bad_stride(y, d->y_stride, d->rows, d->cols))
    return TAC_ERR_BAD_SHAPE;
  const size_t el = bytes_of(d->dtype);
  if (misaligned(x, el) || misaligned(residual, el) || misaligned(h, el) || misaligned(y, el) || misaligned(gain, 4) ||
      misaligned(rstd, 4) || misaligned(codes, 16) || misaligned(scales, 4))
    return TAC_ERR_ALIGN;
  const tac::NormParams p = {x, residual, gain, h, y, codes, scales, rstd, d->rows, d->x_stride, d->residual_stride, d->h_stride,
                             d->y_stride, d->cols, d->dtype == TAC_BF16, d->eps};
  return finish(tac::norm_launch(p, (hipStream_t)stream), "tac_residual_norm");
}

size_t tac_residual_norm_workspace_bytes(const tac_norm_desc_t* d) {
  return check_norm(d) ? 0 : tac::norm_backward_workspace(d->rows, d->cols);
}

int tac_residual_norm_backward(const tac_norm_desc_t* d, const void* h, const float* gain, const float* rstd, const void* grad_y,
                               const void* grad_h, void* grad_x, float* grad_gain, void* workspace, void* stream) {
  const int rc = check_norm(d);
  if (rc) return rc;
  if (!h || !rstd || !grad_y || !grad_x || (grad_gain && !workspace)) return TAC_ERR_NULL;
  if (bad_stride(h, d->h_stride, d->rows, d->cols) || bad_stride(grad_y, d->y_stride, d->rows, d->cols) ||
      bad_stride(grad_h, d->residual_stride, d->rows, d->cols) || bad_stride(grad_x, d->x_stride, d->rows, d->cols))
    return TAC_ERR_BAD_SHAPE;
  const size_t el = bytes_of(d->dtype);
  if (misaligned(h, el) || misaligned(grad_y, el) || misaligned(grad_h, el) || misaligned(grad_x, el) || misaligned(gain, 4) ||
      misaligned(rstd, 4) || misaligned(grad_gain, 4) || misaligned(workspace, 16))
    return TAC_ERR_ALIGN;
  const tac::NormBackwardParams p = {h, gain, rstd, grad_y, grad_h, grad_x, grad_gain, (float*)workspace, d->rows, d->h_stride,
                                     d->y_stride, d->residual_stride, d->x_stride, d->cols, d->dtype == TAC_BF16};
  return finish(tac::norm_backward_launch(p, (hipStream_t)stream), "tac_residual_norm_backward");
}

static int check_product(const tac_product_desc_t* d) {
  if (!d) return TAC_ERR_NULL;
  if (d->M < 1 || d->N < 1 || d->K < 1 || d->M > kMost || d->N > kMost || d->K > kMost) return TAC_ERR_BAD_SHAPE;
  if (d->y_stride < d->N || !in_reach(d->M, d->y_stride)) return TAC_ERR_BAD_SHAPE;
  if (d->K > TAC_PRODUCT_MAX_K) return TAC_ERR_UNSUPPORTED;
  return float_type(d->dtype) ? TAC_OK : TAC_ERR_BAD_PARAM;
}

size_t tac_scaled_product_workspace_bytes(const tac_product_desc_t* d) {
  return check_product(d) ? 0 : tac::product_workspace(d->M, d->N, d->K, d->dtype == TAC_BF16);
}

int tac_scaled_product(const tac_product_desc_t* d, const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* b_codes,
                       const uint8_t* b_scales, const float* bias, void* y, void* workspace, void* stream) {
  const int rc = check_product(d);
  if (rc) return rc;
  if (!a_codes || !a_scales || !b_codes || !b_scales || !y) return TAC_ERR_NULL;
  if (!workspace && tac::product_workspace(d->M, d->N, d->K, d->dtype == TAC_BF16)) return TAC_ERR_NULL;
  if (misaligned(a_codes, 16) || misaligned(b_codes, 16) || misaligned(a_scales, 4) || misaligned(b_scales, 4) ||
      misaligned(bias, 4) || misaligned(y, bytes_of(d->dtype)) || misaligned(workspace, 16))
    return TAC_ERR_ALIGN;
  const tac::ProductParams p = {a_codes, a_scales, b_codes, b_scales, bias, y, (float*)workspace, d->M, d->N, d->K, d->y_stride,
                                d->dtype == TAC_BF16};
  return finish(tac::product_launch(p, (hipStream_t)stream), "tac_scaled_product");
}

size_t tac_gated_scan_workspace_bytes(const tac_scan_desc_t* d) {
  return check_scan(d) ? 0 : tac::scan_workspace(d->T, d->B, d->D, d->dtype == TAC_BF16);
}

int tac_gated_scan(const tac_scan_desc_t* d, const void* gate, const void* value, const int32_t* lengths, const float* h0,
                   void* out, float* h_last, float* states, void* workspace, void* stream) {
  const int rc = check_scan(d);
  if (rc) return rc;
  if (!gate || !value || !out) return TAC_ERR_NULL;
  if (!workspace && tac::scan_workspace(d->T, d->B, d->D, d->dtype == TAC_BF16)) return TAC_ERR_NULL;
  if (bad_layout(d, d->in_stride_t, d->in_stride_b) || bad_layout(d, d->out_stride_t, d->out_stride_b)) return TAC_ERR_BAD_SHAPE;
  const size_t el = bytes_of(d->dtype);
  if (misaligned(gate, el) || misaligned(value, el) || misaligned(out, el) || misaligned(lengths, 4) || misaligned(h0, 4) ||
      misaligned(h_last, 4) || misaligned(states, 4) || misaligned(workspace, 16))
    return TAC_ERR_ALIGN;
  const tac::ScanParams p = {gate, value, lengths, h0, out, h_last, states, (float*)workspace, d->T, d->in_stride_t, d->in_stride_b,
                             d->out_stride_t, d->out_stride_b, d->B, d->D, d->dtype == TAC_BF16};
  return finish(tac::scan_launch(p, (hipStream_t)stream), "tac_gated_scan");
}

int tac_gated_scan_backward(const tac_scan_desc_t* d, const void* gate, const void* value, const int32_t* lengths,
                            const float* states, const void* grad_out, const float* grad_h_last, void* grad_gate, void* grad_value,
                            float* grad_h0, void* workspace, void* stream) {
  const int rc = check_scan(d);
  if (rc) return rc;
  if (!gate || !value || !states || !grad_out || !grad_gate || !grad_value) return TAC_ERR_NULL;
  if (!workspace && tac::scan_workspace(d->T, d->B, d->D, d->dtype == TAC_BF16)) return TAC_ERR_NULL;
  if (bad_layout(d, d->in_stride_t, d->in_stride_b) || bad_layout(d, d->out_stride_t, d->out_stride_b) ||
      bad_layout(d, d->grad_stride_t, d->grad_stride_b))
    return TAC_ERR_BAD_SHAPE;
  const size_t el = bytes_of(d->dtype);
  if (misaligned(gate, el) || misaligned(value, el) || misaligned(grad_out, el) || misaligned(grad_gate, el) ||
      misaligned(grad_value, el) || misaligned(lengths, 4) || misaligned(states, 4) || misaligned(grad_h_last, 4) ||
      misaligned(grad_h0, 4) || misaligned(workspace, 16))
    return TAC_ERR_ALIGN;
  const tac::ScanBackwardParams p = {gate, value, lengths, states, grad_out, grad_h_last, grad_gate, grad_value, grad_h0,
                                     (float*)workspace, d->T, d->in_stride_t, d->in_stride_b, d->out_stride_t, d->out_stride_b,
                                     d->grad_stride_t, d->grad_stride_b, d->B, d->D, d->dtype == TAC_BF16};
  return finish(tac::scan_backward_launch(p, (hipStream_t)stream), "tac_gated_scan_backward");
}

int tac_gated_step(const tac_scan_desc_t* d, const void* gate, const void* value, float* pool, int64_t n_slots,
                   const int32_t* slots, void* out, void* stream) {
  const int rc = check_scan(d);
  if (rc) return rc;
  if (!gate || !value || !pool || !out) return TAC_ERR_NULL;
  if (d->T != 1 || n_slots < 1 || n_slots > kMost || (!slots && n_slots < d->B)) return TAC_ERR_BAD_SHAPE;
  if (bad_layout(d, d->in_stride_t, d->in_stride_b) || bad_layout(d, d->out_stride_t, d->out_stride_b)) return TAC_ERR_BAD_SHAPE;
  const size_t el = bytes_of(d->dtype);
  if (misaligned(gate, el) || misaligned(value, el) || misaligned(out, el) || misaligned(pool, 4) || misaligned(slots, 4))
    return TAC_ERR_ALIGN;
  const tac::StepParams p = {gate, value, pool, slots, out, d->in_stride_b, d->out_stride_b, n_slots, d->B, d->D,
                             d->dtype == TAC_BF16};
  return finish(tac::step_launch(p, (hipStream_t)stream), "tac_gated_step");
}

}  // extern "C"
