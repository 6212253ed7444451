// Shared pieces of the head norm and the gated delta rule: launch parameters, sums over lanes.
#pragma once
#include "tac_delta_plan.h"
#include "tac_head_common.h"

namespace tac {

// sum over LANES (8, 16, 32 or 64) consecutive lanes, every lane gets it: within a row of 16 by exchanges of quads and mirrors, then swaps of rows
template <int CONTROL>
__device__ __forceinline__ float lanes_moved(float v) {
  return bits_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)float_bits(v), CONTROL, 0xf, 0xf, false));
}
template <int LANES>
__device__ __forceinline__ float sum_over_lanes(float v) {
  v += lanes_moved<0xb1>(v);                 // quad_perm 1 0 3 2
  v += lanes_moved<0x4e>(v);                 // quad_perm 2 3 0 1
  v += lanes_moved<0x141>(v);                // row_half_mirror
  if constexpr (LANES >= 16) v += lanes_moved<0x140>(v);       // row_mirror
  if constexpr (LANES >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(float_bits(v), float_bits(v), false, false);
    v = bits_float(r[0]) + bits_float(r[1]);
  }
  if constexpr (LANES >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(float_bits(v), float_bits(v), false, false);
    v = bits_float(r[0]) + bits_float(r[1]);
  }
  return v;
}

// N elements as they stand in memory
template <typename T, int N>
struct Piece;
template <int N>
struct Piece<bf16, N> {
  uint32_t w[N / 2];
  __device__ __forceinline__ void set(int e, bf16 x) {
    const uint32_t v = __builtin_bit_cast(uint16_t, x);
    w[e / 2] = e % 2 ? (w[e / 2] & 0xffffu) | v << 16 : (w[e / 2] & 0xffff0000u) | v;
  }
};
template <int N>
struct Piece<float, N> {
  float w[N];
  __device__ __forceinline__ void set(int e, float x) { w[e] = x; }
};
template <int N>
__device__ __forceinline__ float value_of(const Piece<bf16, N>& v, int e) {
  return bits_float(e % 2 ? v.w[e / 2] & 0xffff0000u : v.w[e / 2] << 16);
}
template <int N>
__device__ __forceinline__ float value_of(const Piece<float, N>& v, int e) {
  return v.w[e];
}

// 1 / (1 + exp(-x)); exp overflows to infinity, whose reciprocal is 0
__device__ __forceinline__ float sigmoid(float x) { return 1.0f / (1.0f + expf(-x)); }

// ---- launch parameters ---------------------------------------------------------------------------
struct HeadTensor {
  const void *x, *grad_out;          // grad_out: backward only
  void* out;                         // the result, or the gradient
  const float* gain;
  tac_head_strides_t x_stride, grad_out_stride, out_stride;
  int heads;
};
struct HeadNormParams {
  HeadTensor q, k;                   // k.heads is 0 without keys
  const int32_t* positions;
  float *partial, *grad_gain_q, *grad_gain_k;
  int64_t rows;
  int D, axes, pairs[TAC_ROTATION_AXES], rotated;      // rotated: pairs in all
  int interleaved, bf16, slices, apart;
  float eps;
  double log2_step[TAC_ROTATION_AXES];      // log2(base) / pairs
};
size_t head_norm_workspace(const HeadNormParams& p);
hipError_t head_norm_launch(const HeadNormParams& p, hipStream_t s);
hipError_t head_norm_backward_launch(const HeadNormParams& p, hipStream_t s);

struct DeltaStepParams {
  const void *q, *k, *v, *gate, *write;
  float* pool;
  const int32_t* slots;
  void* out;
  int64_t n_slots;
  tac_delta_strides_t q_at, k_at, v_at, gate_at, write_at, out_at;
  int B, k_heads, v_heads, Dk, Dv, bf16;
};
hipError_t delta_step_launch(const DeltaStepParams& p, hipStream_t s);

}  // namespace tac
