// Gated linear recurrence h_t = a_t h_{t-1} + (1 - a_t) value_t with a_t = 1 / (1 + exp(-gate_t)), its backward pass, and one step of it
// on a pool of states.
#include "tac_head_common.h"

namespace tac {

namespace {

constexpr int kChunk = TAC_SCAN_CHUNK;

// a and 1 - a, the second without cancellation.  Gates below -80 count as -80 (exp stays finite; a < 2e-35 there).
struct Leak {
  float a, rest;
};
__device__ __forceinline__ Leak leak(float gate) {
  const float e = __expf(-fmaxf(gate, -80.0f));
  const float r = __builtin_amdgcn_rcpf(1.0f + e);
  return Leak{r, e * r};
}

__device__ __forceinline__ int64_t length_of(const int32_t* lengths, int b, int64_t T) {
  return lengths ? min(max((int64_t)lengths[b], (int64_t)0), T) : T;
}

// a thread per channel
template <typename T>
__global__ __launch_bounds__(256) void scan_kernel(const ScanParams p) {
  const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (n >= (int64_t)p.B * p.D) return;
  const int b = (int)(n / p.D), d = (int)(n - (int64_t)b * p.D);
  const int64_t len = length_of(p.lengths, b, p.T);
  float h = p.h0 ? p.h0[n] : 0.0f;
  const T *g = (const T*)p.gate + b * p.in_b + d, *u = (const T*)p.value + b * p.in_b + d;
  T* out = (T*)p.out + b * p.out_b + d;
  for (int64_t t = 0; t < p.T; ++t) {
    if (p.states && t % kChunk == 0) p.states[t / kChunk * p.B * p.D + n] = h;
    float o = 0.0f;
    if (t < len) {
      const Leak k = leak((float)g[t * p.in_t]);
      o = h = fmaf(k.a, h, k.rest * (float)u[t * p.in_t]);
    }
    out[t * p.out_t] = (T)o;
  }
  if (p.h_last) p.h_last[n] = h;
}

template <typename T>
__global__ __launch_bounds__(256) void scan_backward_kernel(const ScanBackwardParams p) {
  const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (n >= (int64_t)p.B * p.D) return;
  const int b = (int)(n / p.D), d = (int)(n - (int64_t)b * p.D);
  const int64_t len = length_of(p.lengths, b, p.T);
  const T *g = (const T*)p.gate + b * p.in_b + d, *u = (const T*)p.value + b * p.in_b + d, *go = (const T*)p.grad_out + b * p.out_b + d;
  T *gg = (T*)p.grad_gate + b * p.grad_b + d, *gv = (T*)p.grad_value + b * p.grad_b + d;
  float c = p.grad_h_last ? p.grad_h_last[n] : 0.0f;
  for (int64_t chunk = (p.T + kChunk - 1) / kChunk - 1; chunk >= 0; --chunk) {
    const int64_t t0 = chunk * kChunk;
    float before[kChunk];
    float h = p.states[chunk * p.B * p.D + n];
#pragma unroll
    for (int i = 0; i < kChunk; ++i) {
      before[i] = h;
      if (t0 + i < len) {
        const Leak k = leak((float)g[(t0 + i) * p.in_t]);
        h = fmaf(k.a, h, k.rest * (float)u[(t0 + i) * p.in_t]);
      }
    }
#pragma unroll
    for (int i = kChunk - 1; i >= 0; --i) {
      const int64_t t = t0 + i;
      if (t >= p.T) continue;
      float dg = 0.0f, dv = 0.0f;
      if (t < len) {
        const Leak k = leak((float)g[t * p.in_t]);
        c += (float)go[t * p.out_t];
        dv = k.rest * c;
        dg = dv * k.a * (before[i] - (float)u[t * p.in_t]);
        c *= k.a;
      }
      gg[t * p.grad_t] = (T)dg;
      gv[t * p.grad_t] = (T)dv;
    }
  }
  if (p.grad_h0) p.grad_h0[n] = c;
}

// a thread per channel of a row
template <typename T>
__global__ __launch_bounds__(256) void step_kernel(const StepParams p) {
  const int d = blockIdx.x * 256 + threadIdx.x, b = blockIdx.y;
  if (d >= p.D) return;
  const int64_t slot = p.slots ? p.slots[b] : b;
  float h = 0.0f;
  if (slot >= 0 && slot < p.n_slots) {
    float* state = p.pool + slot * p.D + d;
    const Leak k = leak((float)((const T*)p.gate)[b * p.in_b + d]);
    h = fmaf(k.a, *state, k.rest * (float)((const T*)p.value)[b * p.in_b + d]);
    *state = h;
  }
  ((T*)p.out)[b * p.out_b + d] = (T)h;
}

}  // namespace

size_t scan_workspace(int64_t, int, int, int) { return 0; }

hipError_t scan_launch(const ScanParams& p, hipStream_t s) {
  const dim3 grid((unsigned)(((int64_t)p.B * p.D + 255) / 256));
  if (p.bf16) hipLaunchKernelGGL(scan_kernel<bf16>, grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL(scan_kernel<float>, grid, dim3(256), 0, s, p);
  return hipGetLastError();
}

hipError_t scan_backward_launch(const ScanBackwardParams& p, hipStream_t s) {
  const dim3 grid((unsigned)(((int64_t)p.B * p.D + 255) / 256));
  if (p.bf16) hipLaunchKernelGGL(scan_backward_kernel<bf16>, grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL(scan_backward_kernel<float>, grid, dim3(256), 0, s, p);
  return hipGetLastError();
}

hipError_t step_launch(const StepParams& p, hipStream_t s) {
  const dim3 grid((unsigned)((p.D + 255) / 256), (unsigned)p.B);
  if (p.bf16) hipLaunchKernelGGL(step_kernel<bf16>, grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL(step_kernel<float>, grid, dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace tac
