// One step of the gated delta rule for running sequences whose states stand in a pool.
//
// Bound by the states' bytes, each read and written once.  A workgroup has 32 columns of one head's state in registers, 8 lanes x 16 bytes along a row and 32 rows at
// a time; the columns' products with the key and the query are sums over rows: within a wave by swaps, over the four waves through LDS.  The query reads
// the new state, S_t^T q = a S^T q + (k . q) u, so that one pass over the rows is enough.
// 128 sequences, 16 heads of 128 x 128: 268 MB in 55.5 us, 4.8 TB/s (through the caches 65.6 a call, past them 57.6); one sequence: 4.7 us, the launch and one trip to memory and back.
#include "tac_delta_common.h"

namespace tac {

namespace {

constexpr int kTile = 32;            // columns of a workgroup
constexpr int kRows = TAC_DELTA_MAX_KEY / 32;

template <bool VEC, bool PAST>
__device__ __forceinline__ f32x4_t load_four(const float* p, int n) {
  if constexpr (VEC && PAST) return __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(p));
  else if constexpr (VEC) return *reinterpret_cast<const f32x4_t*>(p);
  f32x4_t v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < n) v[e] = p[e];
  return v;
}

template <typename T, bool VEC, bool PAST>
__global__ __launch_bounds__(256) void delta_step_kernel(const DeltaStepParams p) {
  __shared__ float room[4][8][9];                      // per wave and lane of a row: four sums with the key, four with the query, k . q
  const int tiles = (p.Dv + kTile - 1) / kTile;
  const int tile = blockIdx.x % tiles, h = blockIdx.x / tiles % p.v_heads, b = blockIdx.x / tiles / p.v_heads;
  const int lane = threadIdx.x % 8, group = threadIdx.x / 8, col = tile * kTile + lane * 4, left = p.Dv - col;
  const int64_t slot = p.slots ? (int64_t)p.slots[b] : (int64_t)b;
  T* out = (T*)p.out + (int64_t)b * p.out_at.b + (int64_t)h * p.out_at.head;
  if (slot < 0 || slot >= p.n_slots) {                 // the same for the whole workgroup
    if (group == 0)
      for (int e = 0; e < 4 && e < left; ++e) out[col + e] = (T)0.0f;
    return;
  }
  const int hk = h / (p.v_heads / p.k_heads);
  const T* q = (const T*)p.q + (int64_t)b * p.q_at.b + (int64_t)hk * p.q_at.head;
  const T* k = (const T*)p.k + (int64_t)b * p.k_at.b + (int64_t)hk * p.k_at.head;
  float* S = p.pool + (slot * p.v_heads + h) * (int64_t)p.Dk * p.Dv;
  f32x4_t s[kRows];
  float kr[kRows], qr[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int r = group + 32 * i;
    s[i] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    kr[i] = qr[i] = 0.0f;
    if (r < p.Dk) {
      if (left > 0) s[i] = load_four<VEC, PAST>(S + (int64_t)r * p.Dv + col, left);
      kr[i] = (float)k[r];
      qr[i] = (float)q[r];
    }
  }
  const float a = sigmoid((float)((const T*)p.gate)[(int64_t)b * p.gate_at.b + h]);
  const float w = sigmoid((float)((const T*)p.write)[(int64_t)b * p.write_at.b + h]);
  float v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = e < left ? (float)((const T*)p.v)[(int64_t)b * p.v_at.b + (int64_t)h * p.v_at.head + col + e] : 0.0f;
  float sums[9];
#pragma unroll
  for (int e = 0; e < 9; ++e) sums[e] = 0.0f;
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s[i][e] *= a;
      sums[e] = fmaf(s[i][e], kr[i], sums[e]);
      sums[4 + e] = fmaf(s[i][e], qr[i], sums[4 + e]);
    }
    sums[8] = fmaf(kr[i], qr[i], sums[8]);
  }
#pragma unroll
  for (int e = 0; e < 9; ++e) {                        // lanes 8, 16 and 32 apart hold other rows of the same columns
    sums[e] += lanes_moved<0x128>(sums[e]);            // row_ror 8
    sums[e] = over_rows(sums[e], [](float x, float y) { return x + y; });
  }
  const int wave = threadIdx.x / 64;
  if (threadIdx.x % 64 < 8) {
#pragma unroll
    for (int e = 0; e < 9; ++e) room[wave][lane][e] = sums[e];
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < 9; ++e) sums[e] = (room[0][lane][e] + room[1][lane][e]) + (room[2][lane][e] + room[3][lane][e]);
  float u[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) u[e] = w * (v[e] - sums[e]);
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int r = group + 32 * i;
    if (r < p.Dk && left > 0) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s[i][e] = fmaf(kr[i], u[e], s[i][e]);
      float* to = S + (int64_t)r * p.Dv + col;
      if constexpr (VEC) {
        store_past<PAST>(reinterpret_cast<f32x4_t*>(to), s[i]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e < left) to[e] = s[i][e];
      }
    }
  }
  if (group == 0) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) out[col + e] = (T)fmaf(sums[8], u[e], sums[4 + e]);
  }
}

}  // namespace

hipError_t delta_step_launch(const DeltaStepParams& p, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)p.B * p.v_heads * ((p.Dv + kTile - 1) / kTile)));
  const bool vec = p.Dv % 4 == 0 && ((uintptr_t)p.pool & 15) == 0;
  // states that would not stay in the last-level cache go past it both ways: 128 sequences of 16 heads x 128 x 128, pools in turn, 65.6 -> 57.6 us
  const bool past = vec && streamed((int64_t)p.B * p.v_heads * p.Dk * p.Dv * 4);
  const auto with = [&](auto type) {
    using T = decltype(type);
    if (past) hipLaunchKernelGGL((delta_step_kernel<T, true, true>), grid, dim3(256), 0, s, p);
    else if (vec) hipLaunchKernelGGL((delta_step_kernel<T, true, false>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((delta_step_kernel<T, false, false>), grid, dim3(256), 0, s, p);
  };
  if (p.bf16) with(bf16());
  else with(float());
  return hipGetLastError();
}

}  // namespace tac
