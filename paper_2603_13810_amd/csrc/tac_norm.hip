// Residual addition and root-mean-square norm of rows, its output also in 8 bits, and its backward pass.
//
// Memory-bound: a row is read once into registers, its sum of squares is one reduction, everything written follows from the registers.
// A lane holds 8 consecutive columns per pass (16 bytes of bf16), so 16 lanes hold the 128 columns that share a scale and the largest
// of them is four exchanges inside a wave.
#include "tac_head_common.h"

namespace tac {

namespace {

constexpr int kCols = 8;       // columns of a lane in one pass
constexpr int64_t kMostGroups = 1 << 20;       // workgroups of a launch; more rows than they take at once are further turns

// sum over the LANES lanes that share a row; `room` is LDS for LANES / 64 floats (unused for one wave)
template <int LANES>
__device__ __forceinline__ float row_sum(float v, float* room) {
  v = sum_over_wave(v);
  if constexpr (LANES > 64) {
    const int wave = threadIdx.x >> 6;
    __syncthreads();                       // the row before has been read
    if ((threadIdx.x & 63) == 0) room[wave] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int w = 0; w < LANES / 64; ++w) v += room[w];
  }
  return v;
}

template <typename T, int LANES, int PASSES, bool VEC, bool PAST>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void norm_kernel(const NormParams p) {
  __shared__ float room[LANES / 64];
  const int lane = threadIdx.x % LANES;
  const int64_t pitch = code_pitch(p.cols), spitch = scale_pitch(p.cols);
  // every lane of a workgroup makes the same number of turns: LANES > 64 has one row a turn, LANES = 64 has no barrier inside
  for (int64_t row = (int64_t)blockIdx.x * (blockDim.x / LANES) + threadIdx.x / LANES; row < p.rows;
       row += (int64_t)gridDim.x * (blockDim.x / LANES)) {
    float v[PASSES][kCols], g[PASSES][kCols];
    float squares = 0.0f;
#pragma unroll
    for (int q = 0; q < PASSES; ++q) {                    // asked for with the row, not after its sum
      const int c = (q * LANES + lane) * kCols;
#pragma unroll
      for (int e = 0; e < kCols; ++e) g[q][e] = 1.0f;
      if (p.gain && (p.y || p.codes) && c < p.cols) load_floats<float, kCols, VEC>(p.gain + c, p.cols - c, g[q]);
    }
#pragma unroll
    for (int q = 0; q < PASSES; ++q) {
      const int c = (q * LANES + lane) * kCols;
      const int n = p.cols - c;
      if (n > 0) {
        load_floats<T, kCols, VEC>((const T*)p.x + row * p.x_stride + c, n, v[q]);
        if (p.residual) {
          float r[kCols];
          load_floats<T, kCols, VEC>((const T*)p.residual + row * p.residual_stride + c, n, r);
#pragma unroll
          for (int e = 0; e < kCols; ++e) v[q][e] += r[e];
        }
        if (p.h) store_floats<T, kCols, VEC, PAST>((T*)p.h + row * p.h_stride + c, n, v[q]);
      } else {
#pragma unroll
        for (int e = 0; e < kCols; ++e) v[q][e] = 0.0f;
      }
#pragma unroll
      for (int e = 0; e < kCols; ++e) squares = fmaf(v[q][e], v[q][e], squares);
    }
    const float rstd = 1.0f / sqrtf(row_sum<LANES>(squares, room) / (float)p.cols + p.eps);
    if (p.rstd && lane == 0) p.rstd[row] = rstd;
    if (!p.y && !p.codes) continue;
#pragma unroll
    for (int q = 0; q < PASSES; ++q) {
      const int c = (q * LANES + lane) * kCols;
      const int n = p.cols - c;
      const float by = !VEC || n > 0 ? rstd : 0.0f;        // pad codes are zero where rstd is NaN too; lanes that are half a pad: below
#pragma unroll
      for (int e = 0; e < kCols; ++e) v[q][e] = v[q][e] * by * g[q][e];
      if (p.y && n > 0) store_floats<T, kCols, VEC, PAST>((T*)p.y + row * p.y_stride + c, n, v[q]);
      if (p.codes) {
        if constexpr (!VEC) {
          if (rstd != rstd) {
#pragma unroll
            for (int e = 0; e < kCols; ++e)
              if (e >= n) v[q][e] = 0.0f;
          }
        }
        float amax = 0.0f;
#pragma unroll
        for (int e = 0; e < kCols; ++e) {
          v[q][e] = finite_or_nan(v[q][e]);
          amax = fmaxf(amax, fabsf(v[q][e]));
        }
        const uint32_t byte = scale_byte(max_over_16(amax));
        const float inv = scale_inverse(byte);
        if (c < pitch) store_codes(p.codes + row * pitch + c, v[q], inv);
        if (lane % 16 == 0 && c / kBlock < spitch) p.scales[row * spitch + c / kBlock] = (uint8_t)byte;
      }
    }
  }
}

// A workgroup takes rows blockIdx, blockIdx + gridDim, ...: a lane keeps its columns from row to row, so the sum over rows of
// grad_y n stays in registers and leaves once per workgroup (partial [workgroup][cols]); gain_sum_kernel adds those up in their order.
template <typename T, int LANES, int PASSES, bool VEC, bool PAST>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void norm_backward_kernel(const NormBackwardParams p) {
  constexpr int kRows = LANES < 256 ? 256 / LANES : 1;      // rows that a workgroup has in hand
  __shared__ float room[LANES / 64];
  __shared__ float sums[kRows > 1 ? kRows : 1][kRows > 1 ? PASSES * LANES * kCols : 1];
  const int lane = threadIdx.x % LANES, sub = threadIdx.x / LANES;
  float gain_sum[PASSES][kCols];
#pragma unroll
  for (int q = 0; q < PASSES; ++q)
#pragma unroll
    for (int e = 0; e < kCols; ++e) gain_sum[q][e] = 0.0f;
  // every lane of a workgroup makes the same number of turns: LANES > 64 has one row a turn, LANES = 64 has no barrier inside
  for (int64_t row = (int64_t)blockIdx.x * kRows + sub; row < p.rows; row += (int64_t)gridDim.x * kRows) {
    const float rstd = p.rstd[row];
    float n[PASSES][kCols], w[PASSES][kCols];
    float dot = 0.0f;
#pragma unroll
    for (int q = 0; q < PASSES; ++q) {
      const int c = (q * LANES + lane) * kCols;
      const int left = p.cols - c;
      if (left > 0) {
        load_floats<T, kCols, VEC>((const T*)p.h + row * p.h_stride + c, left, n[q]);
        load_floats<T, kCols, VEC>((const T*)p.grad_y + row * p.grad_y_stride + c, left, w[q]);
        float g[kCols];
        if (p.gain) {
          load_floats<float, kCols, VEC>(p.gain + c, left, g);
        } else {
#pragma unroll
          for (int e = 0; e < kCols; ++e) g[e] = 1.0f;
        }
#pragma unroll
        for (int e = 0; e < kCols; ++e) {
          n[q][e] *= rstd;
          gain_sum[q][e] = fmaf(w[q][e], n[q][e], gain_sum[q][e]);
          w[q][e] *= g[e];
          dot = fmaf(w[q][e], n[q][e], dot);
        }
      }
    }
    const float mean = row_sum<LANES>(dot, room) / (float)p.cols;
#pragma unroll
    for (int q = 0; q < PASSES; ++q) {
      const int c = (q * LANES + lane) * kCols;
      const int left = p.cols - c;
      if (left > 0) {
        float g[kCols];
        if (p.grad_h) {
          load_floats<T, kCols, VEC>((const T*)p.grad_h + row * p.grad_h_stride + c, left, g);
        } else {
#pragma unroll
          for (int e = 0; e < kCols; ++e) g[e] = 0.0f;
        }
#pragma unroll
        for (int e = 0; e < kCols; ++e) g[e] = fmaf(rstd, w[q][e] - n[q][e] * mean, g[e]);
        store_floats<T, kCols, VEC, PAST>((T*)p.grad_x + row * p.grad_x_stride + c, left, g);
      }
    }
  }
  if (!p.grad_gain) return;
  if constexpr (kRows > 1) {
#pragma unroll
    for (int q = 0; q < PASSES; ++q)
#pragma unroll
      for (int e = 0; e < kCols; ++e) sums[sub][(q * LANES + lane) * kCols + e] = gain_sum[q][e];
    __syncthreads();
    for (int c = threadIdx.x; c < p.cols; c += blockDim.x) {
      float t = 0.0f;
#pragma unroll
      for (int r = 0; r < kRows; ++r) t += sums[r][c];
      p.partial[(int64_t)blockIdx.x * p.cols + c] = t;
    }
  } else {
#pragma unroll
    for (int q = 0; q < PASSES; ++q) {
      const int c = (q * LANES + lane) * kCols;
      if (c < p.cols) store_floats<float, kCols, VEC>(p.partial + (int64_t)blockIdx.x * p.cols + c, p.cols - c, gain_sum[q]);
    }
  }
}

// Column sums of partial [groups][cols]: 16 lanes x 4 columns and 16 slices of the groups a workgroup, then the slices in their order.
template <bool VEC>
__global__ __launch_bounds__(256) void gain_sum_kernel(const float* __restrict__ partial, float* __restrict__ grad_gain, int groups, int cols) {
  __shared__ f32x4_t room[16][16];
  const int lane = threadIdx.x % 16, slice = threadIdx.x / 16, c = (blockIdx.x * 16 + lane) * 4;
  f32x4_t t = {0.0f, 0.0f, 0.0f, 0.0f};
  if (c < cols) {
#pragma unroll 8
    for (int g = slice; g < groups; g += 16) {
      float v[4];
      load_floats<float, 4, VEC>(partial + (int64_t)g * cols + c, cols - c, v);
      t += f32x4_t{v[0], v[1], v[2], v[3]};
    }
  }
  room[slice][lane] = t;
  __syncthreads();
  if (slice || c >= cols) return;
#pragma unroll
  for (int s = 1; s < 16; ++s) t += room[s][lane];
  const float v[4] = {t[0], t[1], t[2], t[3]};
  store_floats<float, 4, VEC>(grad_gain + c, cols - c, v);
}

// Lanes and passes of a row of `cols` columns: f(lanes, passes) with both as constants.
template <typename F>
hipError_t by_columns(int cols, F f) {
  using std::integral_constant;
  if (cols <= 512) return f(integral_constant<int, 64>(), integral_constant<int, 1>());
  if (cols <= 1024) return f(integral_constant<int, 64>(), integral_constant<int, 2>());
  if (cols <= 2048) return f(integral_constant<int, 256>(), integral_constant<int, 1>());
  if (cols <= 4096) return f(integral_constant<int, 256>(), integral_constant<int, 2>());
  if (cols <= 8192) return f(integral_constant<int, 1024>(), integral_constant<int, 1>());
  if (cols <= 16384) return f(integral_constant<int, 1024>(), integral_constant<int, 2>());
  return f(integral_constant<int, 1024>(), integral_constant<int, 4>());
}

int rows_in_hand(int cols) { return cols <= 1024 ? 4 : 1; }

// workgroups of the backward pass: one for each compute unit before any takes a second row, then four rows each, so that the partial sums stay a small part of
// the traffic, up to two waves of every SIMD (1000 x 4096 bfloat16 13.2 us, with up to 1024 workgroups from the start 18.9; 4000 x 777 float32 24 and 36)
int64_t backward_groups(int64_t rows, int cols) {
  const int64_t units = (rows + rows_in_hand(cols) - 1) / rows_in_hand(cols);
  return units <= kFittedUnits ? units : units <= 4 * kFittedUnits ? kFittedUnits : units < 16 * kFittedUnits ? units / 4 : 4 * kFittedUnits;
}

template <typename T, bool VEC, bool PAST>
hipError_t norm_typed(const NormParams& p, hipStream_t s) {
  return by_columns(p.cols, [&](auto lanes, auto passes) {
    constexpr int L = decltype(lanes)::value, P = decltype(passes)::value;
    constexpr int threads = L < 256 ? 256 : L, rows = threads / L;
    const int64_t groups = (p.rows + rows - 1) / rows;
    hipLaunchKernelGGL((norm_kernel<T, L, P, VEC, PAST>), dim3((unsigned)(groups < kMostGroups ? groups : kMostGroups)), dim3(threads), 0, s, p);
    return hipGetLastError();
  });
}

template <typename T, bool VEC, bool PAST>
hipError_t norm_backward_typed(const NormBackwardParams& p, hipStream_t s) {
  const int64_t groups = backward_groups(p.rows, p.cols);
  hipError_t e = by_columns(p.cols, [&](auto lanes, auto passes) {
    constexpr int L = decltype(lanes)::value, P = decltype(passes)::value;
    hipLaunchKernelGGL((norm_backward_kernel<T, L, P, VEC, PAST>), dim3((unsigned)groups), dim3(L < 256 ? 256 : L), 0, s, p);
    return hipGetLastError();
  });
  if (e != hipSuccess || !p.grad_gain) return e;
  const dim3 grid((p.cols + 63) / 64);
  if (p.cols % 4 == 0 && rows_aligned(p.grad_gain, 0, 4)) hipLaunchKernelGGL(gain_sum_kernel<true>, grid, dim3(256), 0, s, p.partial, p.grad_gain, (int)groups, p.cols);
  else hipLaunchKernelGGL(gain_sum_kernel<false>, grid, dim3(256), 0, s, p.partial, p.grad_gain, (int)groups, p.cols);
  return hipGetLastError();
}

}  // namespace

hipError_t norm_launch(const NormParams& p, hipStream_t s) {
  const size_t el = p.bf16 ? 2 : 4;
  const bool past = streamed(p.rows * p.cols * (int64_t)el);
  const bool vec = p.cols % kCols == 0 && rows_aligned(p.x, p.x_stride, el) && rows_aligned(p.residual, p.residual_stride, el) &&
                   rows_aligned(p.h, p.h_stride, el) && rows_aligned(p.y, p.y_stride, el) && rows_aligned(p.gain, 0, 4);
  if (p.bf16) return !vec ? norm_typed<bf16, false, false>(p, s) : past ? norm_typed<bf16, true, true>(p, s) : norm_typed<bf16, true, false>(p, s);
  return !vec ? norm_typed<float, false, false>(p, s) : past ? norm_typed<float, true, true>(p, s) : norm_typed<float, true, false>(p, s);
}

size_t norm_backward_workspace(int64_t rows, int cols) { return (size_t)backward_groups(rows, cols) * (size_t)cols * sizeof(float); }

hipError_t norm_backward_launch(const NormBackwardParams& p, hipStream_t s) {
  const size_t el = p.bf16 ? 2 : 4;
  const bool past = streamed(p.rows * p.cols * (int64_t)el);
  const bool vec = p.cols % kCols == 0 && rows_aligned(p.h, p.h_stride, el) && rows_aligned(p.grad_y, p.grad_y_stride, el) &&
                   rows_aligned(p.grad_h, p.grad_h_stride, el) && rows_aligned(p.grad_x, p.grad_x_stride, el) &&
                   rows_aligned(p.gain, 0, 4);
  if (p.bf16) return !vec ? norm_backward_typed<bf16, false, false>(p, s) : past ? norm_backward_typed<bf16, true, true>(p, s) : norm_backward_typed<bf16, true, false>(p, s);
  return !vec ? norm_backward_typed<float, false, false>(p, s) : past ? norm_backward_typed<float, true, true>(p, s) : norm_backward_typed<float, true, false>(p, s);
}

}  // namespace tac
