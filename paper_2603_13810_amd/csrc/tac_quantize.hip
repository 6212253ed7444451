// Matrices to 8 bits with a power of two per 128 values, along their rows, transposed or both, and back.
//
// Memory-bound.  A workgroup takes a tile of 128 x 128: a thread holds 32 or 64 values of it in registers, so its codes of
// a row are one store of the straight matrix, and its codes of a column go through LDS to become rows of 128 codes of the transposed one.  Tiles along a row
// come first: rows further apart than a few kilobytes share too few memory channels.  8192 x 8192 bfloat16 35 us along the rows and 38 along
// the columns (5.8 and 5.3 TB/s; a copy reaches 5.1).
#include "tac_head_common.h"

namespace tac {

namespace {

constexpr int kPitch = 132;        // bytes of a transposed row in LDS: 16 lanes that write 8 columns further each are 66 words apart

// DT: 0 float32, 1 bfloat16, 2 8-bit codes.  VEC: rows of whole 16-byte pieces.  ROWS: the straight matrix alone, with a scale per row (an activation or
// gradient on its way into a product), which needs nothing of the columns.
// A thread has 4 rows x 8 columns where it looks at rows alone (twice as many waves in flight as with 8: 16 x 4096 3.2 us against 4.6, 8192 x 8192 35 against 37)
// and 8 x 8 for columns, where it then writes 8 codes of one at a time into LDS (8192 x 8192 38 us against 44).
template <int DT, bool VEC, bool ROWS>
__global__ __launch_bounds__(ROWS ? 512 : 256) void quantize_kernel(const QuantizeParams p, int col_tiles) {
  constexpr int RT = ROWS ? 4 : 8, CT = 8, kThreads = kBlock * kBlock / (RT * CT);        // rows and columns of a thread
  __shared__ float col_max[ROWS ? 1 : kThreads / 64][kBlock];
  __shared__ __align__(16) uint8_t turned[ROWS ? 16 : kBlock * kPitch];
  const int64_t r0 = (int64_t)(blockIdx.x / col_tiles) * kBlock, c0 = (int64_t)(blockIdx.x % col_tiles) * kBlock;
  const int rt = threadIdx.x / 16, ct = threadIdx.x % 16;
  const int64_t c = c0 + CT * ct;
  float v[RT][CT];
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const int64_t r = r0 + RT * rt + i;
    if (r < p.rows && c < p.cols) {
      if constexpr (DT == 2) {
        const u32x2_t w = *reinterpret_cast<const u32x2_t*>((const uint8_t*)p.src + r * code_pitch(p.cols) + c);
        const float scale = scale_value(p.src_scales[r * scale_pitch(p.cols) + c / kBlock]);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          float four[4];
          four_values(w[q], four);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[i][4 * q + e] = four[e] * scale;
        }
      } else if constexpr (DT == 1) {
        load_floats<bf16, CT, VEC>((const bf16*)p.src + r * p.src_stride + c, p.cols - c, v[i]);
      } else {
        load_floats<float, CT, VEC>((const float*)p.src + r * p.src_stride + c, p.cols - c, v[i]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < CT; ++e) v[i][e] = 0.0f;
    }
  }
  float col[CT] = {};
  float tile = 0.0f;
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int e = 0; e < CT; ++e) {
      v[i][e] = finite_or_nan(v[i][e]);
      if constexpr (!ROWS) col[e] = fmaxf(col[e], fabsf(v[i][e]));
    }
  // the largest of each column over the row groups of a wave, then over the waves
  if (!ROWS && (p.codes_t || p.tiles)) {
#pragma unroll
    for (int e = 0; e < CT; ++e) {
      col[e] = max_over_rows(col[e]);
      if ((threadIdx.x & 63) < 16) col_max[threadIdx.x >> 6][CT * ct + e] = col[e];
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < CT; ++e) {
      const int at = CT * ct + e;
#pragma unroll
      for (int w = 0; w < kThreads / 64; ++w) col[e] = fmaxf(col[e], col_max[w][at]);
      tile = fmaxf(tile, col[e]);
    }
    if (p.tiles) tile = max_over_16(tile);
  }
  if (ROWS || p.codes) {
    const int64_t pitch = code_pitch(p.cols), spitch = scale_pitch(p.cols);
    const bool last = c0 + kBlock >= p.cols;
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int64_t r = r0 + RT * rt + i;
      float amax = tile;
      if (ROWS || !p.tiles) {
        amax = 0.0f;
#pragma unroll
        for (int e = 0; e < CT; ++e) amax = fmaxf(amax, fabsf(v[i][e]));
        amax = max_over_16(amax);
      }
      const uint32_t byte = scale_byte(amax);
      if (r < p.rows) {
        store_codes(p.codes + r * pitch + c, v[i], scale_inverse(byte));
        const int64_t at = c0 / kBlock + ct;               // the first lane writes the block's byte, the next ones the row's pad bytes
        if (ct == 0 || (last && at < spitch)) p.scales[r * spitch + at] = ct == 0 ? (uint8_t)byte : (uint8_t)0;
      }
    }
  }
  if (!ROWS && p.codes_t) {
    const int64_t pitch = code_pitch(p.rows), spitch = scale_pitch(p.rows);
#pragma unroll
    for (int e = 0; e < CT; ++e) {
      const uint32_t byte = scale_byte(p.tiles ? tile : col[e]);
      const float inv = scale_inverse(byte);
      uint32_t* to = reinterpret_cast<uint32_t*>(turned + (CT * ct + e) * kPitch + RT * rt);
#pragma unroll
      for (int q = 0; q < RT / 4; ++q)
        to[q] = four_codes(v[4 * q][e] * inv, v[4 * q + 1][e] * inv, v[4 * q + 2][e] * inv, v[4 * q + 3][e] * inv);
      const int64_t at = r0 / kBlock + rt;
      const bool last = r0 + kBlock >= p.rows;
      if (c + e < p.cols && (rt == 0 || (last && at < spitch))) p.scales_t[(c + e) * spitch + at] = rt == 0 ? (uint8_t)byte : (uint8_t)0;
    }
    __syncthreads();
    // rows of the transposed matrix: 8 lanes write one row's 128 codes
#pragma unroll
    for (int i = 0; i < 1024 / kThreads; ++i) {
      const int row = i * (kThreads / 8) + threadIdx.x / 8, part = threadIdx.x % 8;
      const uint32_t* from = reinterpret_cast<const uint32_t*>(turned + row * kPitch + 16 * part);
      if (c0 + row < p.cols)
        *reinterpret_cast<u32x4_t*>(p.codes_t + (c0 + row) * pitch + r0 + 16 * part) = u32x4_t{from[0], from[1], from[2], from[3]};
    }
  }
}

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                         T* __restrict__ dst, int64_t rows, int64_t cols, int64_t stride) {
  const int64_t pitch = code_pitch(cols), spitch = scale_pitch(cols), pieces = (cols + 7) / 8;
  const int64_t step = (int64_t)gridDim.x * blockDim.x;
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < rows * pieces; i += step) {
    const int64_t r = i / pieces, c = (i - r * pieces) * 8;
    const u32x2_t w = *reinterpret_cast<const u32x2_t*>(codes + r * pitch + c);
    const float scale = scale_value(scales[r * spitch + c / kBlock]);
    float lo[4], hi[4], v[8];
    four_values(w[0], lo);
    four_values(w[1], hi);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = lo[e] * scale;
      v[4 + e] = hi[e] * scale;
    }
    store_floats<T, 8, VEC>(dst + r * stride + c, cols - c, v);
  }
}

}  // namespace

template <int DT, bool VEC>
static void quantize_typed(const QuantizeParams& p, dim3 grid, int ct, hipStream_t s) {
  if (!p.codes_t && !p.tiles) hipLaunchKernelGGL((quantize_kernel<DT, VEC, true>), grid, dim3(512), 0, s, p, ct);
  else hipLaunchKernelGGL((quantize_kernel<DT, VEC, false>), grid, dim3(256), 0, s, p, ct);
}

hipError_t quantize_launch(const QuantizeParams& p, hipStream_t s) {
  const int64_t rt = (p.rows + kBlock - 1) / kBlock, ct = (p.cols + kBlock - 1) / kBlock;
  const dim3 grid((unsigned)(rt * ct));
  const bool vec = p.dtype != TAC_SCALED && p.cols % 8 == 0 && rows_aligned(p.src, p.src_stride, p.dtype == TAC_BF16 ? 2 : 4);
  if (p.dtype == TAC_SCALED) quantize_typed<2, false>(p, grid, (int)ct, s);
  else if (p.dtype == TAC_BF16 && vec) quantize_typed<1, true>(p, grid, (int)ct, s);
  else if (p.dtype == TAC_BF16) quantize_typed<1, false>(p, grid, (int)ct, s);
  else if (vec) quantize_typed<0, true>(p, grid, (int)ct, s);
  else quantize_typed<0, false>(p, grid, (int)ct, s);
  return hipGetLastError();
}

hipError_t dequantize_launch(const uint8_t* codes, const uint8_t* scales, void* dst, int64_t rows, int64_t cols, int64_t stride,
                             int bf, hipStream_t s) {
  const int64_t work = (rows * ((cols + 7) / 8) + 255) / 256;
  const dim3 grid((unsigned)(work < 256 * 32 ? work : 256 * 32));
  const bool vec = cols % 8 == 0 && rows_aligned(dst, stride, bf ? 2 : 4);
  if (bf && vec) hipLaunchKernelGGL((dequantize_kernel<bf16, true>), grid, dim3(256), 0, s, codes, scales, (bf16*)dst, rows, cols, stride);
  else if (bf) hipLaunchKernelGGL((dequantize_kernel<bf16, false>), grid, dim3(256), 0, s, codes, scales, (bf16*)dst, rows, cols, stride);
  else if (vec) hipLaunchKernelGGL((dequantize_kernel<float, true>), grid, dim3(256), 0, s, codes, scales, (float*)dst, rows, cols, stride);
  else hipLaunchKernelGGL((dequantize_kernel<float, false>), grid, dim3(256), 0, s, codes, scales, (float*)dst, rows, cols, stride);
  return hipGetLastError();
}

}  // namespace tac
