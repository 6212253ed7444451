// Matrices to 8 bits with a power of two per 128 values, along their rows, transposed or both, and back.
//
// Memory-bound.  A workgroup takes a tile of 128 x 128: a thread holds 32 or 64 values of it in registers, so its codes of
// a row are one store of the straight matrix, and its codes of a column go through LDS to become rows of 128 codes of the transposed one.  Tiles along a row
// come first: rows further apart than a few kilobytes share too few memory channels.  8192 x 8192 bfloat16, calls in a row: 32 us along the rows, 31 along
// the columns, 46 both, and 30 from 8-bit codes (6.3, 6.5, 5.8 and 4.5 TB/s with what the last-level cache keeps; a copy from memory reaches 4.9).  In tiles,
// both ways, as weights are laid out: 8192 x 4096 float32 32 us.  Back to bfloat16 31 us, to float32, past what the cache keeps, 88 (3.8 TB/s).
#include "tac_head_common.h"
#include "tac_quantize_plan.h"

namespace tac {

namespace {

constexpr int kPitch = 132;        // bytes of a transposed row in LDS: 16 lanes that write 8 columns further each are 66 words apart

// Eight values of a row as they were read.  Columns are gone over twice, for their largest and for their codes, and what was read takes a half or a quarter
// of the registers of its floats, which leaves room for twice as many waves.  DT: 0 float32, 1 bfloat16, 2 8-bit codes.
template <int DT>
struct Eight {
  uint32_t w[DT == 0 ? 8 : DT == 1 ? 4 : 2];
  float scale;               // of the codes
  // number e, a constant; two neighbours are one instruction
  __device__ __forceinline__ float at(int e) const {
    if constexpr (DT == 2) return (e / 2 % 2 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)w[e / 4], true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)w[e / 4], false))[e % 2] * scale;
    else if constexpr (DT == 1) return bits_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
    else return bits_float(w[e]);
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = at(e);
  }
  // from here on the floats (of e's register) are formed again, not kept
  __device__ __forceinline__ void forget(int e) {
    if constexpr (DT != 0) asm volatile("" : "+v"(w[DT == 1 ? e / 2 : e / 4]));
  }
  __device__ __forceinline__ void forget() {
    if constexpr (DT != 0) {
#pragma unroll
      for (uint32_t& x : w) asm volatile("" : "+v"(x));
    }
  }
};

// VEC: rows of whole 16-byte pieces.  ROWS without COLUMNS: the straight matrix with a scale per row (an activation or gradient on its way into a
// product); COLUMNS without ROWS: the transposed one with a scale per column (the operands of a weight gradient); both: either, and tiles.
// A thread has 4 rows x 8 columns where it looks at rows alone (twice as many waves in flight as with 8: 16 x 4096 3.2 us against 4.6) and 8 x 8 for columns,
// where it then writes 8 codes of one at a time into LDS (8192 x 8192 31 us against 35 with 4).
// Largest values are taken with infinities first, since next to no matrix has one; a workgroup that finds one looks again without them.  The conversion
// turns an infinity into NaN by itself.
template <int DT, bool VEC, bool ROWS, bool COLUMNS>
__global__ __launch_bounds__(COLUMNS ? 256 : 512, COLUMNS && !ROWS && DT ? 5 : 1) void quantize_kernel(const QuantizeParams p, int col_tiles) {
  constexpr int RT = COLUMNS ? 8 : 4, CT = 8, kThreads = kBlock * kBlock / (RT * CT);        // rows and columns of a thread
  __shared__ float col_max[COLUMNS ? kThreads / 64 : 1][kBlock];
  __shared__ __align__(16) uint8_t turned[COLUMNS ? kBlock * kPitch : 16];
  const int64_t r0 = (int64_t)(blockIdx.x / col_tiles) * kBlock, c0 = (int64_t)(blockIdx.x % col_tiles) * kBlock;
  const int rt = threadIdx.x / 16, ct = threadIdx.x % 16;
  const int64_t c = c0 + CT * ct;
  // rows and columns of the tile that are there; addresses are formed once and go on by whole rows (64-bit products cost as much as the values' own work)
  const int rows_here = (int)min(p.rows - r0, (int64_t)kBlock), cols_here = (int)min(p.cols - c0, (int64_t)kBlock), left = cols_here - CT * ct;
  Eight<DT> v[RT];
  const int64_t src_row = DT == 2 ? code_pitch(p.cols) : DT == 1 ? 2 * p.src_stride : 4 * p.src_stride;         // bytes from row to row
  const uint8_t* from = (const uint8_t*)p.src + (r0 + RT * rt) * src_row + (DT == 2 ? c : DT == 1 ? 2 * c : 4 * c);
  const uint8_t* from_scales = DT == 2 ? p.src_scales + (r0 + RT * rt) * scale_pitch(p.cols) + c0 / kBlock : nullptr;
#pragma unroll
  for (int i = 0; i < RT; ++i) {
#pragma unroll
    for (uint32_t& w : v[i].w) w = 0;
    v[i].scale = 0.0f;
    if (RT * rt + i < rows_here && left > 0) {
      if constexpr (DT == 2) {
        const u32x2_t w = *reinterpret_cast<const u32x2_t*>(from + i * src_row);
        v[i].w[0] = w[0];
        v[i].w[1] = w[1];
        v[i].scale = scale_value(from_scales[i * scale_pitch(p.cols)]);
      } else if constexpr (DT == 1) {
        const uint16_t* row = reinterpret_cast<const uint16_t*>(from + i * src_row);
        if constexpr (VEC) {
          const u32x4_t w = *reinterpret_cast<const u32x4_t*>(row);
#pragma unroll
          for (int q = 0; q < 4; ++q) v[i].w[q] = w[q];
        } else if (left >= 8) {
          __builtin_memcpy(v[i].w, row, 16);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (e < left) v[i].w[e / 2] |= (uint32_t)row[e] << (e & 1) * 16;
        }
      } else {
        float f[8];
        load_floats<float, CT, VEC>(reinterpret_cast<const float*>(from + i * src_row), left, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i].w[e] = float_bits(f[e]);
      }
    }
  }
  // the largest magnitudes of the lane's columns (of all its values where rows are all that counts)
  float col[CT];
  auto largest = [&](auto finite) {
#pragma unroll
    for (int e = 0; e < CT; ++e) col[e] = 0.0f;
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      float f[CT];
      if constexpr (COLUMNS) v[i].forget();
      v[i].get(f);
#pragma unroll
      for (int e = 0; e < CT; ++e) col[e] = fmaxf(col[e], fabsf(decltype(finite)::value ? finite_or_nan(f[e]) : f[e]));
    }
  };
  largest(std::false_type());
  float most = 0.0f;
#pragma unroll
  for (int e = 0; e < CT; ++e) most = fmaxf(most, col[e]);
  const bool infinite = __any(most == __builtin_inff());
  if (COLUMNS && infinite) largest(std::true_type());
  float tile = 0.0f;
  // the largest of each column over the row groups of a wave, then over the waves
  if (COLUMNS) {
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
      if constexpr (ROWS) tile = fmaxf(tile, col[e]);
    }
    if (ROWS && p.tiles) tile = max_over_16(tile);
  }
  if (ROWS && p.codes) {
    const int64_t pitch = code_pitch(p.cols), spitch = scale_pitch(p.cols);
    const bool last = c0 + kBlock >= p.cols;
    uint8_t *to = p.codes + (r0 + RT * rt) * pitch + c, *to_scales = p.scales + (r0 + RT * rt) * spitch + c0 / kBlock + ct;
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      float f[CT], amax = tile;
      if constexpr (COLUMNS) {
        __builtin_amdgcn_sched_barrier(0);
        v[i].forget();
      }
      v[i].get(f);
      if (!COLUMNS || !p.tiles) {
        amax = 0.0f;
#pragma unroll
        for (int e = 0; e < CT; ++e) amax = fmaxf(amax, fabsf(f[e]));
        if (infinite) {
          amax = 0.0f;
#pragma unroll
          for (int e = 0; e < CT; ++e) amax = fmaxf(amax, fabsf(finite_or_nan(f[e])));
        }
        amax = max_over_16(amax);
      }
      const uint32_t byte = scale_byte(amax);
      if (RT * rt + i < rows_here) {
        store_codes(to + i * pitch, f, scale_inverse(byte));
        // the first lane writes the block's byte, the next ones the row's pad bytes
        if (ct == 0 || (last && c0 / kBlock + ct < spitch)) to_scales[i * spitch] = ct == 0 ? (uint8_t)byte : (uint8_t)0;
      }
    }
  }
  if (COLUMNS && p.codes_t) {
    const int64_t pitch = code_pitch(p.rows), spitch = scale_pitch(p.rows);
    const bool mine = rt == 0 || (r0 + kBlock >= p.rows && r0 / kBlock + rt < spitch);
    uint8_t* to_scales = p.scales_t + c * spitch + r0 / kBlock + rt;
#pragma unroll
    for (int e = 0; e < CT; ++e) {
      const uint32_t byte = scale_byte(ROWS && p.tiles ? tile : col[e]);
      const float inv = scale_inverse(byte);
      uint32_t* to = reinterpret_cast<uint32_t*>(turned + (CT * ct + e) * kPitch + RT * rt);
      if (e % 2 == 0) {                // two columns at a time, not the loads and floats of all
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < RT; ++i) v[i].forget(e);
      }
#pragma unroll
      for (int q = 0; q < RT / 4; ++q)
        to[q] = four_codes(v[4 * q].at(e) * inv, v[4 * q + 1].at(e) * inv, v[4 * q + 2].at(e) * inv, v[4 * q + 3].at(e) * inv);
      if (mine && e < left) to_scales[e * spitch] = rt == 0 ? (uint8_t)byte : (uint8_t)0;
    }
    __syncthreads();
    // rows of the transposed matrix: 8 lanes write one row's 128 codes
    const int row = threadIdx.x / 8, part = threadIdx.x % 8;
    uint8_t* to = p.codes_t + (c0 + row) * pitch + r0 + 16 * part;
#pragma unroll
    for (int i = 0; i < 1024 / kThreads; ++i) {
      constexpr int kRows = kThreads / 8;
      const uint32_t* codes = reinterpret_cast<const uint32_t*>(turned + (i * kRows + row) * kPitch + 16 * part);
      if (i * kRows + row < cols_here) *reinterpret_cast<u32x4_t*>(to + i * kRows * pitch) = u32x4_t{codes[0], codes[1], codes[2], codes[3]};
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
  if (rows_alone(p.codes_t, p.tiles, grid.x)) hipLaunchKernelGGL((quantize_kernel<DT, VEC, true, false>), grid, dim3(512), 0, s, p, ct);
  else if (!p.codes && !p.tiles) hipLaunchKernelGGL((quantize_kernel<DT, VEC, false, true>), grid, dim3(256), 0, s, p, ct);
  else hipLaunchKernelGGL((quantize_kernel<DT, VEC, true, true>), grid, dim3(256), 0, s, p, ct);
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
