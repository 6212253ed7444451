// Shared pieces of the dense operators that read a stack's features (norm, 8-bit matrices, products, recurrence):
// element types, 8-bit codes and their scales, sums over lanes, launch parameters.
#pragma once
#include "tac_internal.h"
#include "tac_product_plan.h"

namespace tac {

typedef __bf16 bf16;
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

// a row of codes is padded to whole blocks, a row of scales to whole dwords
inline __host__ __device__ int64_t code_pitch(int64_t cols) { return (cols + kBlock - 1) / kBlock * kBlock; }
inline __host__ __device__ int64_t scale_pitch(int64_t cols) { return (cols + 4 * kBlock - 1) / (4 * kBlock) * 4; }

__device__ __forceinline__ float bits_float(uint32_t b) { return __builtin_bit_cast(float, b); }
__device__ __forceinline__ uint32_t float_bits(float f) { return __builtin_bit_cast(uint32_t, f); }

// two floats as bf16, to nearest even (v_cvt_pk_bf16_f32)
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, bf16x2{(bf16)a, (bf16)b});
}

// N consecutive elements as floats.  VEC: the address is a multiple of 16 bytes (or of N elements where those are fewer) and all N
// are there; otherwise `n` of them, the rest zero: where all are there as one piece from any address (memory is read from any byte; 2369 rows of 3841 bfloat16,
// residual norm 17.7 us, element by element 52.6), else element by element.
template <typename T, int N, bool VEC>
__device__ __forceinline__ void load_floats(const T* p, int64_t n, float (&v)[N]) {
  if constexpr (VEC) {
    if constexpr (sizeof(T) == 4) {
      static_assert(N % 4 == 0);
#pragma unroll
      for (int q = 0; q < N / 4; ++q) {
        const f32x4_t t = reinterpret_cast<const f32x4_t*>(p)[q];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * q + e] = t[e];
      }
    } else {
      static_assert(N == 8 || N == 4);
      uint32_t w[N / 2];
      if constexpr (N == 8) {
        const u32x4_t t = *reinterpret_cast<const u32x4_t*>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = t[e];
      } else {
        const u32x2_t t = *reinterpret_cast<const u32x2_t*>(p);
        w[0] = t[0];
        w[1] = t[1];
      }
#pragma unroll
      for (int e = 0; e < N / 2; ++e) {
        v[2 * e] = bits_float(w[e] << 16);
        v[2 * e + 1] = bits_float(w[e] & 0xffff0000u);
      }
    }
  } else if (n >= N) {
    T t[N];
    __builtin_memcpy(t, p, sizeof(t));
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = (float)t[e];
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = e < n ? (float)p[e] : 0.0f;
  }
}

// A tensor of `bytes` bytes is written past the caches: what is larger than a good part of the last-level cache (256 MB) is gone from it before it is read again,
// and takes the place of what the launch still reads.  Smaller ones stay there for the next launch.
// Forward and backward of a norm of 16384 x 4096 bfloat16 206 -> 198 us; norm and product of 16384 x 8192 x 4096 562 -> 541.
constexpr int64_t kStreamed = 32 << 20;
inline bool streamed(int64_t bytes) { return bytes >= kStreamed; }

// PAST is a constant: of two branches whose stores differ in this alone the compiler makes one
template <bool PAST, typename V>
__device__ __forceinline__ void store_past(V* p, V v) {
  if constexpr (PAST) __builtin_nontemporal_store(v, p);
  else *p = v;
}

// the same for stores; one rounding, to nearest even, where T is bf16
template <typename T, int N, bool VEC, bool PAST = false>
__device__ __forceinline__ void store_floats(T* p, int64_t n, const float (&v)[N]) {
  if constexpr (VEC) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int q = 0; q < N / 4; ++q)
        store_past<PAST>(reinterpret_cast<f32x4_t*>(p) + q, f32x4_t{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]});
    } else if constexpr (N == 8) {
      store_past<PAST>(reinterpret_cast<u32x4_t*>(p), u32x4_t{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])});
    } else {
      static_assert(N == 4);
      *reinterpret_cast<u32x2_t*>(p) = u32x2_t{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    }
  } else if (n >= N) {
    T t[N];
#pragma unroll
    for (int e = 0; e < N; ++e) t[e] = (T)v[e];
    __builtin_memcpy(p, t, sizeof(t));
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < n) p[e] = (T)v[e];
  }
}

// ---- 8-bit codes -------------------------------------------------------------------------------
// A block's scale is 2^e with the smallest e for which its largest magnitude is at most 448 * 2^e (448: the largest e4m3 number),
// kept as the byte e + 127.  A power of two because dividing by it rounds nothing, so that a code has one rounding in all, and because
// the matrix instruction takes it as it is.
__device__ __forceinline__ uint32_t scale_byte(float amax) {
  const uint32_t b = float_bits(amax);
  const int at = (int)(b >> 23) - 8 + ((b & 0x7fffffu) > 0x600000u);       // 448 = 1.75 * 2^8
  return (uint32_t)max(at, 0);
}
__device__ __forceinline__ float scale_inverse(uint32_t byte) { return bits_float((254u - byte) << 23); }      // 2^-e; bytes up to 247
__device__ __forceinline__ float scale_value(uint32_t byte) { return byte ? bits_float(byte << 23) : bits_float(1u << 22); }

// Infinities and NaN are stored as NaN and leave their block's scale to its finite values (v_max_f32 passes over a NaN).
__device__ __forceinline__ float finite_or_nan(float v) { return fabsf(v) < __builtin_inff() ? v : __builtin_nanf(""); }

// four values, already divided by their scale, as four codes
__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
__device__ __forceinline__ void four_values(uint32_t codes, float (&v)[4]) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
  v[0] = lo[0];
  v[1] = lo[1];
  v[2] = hi[0];
  v[3] = hi[1];
}

// eight codes of a row
__device__ __forceinline__ void store_codes(uint8_t* to, const float (&v)[8], float inv) {
  *reinterpret_cast<u32x2_t*>(to) = u32x2_t{four_codes(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv),
                                            four_codes(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv)};
}

// largest over 16 consecutive lanes, and sum over a wave; every lane gets it.  Within 16 lanes by rotation (one instruction each, no LDS).
template <int BY>
__device__ __forceinline__ float rotated(float v) {
  return bits_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)float_bits(v), 0x120 + BY, 0xf, 0xf, false));      // row_ror
}
__device__ __forceinline__ float max_over_16(float v) {
  v = fmaxf(v, rotated<8>(v));
  v = fmaxf(v, rotated<4>(v));
  v = fmaxf(v, rotated<2>(v));
  return fmaxf(v, rotated<1>(v));
}
// v of this lane and of those 16, 32 and 48 further: two swaps of lane rows bring the two of a pair (v_permlane16_swap, v_permlane32_swap)
template <class F>
__device__ __forceinline__ float over_rows(float v, F f) {
  auto r = __builtin_amdgcn_permlane16_swap(float_bits(v), float_bits(v), false, false);
  v = f(bits_float(r[0]), bits_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(float_bits(v), float_bits(v), false, false);
  return f(bits_float(r[0]), bits_float(r[1]));
}
__device__ __forceinline__ float max_over_rows(float v) { return over_rows(v, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float sum_over_wave(float v) {
  v += rotated<8>(v);
  v += rotated<4>(v);
  v += rotated<2>(v);
  v += rotated<1>(v);
  return over_rows(v, [](float a, float b) { return a + b; });
}

// whether every row of a matrix starts at a multiple of 16 bytes
inline bool rows_aligned(const void* p, int64_t stride, size_t element) {
  return !p || (((uintptr_t)p | (uintptr_t)(stride * (int64_t)element)) & 15u) == 0;
}

// ---- launch parameters ---------------------------------------------------------------------------
struct NormParams {
  const void *x, *residual;
  const float* gain;
  void *h, *y;
  uint8_t *codes, *scales;
  float* rstd;
  int64_t rows, x_stride, residual_stride, h_stride, y_stride;
  int cols, bf16;
  float eps;
};
hipError_t norm_launch(const NormParams& p, hipStream_t s);

struct NormBackwardParams {
  const void* h;
  const float *gain, *rstd;
  const void *grad_y, *grad_h;
  void* grad_x;
  float *grad_gain, *partial;
  int64_t rows, h_stride, grad_y_stride, grad_h_stride, grad_x_stride;
  int cols, bf16;
};
size_t norm_backward_workspace(int64_t rows, int cols);
hipError_t norm_backward_launch(const NormBackwardParams& p, hipStream_t s);

struct QuantizeParams {
  const void* src;
  const uint8_t* src_scales;
  uint8_t *codes, *scales, *codes_t, *scales_t;
  int64_t rows, cols, src_stride;
  int dtype, tiles;
};
hipError_t quantize_launch(const QuantizeParams& p, hipStream_t s);
hipError_t dequantize_launch(const uint8_t* codes, const uint8_t* scales, void* dst, int64_t rows, int64_t cols, int64_t stride,
                             int bf16, hipStream_t s);

struct ProductParams {
  const uint8_t *a, *a_scales, *b, *b_scales;
  const float* bias;
  void* y;
  float* partial;
  int64_t M, N, K, y_stride;
  int bf16;
  int wide_stores;          // rows of y start at multiples of 16 bytes (set by product_launch): stores past the caches, sums of parts by four
};
size_t product_workspace(int64_t M, int64_t N, int64_t K, int bf16);
hipError_t product_launch(const ProductParams& p, hipStream_t s);

struct ScanParams {
  const void *gate, *value;
  const int32_t* lengths;
  const float* h0;
  void* out;
  float *h_last, *states, *workspace;
  int64_t T, in_t, in_b, out_t, out_b;
  int B, D, bf16;
  int apart;                // no output lies on an input (set by scan_launch): steps can be taken a second time
};
struct ScanBackwardParams {
  const void *gate, *value;
  const int32_t* lengths;
  const float* states;
  const void* grad_out;
  const float* grad_h_last;
  void *grad_gate, *grad_value;
  float *grad_h0, *workspace;
  int64_t T, in_t, in_b, out_t, out_b, grad_t, grad_b;
  int B, D, bf16;
  int apart;
};
size_t scan_workspace(int64_t T, int B, int D, int bf16);
hipError_t scan_launch(const ScanParams& p, hipStream_t s);
hipError_t scan_backward_launch(const ScanBackwardParams& p, hipStream_t s);

struct StepParams {
  const void *gate, *value;
  float* pool;
  const int32_t* slots;
  void* out;
  int64_t in_b, out_b, n_slots;
  int B, D, bf16;
};
hipError_t step_launch(const StepParams& p, hipStream_t s);

}  // namespace tac
