// Pieces of the chunked delta rule: numbers as bfloat16 parts, products on the matrix cores, the workspace of a chunk.
#pragma once
#include "tac_delta_common.h"

namespace tac {

typedef bf16 bf16x8_t __attribute__((ext_vector_type(8)));

constexpr int kChunk = TAC_DELTA_CHUNK;
constexpr int kSteps = kChunk + 8;            // pitch of LDS rows of a chunk's steps in bf16: 16 rows' pieces of 16 bytes fall on all banks

// ---- numbers as sums of bfloat16 parts -----------------------------------------------------------
// A float32 number is the sum of three bfloat16 numbers (3 x 8 digits); the product of two such sums without what is below 2^-24 of it is six products, of a
// bfloat16 number with one three.  Two parts have 16 digits.
template <int PARTS>
struct Parts {
  bf16x8_t p[PARTS];
};

template <int PARTS>
__device__ __forceinline__ Parts<PARTS> split(const float (&v)[8]) {
  Parts<PARTS> r;
  float rest[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) rest[e] = v[e];
#pragma unroll
  for (int q = 0; q < PARTS; ++q) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      r.p[q][e] = (bf16)rest[e];
      if (q + 1 < PARTS) rest[e] -= (float)r.p[q][e];
    }
  }
  return r;
}

// four neighbours of a column, one register quad of the matrix cores' result, as parts
template <int PARTS>
__device__ __forceinline__ void split_quad(const f32x4_t& v, u32x2_t (&out)[PARTS]) {
  float rest[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
  for (int q = 0; q < PARTS; ++q) {
    out[q] = u32x2_t{pack_bf16(rest[0], rest[1]), pack_bf16(rest[2], rest[3])};
    if (q + 1 < PARTS) {
      rest[0] -= bits_float(out[q][0] << 16);
      rest[1] -= bits_float(out[q][0] & 0xffff0000u);
      rest[2] -= bits_float(out[q][1] << 16);
      rest[3] -= bits_float(out[q][1] & 0xffff0000u);
    }
  }
}

// acc += a b, 16 x 16 x 32: parts whose orders add up to less than LIMIT, small ones first.
// Operands: lane l has row (column) l & 15 and the eight summed indices from 8 (l >> 4) on; result: column l & 15, rows from 4 (l >> 4) on.
template <int LIMIT, int PA, int PB>
__device__ __forceinline__ void multiply(f32x4_t& acc, const Parts<PA>& a, const Parts<PB>& b) {
#pragma unroll
  for (int order = LIMIT - 1; order >= 0; --order) {
#pragma unroll
    for (int i = 0; i < PA; ++i) {
      const int j = order - i;
      if (j >= 0 && j < PB) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.p[i], b.p[j], acc, 0, 0, 0);
    }
  }
}

// How element types enter: a bfloat16 tensor's numbers are one part, and results that go to it are formed from two; float32 three and three.
template <typename T>
struct Kind;
template <>
struct Kind<bf16> {
  static constexpr int in = 1, out = 2;
};
template <>
struct Kind<float> {
  static constexpr int in = 3, out = 3;
};

// Eight neighbours of a tensor's row as they stand in memory, and their parts.  `n` of them are there (none: zeros).
template <typename T>
struct Eight;
template <>
struct Eight<bf16> {
  u32x4_t v;
  __device__ __forceinline__ void load(const bf16* p, int n) {
    if (n >= 8) {
      __builtin_memcpy(&v, p, 16);
      return;
    }
    v = u32x4_t{0, 0, 0, 0};
    const uint16_t* at = (const uint16_t*)p;
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < n) v[e / 2] |= (uint32_t)at[e] << 16 * (e % 2);
  }
  __device__ __forceinline__ Parts<1> parts() const { return {__builtin_bit_cast(bf16x8_t, v)}; }
};
template <>
struct Eight<float> {
  float v[8];
  __device__ __forceinline__ void load(const float* p, int n) {
    if (n >= 8) {
      __builtin_memcpy(v, p, 32);
      return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? p[e] : 0.0f;
  }
  __device__ __forceinline__ Parts<3> parts() const { return split<3>(v); }
};

// operand from LDS: rows of `pitch` bfloat16, one plane per part
template <int PARTS>
__device__ __forceinline__ Parts<PARTS> from_planes(const bf16* at, int plane) {
  Parts<PARTS> r;
#pragma unroll
  for (int q = 0; q < PARTS; ++q) r.p[q] = *reinterpret_cast<const bf16x8_t*>(at + q * plane);
  return r;
}
template <int PARTS>
__device__ __forceinline__ void quad_to_planes(bf16* at, int plane, const f32x4_t& v) {
  u32x2_t q[PARTS];
  split_quad<PARTS>(v, q);
#pragma unroll
  for (int i = 0; i < PARTS; ++i) *reinterpret_cast<u32x2_t*>(at + i * plane) = q[i];
}

// The transpose of a 16 x 32 operand by products with the identity: exact, every sum has one term.  to[column][step], 4 steps a store.
struct Identity {
  Parts<1> even, odd;
  __device__ Identity(int lane) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int k = 8 * (lane >> 4) + e;
      even.p[0][e] = (bf16)(k == (lane & 15) ? 1.0f : 0.0f);
      odd.p[0][e] = (bf16)(k - 16 == (lane & 15) ? 1.0f : 0.0f);
    }
  }
};
// `to`: LDS planes [PARTS][columns][kSteps]; the operand holds steps `row`.. (16 of them) and columns col.. (32)
template <int PARTS>
__device__ __forceinline__ void transpose_to(bf16* to, int plane, const Parts<PARTS>& a, int row, int col, const Identity& id, int lane) {
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    bf16* at = to + (col + 16 * half + (lane & 15)) * kSteps + row + 4 * (lane >> 4);
#pragma unroll
    for (int q = 0; q < PARTS; ++q) {
      const f32x4_t t = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.p[q], half ? id.odd.p[0] : id.even.p[0], f32x4_t{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0);
      *reinterpret_cast<u32x2_t*>(at + q * plane) = u32x2_t{pack_bf16(t[0], t[1]), pack_bf16(t[2], t[3])};
    }
  }
}

__device__ __forceinline__ float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896340736f); }

// ---- launch parameters ---------------------------------------------------------------------------
struct DeltaParams {
  const void *q, *k, *v, *gate, *write;
  const int32_t* lengths;
  const float* h0;
  void* out;
  float *h_last, *states, *updates;
  // backward
  const void* grad_out;
  const float* grad_h_last;
  void *grad_q, *grad_k, *grad_v, *grad_gate, *grad_write;
  float* grad_h0;
  tac_delta_strides_t q_at, k_at, v_at, gate_at, write_at, out_at, grad_q_at, grad_k_at, grad_v_at, grad_gate_at, grad_write_at;
  int64_t T;
  int B, k_heads, v_heads, Dk, Dv, bf16, chunks;
  // workspace
  uint8_t* chunk_room;               // [chunks][B][v_heads], ChunkRoom each
  float *back_states, *r, *shared;   // backward: gradients of the states behind every chunk, r as updates are laid out, sums over heads that share a key
};

__device__ __forceinline__ int steps_of(const DeltaParams& p, int b, int64_t from) {      // steps of the chunk that begins at `from`
  const int64_t n = p.lengths ? min((int64_t)max(p.lengths[b], 0), p.T) : p.T;
  return (int)max((int64_t)0, min((int64_t)kChunk, n - from));
}

// What prepare_kernel leaves of a chunk and head: planes of the inverse (three parts) and of the queries' products, then factors of the steps.
// Backwards both matrices stand transposed, so that a row's neighbours are what is summed over.
struct ChunkRoom {
  static constexpr int plane = kChunk * kChunk;
  static constexpr int64_t bytes(int p_parts) { return (int64_t)(3 + p_parts) * plane * 2 + 5 * kChunk * 4; }
  const bf16 *inverse, *products;
  const float *start, *rest, *beta, *high, *low;      // e^G, e^(G_end - G), b, and G in two numbers
  __device__ ChunkRoom(const uint8_t* base, int64_t index, int p_parts) {
    const uint8_t* at = base + index * bytes(p_parts);
    inverse = (const bf16*)at;
    products = inverse + 3 * plane;
    start = (const float*)(products + p_parts * plane);
    rest = start + kChunk;
    beta = rest + kChunk;
    high = beta + kChunk;
    low = high + kChunk;
  }
};

// bytes of LDS, by the features of a key (padded to 32, 64 or 128) and the kind of elements
inline int padded_key(int Dk) { return Dk <= 32 ? 32 : Dk <= 64 ? 64 : 128; }

hipError_t delta_prepare_launch(const DeltaParams& p, bool back, hipStream_t s);
size_t delta_workspace(const DeltaParams& p);
size_t delta_backward_workspace(const DeltaParams& p);
hipError_t delta_scan_launch(const DeltaParams& p, uint8_t* workspace, hipStream_t s);
hipError_t delta_backward_launch(const DeltaParams& p, uint8_t* workspace, hipStream_t s);

}  // namespace tac
