// What the steps of a chunk do to each other, for every chunk and head at once: with G the running sum of log a,
//   A_tj = b_t e^(G_t - G_j) k_t . k_j  (j < t),   (I + A)^-1,   P_tj = e^(G_t - G_j) q_t . k_j  (j <= t).
//
// G is kept in two numbers: a chunk that fades by e^-100 in all may hold neighbours that hardly fade, and one float32 number would have lost their difference.
// A chunk and head is a workgroup of four waves: products of keys and queries, then the inverse, whose steps follow one another; K and Q come as whole rows through LDS (read as operands they took
// a third longer).  With 128 features bf16 it reads 32 KB and writes 31: 8192 chunks of heads 102 us, 5.1 TB/s of which the caches hold a quarter; 4096 with three parts of both, for the
// gradients, 49; 512 of 32 features fp32 11.6, where loads, gates, products and substitution wait for each other.
// The inverse is formed by blocks of 16: the diagonal ones by substitution, one column a lane, those below from them on the float32 matrix cores.  A product
// of powers of A would be shorter, but its terms grow with the number of like keys where the inverse does not.
#include "tac_delta_chunk.h"

namespace tac {

namespace {

constexpr int kPitch = kChunk + 4;       // float32 rows in LDS

// running sum over the wave's lanes of numbers in two parts
__device__ __forceinline__ void scan_pairs(float& high, float& low, int lane) {
#pragma unroll
  for (int by = 1; by < 64; by *= 2) {
    const float h = __shfl_up(high, by), l = __shfl_up(low, by);
    if (lane >= by) {
      const float s = high + h, back = s - high, e = (high - (s - back)) + (h - back);
      const float rest = low + l + e;
      high = s + rest;
      low = rest - (high - s);
    }
  }
}

// A matrix in LDS, or its transpose, to planes; operands that hold nothing are left out.
template <int PARTS, bool BACK>
__device__ __forceinline__ void store_planes(bf16* to, const float (*from)[kPitch]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int operand = threadIdx.x / 64 + 4 * i, lane = threadIdx.x % 64, tile = operand / 2, step = operand % 2;
    if (BACK ? step < tile / 2 : step > tile / 2) continue;
    const int row = 16 * tile + lane % 16, col = 32 * step + 8 * (lane / 16);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = BACK ? from[col + e][row] : from[row][col + e];
    const Parts<PARTS> a = split<PARTS>(v);
#pragma unroll
    for (int part = 0; part < PARTS; ++part) *reinterpret_cast<bf16x8_t*>(to + part * ChunkRoom::plane + ChunkRoom::operand(tile, step, lane)) = a.p[part];
  }
}

// A matrix in LDS as it is, in the same order.
__device__ __forceinline__ void store_numbers(float* to, const float (*from)[kPitch]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int operand = threadIdx.x / 64 + 4 * i, lane = threadIdx.x % 64, tile = operand / 2, step = operand % 2;
    if (step > tile / 2) continue;
    const float* const row = &from[16 * tile + lane % 16][32 * step + 8 * (lane / 16)];
#pragma unroll
    for (int e = 0; e < 8; e += 4) *reinterpret_cast<f32x4_t*>(to + ChunkRoom::operand(tile, step, lane) + e) = *reinterpret_cast<const f32x4_t*>(row + e);
  }
}

// K and Q as they stand, [2][64][DK + 8] elements, give their place to A and P, and P its to the inverse.
template <typename T, int DK>
struct PrepareRoom {
  static constexpr int pitch = DK + 8, inputs = 2 * kChunk * pitch * (int)sizeof(T), matrices = 2 * kChunk * kPitch * 4;
  static constexpr int bytes = inputs > matrices ? inputs : matrices;
};

template <typename T, int DK, bool BACK, int MODE>
__global__ __launch_bounds__(256) void prepare_kernel(const DeltaParams p) {
  using Room = PrepareRoom<T, DK>;
  constexpr int IN = Kind<T>::in, KS = DK / 32;
  __shared__ __align__(16) uint8_t lds[Room::bytes];
  float(*const A)[kPitch] = (float(*)[kPitch])lds;
  float(*const P)[kPitch] = A + kChunk;
  __shared__ float diagonal[4][16][20];
  __shared__ float high[kChunk], low[kChunk], beta[kChunk];
  const int h = blockIdx.x % p.v_heads, b = blockIdx.x / p.v_heads % p.B;
  const int64_t chunk = blockIdx.x / p.v_heads / p.B, from = chunk * kChunk;
  const int n = steps_of(p, b, from);
  if (n == 0) return;
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, low16 = lane & 15, quad = lane >> 4;
  const int hk = h / (p.v_heads / p.k_heads);
  const T* q = (const T*)p.q + from * p.q_at.t + (int64_t)b * p.q_at.b + (int64_t)hk * p.q_at.head;
  const T* k = (const T*)p.k + from * p.k_at.t + (int64_t)b * p.k_at.b + (int64_t)hk * p.k_at.head;

  // whole rows from memory, on their way while the first wave has the gates; what is behind the last step is zero
  constexpr int pieces = DK / 8, each = kChunk * pieces / 256;
  T* const rows_of_k = (T*)lds;
  T* const rows_of_q = rows_of_k + kChunk * Room::pitch;
  Piece<T, 8> a[each], c[each];
#pragma unroll
  for (int i = 0; i < each; ++i) {
    const int piece = threadIdx.x + 256 * i, row = piece / pieces, col = 8 * (piece % pieces);
    load_piece<MODE>(a[i], k + (int64_t)min(row, n - 1) * p.k_at.t, col, p.Dk);
    load_piece<MODE>(c[i], q + (int64_t)min(row, n - 1) * p.q_at.t, col, p.Dk);
  }
  in_this_order();
  if (wave == 0) {
    float hi = 0.0f, lo = 0.0f, w = 0.0f;
    if (lane < n) {
      const float x = (float)((const T*)p.gate)[(from + lane) * p.gate_at.t + (int64_t)b * p.gate_at.b + h];
      hi = fminf(x, 0.0f) - log1pf(expf(-fabsf(x)));
      if (x < -128.0f) hi = -128.0f;                  // e^-128 is 0 in float32; keeps -inf out of the differences
      if (x != x) hi = x;
      w = sigmoid((float)((const T*)p.write)[(from + lane) * p.write_at.t + (int64_t)b * p.write_at.b + h]);
    }
    scan_pairs(hi, lo, lane);
    high[lane] = hi;
    low[lane] = lo;
    beta[lane] = w;
  }
#pragma unroll
  for (int i = 0; i < each; ++i) {
    const int piece = threadIdx.x + 256 * i, row = piece / pieces, col = 8 * (piece % pieces), left = row < n ? p.Dk - col : 0;
    a[i] = arranged<MODE>(a[i], col, p.Dk);
    c[i] = arranged<MODE>(c[i], col, p.Dk);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (e >= left) {
        a[i].set(e, (T)0.0f);
        c[i].set(e, (T)0.0f);
      }
    }
    store_aligned(rows_of_k + row * Room::pitch + col, a[i]);
    store_aligned(rows_of_q + row * Room::pitch + col, c[i]);
  }
  __syncthreads();
  const ChunkRoom room(p.chunk_room, blockIdx.x, BACK ? ChunkRoom::kBackward : ChunkRoom::kForward);
  f32x4_t kk[4], qk[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) kk[j] = qk[j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const int at = (16 * wave + low16) * Room::pitch + 32 * s + 8 * quad;
    const Parts<IN> own_k = parts_of(load_aligned<T, 8>(rows_of_k + at)), own_q = parts_of(load_aligned<T, 8>(rows_of_q + at));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (j > wave) continue;
      const Parts<IN> other = parts_of(load_aligned<T, 8>(rows_of_k + (16 * j + low16) * Room::pitch + 32 * s + 8 * quad));
      multiply<IN>(kk[j], own_k, other);
      multiply<IN>(qk[j], own_q, other);
    }
  }
  __syncthreads();                                    // K and Q have been read
  // e^(G_t - G_c) of blocks below the diagonal is two factors, to the step in front of the block's rows and from there on, neither above 1
  float since[4], with_beta[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int t = 16 * wave + 4 * quad + r, from_step = max(16 * wave - 1, 0);
    since[r] = fast_exp((high[t] - high[from_step]) + (low[t] - low[from_step]));
    with_beta[r] = since[r] * beta[t];
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (j / 2 > wave / 2) continue;
    const int c = 16 * j + low16;
    if (j < wave) {
      const float until = fast_exp((high[16 * wave - 1] - high[c]) + (low[16 * wave - 1] - low[c]));
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int t = 16 * wave + 4 * quad + r;
        A[t][c] = with_beta[r] * until * kk[j][r];
        P[t][c] = since[r] * until * qk[j][r];
      }
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int t = 16 * wave + 4 * quad + r;
        const float decay = fast_exp((high[t] - high[c]) + (low[t] - low[c]));
        A[t][c] = c < t ? beta[t] * decay * kk[j][r] : 0.0f;
        P[t][c] = c <= t ? decay * qk[j][r] : 0.0f;
      }
    }
  }
  __syncthreads();
  if constexpr (BACK) store_planes<3, true>(room.products, P);
  else store_numbers(room.products32(), P);
  // a diagonal block's inverse: column low16 of x, row by row
  float x[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    x[i] = i == low16 ? 1.0f : 0.0f;
#pragma unroll
    for (int j = 0; j < i; ++j) x[i] = fmaf(-A[16 * wave + i][16 * wave + j], x[j], x[i]);
  }
  f32x4_t block[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) block[i] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  f32x4_t mine;
#pragma unroll
  for (int r = 0; r < 4; ++r) mine[r] = quad == 0 ? x[r] : quad == 1 ? x[4 + r] : quad == 2 ? x[8 + r] : x[12 + r];
#pragma unroll
  for (int r = 0; r < 4; ++r) diagonal[wave][4 * quad + r][low16] = mine[r];
  __syncthreads();
  // block column `wave`, downwards: T_ij = -T_ii sum_k A_ik T_kj.  A result's registers are the next product's second operand as they are (rows 4 quad + r in step r).
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (i == wave) block[i] = mine;
    if (i <= wave) continue;
    f32x4_t sum = {0.0f, 0.0f, 0.0f, 0.0f}, result = sum;
#pragma unroll
    for (int m = 0; m < 3; ++m) {
      if (m < wave || m >= i) continue;
      const f32x4_t a = *reinterpret_cast<const f32x4_t*>(&A[16 * i + low16][16 * m + 4 * quad]);
#pragma unroll
      for (int r = 0; r < 4; ++r) sum = __builtin_amdgcn_mfma_f32_16x16x4f32(a[r], block[m][r], sum, 0, 0, 0);
    }
    const f32x4_t d = *reinterpret_cast<const f32x4_t*>(&diagonal[i][low16][4 * quad]);
#pragma unroll
    for (int r = 0; r < 4; ++r) result = __builtin_amdgcn_mfma_f32_16x16x4f32(-d[r], sum[r], result, 0, 0, 0);
    block[i] = result;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (wave / 2 <= i / 2) {
#pragma unroll
      for (int r = 0; r < 4; ++r) P[16 * i + 4 * quad + r][16 * wave + low16] = block[i][r];
    }
  __syncthreads();
  store_planes<3, BACK>(room.inverse, P);
  if (threadIdx.x < kChunk) {
    const int t = threadIdx.x;
    room.start[t] = fast_exp(high[t] + low[t]);
    room.rest[t] = fast_exp((high[kChunk - 1] - high[t]) + (low[kChunk - 1] - low[t]));
    room.beta[t] = beta[t];
    room.high[t] = high[t];
    room.low[t] = low[t];
  }
}

template <typename T, bool BACK>
hipError_t prepare_typed(const DeltaParams& p, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)p.chunks * p.B * p.v_heads));
  const auto with = [&](auto mode) {
    constexpr int MODE = decltype(mode)::value;
    switch (padded_key(p.Dk)) {
      case 32: hipLaunchKernelGGL((prepare_kernel<T, 32, BACK, MODE>), grid, dim3(256), 0, s, p); break;
      case 64: hipLaunchKernelGGL((prepare_kernel<T, 64, BACK, MODE>), grid, dim3(256), 0, s, p); break;
      default: hipLaunchKernelGGL((prepare_kernel<T, 128, BACK, MODE>), grid, dim3(256), 0, s, p);
    }
    return hipGetLastError();
  };
  return by_mode(piece_mode(p.Dk, 8), with);
}

}  // namespace

hipError_t delta_prepare_launch(const DeltaParams& p, bool back, hipStream_t s) {
  if (p.bf16) return back ? prepare_typed<bf16, true>(p, s) : prepare_typed<bf16, false>(p, s);
  return back ? prepare_typed<float, true>(p, s) : prepare_typed<float, false>(p, s);
}

}  // namespace tac
