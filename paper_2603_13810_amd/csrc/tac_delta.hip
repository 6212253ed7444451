// Gated delta rule over sequences: the states from chunk to chunk and the outputs.
//
// Columns of a state do not touch each other: a workgroup takes 16 or 32 of a head's and goes through the chunks, four waves side by side.  Of a chunk, with S its
// first state and what prepare_kernel left,
//   U = (I + A)^-1 b (V - e^G K S),   O = e^G Q S + P U,   S <- e^G_end S + K^T (e^(G_end - G) U).
// S, the right-hand sides and U go from one product's result to the next one's operand through LDS as bfloat16 parts; S itself stays in registers in float32.
#include "tac_delta_chunk.h"

namespace tac {

namespace {

// LDS of scan_kernel in bfloat16 numbers: S [3][columns][DK + 8], right-hand sides [3][columns][kSteps], U faded [3], U [OUT], K transposed [IN][DK][kSteps]
template <typename T, int DK, int NT>
struct ScanRoom {
  static constexpr int columns = 16 * NT, key = DK + 8;
  static constexpr int s_plane = columns * key, u_plane = columns * kSteps, k_plane = DK * kSteps;
  static constexpr int s = 0, rhs = s + 3 * s_plane, faded = rhs + 3 * u_plane, u = faded + 3 * u_plane, k = u + Kind<T>::out * u_plane;
  static constexpr int size = k + Kind<T>::in * k_plane;
};

template <typename T, int DK, int NT>
__global__ __launch_bounds__(256) void scan_kernel(const DeltaParams p, int tiles) {
  using Room = ScanRoom<T, DK, NT>;
  constexpr int IN = Kind<T>::in, OUT = Kind<T>::out, KS = DK / 32, MT = DK / 16, OWN = MT > 4 ? MT / 4 : 1;
  extern __shared__ __align__(16) uint8_t lds[];
  bf16* const L = (bf16*)lds;
  const int index = blockIdx.x, tile = index % tiles, h = index / tiles % p.v_heads, b = index / tiles / p.v_heads;
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, low16 = lane & 15, quad = lane >> 4;
  const int hk = h / (p.v_heads / p.k_heads), first = tile * Room::columns;
  const int64_t length = p.lengths ? min((int64_t)max(p.lengths[b], 0), p.T) : p.T;
  const T* const q = (const T*)p.q + (int64_t)b * p.q_at.b + (int64_t)hk * p.q_at.head;
  const T* const k = (const T*)p.k + (int64_t)b * p.k_at.b + (int64_t)hk * p.k_at.head;
  const T* const v = (const T*)p.v + (int64_t)b * p.v_at.b + (int64_t)h * p.v_at.head;
  T* const out = (T*)p.out + (int64_t)b * p.out_at.b + (int64_t)h * p.out_at.head;
  const int64_t head = (int64_t)b * p.v_heads + h, state = (int64_t)p.Dk * p.Dv;
  const Identity id(lane);
  const bool owner = MT >= 4 || wave < MT;             // waves that have rows of S
  int col[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) col[t] = first + 16 * t + low16;

  f32x4_t S[OWN][NT];
#pragma unroll
  for (int m = 0; m < OWN; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * (wave * OWN + m) + 4 * quad + r;
        S[m][t][r] = p.h0 && row < p.Dk && col[t] < p.Dv ? p.h0[head * state + (int64_t)row * p.Dv + col[t]] : 0.0f;
      }

  const int chunks = (int)((length + kChunk - 1) / kChunk);
  for (int c = 0; c < chunks; ++c) {
    const int64_t from = (int64_t)c * kChunk;
    const int n = (int)min((int64_t)kChunk, length - from);
    const int64_t index_of_chunk = (int64_t)c * p.B * p.v_heads + head;
    const ChunkRoom room(p.chunk_room, index_of_chunk, OUT);
    // operands with the chunk's steps as rows
    Parts<IN> key[KS], query[KS];
    {
      const int row = 16 * wave + low16;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int at = 32 * s + 8 * quad, left = row < n ? p.Dk - at : 0;
        Eight<T> e;
        e.load(k + (from + row) * p.k_at.t + at, left);
        key[s] = e.parts();
        e.load(q + (from + row) * p.q_at.t + at, left);
        query[s] = e.parts();
      }
    }
    f32x4_t value[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * wave + 4 * quad + r;
        value[t][r] = row < n && col[t] < p.Dv ? (float)v[(from + row) * p.v_at.t + col[t]] : 0.0f;
      }
    const f32x4_t start = *reinterpret_cast<const f32x4_t*>(room.start + 16 * wave + 4 * quad);
    const f32x4_t rest = *reinterpret_cast<const f32x4_t*>(room.rest + 16 * wave + 4 * quad);
    const f32x4_t beta = *reinterpret_cast<const f32x4_t*>(room.beta + 16 * wave + 4 * quad);
    const float whole = room.start[kChunk - 1];

    if (owner) {
#pragma unroll
      for (int m = 0; m < OWN; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const int row = 16 * (wave * OWN + m) + 4 * quad;
          quad_to_planes<3>(L + Room::s + (16 * t + low16) * Room::key + row, Room::s_plane, S[m][t]);
          if (p.states && col[t] < p.Dv) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (row + r < p.Dk) p.states[index_of_chunk * state + (int64_t)(row + r) * p.Dv + col[t]] = S[m][t][r];
          }
        }
    }
    __syncthreads();

    f32x4_t ks[NT], qs[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      ks[t] = qs[t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const Parts<3> op = from_planes<3>(L + Room::s + (16 * t + low16) * Room::key + 32 * s + 8 * quad, Room::s_plane);
        multiply<3>(ks[t], key[s], op);
        multiply<OUT>(qs[t], query[s], op);
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      f32x4_t rhs;
#pragma unroll
      for (int r = 0; r < 4; ++r) rhs[r] = beta[r] * fmaf(-start[r], ks[t][r], value[t][r]);
      quad_to_planes<3>(L + Room::rhs + (16 * t + low16) * kSteps + 16 * wave + 4 * quad, Room::u_plane, rhs);
    }
#pragma unroll
    for (int s = 0; s < KS; ++s) transpose_to<IN>(L + Room::k, Room::k_plane, key[s], 16 * wave, 32 * s, id, lane);
    __syncthreads();

    f32x4_t u[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) u[t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (32 * s > 16 * wave + 15) continue;           // nothing above the diagonal
      const Parts<3> a = from_planes<3>(room.inverse + (16 * wave + low16) * kChunk + 32 * s + 8 * quad, ChunkRoom::plane);
#pragma unroll
      for (int t = 0; t < NT; ++t) multiply<3>(u[t], a, from_planes<3>(L + Room::rhs + (16 * t + low16) * kSteps + 32 * s + 8 * quad, Room::u_plane));
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int at = (16 * t + low16) * kSteps + 16 * wave + 4 * quad;
      f32x4_t faded;
#pragma unroll
      for (int r = 0; r < 4; ++r) faded[r] = rest[r] * u[t][r];
      quad_to_planes<3>(L + Room::faded + at, Room::u_plane, faded);
      quad_to_planes<OUT>(L + Room::u + at, Room::u_plane, u[t]);
      if (p.updates && col[t] < p.Dv) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = 16 * wave + 4 * quad + r;
          if (from + row < p.T) p.updates[((from + row) * p.B * p.v_heads + head) * p.Dv + col[t]] = u[t][r];
        }
      }
    }
    __syncthreads();

    if (owner) {
#pragma unroll
      for (int m = 0; m < OWN; ++m) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) S[m][t][r] *= whole;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const Parts<IN> a = from_planes<IN>(L + Room::k + (16 * (wave * OWN + m) + low16) * kSteps + 32 * s + 8 * quad, Room::k_plane);
#pragma unroll
          for (int t = 0; t < NT; ++t)
            multiply<3>(S[m][t], a, from_planes<3>(L + Room::faded + (16 * t + low16) * kSteps + 32 * s + 8 * quad, Room::u_plane));
        }
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) qs[t][r] *= start[r];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (32 * s > 16 * wave + 15) continue;
      const Parts<OUT> a = from_planes<OUT>(room.products + (16 * wave + low16) * kChunk + 32 * s + 8 * quad, ChunkRoom::plane);
#pragma unroll
      for (int t = 0; t < NT; ++t) multiply<OUT>(qs[t], a, from_planes<OUT>(L + Room::u + (16 * t + low16) * kSteps + 32 * s + 8 * quad, Room::u_plane));
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if (col[t] >= p.Dv) continue;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * wave + 4 * quad + r;
        if (from + row < p.T) out[(from + row) * p.out_at.t + col[t]] = (T)(row < n ? qs[t][r] : 0.0f);
      }
    }
  }
  // behind the last chunk's steps
  for (int64_t t = (int64_t)chunks * kChunk + threadIdx.x / Room::columns; t < p.T; t += 256 / Room::columns) {
    const int at = first + threadIdx.x % Room::columns;
    if (at < p.Dv) out[t * p.out_at.t + at] = (T)0.0f;
  }
  if (!p.h_last || !owner) return;
#pragma unroll
  for (int m = 0; m < OWN; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * (wave * OWN + m) + 4 * quad + r;
        if (row < p.Dk && col[t] < p.Dv) p.h_last[head * state + (int64_t)row * p.Dv + col[t]] = S[m][t][r];
      }
}

template <typename T, int DK, int NT>
hipError_t scan_shaped(const DeltaParams& p, hipStream_t s) {
  const int tiles = (p.Dv + 16 * NT - 1) / (16 * NT);
  constexpr int bytes = ScanRoom<T, DK, NT>::size * 2;
  if (bytes > 64 << 10) {
    const hipError_t e = hipFuncSetAttribute((const void*)scan_kernel<T, DK, NT>, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((scan_kernel<T, DK, NT>), dim3((unsigned)((int64_t)p.B * p.v_heads * tiles)), dim3(256), bytes, s, p, tiles);
  return hipGetLastError();
}

template <typename T, int NT>
hipError_t scan_typed(const DeltaParams& p, hipStream_t s) {
  switch (padded_key(p.Dk)) {
    case 32: return scan_shaped<T, 32, NT>(p, s);
    case 64: return scan_shaped<T, 64, NT>(p, s);
    default: return scan_shaped<T, 128, NT>(p, s);
  }
}

}  // namespace

size_t delta_workspace(const DeltaParams& p) {
  return (size_t)p.chunks * p.B * p.v_heads * (size_t)ChunkRoom::bytes(p.bf16 ? Kind<bf16>::out : Kind<float>::out);
}

hipError_t delta_scan_launch(const DeltaParams& given, uint8_t* workspace, hipStream_t s) {
  DeltaParams p = given;
  p.chunk_room = workspace;
  const hipError_t e = delta_prepare_launch(p, false, s);
  if (e != hipSuccess) return e;
  const bool narrow = delta_narrow(p.B, p.v_heads, p.Dv);
  if (p.bf16) return narrow ? scan_typed<bf16, 1>(p, s) : scan_typed<bf16, 2>(p, s);
  return narrow ? scan_typed<float, 1>(p, s) : scan_typed<float, 2>(p, s);
}

}  // namespace tac
