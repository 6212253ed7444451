// Gated delta rule over sequences: the states from chunk to chunk and the outputs.
//
// Columns of a state do not touch each other: a workgroup takes 16 or 32 of a head's and goes through the chunks.  Of a chunk, with S its
// first state and what prepare_kernel left,
//   U = (I + A)^-1 b (V - e^G K S),   O = e^G Q S + P U,   S <- e^G_end S + K^T (e^(G_end - G) U).
// S, the right-hand sides and U go from one product's result to the next one's operand through LDS as bfloat16 parts; S itself stays in registers in float32.
//
// Bound by the chain: a chunk waits for the state that the one before leaves, and what is in between (parts of S, K S over LDS, the right-hand sides, the inverse, U over LDS, K^T U) is some 4500
// cycles, of which the matrix cores work 300.  32768 steps, 16 heads of 128 x 128 bf16: 953 us for 512 chunks, 1.9 us each, on 128 workgroups (865 where the outputs' products had 16
// digits); 8 sequences of 2048 steps with what training keeps: 188 us.  What shortened it: outputs on waves of their own, S as an operand from registers, loads a chunk ahead, whole lines, a head's tiles on one die (3020 us at first).
#include "tac_delta_chunk.h"

namespace tac {

namespace {

// Eight waves: four take the states from chunk to chunk, and four form the outputs from what those leave in LDS.

// LDS of scan_kernel.  float32: the waves' shares of K S; then in bfloat16 numbers, each in three parts, S [columns][DK + 8] and U [columns][kSteps] for the outputs, right-hand sides
// [columns][kSteps], U faded, K transposed [IN][DK][kSteps]; and K as it stands, [64][DK + 8] elements.
// With 16 columns and bfloat16 keys of 128 features that is half of a compute unit's 160 KB, so that two workgroups are there at once (6 sequences of 2048, 16 heads of 128 x 128: 203 us,
// one at a time 237): a wave keeps the share that it needs itself, and the shares' rows are not padded, their quads change places instead.
template <typename T, int DK, int NT>
struct ScanRoom {
  static constexpr int columns = 16 * NT, key = DK + 8;
  static constexpr bool tight = NT == 1;      // with 32 columns one workgroup fits, and the selection costs more (16 sequences of 2048: 484 us, 514)
  static constexpr int s_plane = columns * key, u_plane = columns * kSteps, k_plane = DK * kSteps;
  static constexpr int s = (tight ? 3 * columns * kChunk : 4 * columns * kSums) * 2, u = s + 3 * s_plane, rhs = u + 3 * u_plane, faded = rhs + 3 * u_plane, k = faded + 3 * u_plane;
  static constexpr int rows = k + Kind<T>::in * k_plane;
  static constexpr int bytes = 2 * rows + kChunk * key * (int)sizeof(T);
  // where wave `of`'s share for the steps from `step` on (four of them, wave `to`'s) of a column stands
  static __device__ __forceinline__ int share(int of, int to, int t, int low16, int step) {
    if constexpr (tight) return ((of < to ? of : of - 1) * 16 + low16) * kChunk + (step ^ (4 * low16));
    else return (of * columns + 16 * t + low16) * kSums + step;
  }
};

// a row of the inverse; nothing stands above the diagonal
template <typename T, int NT>
__device__ __forceinline__ void load_rows_of(Parts<3> (&m)[2], const bf16* from, const ScanPlace<T, NT>& at) {
  m[0] = from_planes<3>(from + ChunkRoom::operand(at.wave, 0, at.lane), ChunkRoom::plane);
  m[1] = from_planes<3>(from + ChunkRoom::operand(at.wave, at.wave >= 2 ? 1 : 0, at.lane), ChunkRoom::plane);
}

// Loads of the next chunk are asked for as soon as this one's have been used, a chunk before they are waited for; memory operations come in the same number whatever
// the sizes (behind a branch the compiler waits for all of them), so what is not to be stored goes to a place of the workspace that nobody reads.

// The chain that everything waits for: the states from chunk to chunk.  A wave has 32 rows of S (16 where Dk is at most 64).  As the first product's operand they stay in the wave's
// registers: the summed index may come in any order, so the result's layout is taken as it is, and K is read to match; the waves' shares of K S are
// added up through LDS, which moves a third of what S in parts would.  Of the chunk's K the wave reads every step, from LDS: a compute unit takes 64 bytes a cycle from the
// caches, and every load that is not asked for twice counts.
template <typename T, int DK, int NT, int MODE, bool KEEP>
__device__ __forceinline__ void scan_states(const DeltaParams& p, const ScanPlace<T, NT>& at, uint8_t* lds) {
  using Room = ScanRoom<T, DK, NT>;
  constexpr int IN = Kind<T>::in, MT = DK / 16, OWN = MT > 4 ? 2 : 1;
  float* const sums = (float*)lds;
  bf16* const L = (bf16*)lds;
  const int low16 = at.low16, quad = at.quad, rows = at.rows;
  const bool owner = MT >= 4 || at.wave < MT;             // waves that have rows of S; the others' are zeros behind Dk
  int state_row[OWN];
#pragma unroll
  for (int m = 0; m < OWN; ++m) state_row[m] = 16 * (at.wave * OWN + m) + 4 * quad;
  f32x4_t S[OWN][NT];
#pragma unroll
  for (int m = 0; m < OWN; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        S[m][t][r] = p.h0 && state_row[m] + r < p.Dk && at.col[t] < p.Dv ? p.h0[at.head * at.state + (int64_t)(state_row[m] + r) * p.Dv + at.col[t]] : 0.0f;

  Parts<3> inverse[2];
  T value[NT][4];
  f32x4_t start, rest, beta;
  float whole;
  const auto load_values = [&](int c) {
    const ChunkRoom room = at.room(p, c);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const T* from = at.step(at.v, p.v_at.t, c, rows + r);
#pragma unroll
      for (int t = 0; t < NT; ++t) value[t][r] = from[min(at.col[t], p.Dv - 1)];
    }
    start = *reinterpret_cast<const f32x4_t*>(room.start + rows);
    beta = *reinterpret_cast<const f32x4_t*>(room.beta + rows);
  };
  const auto load_matrix = [&](int c) {
    const ChunkRoom room = at.room(p, c);
    load_rows_of(inverse, room.inverse, at);
    rest = *reinterpret_cast<const f32x4_t*>(room.rest + rows);
  };
  const auto load_whole = [&](int c) { whole = at.room(p, c).start[kChunk - 1]; };
  loads_arrive();
  if (at.chunks) {
    load_values(0);
    load_matrix(0);
    load_whole(0);
  }
  __syncthreads();                                        // the first chunk's K
  for (int c = 0; c < at.chunks; ++c) {
    const int64_t from = (int64_t)c * kChunk;
    const int next = c + 1 < at.chunks ? c + 1 : c;
    float* const nowhere = at.room(p, c).nowhere;
    f32x4_t mine[NT];                                     // the share of K S for this wave's steps
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float own[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) own[e] = e / 4 < OWN ? S[e / 4 < OWN ? e / 4 : 0][t][e % 4] : 0.0f;
      const Parts<3> op = split<3, false>(own);
      if (owner) {
#pragma unroll
        for (int m = 0; m < OWN; ++m)
#pragma unroll
          for (int i = 0; i < 3; ++i) {
            const u32x4_t w = __builtin_bit_cast(u32x4_t, op.p[i]);
            *reinterpret_cast<u32x2_t*>(L + Room::s + i * Room::s_plane + (16 * t + low16) * Room::key + state_row[m]) = u32x2_t{w[2 * m], w[2 * m + 1]};
          }
      }
      if constexpr (KEEP) {
#pragma unroll
        for (int m = 0; m < OWN; ++m) {
          float* to = p.states + ((int64_t)c * p.B * p.v_heads + at.head) * at.state + (int64_t)state_row[m] * p.Dv + at.col[t];
#pragma unroll
          for (int r = 0; r < 4; ++r) store_device(state_row[m] + r < p.Dk && at.col[t] < p.Dv ? to + r * p.Dv : nowhere, S[m][t][r]);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f32x4_t share = {0.0f, 0.0f, 0.0f, 0.0f};
        const T* const from = (const T*)(L + Room::rows) + (16 * i + low16) * Room::key;
        const Piece<T, 4> a = load_aligned<T, 4>(from + (owner ? state_row[0] : 0));
        if constexpr (OWN == 2) multiply<3>(share, parts_of(a, load_aligned<T, 4>(from + state_row[1])), op);
        else multiply<3>(share, parts_of(a, a), op);          // the other half of S's operand is zero
        if (Room::tight && i == at.wave) mine[t] = share;
        else *reinterpret_cast<f32x4_t*>(sums + Room::share(at.wave, i, t, low16, 16 * i + 4 * quad)) = share;
      }
    }
    __syncthreads();                                      // S, the shares of K S
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      f32x4_t ks = {0.0f, 0.0f, 0.0f, 0.0f}, rhs;
#pragma unroll
      for (int w = 0; w < 4; ++w) ks += Room::tight && w == at.wave ? mine[t] : *reinterpret_cast<const f32x4_t*>(sums + Room::share(w, at.wave, t, low16, rows));
#pragma unroll
      for (int r = 0; r < 4; ++r) rhs[r] = beta[r] * fmaf(-start[r], ks[r], (float)value[t][r]);
      quad_to_planes<3>(L + Room::rhs + (16 * t + low16) * kSteps + rows, Room::u_plane, rhs);
    }
    in_this_order();
    load_values(next);
    __syncthreads();                                      // right-hand sides, K transposed
    f32x4_t u[NT], faded[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) u[t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (s && at.wave < 2) continue;
#pragma unroll
      for (int t = 0; t < NT; ++t) multiply<3>(u[t], inverse[s], from_planes<3>(L + Room::rhs + (16 * t + low16) * kSteps + 32 * s + 8 * quad, Room::u_plane));
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) faded[t][r] = rest[r] * u[t][r];
    computed(faded);
    in_this_order();
    load_matrix(next);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int place = (16 * t + low16) * kSteps + rows;
      quad_to_planes<3>(L + Room::faded + place, Room::u_plane, faded[t]);
      quad_to_planes<3>(L + Room::u + place, Room::u_plane, u[t]);
      if constexpr (KEEP) {
        float* to = p.updates + ((from + rows) * p.B * p.v_heads + at.head) * p.Dv + at.col[t];
#pragma unroll
        for (int r = 0; r < 4; ++r) store_device(from + rows + r < p.T && at.col[t] < p.Dv ? to + (int64_t)r * p.B * p.v_heads * p.Dv : nowhere, u[t][r]);
      }
    }
    __syncthreads();                                      // U, the next chunk's K
#pragma unroll
    for (int m = 0; m < OWN; ++m) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) S[m][t][r] *= whole;
      computed(S[m]);
    }
    in_this_order();
    load_whole(next);
    if (owner) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        Parts<3> op[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) op[t] = from_planes<3>(L + Room::faded + (16 * t + low16) * kSteps + 32 * s + 8 * quad, Room::u_plane);
#pragma unroll
        for (int m = 0; m < OWN; ++m) {
          const Parts<IN> a = from_planes<IN>(L + Room::k + (16 * (at.wave * OWN + m) + low16) * kSteps + 32 * s + 8 * quad, Room::k_plane);
#pragma unroll
          for (int t = 0; t < NT; ++t) multiply<3>(S[m][t], a, op[t]);
        }
      }
    }
  }
  if (!p.h_last || !owner) return;
#pragma unroll
  for (int m = 0; m < OWN; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (state_row[m] + r < p.Dk && at.col[t] < p.Dv) p.h_last[at.head * at.state + (int64_t)(state_row[m] + r) * p.Dv + at.col[t]] = S[m][t][r];
}

// The outputs, from what the chain leaves in LDS.  And its K: the next chunk's as it stands, this one's transposed, zero behind Dk, so that S is.
template <typename T, int DK, int NT, int MODE>
__device__ __forceinline__ void scan_outputs(const DeltaParams& p, const ScanPlace<T, NT>& at, uint8_t* lds) {
  using Room = ScanRoom<T, DK, NT>;
  constexpr int IN = Kind<T>::in, KS = DK / 32;
  bf16* const L = (bf16*)lds;
  T* const key_row = (T*)(L + Room::rows) + at.row * Room::key + 8 * at.quad;
  const int low16 = at.low16, quad = at.quad, rows = at.rows;
  const Identity id(at.lane);
  Piece<T, 8> key[KS], query[KS];
  f32x4_t products[2][2];                                 // float32 numbers
  f32x4_t start;
  const auto load_queries = [&](int c) {
    const T* from = at.step(at.q, p.q_at.t, c, at.row);
#pragma unroll
    for (int s = 0; s < KS; ++s) load_piece<MODE>(query[s], from, 32 * s + 8 * quad, p.Dk);
    start = *reinterpret_cast<const f32x4_t*>(at.room(p, c).start + rows);
  };
  const auto load_products = [&](int c) {
    const float* const from = at.room(p, c).products32();
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < 2; ++i) products[s][i] = reinterpret_cast<const f32x4_t*>(from + ChunkRoom::operand(at.wave, at.wave >= 2 ? s : 0, at.lane))[i];
  };
  // whole rows at a time on the way from memory
  constexpr int pieces = DK / 8;
  const int key_at = 16 * at.wave + at.lane / pieces, key_col = 8 * (at.lane % pieces);
  const auto load_keys = [&](int c) {
#pragma unroll
    for (int s = 0; s < KS; ++s) load_piece<MODE>(key[s], at.step(at.k, p.k_at.t, c, key_at + s * (64 / pieces)), key_col, p.Dk);
  };
  const auto keep_keys = [&] {
#pragma unroll
    for (int s = 0; s < KS; ++s) store_aligned((T*)(L + Room::rows) + (key_at + s * (64 / pieces)) * Room::key + key_col, arranged<MODE>(key[s], key_col, p.Dk));
  };
  if (at.chunks) {
    load_keys(0);
    keep_keys();
    in_this_order();
    load_keys(at.chunks > 1 ? 1 : 0);                     // in the loop's order: waits count what was asked for behind
    in_this_order();
    load_products(0);
    load_queries(0);
  }
  __syncthreads();                                        // the first chunk's K
  for (int c = 0; c < at.chunks; ++c) {
    const int64_t from = (int64_t)c * kChunk;
    const int n = at.steps(c), next = c + 1 < at.chunks ? c + 1 : c, after = c + 2 < at.chunks ? c + 2 : next;
    __syncthreads();                                      // S, the shares of K S
#pragma unroll
    for (int s = 0; s < KS; ++s) transpose_to<IN>(L + Room::k, Room::k_plane, parts_of(load_aligned<T, 8>(key_row + 32 * s)), 16 * at.wave, 32 * s, id, at.lane, p.Dk);
    __syncthreads();                                      // right-hand sides, K transposed
    keep_keys();
    in_this_order();
    load_keys(after);
    f32x4_t o[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) o[t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const Parts<IN> a = parts_of(arranged<MODE>(query[s], 32 * s + 8 * quad, p.Dk));
#pragma unroll
      for (int t = 0; t < NT; ++t) multiply<3>(o[t], a, from_planes<3>(L + Room::s + (16 * t + low16) * Room::key + 32 * s + 8 * quad, Room::s_plane));
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) o[t][r] *= start[r];
    __syncthreads();                                      // U, the next chunk's K
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (s && at.wave < 2) continue;
      const Parts<3> a = parts_of(products[s][0], products[s][1]);
#pragma unroll
      for (int t = 0; t < NT; ++t) multiply<3>(o[t], a, from_planes<3>(L + Room::u + (16 * t + low16) * kSteps + 32 * s + 8 * quad, Room::u_plane));
    }
    computed(o);
    in_this_order();
    T* to[NT][4];
    T* const nowhere = (T*)at.room(p, c).nowhere;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      T* const line = at.out + (from + rows + r) * p.out_at.t;
#pragma unroll
      for (int t = 0; t < NT; ++t) to[t][r] = line + at.col[t];
    }
    if (n < kChunk || at.first + Room::columns > p.Dv) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          if (rows + r >= n) o[t][r] = 0.0f;
          if (from + rows + r >= p.T || at.col[t] >= p.Dv) to[t][r] = nowhere;
        }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) store_device(to[t][r], (T)o[t][r]);
    load_products(next);
    load_queries(next);
  }
  // behind the last chunk's steps
  for (int64_t t = (int64_t)at.chunks * kChunk + threadIdx.x % 256 / Room::columns; t < p.T; t += 256 / Room::columns) {
    const int c = at.first + threadIdx.x % Room::columns;
    if (c < p.Dv) at.out[t * p.out_at.t + c] = (T)0.0f;
  }
}

template <typename T, int DK, int NT, int MODE, bool KEEP>
__global__ __launch_bounds__(512) void scan_kernel(const DeltaParams p, int tiles) {
  extern __shared__ __align__(16) uint8_t lds[];
  const ScanPlace<T, NT> at(p, tiles, p.v, p.v_at, p.out, p.out_at);
  // both meet at the same barriers: one, then three a chunk
  if (__builtin_amdgcn_readfirstlane(threadIdx.x / 256) == 0) scan_states<T, DK, NT, MODE, KEEP>(p, at, lds);
  else scan_outputs<T, DK, NT, MODE>(p, at, lds);
}

template <typename T, int DK, int NT, int MODE, bool KEEP>
hipError_t scan_shaped(const DeltaParams& p, hipStream_t s) {
  const int tiles = (p.Dv + 16 * NT - 1) / (16 * NT);
  constexpr int bytes = ScanRoom<T, DK, NT>::bytes;
  if (bytes > 64 << 10) {
    const hipError_t e = hipFuncSetAttribute((const void*)scan_kernel<T, DK, NT, MODE, KEEP>, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((scan_kernel<T, DK, NT, MODE, KEEP>), dim3((unsigned)((int64_t)p.B * p.v_heads * tiles)), dim3(512), bytes, s, p, tiles);
  return hipGetLastError();
}

template <typename T, int DK, int NT, int MODE, bool KEEP>
hipError_t scan_fitting(const DeltaParams& p, hipStream_t s) {      // float32 keys of 128 features in three parts leave LDS for 16 columns
  return scan_shaped<T, DK, (ScanRoom<T, DK, NT>::bytes <= 160 << 10 ? NT : 1), MODE, KEEP>(p, s);
}

template <typename T, int NT, bool KEEP>
hipError_t scan_typed(const DeltaParams& p, hipStream_t s) {
  return by_mode(piece_mode(p.Dk, 8), [&](auto mode) {
    constexpr int MODE = decltype(mode)::value;
    switch (padded_key(p.Dk)) {
      case 32: return scan_fitting<T, 32, NT, MODE, KEEP>(p, s);
      case 64: return scan_fitting<T, 64, NT, MODE, KEEP>(p, s);
      default: return scan_fitting<T, 128, NT, MODE, KEEP>(p, s);
    }
  });
}

}  // namespace

size_t delta_workspace(const DeltaParams& p) {
  return (size_t)p.chunks * p.B * p.v_heads * (size_t)ChunkRoom::bytes(ChunkRoom::kForward);
}

hipError_t delta_scan_launch(const DeltaParams& given, uint8_t* workspace, hipStream_t s) {
  DeltaParams p = given;
  p.chunk_room = workspace;
  const hipError_t e = delta_prepare_launch(p, false, s);
  if (e != hipSuccess) return e;
  const auto with = [&](auto keep) {
    constexpr bool KEEP = decltype(keep)::value;
    const bool narrow = delta_narrow(p.B, p.v_heads, p.Dv);
    if (p.bf16) return narrow ? scan_typed<bf16, 1, KEEP>(p, s) : scan_typed<bf16, 2, KEEP>(p, s);
    return narrow ? scan_typed<float, 1, KEEP>(p, s) : scan_typed<float, 2, KEEP>(p, s);
  };
  return p.states ? with(std::true_type()) : with(std::false_type());
}

}  // namespace tac
