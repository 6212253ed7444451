// Backward pass of the gated delta rule over sequences.
//
// With the forward's names and dO the outputs' gradients, of a chunk behind whose last step the state has the gradient dS:
//   X = P^T dO + e^(G_end - G) K dS,   R = (I + A)^-T X,   dV = b R,
//   dS <- e^G_end dS + Q^T (e^G dO) - K^T (b e^G R):
// back_scan_kernel, the forward's walk in the other direction, columns by columns; it leaves R and every chunk's dS.  Then every chunk by itself (gradient_kernel), with
// Y = e^(G_t - G_j) dO U^T (j <= t) and Z = -b_t e^(G_t - G_j) R U^T (j < t) and S the state before the chunk:
//   dQ = Y K + e^G dO S^T,   dK = [Z K - b e^G R S^T] + [Z^T K + Y^T Q + e^(G_end - G) U dS^T],   dwrite = (1 - b) R . U.
// e^G_t stands beside every q_t and every k_t that reads (first bracket), e^-G_j beside every k_j that writes (second), e^G_end beside what leaves the chunk, so
//   dG_t = q_t . dQ_t + k_t . [first]_t - k_t . [second]_t  (+ e^G_end <S, dS> + sum_j k_j . (e^(G_end - G_j) dS u_j) at the last),
// and the gradient of log a_t is the sum of dG over the steps from t on.
//
// 8 sequences of 2048 steps, 16 heads of 128 x 128 bf16: back_scan_kernel 200 us, bound by its chain as the forward's walk is (455 with everything on the same four waves);
// gradient_kernel 351 us (300 where its products had 16 digits, three matrix instructions in the place of six): it reads S, dS, U, R (1.0 GB, 2.9 TB/s) while values are summed over, and
// nothing while it then multiplies what is in LDS, with one workgroup a compute unit.
#include "tac_delta_chunk.h"

namespace tac {

namespace {

// LDS of back_scan_kernel.  float32 [5][columns][kSums]: the waves' shares of K dS, and P^T dO; [columns][DK + 4]: Q^T (e^G dO); then in bfloat16 numbers X
// [3][columns][kSteps], b e^G R [3], dO [IN], e^G dO [3], K transposed [IN][DK][kSteps]; and K as it stands, [64][DK + 8] elements.
template <typename T, int DK, int NT>
struct BackRoom {
  static constexpr int columns = 16 * NT, key = DK + 8, fed_pitch = DK + 4;
  static constexpr int u_plane = columns * kSteps, k_plane = DK * kSteps;
  static constexpr int fed = 5 * columns * kSums;                            // float32 numbers before it
  static constexpr int x = 2 * (fed + columns * fed_pitch), r = x + 3 * u_plane, grad = r + 3 * u_plane, fading = grad + Kind<T>::in * u_plane;
  static constexpr int k = fading + 3 * u_plane, rows = k + Kind<T>::in * k_plane;
  static constexpr int bytes = 2 * rows + kChunk * key * (int)sizeof(T);
};

// The chain: the gradients of the states from chunk to chunk, last to first, as scan_states has the states.
template <typename T, int DK, int NT, int MODE>
__device__ __forceinline__ void back_states(const DeltaParams& p, const ScanPlace<T, NT>& at, uint8_t* lds) {
  using Room = BackRoom<T, DK, NT>;
  constexpr int IN = Kind<T>::in, MT = DK / 16, OWN = MT > 4 ? 2 : 1;
  float* const sums = (float*)lds;
  bf16* const L = (bf16*)lds;
  const int low16 = at.low16, quad = at.quad, rows = at.rows;
  const bool owner = MT >= 4 || at.wave < MT;
  int state_row[OWN];
#pragma unroll
  for (int m = 0; m < OWN; ++m) state_row[m] = 16 * (at.wave * OWN + m) + 4 * quad;
  f32x4_t S[OWN][NT];                                     // dS
#pragma unroll
  for (int m = 0; m < OWN; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        S[m][t][r] = p.grad_h_last && state_row[m] + r < p.Dk && at.col[t] < p.Dv ? p.grad_h_last[at.head * at.state + (int64_t)(state_row[m] + r) * p.Dv + at.col[t]] : 0.0f;

  Parts<3> inverse[2];                                    // transposed: rows begin at the diagonal
  f32x4_t start, rest, beta;
  float whole;
  const auto load_rest = [&](int c) { rest = *reinterpret_cast<const f32x4_t*>(at.room(p, c, 3).rest + rows); };
  const auto load_matrix = [&](int c) {
    const ChunkRoom room = at.room(p, c, 3);
    inverse[0] = from_planes<3>(room.inverse + ChunkRoom::operand(at.wave, at.wave >= 2 ? 1 : 0, at.lane), ChunkRoom::plane);
    inverse[1] = from_planes<3>(room.inverse + ChunkRoom::operand(at.wave, 1, at.lane), ChunkRoom::plane);
    start = *reinterpret_cast<const f32x4_t*>(room.start + rows);
    beta = *reinterpret_cast<const f32x4_t*>(room.beta + rows);
  };
  const auto load_whole = [&](int c) { whole = at.room(p, c, 3).start[kChunk - 1]; };
  loads_arrive();
  if (at.chunks) {
    load_rest(at.chunks - 1);
    load_matrix(at.chunks - 1);
    load_whole(at.chunks - 1);
  }
  __syncthreads();                                        // the last chunk's K, dO
  for (int c = at.chunks - 1; c >= 0; --c) {
    const int64_t from = (int64_t)c * kChunk;
    const int n = at.steps(c), next = c ? c - 1 : 0;
    float* const nowhere = at.room(p, c, 3).nowhere;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float own[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) own[e] = e / 4 < OWN ? S[e / 4 < OWN ? e / 4 : 0][t][e % 4] : 0.0f;
      const Parts<3> op = split<3>(own);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f32x4_t share = {0.0f, 0.0f, 0.0f, 0.0f};
        const T* const key = (const T*)(L + Room::rows) + (16 * i + low16) * Room::key;
        const Piece<T, 4> a = load_aligned<T, 4>(key + (owner ? state_row[0] : 0));
        if constexpr (OWN == 2) multiply<3>(share, parts_of(a, load_aligned<T, 4>(key + state_row[1])), op);
        else multiply<3>(share, parts_of(a, a), op);          // the other half of S's operand is zero
        *reinterpret_cast<f32x4_t*>(sums + (at.wave * Room::columns + 16 * t + low16) * kSums + 16 * i + 4 * quad) = share;
      }
    }
    __syncthreads();                                      // shares of K dS, P^T dO
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      f32x4_t x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < 4; ++w) x += *reinterpret_cast<const f32x4_t*>(sums + (w * Room::columns + 16 * t + low16) * kSums + rows);
      const f32x4_t y = *reinterpret_cast<const f32x4_t*>(sums + (4 * Room::columns + 16 * t + low16) * kSums + rows);
#pragma unroll
      for (int r = 0; r < 4; ++r) x[r] = fmaf(rest[r], x[r], y[r]);
      quad_to_planes<3>(L + Room::x + (16 * t + low16) * kSteps + rows, Room::u_plane, x);
    }
    in_this_order();
    load_rest(next);
#pragma unroll
    for (int m = 0; m < OWN; ++m)
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float* to = p.back_states + ((int64_t)c * p.B * p.v_heads + at.head) * at.state + (int64_t)state_row[m] * p.Dv + at.col[t];
#pragma unroll
        for (int r = 0; r < 4; ++r) store_device(state_row[m] + r < p.Dk && at.col[t] < p.Dv ? to + r * p.Dv : nowhere, S[m][t][r]);
      }
    __syncthreads();                                      // X
    f32x4_t R[NT], faded[NT], scaled[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) R[t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (!s && at.wave >= 2) continue;
#pragma unroll
      for (int t = 0; t < NT; ++t) multiply<3>(R[t], inverse[s], from_planes<3>(L + Room::x + (16 * t + low16) * kSteps + 32 * s + 8 * quad, Room::u_plane));
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        scaled[t][r] = beta[r] * R[t][r];
        faded[t][r] = -start[r] * scaled[t][r];
      }
    computed(scaled);
    computed(faded);
    in_this_order();
    load_matrix(next);
#pragma unroll
    for (int t = 0; t < NT; ++t) quad_to_planes<3>(L + Room::r + (16 * t + low16) * kSteps + rows, Room::u_plane, faded[t]);
    {
      float* r_to[NT][4];
      T* v_to[NT][4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float* const line = p.r + ((from + rows + r) * p.B * p.v_heads + at.head) * p.Dv;
        T* const value = at.out + (from + rows + r) * p.grad_v_at.t;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          r_to[t][r] = line + at.col[t];
          v_to[t][r] = value + at.col[t];
        }
      }
      if (n < kChunk || at.first + Room::columns > p.Dv) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            if (rows + r >= n) scaled[t][r] = 0.0f;
            if (from + rows + r >= p.T || at.col[t] >= p.Dv) {
              r_to[t][r] = nowhere;
              v_to[t][r] = (T*)nowhere;
            }
          }
      }
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          store_device(r_to[t][r], R[t][r]);
          store_device(v_to[t][r], (T)scaled[t][r]);
        }
    }
    __syncthreads();                                      // b e^G R, K transposed, Q^T (e^G dO), the next chunk's K and dO
#pragma unroll
    for (int m = 0; m < OWN; ++m) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const f32x4_t fed = *reinterpret_cast<const f32x4_t*>(sums + Room::fed + (16 * t + low16) * Room::fed_pitch + (owner ? state_row[m] : 0));
#pragma unroll
        for (int r = 0; r < 4; ++r) S[m][t][r] = owner ? fmaf(whole, S[m][t][r], fed[r]) : 0.0f;
      }
      computed(S[m]);
    }
    in_this_order();
    load_whole(next);
    if (owner) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        Parts<3> op[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) op[t] = from_planes<3>(L + Room::r + (16 * t + low16) * kSteps + 32 * s + 8 * quad, Room::u_plane);
#pragma unroll
        for (int m = 0; m < OWN; ++m) {
          const Parts<IN> a = from_planes<IN>(L + Room::k + (16 * (at.wave * OWN + m) + low16) * kSteps + 32 * s + 8 * quad, Room::k_plane);
#pragma unroll
          for (int t = 0; t < NT; ++t) multiply<3>(S[m][t], a, op[t]);
        }
      }
    }
  }
  if (!p.grad_h0 || !owner) return;
#pragma unroll
  for (int m = 0; m < OWN; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (state_row[m] + r < p.Dk && at.col[t] < p.Dv) p.grad_h0[at.head * at.state + (int64_t)(state_row[m] + r) * p.Dv + at.col[t]] = S[m][t][r];
}

// What the chain takes that does not wait for it: of this chunk Q^T (e^G dO) and K transposed, of the one in front of it K, dO and P^T dO.
template <typename T, int DK, int NT, int MODE>
__device__ __forceinline__ void back_inputs(const DeltaParams& p, const ScanPlace<T, NT>& at, uint8_t* lds) {
  using Room = BackRoom<T, DK, NT>;
  constexpr int IN = Kind<T>::in, KS = DK / 32, MT = DK / 16, OWN = MT > 4 ? 2 : 1;
  float* const sums = (float*)lds;
  bf16* const L = (bf16*)lds;
  const int low16 = at.low16, quad = at.quad, rows = at.rows;
  const Identity id(at.lane);
  const T* const key_row = (const T*)(L + Room::rows) + at.row * Room::key + 8 * quad;
  const int own_col = 32 * (at.wave * OWN / 2);           // the 32 features that hold the wave's rows of dS
  const bool owner = MT >= 4 || at.wave < MT;
  Piece<T, 8> key[KS], query[4];                          // queries: all steps, the wave's 32 features
  Parts<3> products[2];
  T grad[NT][4];
  f32x4_t start;
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
  const auto load_queries = [&](int c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) load_piece<MODE>(query[i], at.step(at.q, p.q_at.t, c, 16 * i + low16), own_col + 8 * quad, p.Dk);
  };
  const auto load_grads = [&](int c) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const T* from = at.step(at.v, p.out_at.t, c, rows + r);
#pragma unroll
      for (int t = 0; t < NT; ++t) grad[t][r] = from[min(at.col[t], p.Dv - 1)];
    }
    start = *reinterpret_cast<const f32x4_t*>(at.room(p, c, 3).start + rows);
  };
  const auto keep_grads = [&](int c) {
    const int n = at.steps(c);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      f32x4_t g, fading;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        g[r] = rows + r < n ? (float)grad[t][r] : 0.0f;
        fading[r] = start[r] * g[r];
      }
      const int place = (16 * t + low16) * kSteps + rows;
      quad_to_planes<IN>(L + Room::grad + place, Room::u_plane, g);
      quad_to_planes<3>(L + Room::fading + place, Room::u_plane, fading);
    }
  };
  const auto load_matrix = [&](int c) {
    const ChunkRoom room = at.room(p, c, 3);
    products[0] = from_planes<3>(room.products + ChunkRoom::operand(at.wave, at.wave >= 2 ? 1 : 0, at.lane), ChunkRoom::plane);
    products[1] = from_planes<3>(room.products + ChunkRoom::operand(at.wave, 1, at.lane), ChunkRoom::plane);
  };
  const auto from_outputs = [&] {                         // P^T dO
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      f32x4_t x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if (!s && at.wave >= 2) continue;
        multiply<3>(x, products[s], from_planes<IN>(L + Room::grad + (16 * t + low16) * kSteps + 32 * s + 8 * quad, Room::u_plane));
      }
      *reinterpret_cast<f32x4_t*>(sums + (4 * Room::columns + 16 * t + low16) * kSums + rows) = x;
    }
  };
  const int top = at.chunks - 1;
  if (at.chunks) {
    load_keys(top);
    load_grads(top);
    keep_keys();
    keep_grads(top);
    in_this_order();
    load_queries(top);
    load_keys(top ? top - 1 : 0);
    load_grads(top ? top - 1 : 0);
    load_matrix(top);
  }
  __syncthreads();                                        // the last chunk's K, dO
  if (at.chunks) {
    from_outputs();
    in_this_order();
    load_matrix(top ? top - 1 : 0);
  }
  for (int c = top; c >= 0; --c) {
    const int next = c ? c - 1 : 0, after = c > 1 ? c - 2 : 0;
    __syncthreads();                                      // shares of K dS, P^T dO
    // Q^T (e^G dO) for the wave's rows.  A transpose by the identity leaves a column's steps in fours as the summed index wants them; e^G dO is read to match
    f32x4_t fed[OWN][NT];
#pragma unroll
    for (int m = 0; m < OWN; ++m)
#pragma unroll
      for (int t = 0; t < NT; ++t) fed[m][t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      Parts<IN> turned[OWN];
      const Parts<IN> a = parts_of(arranged<MODE>(query[2 * s], own_col + 8 * quad, p.Dk)), b = parts_of(arranged<MODE>(query[2 * s + 1], own_col + 8 * quad, p.Dk));
#pragma unroll
      for (int m = 0; m < OWN; ++m) {
        Parts<1> which = m ? id.odd : id.even;
        if (OWN == 1) which = id.of(at.wave % 2);
#pragma unroll
        for (int i = 0; i < IN; ++i) {
          const f32x4_t zero = {0.0f, 0.0f, 0.0f, 0.0f};
          const f32x4_t x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.p[i], which.p[0], zero, 0, 0, 0);
          const f32x4_t y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.p[i], which.p[0], zero, 0, 0, 0);
          turned[m].p[i] = __builtin_bit_cast(bf16x8_t, u32x4_t{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])});
        }
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        Parts<3> op;
#pragma unroll
        for (int i = 0; i < 3; ++i) {
          const bf16* const f = L + Room::fading + i * Room::u_plane + (16 * t + low16) * kSteps + 32 * s + 4 * quad;
          const u32x2_t x = *reinterpret_cast<const u32x2_t*>(f), y = *reinterpret_cast<const u32x2_t*>(f + 16);
          op.p[i] = __builtin_bit_cast(bf16x8_t, u32x4_t{x[0], x[1], y[0], y[1]});
        }
#pragma unroll
        for (int m = 0; m < OWN; ++m) multiply<3>(fed[m][t], turned[m], op);
      }
    }
    if (owner) {
#pragma unroll
      for (int m = 0; m < OWN; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const int first = 16 * (at.wave * OWN + m) + 4 * quad;
          f32x4_t v = fed[m][t];
#pragma unroll
          for (int r = 0; r < 4; ++r) v[r] = first + r < p.Dk ? v[r] : 0.0f;
          *reinterpret_cast<f32x4_t*>(sums + Room::fed + (16 * t + low16) * Room::fed_pitch + first) = v;
        }
    }
    in_this_order();
    load_queries(next);
    __syncthreads();                                      // X
#pragma unroll
    for (int s = 0; s < KS; ++s) transpose_to<IN>(L + Room::k, Room::k_plane, parts_of(load_aligned<T, 8>(key_row + 32 * s)), 16 * at.wave, 32 * s, id, at.lane, p.Dk);
    keep_keys();
    keep_grads(next);
    in_this_order();
    load_keys(after);
    load_grads(after);
    __syncthreads();                                      // b e^G R, K transposed, Q^T (e^G dO), the next chunk's K and dO
    from_outputs();
    in_this_order();
    load_matrix(after);
  }
  // behind the last chunk's steps
  for (int64_t t = (int64_t)at.chunks * kChunk + threadIdx.x % 256 / Room::columns; t < p.T; t += 256 / Room::columns) {
    const int c = at.first + threadIdx.x % Room::columns;
    if (c < p.Dv) at.out[t * p.grad_v_at.t + c] = (T)0.0f;
  }
}

template <typename T, int DK, int NT, int MODE>
__global__ __launch_bounds__(512) void back_scan_kernel(const DeltaParams p, int tiles) {
  extern __shared__ __align__(16) uint8_t lds[];
  const ScanPlace<T, NT> at(p, tiles, p.grad_out, p.out_at, p.grad_v, p.grad_v_at);
  if (__builtin_amdgcn_readfirstlane(threadIdx.x / 256) == 0) back_states<T, DK, NT, MODE>(p, at, lds);
  else back_inputs<T, DK, NT, MODE>(p, at, lds);
}

// LDS of gradient_kernel in bfloat16 numbers.  While values' features are summed over, 32 at a time: S and dS [3][DK][40], U and R [3][64][40], dO [IN][64][40]; then K or Q
// [IN][64][turned_pitch], Z and Y transposed [3][64][kSteps] each; at last the gradients, [2][64][DK + 8] elements.
template <typename T, int DK>
struct GradientRoom {
  static constexpr int IN = Kind<T>::in, pitch = 40, out_pitch = DK + 8;
  static constexpr int s_plane = DK * pitch, u_plane = kChunk * pitch, k_pitch = turned_pitch(DK), k_plane = kChunk * k_pitch, y_plane = kChunk * kSteps;
  static constexpr int s = 0, back = s + 3 * s_plane, u = back + 3 * s_plane, r = u + 3 * u_plane, g = r + 3 * u_plane, first_size = g + IN * u_plane;
  static constexpr int k = 0, z = k + IN * k_plane, y = z + 3 * y_plane, second_size = y + 3 * y_plane;
  static constexpr int third_size = 2 * kChunk * out_pitch * (int)sizeof(T) / 2;
  static constexpr int most = first_size > second_size ? first_size : second_size, bytes = 2 * (most > third_size ? most : third_size);
};

// four steps of a feature, from what stands as rows
template <int PARTS>
__device__ __forceinline__ f32x4_t steps_of_rows(const bf16* rows, int plane, int pitch, int step, int col, int lane) {
  u32x2_t w[PARTS];
  turned_quad(w, rows, plane, pitch, step, col, lane);
  f32x4_t v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int i = PARTS - 1; i >= 0; --i) v += f32x4_t{bits_float(w[i][0] << 16), bits_float(w[i][0] & 0xffff0000u), bits_float(w[i][1] << 16), bits_float(w[i][1] & 0xffff0000u)};
  return v;
}

// One chunk of a head of queries and keys, the heads of values that share it one after the other.  Eight waves: wave w of either four has the steps from 16 w on as rows and half of a
// key's features as columns, the first four form Y, the others Z.  All that is summed over values comes through LDS, whole lines at a time and two steps ahead.
// MODE: of pieces of 8 of a key and of 4 of a value.
template <typename T, int DK, int MODE>
__global__ __launch_bounds__(512) void gradient_kernel(const DeltaParams p) {
  using Room = GradientRoom<T, DK>;
  constexpr int IN = Kind<T>::in, NT = DK / 32, KS = NT > 1 ? NT / 2 : 1;      // tiles and pieces of this half of the features
  extern __shared__ __align__(16) uint8_t lds[];
  __shared__ float high[kChunk], low[kChunk], change[2][kChunk], both[8];
  bf16* const L = (bf16*)lds;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64 % 4), half = __builtin_amdgcn_readfirstlane(threadIdx.x / 256);
  const int group = p.v_heads / p.k_heads;
  const int hk = blockIdx.x % p.k_heads, b = blockIdx.x / p.k_heads % p.B;
  const int64_t chunk = blockIdx.x / p.k_heads / p.B, from = chunk * kChunk;
  const int n = steps_of(p, b, from), here = (int)min((int64_t)kChunk, p.T - from);
  T* const gq = (T*)p.grad_q + from * p.grad_q_at.t + (int64_t)b * p.grad_q_at.b + (int64_t)hk * p.grad_q_at.head;
  T* const gk = (T*)p.grad_k + from * p.grad_k_at.t + (int64_t)b * p.grad_k_at.b + (int64_t)hk * p.grad_k_at.head;
  T* const gg = (T*)p.grad_gate + from * p.grad_gate_at.t + (int64_t)b * p.grad_gate_at.b;
  T* const gw = (T*)p.grad_write + from * p.grad_write_at.t + (int64_t)b * p.grad_write_at.b;
  if (n == 0) {
    const int tid = threadIdx.x;
    for (int i = tid; i < here * p.Dk; i += 512) {
      gq[(int64_t)(i / p.Dk) * p.grad_q_at.t + i % p.Dk] = (T)0.0f;
      gk[(int64_t)(i / p.Dk) * p.grad_k_at.t + i % p.Dk] = (T)0.0f;
    }
    for (int i = tid; i < here * group; i += 512) {
      gg[(int64_t)(i / group) * p.grad_gate_at.t + hk * group + i % group] = (T)0.0f;
      gw[(int64_t)(i / group) * p.grad_write_at.t + hk * group + i % group] = (T)0.0f;
    }
    return;
  }
  // the features of this half: tiles of 16, and pieces of 32 that hold them
  const int tile0 = half * NT, piece0 = tile0 / 2;
  Piece<T, 8> key[KS], query[KS];
  const auto load_rows = [&] {
    const int lane = fresh(threadIdx.x) % 64, row = 16 * wave + lane % 16, quad = lane / 16;
    const T* const k = (const T*)p.k + (from + min(row, n - 1)) * p.k_at.t + (int64_t)b * p.k_at.b + (int64_t)hk * p.k_at.head;
    const T* const q = (const T*)p.q + (from + min(row, n - 1)) * p.q_at.t + (int64_t)b * p.q_at.b + (int64_t)hk * p.q_at.head;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      load_piece<MODE>(key[s], k, 32 * (piece0 + s) + 8 * quad, p.Dk);
      load_piece<MODE>(query[s], q, 32 * (piece0 + s) + 8 * quad, p.Dk);
    }
  };
  const auto keep = [&](const Piece<T, 8>(&x)[KS], int lane) {      // this half's features
    const int row = 16 * wave + lane % 16;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int col = 32 * (piece0 + s) + 8 * (lane / 16);
      if (NT == 1 && lane / 32 != half) continue;
      const Parts<IN> a = parts_of(zero_ended<MODE>(x[s], col, p.Dk));
#pragma unroll
      for (int i = 0; i < IN; ++i) *reinterpret_cast<bf16x8_t*>(L + Room::k + i * Room::k_plane + row * Room::k_pitch + col) = a.p[i];
    }
  };

  // What a thread brings of S and dS (eight of a row), U, R and dO (four of a row): two steps of 32 values are on their way, of the next head too.
  struct Brought {
    Piece<float, 4> s[2], d[2], u, r;
    Piece<T, 4> g;
  } brought[2];
  const int steps = (p.Dv + 31) / 32, even_steps = (steps + 1) / 2 * 2;
  // where its rows are in the chunk's head: products of 64 bits once for many pieces
  const int state_row = min((int)threadIdx.x / 4, p.Dk - 1) * p.Dv;
  const int64_t own_row = min((int)threadIdx.x / 8, n - 1), update_row = own_row * p.B * p.v_heads * p.Dv, grad_row = own_row * p.out_at.t;
  const auto bring = [&](Brought& x, int h, int step) {
    const int tid = fresh(threadIdx.x), s_col = 8 * (tid % 4), u_col = 4 * (tid % 8);
    const int64_t head = (int64_t)b * p.v_heads + h;
    const int64_t state = (chunk * p.B * p.v_heads + head) * (int64_t)p.Dk * p.Dv + state_row;
    const int64_t update = (from * p.B * p.v_heads + head) * p.Dv + update_row;
    const T* const go = (const T*)p.grad_out + (from * p.out_at.t + (int64_t)b * p.out_at.b + (int64_t)h * p.out_at.head) + grad_row;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      load_piece<MODE>(x.s[i], p.states + state, 32 * step + s_col + 4 * i, p.Dv);
      load_piece<MODE>(x.d[i], p.back_states + state, 32 * step + s_col + 4 * i, p.Dv);
    }
    load_piece<MODE>(x.u, p.updates + update, 32 * step + u_col, p.Dv);
    load_piece<MODE>(x.r, p.r + update, 32 * step + u_col, p.Dv);
    load_piece<MODE>(x.g, go, 32 * step + u_col, p.Dv);
  };
  bring(brought[0], hk * group, 0);
  bring(brought[1], hk * group, 1);
  f32x4_t* const shared = (f32x4_t*)p.shared + (int64_t)blockIdx.x * (2 * NT * 512);      // [2 NT][threads]: a thread's sums over the values' heads before

  for (int member = 0; member < group; ++member) {
    const int h = hk * group + member;
    const ChunkRoom room(p.chunk_room, chunk * p.B * p.v_heads + (int64_t)b * p.v_heads + h, 3);
    const int tid = fresh(threadIdx.x), lane = tid % 64, low16 = lane & 15, quad = lane >> 4, row = 16 * wave + low16, rows = 16 * wave + 4 * quad;
    const int s_row = tid / 4, s_col = 8 * (tid % 4), u_row = tid / 8, u_col = 4 * (tid % 8);
    const f32x4_t start = *reinterpret_cast<const f32x4_t*>(room.start + rows);
    const f32x4_t rest = *reinterpret_cast<const f32x4_t*>(room.rest + rows);
    const f32x4_t beta = *reinterpret_cast<const f32x4_t*>(room.beta + rows);
    const float whole = room.start[kChunk - 1];
    const T gate = ((const T*)p.gate)[(from + min(kChunk - 1 - lane, n - 1)) * p.gate_at.t + (int64_t)b * p.gate_at.b + h];
    const T write = ((const T*)p.write)[(from + min(u_row, n - 1)) * p.write_at.t + (int64_t)b * p.write_at.b + h];
    const float own_high = room.high[tid % kChunk], own_low = room.low[tid % kChunk];      // used behind the products: to wait for them here is to wait for what was brought
    load_rows();
    f32x4_t w[4], dq[NT], reads[NT], writes[NT];      // w: Y or Z
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < NT; ++i) dq[i] = reads[i] = writes[i] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    float written = 0.0f, kept = 0.0f;               // R . U of step u_row, <S, dS>: this thread's parts

    int pair = 0;
    do {                                               // at least once, and known to be: otherwise what is loaded around it would be waited for together
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int step = pair + k, v = 32 * step;
        const bool there_is = step < steps;            // for everybody
        if (there_is) {
          __syncthreads();                             // the features before have been read
          Brought& x = brought[k];
          float s[8], d[8];
          Piece<float, 4> ps[2], pd[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            ps[i] = arranged<MODE>(x.s[i], v + s_col + 4 * i, p.Dv);
            pd[i] = arranged<MODE>(x.d[i], v + s_col + 4 * i, p.Dv);
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            s[e] = ps[e / 4].w[e % 4];               // behind the last value stand numbers of the row, beside zeros of U, R and dO
            d[e] = pd[e / 4].w[e % 4];
          }
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float one = s[4 * i + e] * d[4 * i + e];
              sum += MODE == WHOLE || v + s_col + 4 * i + e < p.Dv ? one : 0.0f;
            }
            kept += MODE != WHOLE || v + s_col + 4 * i < p.Dv ? sum : 0.0f;
          }
          if (s_row < DK) {
            const Parts<3> a = split<3>(s), c = split<3>(d);
#pragma unroll
            for (int i = 0; i < 3; ++i) {
              *reinterpret_cast<bf16x8_t*>(L + Room::s + i * Room::s_plane + s_row * Room::pitch + s_col) = a.p[i];
              *reinterpret_cast<bf16x8_t*>(L + Room::back + i * Room::s_plane + s_row * Room::pitch + s_col) = c.p[i];
            }
          }
          f32x4_t u, r, g;
          const Piece<float, 4> pu = arranged<MODE>(x.u, v + u_col, p.Dv), pr = arranged<MODE>(x.r, v + u_col, p.Dv);
          const Piece<T, 4> pg = arranged<MODE>(x.g, v + u_col, p.Dv);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool there = u_row < n && v + u_col + e < p.Dv;
            u[e] = there ? pu.w[e] : 0.0f;
            r[e] = there ? pr.w[e] : 0.0f;
            g[e] = there ? value_of(pg, e) : 0.0f;
            written = fmaf(u[e], r[e], written);
          }
          const int place = u_row * Room::pitch + u_col;
          quad_to_planes<3>(L + Room::u + place, Room::u_plane, u);
          quad_to_planes<3>(L + Room::r + place, Room::u_plane, r);
          quad_to_planes<IN>(L + Room::g + place, Room::u_plane, g);
        }
        in_this_order();
        bring(brought[k], step + 2 < even_steps || member + 1 == group ? h : h + 1, step + 2 < even_steps ? step + 2 : k);
        if (there_is) {
          __syncthreads();
          const int place = row * Room::pitch + 8 * quad;
          const Parts<IN> own_g = from_planes<IN>(L + Room::g + place, Room::u_plane);
          const Parts<3> own_r = from_planes<3>(L + Room::r + place, Room::u_plane), own_u = from_planes<3>(L + Room::u + place, Room::u_plane);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (i > wave) continue;
            const Parts<3> o = from_planes<3>(L + Room::u + (16 * i + low16) * Room::pitch + 8 * quad, Room::u_plane);
            if (half) multiply<3>(w[i], own_r, o);
            else multiply<3>(w[i], own_g, o);
          }
#pragma unroll
          for (int i = 0; i < NT; ++i) {
            const int feature = (16 * (tile0 + i) + low16) * Room::pitch + 8 * quad;
            const Parts<3> s = from_planes<3>(L + Room::s + feature, Room::s_plane);
            multiply<3>(dq[i], own_g, s);
            multiply<3>(reads[i], own_r, s);
            multiply<3>(writes[i], own_u, from_planes<3>(L + Room::back + feature, Room::s_plane));
            in_this_order();
          }
        }
      }
      pair += 2;
    } while (pair < even_steps);
    if (tid < kChunk) {
      high[tid] = own_high;
      low[tid] = own_low;
    }
    __syncthreads();                                 // S, dS, U, R and dO have been read: K, Z and Y take their place
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        dq[i][r] *= start[r];
        reads[i][r] *= -(beta[r] * start[r]);
        writes[i][r] *= rest[r];
      }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i > wave) continue;                        // above the diagonal: zeros
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int t = rows + r, j = 16 * i + low16;
        const float decay = fast_exp((high[t] - high[j]) + (low[t] - low[j]));
        w[i][r] *= half ? -beta[r] * decay : decay;
        if (half ? j >= t : j > t) w[i][r] = 0.0f;
      }
    }
    keep(key, lane);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = 16 * i + low16;
      quad_to_planes<3>(L + (half ? Room::z : Room::y) + j * kSteps + rows, Room::y_plane, w[i]);
    }
    __syncthreads();
    f32x4_t dG = {0.0f, 0.0f, 0.0f, 0.0f}, leaves = dG, kept_key[NT];      // of the four steps of this lane's results: a part over the features
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      kept_key[i] = steps_of_rows<IN>(L + Room::k, Room::k_plane, Room::k_pitch, rows, 16 * (tile0 + i), lane);
      leaves += kept_key[i] * writes[i];
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int at = 32 * s + 8 * quad;
      const bool lower = 2 * s <= wave, upper = 2 * s + 1 >= wave;      // whether these 32 columns of Y and Z, and of Z transposed, hold something
      Parts<3> a, c, d;
      if (lower) {
        a = turned<3>(L + Room::y, Room::y_plane, kSteps, 32 * s, 16 * wave, lane);
        c = turned<3>(L + Room::z, Room::y_plane, kSteps, 32 * s, 16 * wave, lane);
      }
      if (upper) d = from_planes<3>(L + Room::z + row * kSteps + at, Room::y_plane);
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const Parts<IN> o = turned<IN>(L + Room::k, Room::k_plane, Room::k_pitch, 32 * s, 16 * (tile0 + i), lane);
        if (lower) {
          multiply<3>(dq[i], a, o);
          multiply<3>(reads[i], c, o);
        }
        if (upper) multiply<3>(writes[i], d, o);
      }
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) dG += kept_key[i] * reads[i];
    __syncthreads();                                 // K has been read: Q takes its place
    keep(query, lane);
    __syncthreads();
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (2 * s + 1 < wave) continue;
      const int at = 32 * s + 8 * quad;
      const Parts<3> a = from_planes<3>(L + Room::y + row * kSteps + at, Room::y_plane);
#pragma unroll
      for (int i = 0; i < NT; ++i) multiply<3>(writes[i], a, turned<IN>(L + Room::k, Room::k_plane, Room::k_pitch, 32 * s, 16 * (tile0 + i), lane));
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      dG += steps_of_rows<IN>(L + Room::k, Room::k_plane, Room::k_pitch, rows, 16 * (tile0 + i), lane) * dq[i];
      dG -= kept_key[i] * writes[i];
    }
    // sums over this half's features: 16 lanes; over a step's values: 8 threads; over everything
    kept = sum_over_lanes<64>(s_row < p.Dk ? kept : 0.0f);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      dG[r] = sum_over_lanes<16>(dG[r]);
      leaves[r] = sum_over_lanes<16>(leaves[r]);
    }
    const float out = sum_over_lanes<64>(low16 == 0 ? (leaves[0] + leaves[1]) + (leaves[2] + leaves[3]) : 0.0f);
    written = sum_over_lanes<8>(written);
    if (low16 == 0) {
#pragma unroll
      for (int r = 0; r < 4; ++r) change[half][rows + r] = dG[r];
    }
    if (lane == 0) both[tid / 64] = fmaf(whole, kept, out);
    if (tid % 8 == 0 && u_row < here) {
      float d = 0.0f;                                // 1 - b by itself: from a rounded b near 1 nothing would be left of it
      if (u_row < n) d = sigmoid(-(float)write) * written;
      gw[(int64_t)u_row * p.grad_write_at.t + h] = (T)d;
    }
    __syncthreads();
    if (tid < 64) {
      // the sum from every step on, in 64 bits: its terms are far larger than what is left of them
      double total = (double)change[0][kChunk - 1 - lane] + (double)change[1][kChunk - 1 - lane];
      if (lane == 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) total += (double)both[i];
      }
#pragma unroll
      for (int by = 1; by < 64; by *= 2) {
        const double before = __shfl_up(total, by);
        if (lane >= by) total += before;
      }
      const int t = kChunk - 1 - lane;
      if (t < here) {
        float d = 0.0f;
        if (t < n) d = sigmoid(-(float)gate) * (float)total;
        gg[(int64_t)t * p.grad_gate_at.t + h] = (T)d;
      }
    }
    const bool last = member + 1 == group;
#pragma unroll
    for (int i = 0; i < NT; ++i) reads[i] += writes[i];
    if (member) {
      f32x4_t before[2 * NT];                        // all on their way together
#pragma unroll
      for (int i = 0; i < 2 * NT; ++i) before[i] = shared[i * 512 + tid];
      in_this_order();
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        dq[i] += before[2 * i];
        reads[i] += before[2 * i + 1];
      }
    }
    if (!last) {
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        shared[2 * i * 512 + tid] = dq[i];
        shared[(2 * i + 1) * 512 + tid] = reads[i];
      }
    } else {                                         // every wave has read Q and Y
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          T* const to = (T*)lds + (rows + r) * Room::out_pitch + 16 * (tile0 + i) + low16;
          to[0] = (T)dq[i][r];
          to[kChunk * Room::out_pitch] = (T)reads[i][r];
        }
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * kChunk * (DK / 8); i += 512) {
    const int which = i / (kChunk * (DK / 8)), t = i / (DK / 8) % kChunk, c = 8 * (i % (DK / 8)), left = p.Dk - c;
    if (t >= here || left <= 0) continue;
    Piece<T, 8> v = load_aligned<T, 8>((const T*)lds + (which * kChunk + t) * Room::out_pitch + c);
    if (t >= n) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v.set(e, (T)0.0f);
    }
    T* const to = which ? gk + (int64_t)t * p.grad_k_at.t + c : gq + (int64_t)t * p.grad_q_at.t + c;
    if (left >= 8) {
      __builtin_memcpy(to, v.w, 8 * sizeof(T));
    } else {
      const T* const at = (const T*)lds + (which * kChunk + t) * Room::out_pitch + c;
      for (int e = 0; e < left; ++e) to[e] = t < n ? at[e] : (T)0.0f;
    }
  }
}

template <typename K>
hipError_t with_lds(K kernel, int bytes) {
  return bytes > 64 << 10 ? hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) : hipSuccess;
}

template <typename T, int DK, int NT, int MODE>
hipError_t back_scan_shaped(const DeltaParams& p, hipStream_t s) {
  if constexpr (NT > 1 && BackRoom<T, DK, NT>::bytes > 160 << 10) {      // float32 keys in three parts leave LDS for 16 columns
    return back_scan_shaped<T, DK, 1, MODE>(p, s);
  } else {
    const int tiles = (p.Dv + 16 * NT - 1) / (16 * NT);
    constexpr int bytes = BackRoom<T, DK, NT>::bytes;
    const hipError_t e = with_lds(back_scan_kernel<T, DK, NT, MODE>, bytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((back_scan_kernel<T, DK, NT, MODE>), dim3((unsigned)((int64_t)p.B * p.v_heads * tiles)), dim3(512), bytes, s, p, tiles);
    return hipGetLastError();
  }
}

template <typename T, int DK>
hipError_t backward_shaped(const DeltaParams& p, hipStream_t s) {
  const bool narrow = delta_narrow(p.B, p.v_heads, p.Dv);
  const int key = piece_mode(p.Dk, 8), value = piece_mode(p.Dv, 4);
  const hipError_t e = by_mode(key, [&](auto mode) {
    constexpr int MODE = decltype(mode)::value;
    return narrow ? back_scan_shaped<T, DK, 1, MODE>(p, s) : back_scan_shaped<T, DK, 2, MODE>(p, s);
  });
  if (e != hipSuccess) return e;
  // whole pieces of a row that is long enough may be read as shifted ones, by nothing
  const int both = key == EACH || value == EACH ? EACH : key == WHOLE && value == WHOLE ? WHOLE : p.Dk >= 8 && p.Dv >= 4 ? SHIFTED : EACH;
  return by_mode(both, [&](auto mode) {
    constexpr int MODE = decltype(mode)::value, bytes = GradientRoom<T, DK>::bytes;
    const hipError_t e = with_lds(gradient_kernel<T, DK, MODE>, bytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((gradient_kernel<T, DK, MODE>), dim3((unsigned)((int64_t)p.chunks * p.B * p.k_heads)), dim3(512), bytes, s, p);
    return hipGetLastError();
  });
}

template <typename T>
hipError_t backward_typed(const DeltaParams& p, hipStream_t s) {
  switch (padded_key(p.Dk)) {
    case 32: return backward_shaped<T, 32>(p, s);
    case 64: return backward_shaped<T, 64>(p, s);
    default: return backward_shaped<T, 128>(p, s);
  }
}

// parts of the workspace, each a multiple of 16 bytes
struct BackWorkspace {
  size_t room, states, r, shared, size;
  explicit BackWorkspace(const DeltaParams& p) {
    const auto up = [](size_t n) { return (n + 15) / 16 * 16; };
    const size_t heads = (size_t)p.chunks * p.B * p.v_heads;
    room = 0;
    states = room + heads * (size_t)ChunkRoom::bytes(3);
    r = states + up(heads * (size_t)p.Dk * p.Dv * 4);
    shared = r + up((size_t)p.T * p.B * p.v_heads * p.Dv * 4);
    size = shared + (p.v_heads > p.k_heads ? (size_t)p.chunks * p.B * p.k_heads * 2 * kChunk * padded_key(p.Dk) * 4 : 0);
  }
};

}  // namespace

size_t delta_backward_workspace(const DeltaParams& p) { return BackWorkspace(p).size; }

hipError_t delta_backward_launch(const DeltaParams& given, uint8_t* workspace, hipStream_t s) {
  DeltaParams p = given;
  const BackWorkspace w(p);
  p.chunk_room = workspace + w.room;
  p.back_states = (float*)(workspace + w.states);
  p.r = (float*)(workspace + w.r);
  p.shared = (float*)(workspace + w.shared);
  const hipError_t e = delta_prepare_launch(p, true, s);
  if (e != hipSuccess) return e;
  return p.bf16 ? backward_typed<bf16>(p, s) : backward_typed<float>(p, s);
}

}  // namespace tac
