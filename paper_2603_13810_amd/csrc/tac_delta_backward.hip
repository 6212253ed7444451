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
#include "tac_delta_chunk.h"

namespace tac {

namespace {

// LDS of back_scan_kernel in bfloat16 numbers: dS [3][columns][DK + 8], dO [IN][columns][kSteps], e^G dO [3], X [3], b e^G R [3], K and Q transposed [IN][DK][kSteps]
template <typename T, int DK, int NT>
struct BackRoom {
  static constexpr int columns = 16 * NT, key = DK + 8;
  static constexpr int s_plane = columns * key, u_plane = columns * kSteps, k_plane = DK * kSteps;
  static constexpr int s = 0, grad = s + 3 * s_plane, fading = grad + Kind<T>::in * u_plane, x = fading + 3 * u_plane, r = x + 3 * u_plane, k = r + 3 * u_plane;
  static constexpr int q = k + Kind<T>::in * k_plane, size = q + Kind<T>::in * k_plane;
};

template <typename T, int DK, int NT>
__global__ __launch_bounds__(256) void back_scan_kernel(const DeltaParams p, int tiles) {
  using Room = BackRoom<T, DK, NT>;
  constexpr int IN = Kind<T>::in, KS = DK / 32, MT = DK / 16, OWN = MT > 4 ? MT / 4 : 1;
  extern __shared__ __align__(16) uint8_t lds[];
  bf16* const L = (bf16*)lds;
  const HeadTile place(blockIdx.x, p.B * p.v_heads, tiles);
  const int tile = place.tile, h = place.head % p.v_heads, b = place.head / p.v_heads;
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, low16 = lane & 15, quad = lane >> 4;
  const int hk = h / (p.v_heads / p.k_heads), first = tile * Room::columns;
  const int64_t length = p.lengths ? min((int64_t)max(p.lengths[b], 0), p.T) : p.T;
  const T* const q = (const T*)p.q + (int64_t)b * p.q_at.b + (int64_t)hk * p.q_at.head;
  const T* const k = (const T*)p.k + (int64_t)b * p.k_at.b + (int64_t)hk * p.k_at.head;
  const T* const go = (const T*)p.grad_out + (int64_t)b * p.out_at.b + (int64_t)h * p.out_at.head;
  T* const gv = (T*)p.grad_v + (int64_t)b * p.grad_v_at.b + (int64_t)h * p.grad_v_at.head;
  const int64_t head = (int64_t)b * p.v_heads + h, state = (int64_t)p.Dk * p.Dv;
  const Identity id(lane);
  const bool owner = MT >= 4 || wave < MT;
  int col[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) col[t] = first + 16 * t + low16;

  f32x4_t S[OWN][NT];                 // dS
#pragma unroll
  for (int m = 0; m < OWN; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * (wave * OWN + m) + 4 * quad + r;
        S[m][t][r] = p.grad_h_last && row < p.Dk && col[t] < p.Dv ? p.grad_h_last[head * state + (int64_t)row * p.Dv + col[t]] : 0.0f;
      }

  const int chunks = (int)((length + kChunk - 1) / kChunk);
  for (int c = chunks - 1; c >= 0; --c) {
    const int64_t from = (int64_t)c * kChunk;
    const int n = (int)min((int64_t)kChunk, length - from);
    const int64_t index_of_chunk = (int64_t)c * p.B * p.v_heads + head;
    const ChunkRoom room(p.chunk_room, index_of_chunk, 3);
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
    const f32x4_t start = *reinterpret_cast<const f32x4_t*>(room.start + 16 * wave + 4 * quad);
    const f32x4_t rest = *reinterpret_cast<const f32x4_t*>(room.rest + 16 * wave + 4 * quad);
    const f32x4_t beta = *reinterpret_cast<const f32x4_t*>(room.beta + 16 * wave + 4 * quad);
    const float whole = room.start[kChunk - 1];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      f32x4_t grad, fading;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * wave + 4 * quad + r;
        grad[r] = row < n && col[t] < p.Dv ? (float)go[(from + row) * p.out_at.t + col[t]] : 0.0f;
        fading[r] = start[r] * grad[r];
      }
      const int at = (16 * t + low16) * kSteps + 16 * wave + 4 * quad;
      quad_to_planes<IN>(L + Room::grad + at, Room::u_plane, grad);
      quad_to_planes<3>(L + Room::fading + at, Room::u_plane, fading);
    }
    if (owner) {
#pragma unroll
      for (int m = 0; m < OWN; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const int row = 16 * (wave * OWN + m) + 4 * quad;
          quad_to_planes<3>(L + Room::s + (16 * t + low16) * Room::key + row, Room::s_plane, S[m][t]);
          if (col[t] < p.Dv) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (row + r < p.Dk) p.back_states[index_of_chunk * state + (int64_t)(row + r) * p.Dv + col[t]] = S[m][t][r];
          }
        }
    }
    __syncthreads();

    f32x4_t x[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      x[t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int s = 0; s < KS; ++s) multiply<3>(x[t], key[s], from_planes<3>(L + Room::s + (16 * t + low16) * Room::key + 32 * s + 8 * quad, Room::s_plane));
#pragma unroll
      for (int r = 0; r < 4; ++r) x[t][r] *= rest[r];
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (32 * s + 31 < 16 * wave) continue;           // rows of the transposed matrices begin at the diagonal
      const Parts<3> a = from_planes<3>(room.products + ChunkRoom::operand(wave, s, lane), ChunkRoom::plane);
#pragma unroll
      for (int t = 0; t < NT; ++t) multiply<3>(x[t], a, from_planes<IN>(L + Room::grad + (16 * t + low16) * kSteps + 32 * s + 8 * quad, Room::u_plane));
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) quad_to_planes<3>(L + Room::x + (16 * t + low16) * kSteps + 16 * wave + 4 * quad, Room::u_plane, x[t]);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      transpose_to<IN>(L + Room::k, Room::k_plane, key[s], 16 * wave, 32 * s, id, lane, p.Dk);
      transpose_to<IN>(L + Room::q, Room::k_plane, query[s], 16 * wave, 32 * s, id, lane, p.Dk);
    }
    __syncthreads();

    f32x4_t R[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) R[t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (32 * s + 31 < 16 * wave) continue;
      const Parts<3> a = from_planes<3>(room.inverse + ChunkRoom::operand(wave, s, lane), ChunkRoom::plane);
#pragma unroll
      for (int t = 0; t < NT; ++t) multiply<3>(R[t], a, from_planes<3>(L + Room::x + (16 * t + low16) * kSteps + 32 * s + 8 * quad, Room::u_plane));
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      f32x4_t faded;
#pragma unroll
      for (int r = 0; r < 4; ++r) faded[r] = -(beta[r] * start[r]) * R[t][r];
      quad_to_planes<3>(L + Room::r + (16 * t + low16) * kSteps + 16 * wave + 4 * quad, Room::u_plane, faded);
      if (col[t] < p.Dv) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = 16 * wave + 4 * quad + r;
          if (from + row >= p.T) continue;
          p.r[((from + row) * p.B * p.v_heads + head) * p.Dv + col[t]] = R[t][r];
          gv[(from + row) * p.grad_v_at.t + col[t]] = (T)(row < n ? beta[r] * R[t][r] : 0.0f);
        }
      }
    }
    __syncthreads();

    if (owner) {
#pragma unroll
      for (int m = 0; m < OWN; ++m) {
        const int row = (16 * (wave * OWN + m) + low16) * kSteps;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) S[m][t][r] *= whole;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const Parts<IN> a = from_planes<IN>(L + Room::q + row + 32 * s + 8 * quad, Room::k_plane), d = from_planes<IN>(L + Room::k + row + 32 * s + 8 * quad, Room::k_plane);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const int at = (16 * t + low16) * kSteps + 32 * s + 8 * quad;
            multiply<3>(S[m][t], a, from_planes<3>(L + Room::fading + at, Room::u_plane));
            multiply<3>(S[m][t], d, from_planes<3>(L + Room::r + at, Room::u_plane));
          }
        }
      }
    }
    __syncthreads();                                   // the next chunk's gradients take the place of these
  }
  for (int64_t t = (int64_t)chunks * kChunk + threadIdx.x / Room::columns; t < p.T; t += 256 / Room::columns) {
    const int at = first + threadIdx.x % Room::columns;
    if (at < p.Dv) gv[t * p.grad_v_at.t + at] = (T)0.0f;
  }
  if (!p.grad_h0 || !owner) return;
#pragma unroll
  for (int m = 0; m < OWN; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * (wave * OWN + m) + 4 * quad + r;
        if (row < p.Dk && col[t] < p.Dv) p.grad_h0[head * state + (int64_t)row * p.Dv + col[t]] = S[m][t][r];
      }
}

// LDS of gradient_kernel in bytes.  While values' features are summed over, 32 at a time: S and dS [OUT][DK][40], U [OUT][64][40]; then K or Q transposed [IN][DK][kSteps],
// Z and its transpose, Y or its transpose [OUT][64][kSteps] each.
template <typename T, int DK>
struct GradientRoom {
  static constexpr int IN = Kind<T>::in, OUT = Kind<T>::out, pitch = 40;
  static constexpr int s_plane = DK * pitch, u_plane = kChunk * pitch, k_plane = DK * kSteps, y_plane = kChunk * kSteps;
  static constexpr int s = 0, back = s + OUT * s_plane, u = back + OUT * s_plane, first_size = u + OUT * u_plane;
  static constexpr int k = 0, z = k + IN * k_plane, z_turned = z + OUT * y_plane, y = z_turned + OUT * y_plane, second_size = y + OUT * y_plane;
  static constexpr int size = first_size > second_size ? first_size : second_size;
};

// rows 4 quad .. of column `col` of a 16 x 16 result, to planes [rows][kSteps]: as it stands, or transposed (a column's rows are neighbours)
template <int PARTS>
__device__ __forceinline__ void result_to_planes(bf16* to, int plane, const f32x4_t& v, int row, int col) {
  u32x2_t q[PARTS];
  split_quad<PARTS>(v, q);
#pragma unroll
  for (int i = 0; i < PARTS; ++i) {
    uint16_t* at = (uint16_t*)(to + i * plane) + row * kSteps + col;
    at[0] = (uint16_t)q[i][0];
    at[kSteps] = (uint16_t)(q[i][0] >> 16);
    at[2 * kSteps] = (uint16_t)q[i][1];
    at[3 * kSteps] = (uint16_t)(q[i][1] >> 16);
  }
}

// four steps of one feature from planes [features][kSteps], whole numbers again
template <int PARTS>
__device__ __forceinline__ f32x4_t steps_from_planes(const bf16* at, int plane) {
  f32x4_t v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int i = PARTS - 1; i >= 0; --i) {
    const u32x2_t w = *reinterpret_cast<const u32x2_t*>(at + i * plane);
    v += f32x4_t{bits_float(w[0] << 16), bits_float(w[0] & 0xffff0000u), bits_float(w[1] << 16), bits_float(w[1] & 0xffff0000u)};
  }
  return v;
}

template <typename T, int DK>
__global__ __launch_bounds__(256) void gradient_kernel(const DeltaParams p) {
  using Room = GradientRoom<T, DK>;
  constexpr int IN = Kind<T>::in, OUT = Kind<T>::out, KS = DK / 32, NT = DK / 16;
  extern __shared__ __align__(16) uint8_t lds[];
  __shared__ float high[kChunk], low[kChunk], change[kChunk], both[4];
  bf16* const L = (bf16*)lds;
  const int hk = blockIdx.x % p.k_heads, b = blockIdx.x / p.k_heads % p.B;
  const int64_t chunk = blockIdx.x / p.k_heads / p.B, from = chunk * kChunk;
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, low16 = lane & 15, quad = lane >> 4;
  const int group = p.v_heads / p.k_heads;
  const int n = steps_of(p, b, from), here = (int)min((int64_t)kChunk, p.T - from);
  T* const gq = (T*)p.grad_q + from * p.grad_q_at.t + (int64_t)b * p.grad_q_at.b + (int64_t)hk * p.grad_q_at.head;
  T* const gk = (T*)p.grad_k + from * p.grad_k_at.t + (int64_t)b * p.grad_k_at.b + (int64_t)hk * p.grad_k_at.head;
  T* const gg = (T*)p.grad_gate + from * p.grad_gate_at.t + (int64_t)b * p.grad_gate_at.b;
  T* const gw = (T*)p.grad_write + from * p.grad_write_at.t + (int64_t)b * p.grad_write_at.b;
  if (n == 0) {
    for (int i = threadIdx.x; i < here * p.Dk; i += 256) {
      gq[(int64_t)(i / p.Dk) * p.grad_q_at.t + i % p.Dk] = (T)0.0f;
      gk[(int64_t)(i / p.Dk) * p.grad_k_at.t + i % p.Dk] = (T)0.0f;
    }
    for (int i = threadIdx.x; i < here * group; i += 256) {
      gg[(int64_t)(i / group) * p.grad_gate_at.t + hk * group + i % group] = (T)0.0f;
      gw[(int64_t)(i / group) * p.grad_write_at.t + hk * group + i % group] = (T)0.0f;
    }
    return;
  }
  const T* const q = (const T*)p.q + from * p.q_at.t + (int64_t)b * p.q_at.b + (int64_t)hk * p.q_at.head;
  const T* const k = (const T*)p.k + from * p.k_at.t + (int64_t)b * p.k_at.b + (int64_t)hk * p.k_at.head;
  float* const shared = p.shared + (int64_t)blockIdx.x * 2 * kChunk * DK;       // sums of this head's queries and keys over the values' heads before
  const int own = 16 * wave + low16;                 // the step whose rows this lane has as an operand
  const Identity id(lane);

  for (int member = 0; member < group; ++member) {
    const int h = hk * group + member;
    const int64_t head = (int64_t)b * p.v_heads + h, index_of_chunk = chunk * p.B * p.v_heads + head;
    const ChunkRoom room(p.chunk_room, index_of_chunk, 3);
    const float* const S = p.states + index_of_chunk * (int64_t)p.Dk * p.Dv;
    const float* const back = p.back_states + index_of_chunk * (int64_t)p.Dk * p.Dv;
    const T* const go = (const T*)p.grad_out + (from + own) * p.out_at.t + (int64_t)b * p.out_at.b + (int64_t)h * p.out_at.head;
    const float* const U = p.updates + (from * p.B * p.v_heads + head) * (int64_t)p.Dv;
    const float* const R = p.r + (from * p.B * p.v_heads + head) * (int64_t)p.Dv;
    const int64_t step = (int64_t)p.B * p.v_heads * p.Dv;
    __syncthreads();                                 // the member before has been done with LDS
    if (threadIdx.x < kChunk) {
      high[threadIdx.x] = room.high[threadIdx.x];
      low[threadIdx.x] = room.low[threadIdx.x];
    }
    f32x4_t y[4], z[4], dq[NT], reads[NT], writes[NT];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = z[i] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < NT; ++i) dq[i] = reads[i] = writes[i] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    float written = 0.0f, kept = 0.0f;               // R . U of the own step (a part), <S, dS> (this thread's part)

    for (int v = 0; v < p.Dv; v += 32) {
      const int at = v + 8 * quad;
      __syncthreads();                               // the features before have been read
#pragma unroll
      for (int i = 0; i < DK * 4 / 256 + (DK * 4 % 256 != 0); ++i) {
        const int piece = threadIdx.x + 256 * i, row = piece / 4, c = 8 * (piece % 4);
        if (row >= DK) break;
        Eight<float> s, d;
        s.load(S + (int64_t)row * p.Dv + v + c, row < p.Dk ? p.Dv - v - c : 0);
        d.load(back + (int64_t)row * p.Dv + v + c, row < p.Dk ? p.Dv - v - c : 0);
        const Parts<OUT> a = split<OUT>(s.v), e = split<OUT>(d.v);
#pragma unroll
        for (int m = 0; m < 8; ++m) kept = fmaf(s.v[m], d.v[m], kept);
#pragma unroll
        for (int m = 0; m < OUT; ++m) {
          *reinterpret_cast<bf16x8_t*>(L + Room::s + m * Room::s_plane + row * Room::pitch + c) = a.p[m];
          *reinterpret_cast<bf16x8_t*>(L + Room::back + m * Room::s_plane + row * Room::pitch + c) = e.p[m];
        }
      }
      Eight<float> u, r;
      u.load(U + own * step + at, own < n ? p.Dv - at : 0);
      r.load(R + own * step + at, own < n ? p.Dv - at : 0);
#pragma unroll
      for (int m = 0; m < 8; ++m) written = fmaf(u.v[m], r.v[m], written);
      const Parts<OUT> own_u = split<OUT>(u.v), own_r = split<OUT>(r.v);
#pragma unroll
      for (int m = 0; m < OUT; ++m) *reinterpret_cast<bf16x8_t*>(L + Room::u + m * Room::u_plane + own * Room::pitch + 8 * quad) = own_u.p[m];
      Eight<T> g;
      g.load(go + at, own < n ? p.Dv - at : 0);
      const Parts<IN> own_g = g.parts();
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i > wave) continue;
        const Parts<OUT> o = from_planes<OUT>(L + Room::u + (16 * i + low16) * Room::pitch + 8 * quad, Room::u_plane);
        multiply<OUT>(y[i], own_g, o);
        multiply<OUT>(z[i], own_r, o);
      }
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const Parts<OUT> s = from_planes<OUT>(L + Room::s + (16 * i + low16) * Room::pitch + 8 * quad, Room::s_plane);
        multiply<OUT>(dq[i], own_g, s);
        multiply<OUT>(reads[i], own_r, s);
        multiply<OUT>(writes[i], own_u, from_planes<OUT>(L + Room::back + (16 * i + low16) * Room::pitch + 8 * quad, Room::s_plane));
      }
    }

    const f32x4_t start = *reinterpret_cast<const f32x4_t*>(room.start + 16 * wave + 4 * quad);
    const f32x4_t rest = *reinterpret_cast<const f32x4_t*>(room.rest + 16 * wave + 4 * quad);
    const f32x4_t beta = *reinterpret_cast<const f32x4_t*>(room.beta + 16 * wave + 4 * quad);
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        dq[i][r] *= start[r];
        reads[i][r] *= -(beta[r] * start[r]);
        writes[i][r] *= rest[r];
      }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int t = 16 * wave + 4 * quad + r, j = 16 * i + low16;
        const float decay = fast_exp((high[t] - high[j]) + (low[t] - low[j]));
        y[i][r] = j <= t ? decay * y[i][r] : 0.0f;
        z[i][r] = j < t ? -beta[r] * decay * z[i][r] : 0.0f;
      }
    __syncthreads();                                 // S, dS and U have been read: K, Z and Y take their place
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = 16 * wave + 4 * quad, j = 16 * i + low16;
      result_to_planes<OUT>(L + Room::z, Room::y_plane, z[i], t, j);
      result_to_planes<OUT>(L + Room::y, Room::y_plane, y[i], t, j);
      quad_to_planes<OUT>(L + Room::z_turned + j * kSteps + t, Room::y_plane, z[i]);
    }
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int at = 32 * s + 8 * quad;
      Eight<T> e;
      e.load(k + (int64_t)own * p.k_at.t + at, own < n ? p.Dk - at : 0);
      transpose_to<IN>(L + Room::k, Room::k_plane, e.parts(), 16 * wave, 32 * s, id, lane, p.Dk);
    }
    __syncthreads();
    f32x4_t dG = {0.0f, 0.0f, 0.0f, 0.0f}, leaves = dG;      // of the four steps of this lane's results: a part over the features
#pragma unroll
    for (int i = 0; i < NT; ++i) leaves += steps_from_planes<IN>(L + Room::k + (16 * i + low16) * kSteps + 16 * wave + 4 * quad, Room::k_plane) * writes[i];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int at = 32 * s + 8 * quad;
      const Parts<OUT> a = from_planes<OUT>(L + Room::y + own * kSteps + at, Room::y_plane), c = from_planes<OUT>(L + Room::z + own * kSteps + at, Room::y_plane),
                       d = from_planes<OUT>(L + Room::z_turned + own * kSteps + at, Room::y_plane);
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const Parts<IN> o = from_planes<IN>(L + Room::k + (16 * i + low16) * kSteps + at, Room::k_plane);
        multiply<OUT>(dq[i], a, o);
        multiply<OUT>(reads[i], c, o);
        multiply<OUT>(writes[i], d, o);
      }
    }
    __syncthreads();                                 // K and Y have been read: Q and Y transposed take their place
#pragma unroll
    for (int i = 0; i < NT; ++i) dG += steps_from_planes<IN>(L + Room::k + (16 * i + low16) * kSteps + 16 * wave + 4 * quad, Room::k_plane) * reads[i];
    f32x4_t key[NT];                                 // the writing keys' products wait for the queries'
#pragma unroll
    for (int i = 0; i < NT; ++i) key[i] = steps_from_planes<IN>(L + Room::k + (16 * i + low16) * kSteps + 16 * wave + 4 * quad, Room::k_plane);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) quad_to_planes<OUT>(L + Room::y + (16 * i + low16) * kSteps + 16 * wave + 4 * quad, Room::y_plane, y[i]);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int at = 32 * s + 8 * quad;
      Eight<T> e;
      e.load(q + (int64_t)own * p.q_at.t + at, own < n ? p.Dk - at : 0);
      transpose_to<IN>(L + Room::k, Room::k_plane, e.parts(), 16 * wave, 32 * s, id, lane, p.Dk);
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int at = 32 * s + 8 * quad;
      const Parts<OUT> a = from_planes<OUT>(L + Room::y + own * kSteps + at, Room::y_plane);
#pragma unroll
      for (int i = 0; i < NT; ++i) multiply<OUT>(writes[i], a, from_planes<IN>(L + Room::k + (16 * i + low16) * kSteps + at, Room::k_plane));
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      dG += steps_from_planes<IN>(L + Room::k + (16 * i + low16) * kSteps + 16 * wave + 4 * quad, Room::k_plane) * dq[i];
      dG -= key[i] * writes[i];
    }
    // sums over the features: 16 lanes; over the own step's values: four lanes 16 apart; over everything
    kept = sum_over_lanes<64>(kept);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      dG[r] = sum_over_lanes<16>(dG[r]);
      leaves[r] = sum_over_lanes<16>(leaves[r]);
    }
    float out = sum_over_lanes<64>(low16 == 0 ? (leaves[0] + leaves[1]) + (leaves[2] + leaves[3]) : 0.0f);
    written = over_rows(written, [](float a, float c) { return a + c; });
    if (low16 == 0) {
#pragma unroll
      for (int r = 0; r < 4; ++r) change[16 * wave + 4 * quad + r] = dG[r];
    }
    if (lane == 0) both[wave] = fmaf(room.start[kChunk - 1], kept, out);
    if (quad == 0 && own < here) {
      float d = 0.0f;                                // 1 - b by itself: from a rounded b near 1 nothing would be left of it
      if (own < n) d = sigmoid(-(float)((const T*)p.write)[(from + own) * p.write_at.t + (int64_t)b * p.write_at.b + h]) * written;
      gw[(int64_t)own * p.grad_write_at.t + h] = (T)d;
    }
    __syncthreads();
    if (wave == 0) {
      // the sum from every step on, in 64 bits: its terms are far larger than what is left of them
      double total = (double)change[kChunk - 1 - lane];
      if (lane == 0) total += ((double)both[0] + both[1]) + ((double)both[2] + both[3]);
#pragma unroll
      for (int by = 1; by < 64; by *= 2) {
        const double before = __shfl_up(total, by);
        if (lane >= by) total += before;
      }
      const int t = kChunk - 1 - lane;
      if (t < here) {
        float d = 0.0f;
        if (t < n) d = sigmoid(-(float)((const T*)p.gate)[(from + t) * p.gate_at.t + (int64_t)b * p.gate_at.b + h]) * (float)total;
        gg[(int64_t)t * p.grad_gate_at.t + h] = (T)d;
      }
    }
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int t = 16 * wave + 4 * quad + r, c = 16 * i + low16;
        float a = dq[i][r], d = reads[i][r] + writes[i][r];
        float* const kept_q = shared + t * DK + c;
        float* const kept_k = kept_q + kChunk * DK;
        if (member) {                                // the same lane's sums
          a += *kept_q;
          d += *kept_k;
        }
        if (member + 1 < group) {
          *kept_q = a;
          *kept_k = d;
        } else if (t < here && c < p.Dk) {
          gq[(int64_t)t * p.grad_q_at.t + c] = (T)(t < n ? a : 0.0f);
          gk[(int64_t)t * p.grad_k_at.t + c] = (T)(t < n ? d : 0.0f);
        }
      }
  }
}

template <typename K>
hipError_t with_lds(K kernel, int bytes) {
  return bytes > 64 << 10 ? hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) : hipSuccess;
}

template <typename T, int DK, int NT>
hipError_t back_scan_shaped(const DeltaParams& p, hipStream_t s) {
  const int tiles = (p.Dv + 16 * NT - 1) / (16 * NT);
  constexpr int bytes = BackRoom<T, DK, NT>::size * 2;
  const hipError_t e = with_lds(back_scan_kernel<T, DK, NT>, bytes);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((back_scan_kernel<T, DK, NT>), dim3((unsigned)((int64_t)p.B * p.v_heads * tiles)), dim3(256), bytes, s, p, tiles);
  return hipGetLastError();
}

template <typename T, int DK>
hipError_t backward_shaped(const DeltaParams& p, hipStream_t s) {
  // float32 keys of 128 features in three parts leave LDS for 16 columns
  const bool narrow = delta_narrow(p.B, p.v_heads, p.Dv) || BackRoom<T, DK, 2>::size * 2 > 160 << 10;
  hipError_t e;
  if constexpr (BackRoom<T, DK, 2>::size * 2 <= 160 << 10) e = narrow ? back_scan_shaped<T, DK, 1>(p, s) : back_scan_shaped<T, DK, 2>(p, s);
  else e = back_scan_shaped<T, DK, 1>(p, s);
  if (e != hipSuccess) return e;
  constexpr int bytes = GradientRoom<T, DK>::size * 2;
  e = with_lds(gradient_kernel<T, DK>, bytes);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((gradient_kernel<T, DK>), dim3((unsigned)((int64_t)p.chunks * p.B * p.k_heads)), dim3(256), bytes, s, p);
  return hipGetLastError();
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
