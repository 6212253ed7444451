// Pieces of the chunked delta rule: numbers as bfloat16 parts, products on the matrix cores, the workspace of a chunk.
#pragma once
#include "tac_delta_common.h"

namespace tac {

typedef bf16 bf16x8_t __attribute__((ext_vector_type(8)));

constexpr int kChunk = TAC_DELTA_CHUNK;
constexpr int kSteps = kChunk + 8;            // pitch of LDS rows of a chunk's steps in bf16: 16 rows' pieces of 16 bytes fall on all banks

// ---- numbers as sums of bfloat16 parts -----------------------------------------------------------
// A float32 number is the sum of three bfloat16 numbers (3 x 8 digits); the product of two such sums without what is below 2^-24 of it is six products, of a
// bfloat16 number with one three.
template <int PARTS>
struct Parts {
  bf16x8_t p[PARTS];
};

// PAIRS: two numbers an instruction, a fifth fewer of them; one by one each waits for less, for the chain of states (32768 steps: 991 us, in pairs 1014)
template <int PARTS, bool PAIRS = true>
__device__ __forceinline__ Parts<PARTS> split(const float (&v)[8]) {
  Parts<PARTS> r;
  float rest[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) rest[e] = v[e];
#pragma unroll
  for (int q = 0; q < PARTS; ++q) {
    if constexpr (PAIRS) {
      u32x4_t w;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t two = pack_bf16(rest[2 * e], rest[2 * e + 1]);
        w[e] = two;
        if (q + 1 < PARTS) {
          rest[2 * e] -= bits_float(two << 16);
          rest[2 * e + 1] -= bits_float(two & 0xffff0000u);
        }
      }
      r.p[q] = __builtin_bit_cast(bf16x8_t, w);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        r.p[q][e] = (bf16)rest[e];
        if (q + 1 < PARTS) rest[e] -= (float)r.p[q][e];
      }
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

// In how many parts numbers enter that come from tensors of a type.  What is formed from them has three, also on its way to bfloat16 results: those are often what is left of far larger terms.
template <typename T>
struct Kind;
template <>
struct Kind<bf16> {
  static constexpr int in = 1;
};
template <>
struct Kind<float> {
  static constexpr int in = 3;
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
  __device__ __forceinline__ Parts<1> of(int second) const {      // by value: a reference to one of the two would put both into memory
    const u32x4_t a = __builtin_bit_cast(u32x4_t, even.p[0]), b = __builtin_bit_cast(u32x4_t, odd.p[0]);
    u32x4_t r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = second ? b[e] : a[e];
    return {__builtin_bit_cast(bf16x8_t, r)};
  }
  __device__ Identity(int lane) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int k = 8 * (lane >> 4) + e;
      even.p[0][e] = (bf16)(k == (lane & 15) ? 1.0f : 0.0f);
      odd.p[0][e] = (bf16)(k - 16 == (lane & 15) ? 1.0f : 0.0f);
    }
  }
};
// `to`: LDS planes [PARTS][columns][kSteps]; the operand holds steps `row`.. (16 of them) and columns col.. (32), of which those from `cols` on are taken as zero
template <int PARTS>
__device__ __forceinline__ void transpose_to(bf16* to, int plane, const Parts<PARTS>& a, int row, int col, const Identity& id, int lane, int cols) {
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    bf16* at = to + (col + 16 * half + (lane & 15)) * kSteps + row + 4 * (lane >> 4);
#pragma unroll
    for (int q = 0; q < PARTS; ++q) {
      f32x4_t t = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.p[q], half ? id.odd.p[0] : id.even.p[0], f32x4_t{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0);
      if (col + 16 * half + (lane & 15) >= cols) t = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
      *reinterpret_cast<u32x2_t*>(at + q * plane) = u32x2_t{pack_bf16(t[0], t[1]), pack_bf16(t[2], t[3])};
    }
  }
}

// What stands in LDS as rows of steps (planes of bfloat16 parts), read turned.  Of the 16 lanes that read together each brings four neighbours of a row, four lanes a row, and gets four
// rows of its own column: here steps from `step` on of column `col` + lane % 16.
constexpr int turned_pitch(int features) { return features + (features == 64 ? 8 : 24); }      // of 32, 64, 128: four rows' 32 bytes meet on no bank
typedef short s16x4_t __attribute__((ext_vector_type(4)));
template <int PARTS>
__device__ __forceinline__ void turned_quad(u32x2_t (&to)[PARTS], const bf16* rows, int plane, int pitch, int step, int col, int lane) {
  const bf16* const at = rows + (step + (lane & 15) / 4) * pitch + col + 4 * (lane & 3);
#pragma unroll
  for (int i = 0; i < PARTS; ++i) to[i] = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(at + i * plane)));
}
// as an operand: rows are the columns from `col` on, summed indices the steps from `step` on
template <int PARTS>
__device__ __forceinline__ Parts<PARTS> turned(const bf16* rows, int plane, int pitch, int step, int col, int lane) {
  u32x2_t a[PARTS], b[PARTS];
  turned_quad(a, rows, plane, pitch, step + 8 * (lane >> 4), col, lane);
  turned_quad(b, rows, plane, pitch, step + 8 * (lane >> 4) + 4, col, lane);
  Parts<PARTS> r;
#pragma unroll
  for (int i = 0; i < PARTS; ++i) r.p[i] = __builtin_bit_cast(bf16x8_t, u32x4_t{a[i][0], a[i][1], b[i][0], b[i][1]});
  return r;
}

// Everything that was asked for from memory is there.  In front of a loop whose loads stay on their way: the compiler would otherwise keep the wait for what was
// loaded before the loop at its first use inside, where it waits for the loop's own loads in every turn.
__device__ __forceinline__ void loads_arrive() { __builtin_amdgcn_s_waitcnt(0x0f70); }      // vmcnt(0)

// keeps the loads behind it behind it, so that they can take the registers of what was used before it
__device__ __forceinline__ void in_this_order() { __builtin_amdgcn_sched_barrier(0); }
template <int N>
__device__ __forceinline__ void computed(f32x4_t (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(v[i]));
}

// The same number, of which the compiler does not know that it is: what is computed from it is computed here, not kept in registers around a loop.
__device__ __forceinline__ int fresh(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// a store to device memory, also where the compiler cannot tell from a chosen address that it is
template <typename T>
__device__ __forceinline__ void store_device(T* to, T v) {
  *(__attribute__((address_space(1))) T*)(uintptr_t)to = v;
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

// Which head and which tile of its columns a workgroup takes.  Consecutive workgroups go to the eight dies in turn: a head's tiles, which read the same queries, keys and matrices,
// are eight apart, so that one die's cache holds them (a sequence of 32768 steps, 16 heads: before, the loads of one chunk took longer than the chunk before it).
struct HeadTile {
  int head, tile;
  __device__ __forceinline__ HeadTile(int index, int heads, int tiles) {
    const int group = index / (8 * tiles), at = index - group * 8 * tiles, wide = min(8, heads - 8 * group);
    head = 8 * group + at % wide;
    tile = at / wide;
  }
};

__device__ __forceinline__ int steps_of(const DeltaParams& p, int b, int64_t from) {      // steps of the chunk that begins at `from`
  // by a scalar load: to wait for a vector one is to wait for all that were asked for before it
  const int64_t n = p.lengths ? min((int64_t)max(*(const __attribute__((address_space(4))) int32_t*)(uintptr_t)(p.lengths + b), 0), p.T) : p.T;
  return (int)max((int64_t)0, min((int64_t)kChunk, n - from));
}

// What prepare_kernel leaves of a chunk and head: the inverse in three parts, [64][64] each; the queries' products, forwards as float32 numbers, a third less than three parts (which spare one
// long sequence 4 % and cost a batch of them 2 %), backwards in three parts; float32 factors of the steps.
// Backwards both matrices stand transposed, so that a row's neighbours are what is summed over.  A plane is in the order in which it is read, the operand of 16 rows and 32
// columns in one piece, a lane's eight numbers after the other's; of the operands only those that hold something are written.
struct ChunkRoom {
  // operand of rows 16 tile.. and columns 32 step..
  static __device__ __forceinline__ int operand(int tile, int step, int lane) { return ((tile * 2 + step) * 64 + lane) * 8; }
  static constexpr int plane = kChunk * kChunk;
  static constexpr int kForward = 2, kBackward = 3;      // what the products take, in planes of 16 bits
  static constexpr int64_t bytes(int p_planes) { return (int64_t)(3 + p_planes) * plane * 2 + 6 * kChunk * 4; }
  bf16 *inverse, *products;                     // forwards the products are float32 numbers: products32()
  float *start, *rest, *beta, *high, *low;      // e^G, e^(G_end - G), b, and G in two numbers
  float* nowhere;                               // takes what is not to be stored
  __device__ __forceinline__ float* products32() const { return (float*)products; }
  __device__ __forceinline__ ChunkRoom(uint8_t* base, int64_t index, int p_planes) {
    inverse = (bf16*)(base + index * bytes(p_planes));
    products = inverse + 3 * plane;
    start = (float*)(products + p_planes * plane);
    rest = start + kChunk;
    beta = rest + kChunk;
    high = beta + kChunk;
    low = high + kChunk;
    nowhere = low + kChunk;
  }
};

// A piece of a row of n elements, N neighbours from `at` on, as it stands in memory.  Loads of the next chunk are on their way while this one is worked on: nothing here looks
// at what is loaded, and nothing branches, since behind a branch the compiler waits for everything.
//   WHOLE    n is a multiple of N: a piece is there or not
//   SHIFTED  n is at least N: the last piece is read so that it ends with the row, and arranged() moves its elements to their places
//   EACH     element by element
// Of what is not there something of the row is read instead, which is no zero.
enum { EACH = 0, SHIFTED = 1, WHOLE = 2 };
inline int piece_mode(int n, int N) { return n % N == 0 ? WHOLE : n > N ? SHIFTED : EACH; }

// f(mode) with it as a constant
template <typename F>
hipError_t by_mode(int mode, F f) {
  using std::integral_constant;
  return mode == WHOLE ? f(integral_constant<int, WHOLE>()) : mode == SHIFTED ? f(integral_constant<int, SHIFTED>()) : f(integral_constant<int, EACH>());
}

template <int MODE, typename T, int N>
__device__ __forceinline__ void load_piece(Piece<T, N>& v, const T* row, int at, int n) {
  if constexpr (MODE == WHOLE) {
    __builtin_memcpy(v.w, row + (at < n ? at : 0), N * sizeof(T));
  } else if constexpr (MODE == SHIFTED) {
    __builtin_memcpy(v.w, row + min(at, n - N), N * sizeof(T));
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) v.set(e, row[min(at + e, n - 1)]);
  }
}
template <int MODE, typename T, int N>
__device__ __forceinline__ Piece<T, N> arranged(const Piece<T, N>& v, int at, int n) {
  if constexpr (MODE != SHIFTED) return v;
  const int by = at - min(at, n - N);                 // elements; N and more: nothing of the piece is there, and what is returned is of the row
  constexpr int words = N * sizeof(T) / 4, per = 4 / sizeof(T);
  Piece<T, N> r = v;
  if constexpr (per == 2) {
#pragma unroll
    for (int i = 0; i < words; ++i) r.w[i] = __builtin_amdgcn_alignbit(i + 1 < words ? v.w[i + 1] : 0u, v.w[i], (by & 1) * 16);
  }
#pragma unroll
  for (int step = 1; step < words; step *= 2) {
    const bool on = (by / per) & step;
#pragma unroll
    for (int i = 0; i < words; ++i) r.w[i] = on ? (i + step < words ? r.w[i + step] : std::remove_reference_t<decltype(r.w[0])>()) : r.w[i];
  }
  return r;
}

// zeros behind the row's end
template <int MODE, typename T, int N>
__device__ __forceinline__ Piece<T, N> zero_ended(const Piece<T, N>& v, int at, int n) {
  Piece<T, N> r = arranged<MODE>(v, at, n);
  if constexpr (MODE != EACH) {
#pragma unroll
    for (int i = 0; i < (int)(N * sizeof(T) / 4); ++i) r.w[i] = at < n ? r.w[i] : std::remove_reference_t<decltype(r.w[0])>();
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (at + e >= n) r.set(e, (T)0.0f);
  }
  return r;
}

// the same in LDS, aligned
template <typename T, int N>
__device__ __forceinline__ void store_aligned(T* to, const Piece<T, N>& v) {
  constexpr int words = N * sizeof(T) / 4;
  if constexpr (words == 2) {
    *reinterpret_cast<u32x2_t*>(to) = u32x2_t{v.w[0], v.w[1]};
  } else {
#pragma unroll
    for (int i = 0; i < words; i += 4) {
      u32x4_t w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = __builtin_bit_cast(uint32_t, v.w[i + e]);
      reinterpret_cast<u32x4_t*>(to)[i / 4] = w;
    }
  }
}
template <typename T, int N>
__device__ __forceinline__ Piece<T, N> load_aligned(const T* from) {
  constexpr int words = N * sizeof(T) / 4;
  Piece<T, N> v;
  if constexpr (words == 2) {
    const u32x2_t w = *reinterpret_cast<const u32x2_t*>(from);
    v.w[0] = w[0];
    v.w[1] = w[1];
  } else {
#pragma unroll
    for (int i = 0; i < words; i += 4) {
      const u32x4_t w = reinterpret_cast<const u32x4_t*>(from)[i / 4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t one = w[e];             // a vector's element itself is not what a bit cast takes
        v.w[i + e] = __builtin_bit_cast(std::remove_reference_t<decltype(v.w[0])>, one);
      }
    }
  }
  return v;
}
// eight summed indices as an operand: one piece of eight, or two of four
__device__ __forceinline__ Parts<1> parts_of(const Piece<bf16, 8>& v) { return {__builtin_bit_cast(bf16x8_t, v)}; }
__device__ __forceinline__ Parts<1> parts_of(const Piece<bf16, 4>& a, const Piece<bf16, 4>& b) {
  return {__builtin_bit_cast(bf16x8_t, u32x4_t{a.w[0], a.w[1], b.w[0], b.w[1]})};
}
__device__ __forceinline__ Parts<3> parts_of(const Piece<float, 8>& v) { return split<3>(v.w); }
__device__ __forceinline__ Parts<3> parts_of(const Piece<float, 4>& a, const Piece<float, 4>& b) {
  const float v[8] = {a.w[0], a.w[1], a.w[2], a.w[3], b.w[0], b.w[1], b.w[2], b.w[3]};
  return split<3>(v);
}
__device__ __forceinline__ Parts<3> parts_of(const f32x4_t& a, const f32x4_t& b) {
  const float v[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  return split<3>(v);
}
constexpr int kSums = kChunk + 4;             // pitch of LDS rows of a chunk's steps in float32

// What a workgroup of a walk over the chunks works on, and where this lane stands: of its eight waves, wave w of either four has the chunk's steps from 16 w on as rows.
template <typename T, int NT>
struct ScanPlace {
  int wave, lane, low16, quad, row, rows;      // row: of operands; rows: the first of four of results
  int first, chunks, last;                     // last: steps of the last chunk
  int col[NT];
  int64_t head, state;
  const T *q, *k, *v;
  T* out;
  // v, out: what is read and written in the layout of values
  __device__ ScanPlace(const DeltaParams& p, int tiles, const void* v_base, const tac_delta_strides_t& v_at, void* out_base, const tac_delta_strides_t& out_at) {
    const HeadTile place(blockIdx.x, p.B * p.v_heads, tiles);
    const int tile = place.tile, h = place.head % p.v_heads, b = place.head / p.v_heads, hk = h / (p.v_heads / p.k_heads);
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64 % 4);
    lane = threadIdx.x % 64;
    low16 = lane & 15;
    quad = lane >> 4;
    row = 16 * wave + low16;
    rows = 16 * wave + 4 * quad;
    first = tile * 16 * NT;
#pragma unroll
    for (int t = 0; t < NT; ++t) col[t] = first + 16 * t + low16;
    const int64_t length = p.lengths ? min((int64_t)max(p.lengths[b], 0), p.T) : p.T;
    chunks = (int)((length + kChunk - 1) / kChunk);
    last = (int)(length - (int64_t)(chunks - 1) * kChunk);
    head = (int64_t)b * p.v_heads + h;
    state = (int64_t)p.Dk * p.Dv;
    q = (const T*)p.q + (int64_t)b * p.q_at.b + (int64_t)hk * p.q_at.head;
    k = (const T*)p.k + (int64_t)b * p.k_at.b + (int64_t)hk * p.k_at.head;
    v = (const T*)v_base + (int64_t)b * v_at.b + (int64_t)h * v_at.head;
    out = (T*)out_base + (int64_t)b * out_at.b + (int64_t)h * out_at.head;
  }
  __device__ __forceinline__ ChunkRoom room(const DeltaParams& p, int c, int p_planes = ChunkRoom::kForward) const { return ChunkRoom(p.chunk_room, (int64_t)c * p.B * p.v_heads + head, p_planes); }
  __device__ __forceinline__ int steps(int c) const { return c + 1 < chunks ? kChunk : last; }
  // step `i` of chunk c, of a tensor whose steps are `stride` apart.  What is behind the last step is read from there: it stands beside b = 0, or is not stored.
  template <typename E>
  __device__ __forceinline__ E* step(E* base, int64_t stride, int c, int i) const {
    base += (int64_t)c * kChunk * stride;
    return base + (steps(c) == kChunk ? (int64_t)i * stride : (int64_t)min(i, last - 1) * stride);
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
