// Product of two 8-bit matrices with a power of two per 128 columns, on the matrix cores.
//
// v_mfma_scale_f32_32x32x64_f8f6f4 multiplies 32 rows by 32 rows over 64 columns and applies, per row and 32 columns, a power of two that each
// lane passes in a byte: a block's scale costs no instruction of its own, and all blocks of a sum stay in one accumulator.  Lane l holds 32
// consecutive codes of row l % 32.
//
// That instruction adds eight consecutive products at a time and keeps only what reaches 2^-13 of the largest of them (measured: 2^16 and
// one smaller term; the root mean square of a sum's error is 1.3e-5 to 1.7e-5 of the sums' for normal operands of 512 to 16384 columns, 4e-5 to 7e-5 where
// their columns' sizes spread by a factor e).  A bfloat16 result rounds by 2^-8 and does not notice; for a float32 result the codes are turned into bfloat16 in registers, exactly and with their scale (v_cvt_scalef32_pk_bf16_fp8),
// and multiplied by v_mfma_f32_32x32x16_bf16, which keeps float32 sums (1e-8), at half the rate.
//
// The rows of b are the instruction's first operand: a lane then ends with four consecutive n of one m.
#include "tac_head_common.h"
#include "tac_mfma_common.h"
#include "tac_plan_memo.h"
#include "tac_product_plan.h"

namespace tac {

namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef bf16 bf16x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ i32x8_t join_codes(u32x4_t lo, u32x4_t hi) {
  return i32x8_t{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}

// the 8 q-th to 8 q + 7-th of 32 codes as bfloat16 times 2^e (its float in `scale`)
__device__ __forceinline__ bf16x8_t widen(i32x8_t codes, int q, float scale) {
  const uint32_t lo = (uint32_t)codes[2 * q], hi = (uint32_t)codes[2 * q + 1];
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// 16 bytes a lane from a buffer into LDS at lds_base + 16 lane, and 4 bytes a lane from an address of its own to lds_base + 4 lane.  Addresses beyond the
// buffer are not read and bring zeros: a load that is not wanted has a buffer of no bytes, which takes no branch (a branch would let the compiler
// move the multiplications around it behind it) and counts like the others.  Like lds_dma16 they are not known to the compiler: the reader
// waits (dma_wait) in front of the barrier that parts it from the loads.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void lds_dma_rows(uint32_t offset, u32x4_t buffer, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" :: "v"(offset), "s"(buffer), "s"(lds_base) : "m0", "memory");
}
__device__ __forceinline__ void lds_dma_dword(const void* from, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" :: "v"(from), "s"(lds_base) : "m0", "memory");
}
#pragma clang diagnostic pop
// until all but the last N of the wave's loads have arrived
template <int N>
__device__ __forceinline__ void dma_wait() {
  static_assert(N < 64);
  __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | (N >> 4) << 14);
}

// a buffer of `bytes` bytes (at most 2^32 - 1 are asked for) from `at` on
__device__ __forceinline__ u32x4_t buffer_at(uint64_t at, int64_t bytes) {
  return u32x4_t{(uint32_t)__builtin_amdgcn_readfirstlane((int)at), (uint32_t)__builtin_amdgcn_readfirstlane((int)(at >> 32)) & 0xffffu,
                 (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes), 0x00020000u};
}

// Tiles of TM rows of a x TN rows of b, WM x WN waves.  One block of 128 columns of the tile's rows (128 bytes each) is a stage in LDS: while the waves
// multiply one, direct-to-LDS loads fill the others.  Fragments are read two steps ahead of their use, across blocks too: the one
// barrier a block stands two steps before its end, where all of the stage has been read and the next one is there.  A row's eight pieces of 16
// bytes stand at their number XOR bits 1 to 3 of the row, so that the 16 rows that a fragment read takes at once fall into different
// banks.  A workgroup takes items (a tile, or one of `parts` parts of a tile's columns, whose results are [part][M][N]) until there are
// none, and has the next item's first blocks on their way while it writes the results of the one before: they are turned through LDS, so that
// rows leave in pieces of up to 256 bytes.
template <int TM, int TN, int WM, int WN, int STAGES, bool EXACT, bool PAST, typename U>
__global__ __launch_bounds__(64 * WM * WN, 2) void product_tile_kernel(const ProductParams p, int parts) {
  constexpr int kWaves = WM * WN, FM = TM / WM / 32, FN = TN / WN / 32, kStage = (TM + TN) * kBlock;
  constexpr int kLoadsM = TM / 8 / kWaves, kLoadsN = TN / 8 / kWaves;         // a load instruction brings 8 rows
  static_assert(TM % (32 * WM) == 0 && TN % (32 * WN) == 0 && TM % (8 * kWaves) == 0 && TN % (8 * kWaves) == 0 && kWaves % 2 == 0);
  static_assert(TM + TN <= 64 * kWaves);
  constexpr int kScales = tile_scales_at(TM, TN, kWaves, STAGES), kLoads = kLoadsM + kLoadsN + 1;
  extern __shared__ __align__(1024) uint8_t stages[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave % WM, wn = wave / WM;
  const int64_t pitch = code_pitch(p.K), spitch = scale_pitch(p.K);
  const int blocks = (int)(pitch / kBlock);
  const int tiles_m = (int)((p.M + TM - 1) / TM), tiles_n = (int)((p.N + TN - 1) / TN), items = tiles_m * tiles_n * parts;

  // the item in hand: its rows and blocks of columns
  int64_t m0, n0;
  int part, first, last;
  uint64_t am_at, bn_at;             // the tile's rows of either matrix: those that are there, from their first byte (rows of at most
  uint32_t am_bytes, bn_bytes;       // 2^23 codes: 32-bit offsets)
  const uint8_t* scales_from;        // a lane brings one row's scales; rows beyond the matrices take the last one's, what comes of them is not stored
  auto take = [&](int item) {
    // Workgroups i, i + 8, i + 16 ... run on one of the eight dies, which have an L2 each: a die takes consecutive tiles, in strips of four tile
    // rows of a, so that the tiles that it has in hand at a time share their rows.
    const int die = item % 8, at = item / 8, whole = items / 8, more = items % 8;
    item = die * whole + min(die, more) + at;
    part = item / (tiles_m * tiles_n);
    const int tile = item - part * (tiles_m * tiles_n);
    const int strip = tile / (4 * tiles_n), rows = min(4, tiles_m - 4 * strip), in = tile - strip * 4 * tiles_n;
    m0 = (int64_t)(4 * strip + in % rows) * TM;
    n0 = (int64_t)(in / rows) * TN;
    first = (int)((int64_t)blocks * part / parts);
    last = (int)((int64_t)blocks * (part + 1) / parts);
    am_at = (uint64_t)(uintptr_t)p.a + (uint64_t)(m0 * pitch);
    bn_at = (uint64_t)(uintptr_t)p.b + (uint64_t)(n0 * pitch);
    am_bytes = (uint32_t)(min((int64_t)TM, p.M - m0) * pitch);
    bn_bytes = (uint32_t)(min((int64_t)TN, p.N - n0) * pitch);
    const int64_t row = (64 * wave + lane) % (TM + TN);      // waves that have none of their own bring others' again, to a place that nobody reads
    scales_from = row < TM ? p.a_scales + min(m0 + row, p.M - 1) * spitch : p.b_scales + min(n0 + row - TM, p.N - 1) * spitch;
  };

  const uint32_t offset = (uint32_t)((8 * wave + lane / 8) * pitch) + 16 * ((lane % 8) ^ ((4 * wave + (lane >> 4)) & 7));
  const uint32_t step = (uint32_t)(8 * kWaves * pitch);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)stages;
  auto load = [&](int k) {
    const int slot = (uint32_t)(k - first) % STAGES, at = min(k, last - 1);
    const u32x4_t am = buffer_at(am_at + (uint32_t)at * kBlock, k < last ? am_bytes - at * kBlock : 0);
    const u32x4_t bn = buffer_at(bn_at + (uint32_t)at * kBlock, k < last ? bn_bytes - at * kBlock : 0);
    const uint32_t to = lds0 + wave * 1024 + slot * kStage;
#pragma unroll
    for (int j = 0; j < kLoadsM; ++j) lds_dma_rows(offset + j * step, am, to + j * kWaves * 1024);
#pragma unroll
    for (int j = 0; j < kLoadsN; ++j) lds_dma_rows(offset + j * step, bn, to + TM * kBlock + j * kWaves * 1024);
    lds_dma_dword(scales_from + (at & ~3), lds0 + kScales + (slot * kWaves + wave) * 256);
  };

  uint32_t em[FM], en[FN];                                // scale bytes of the block in hand
  auto fetch_scales = [&](int k, uint32_t (&m)[FM], uint32_t (&n)[FN]) {
    const uint8_t* at = stages + kScales + (uint32_t)(k - first) % STAGES * (256 * kWaves) + (k & 3) + 4 * (lane % 32);
#pragma unroll
    for (int f = 0; f < FM; ++f) m[f] = at[(wm * FM + f) * 128];
#pragma unroll
    for (int f = 0; f < FN; ++f) n[f] = at[4 * TM + (wn * FN + f) * 128];
  };

  f32x16_t sum[FN][FM];

  // A block is kSteps steps, each a fragment of b against all of the wave's fragments of a; every step first reads what the step after next needs.
  constexpr int kSteps = 2 * FN, kRing = kSteps < 4 ? kSteps : 4;
  static_assert(kSteps % kRing == 0);
  i32x8_t a[2][FM], b[kRing];
  bf16x8_t wide[EXACT ? FM : 1][4];
  const int x = (lane >> 1) & 7, at_m = (wm * FM * 32 + lane % 32) * kBlock, at_n = (TM + wn * FN * 32 + lane % 32) * kBlock;
  const int piece[2][2] = {{16 * ((2 * (lane / 32)) ^ x), 16 * ((2 * (lane / 32) + 1) ^ x)},
                           {16 * ((2 * (lane / 32) + 4) ^ x), 16 * ((2 * (lane / 32) + 5) ^ x)}};
  auto fetch = [&](const uint8_t* at, auto step_number) {
    constexpr int S = decltype(step_number)::value, H = S / FN, I = S % FN;
    if constexpr (I == 0) {
#pragma unroll
      for (int f = 0; f < FM; ++f)
        a[H][f] = join_codes(*reinterpret_cast<const u32x4_t*>(at + at_m + f * 32 * kBlock + piece[H][0]),
                             *reinterpret_cast<const u32x4_t*>(at + at_m + f * 32 * kBlock + piece[H][1]));
    }
    b[S % kRing] = join_codes(*reinterpret_cast<const u32x4_t*>(at + at_n + I * 32 * kBlock + piece[H][0]),
                          *reinterpret_cast<const u32x4_t*>(at + at_n + I * 32 * kBlock + piece[H][1]));
  };

  auto block = [&](int k, auto more) {
    const uint8_t *here = stages + (uint32_t)(k - first) % STAGES * kStage, *there = stages + (uint32_t)(k - first + 1) % STAGES * kStage;
    uint32_t next_m[FM], next_n[FN];
    static_for<0, kSteps>([&](auto step_number) {
      constexpr int S = decltype(step_number)::value, H = S / FN, I = S % FN;
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (S == kSteps - 2 && decltype(more)::value) {          // all of this stage has been read: its place takes the next block that is not on its way
        dma_wait<(STAGES - 2) * kLoads>();
        __syncthreads();
        load(k + STAGES);
        fetch_scales(k + 1, next_m, next_n);
      }
      auto ahead = [&] {
        if constexpr (S < kSteps - 2) fetch(here, std::integral_constant<int, (S + 2) % kSteps>());
        else if constexpr (decltype(more)::value) fetch(there, std::integral_constant<int, (S + 2) % kSteps>());
      };
      if constexpr (kSteps > 2) ahead();                  // with two steps a block the step after next has this step's registers
      if constexpr (EXACT) {
        if constexpr (I == 0) {
#pragma unroll
          for (int f = 0; f < FM; ++f)
#pragma unroll
            for (int q = 0; q < 4; ++q) wide[f][q] = widen(a[H][f], q, scale_value(em[f]));
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const bf16x8_t bv = widen(b[S % kRing], q, scale_value(en[I]));
#pragma unroll
          for (int j = 0; j < FM; ++j) sum[I][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bv, wide[j][q], sum[I][j], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int j = 0; j < FM; ++j)
          sum[I][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b[S % kRing], a[H][j], sum[I][j], 0, 0, 0, (int)en[I], 0, (int)em[j]);
      }
      if constexpr (kSteps == 2) ahead();
    });
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (decltype(more)::value) {
#pragma unroll
      for (int f = 0; f < FM; ++f) em[f] = next_m[f];
#pragma unroll
      for (int f = 0; f < FN; ++f) en[f] = next_n[f];
    }
  };
  // Results of 32 m x 32 FN n through the wave's own piece of LDS: element e of a lane is n = 8 (e / 4) + 4 (lane / 32) + e % 4, m = lane % 32.
  auto store_rows = [&](int64_t mw, int64_t nw, U* y, auto fragment) {
    constexpr int J = decltype(fragment)::value;
    constexpr int kPerPass = sizeof(U) == 4 ? (FN + 1) / 2 : FN;                    // fragments that fit
    constexpr int kRow = kPerPass * 32 * (int)sizeof(U) + 16, kPieces = kPerPass * 32 * (int)sizeof(U) / 16, kIn = 16 / (int)sizeof(U);
    static_assert(kRow <= 256 + 16 && 64 % kPieces == 0);
    uint8_t* room = stages + (STAGES - 1) * kStage + wave * (32 * kRow);
    const int rows_left = (int)min(p.M - mw, (int64_t)32), cols_left = (int)min(p.N - nw, (int64_t)(32 * FN));
    if (rows_left <= 0 || cols_left <= 0) return;
    // columns beyond the matrix read zeros
    const auto bias = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(p.bias + (p.bias ? nw : 0)), 0, 4 * cols_left, 0x00020000);
    static_for<0, FN / kPerPass>([&](auto pass) {
      constexpr int I0 = decltype(pass)::value * kPerPass;
      __builtin_amdgcn_sched_barrier(0);
      static_for<0, kPerPass * 4>([&](auto quarter) {
        constexpr int I = I0 + decltype(quarter)::value / 4, Q = decltype(quarter)::value % 4;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = sum[I][J][4 * Q + e];
        if (p.bias) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            v[e] += bits_float((uint32_t)__builtin_amdgcn_raw_buffer_load_b32(bias, 16 * (lane / 32) + 4 * (32 * I + 8 * Q + e), 0, 0));
        }
        store_floats<U, 4, true>(reinterpret_cast<U*>(room + (lane % 32) * kRow) + 32 * (I - I0) + 8 * Q + 4 * (lane / 32), 4, v);
      });
      __builtin_amdgcn_sched_barrier(0);
      const int piece = lane % kPieces, left = cols_left - 32 * I0 - kIn * piece;
      int row = lane / kPieces;
      U* to = y + (mw + row) * p.y_stride + nw + 32 * I0 + kIn * piece;
      const uint8_t* from = room + row * kRow + 16 * piece;
      // pieces of 16 bytes wherever a row starts: memory is written from any byte (4100 x 3001 x 512 bfloat16 15.4 us, element by element 31.6)
      if (cols_left == 32 * FN && rows_left == 32) {
#pragma unroll 4
        for (int r = 0; r < 32 * kPieces / 64; ++r) {
          if constexpr (PAST) store_past<true>(reinterpret_cast<u32x4_t*>(to), *reinterpret_cast<const u32x4_t*>(from));
          else __builtin_memcpy(to, __builtin_assume_aligned(from, 16), 16);
          to += (64 / kPieces) * p.y_stride;
          from += (64 / kPieces) * kRow;
        }
      } else {
#pragma unroll 1
        for (; row < rows_left; row += 64 / kPieces) {
          if (left >= kIn) {
            __builtin_memcpy(to, __builtin_assume_aligned(from, 16), 16);
          } else {
#pragma unroll 1
            for (int e = 0; e < min(kIn, left); ++e) to[e] = reinterpret_cast<const U*>(from)[e];
          }
          to += (64 / kPieces) * p.y_stride;
          from += (64 / kPieces) * kRow;
        }
      }
    });
  };

  int item = blockIdx.x;
  take(item);
  for (int i = 0; i < STAGES - 1; ++i) load(first + i);
  while (true) {
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
      for (int j = 0; j < FM; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) sum[i][j][e] = 0.0f;
    dma_wait<0>();
    __syncthreads();
    load(first + STAGES - 1);
    fetch_scales(first, em, en);
    fetch(stages, std::integral_constant<int, 0>());
    fetch(stages, std::integral_constant<int, 1>());
    for (int k = first; k + 1 < last; ++k) block(k, std::true_type());
    block(last - 1, std::false_type());
    dma_wait<0>();                                        // the empty loads behind the last block write zeros: they have to be there
    __syncthreads();                                      // before the stages are used again, and all stages have been read
    const int64_t mw = m0 + wm * FM * 32, nw = n0 + wn * FN * 32;
    U* y = (U*)p.y + (int64_t)part * p.M * p.N;
    item += gridDim.x;
    if (item < items) {
      take(item);
      for (int i = 0; i < STAGES - 1; ++i) load(first + i);
    }
    static_for<0, FM>([&](auto j) { store_rows(mw + 32 * decltype(j)::value, nw, y, j); });
    if (item >= items) return;
  }
}

// `parts` > 1: float32 results of every part
template <int TM, int TN, int WM, int WN, int STAGES, bool EXACT, bool PAST, typename U>
hipError_t tile_launch(const ProductParams& p, int parts, hipStream_t s) {
  const int64_t items = ((p.M + TM - 1) / TM) * ((p.N + TN - 1) / TN) * parts;
  auto* kernel = product_tile_kernel<TM, TN, WM, WN, STAGES, EXACT, PAST, U>;
  constexpr int lds = tile_lds(TM, TN, WM * WN, STAGES);
  constexpr int at_once = kFittedUnits * (160 * 1024 / lds);       // workgroups that the LDS holds
  static const hipError_t room = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (room != hipSuccess) return room;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(items < at_once ? items : at_once)), dim3(64 * WM * WN), lds, s, p, parts);
  return hipGetLastError();
}

// sums of the parts, in their order; four n a thread where the rows allow it
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void join_kernel(const ProductParams p, int parts) {
  constexpr int E = VEC ? 4 : 1;
  const int64_t per_row = (p.N + E - 1) / E, all = p.M * per_row, step = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += step) {
    const int64_t m = i / per_row, n = (i - m * per_row) * E;
    float v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = p.bias ? p.bias[n + e] : 0.0f;
    const float* from = p.partial + m * p.N + n;
    for (int first = 0; first < parts; first += 8) {      // eight loads on their way, their sums in order
      float t[8][E];
#pragma unroll
      for (int q = 0; q < 8; ++q) load_floats<float, E, VEC>(from + min(first + q, parts - 1) * (p.M * p.N), E, t[q]);
#pragma unroll
      for (int q = 0; q < 8; ++q)
        if (first + q < parts) {
#pragma unroll
          for (int e = 0; e < E; ++e) v[e] += t[q][e];
        }
    }
    T* to = (T*)p.y + m * p.y_stride + n;
    if constexpr (VEC) store_floats<T, 4, true>(to, 4, v);
    else *to = (T)v[0];
  }
}

// a tile with results of type T
template <typename T, int TM, int TN, int WM, int WN, int STAGES>
hipError_t tiles(const ProductParams& p, int parts, hipStream_t s) {
  constexpr bool exact = sizeof(T) == 4;
  if constexpr (TM == 256)
    if (parts == 1 && p.wide_stores && streamed(p.M * p.N * (int64_t)sizeof(T))) return tile_launch<TM, TN, WM, WN, STAGES, exact, true, T>(p, 1, s);
  if (parts == 1) return tile_launch<TM, TN, WM, WN, STAGES, exact, false, T>(p, 1, s);
  ProductParams q = p;
  q.y = p.partial;
  q.y_stride = p.N;
  q.bias = nullptr;
  const hipError_t e = tile_launch<TM, TN, WM, WN, STAGES, exact, false, float>(q, parts, s);
  if (e != hipSuccess) return e;
  const bool vec = p.N % 4 == 0 && p.wide_stores;
  const int64_t work = (p.M * ((p.N + 3) / 4) + 255) / 256;
  const dim3 grid((unsigned)(work < 8192 ? work : 8192));
  if (vec) hipLaunchKernelGGL((join_kernel<T, true>), grid, dim3(256), 0, s, p, parts);
  else hipLaunchKernelGGL((join_kernel<T, false>), grid, dim3(256), 0, s, p, parts);
  return hipGetLastError();
}

hipError_t launch_plan(const ProductPlan& plan, const ProductParams& p, hipStream_t s) {
  if (p.bf16) switch (plan.tile) {
    case 0: return tiles<bf16, 256, 256, 4, 2, 2>(p, plan.parts, s);
    case 1: return tiles<bf16, 128, 128, 2, 2, 4>(p, plan.parts, s);
    case 2: return tiles<bf16, 128, 128, 2, 2, 2>(p, plan.parts, s);
    case 4: return tiles<bf16, 64, 64, 2, 1, 2>(p, plan.parts, s);
    case 5: return tiles<bf16, 64, 64, 2, 1, 4>(p, plan.parts, s);
    case 6: return tiles<bf16, 64, 64, 2, 2, 4>(p, plan.parts, s);
    default: return tiles<bf16, 64, 32, 2, 1, 8>(p, plan.parts, s);
  }
  switch (plan.tile) {
    case 0: return tiles<float, 256, 256, 4, 2, 2>(p, plan.parts, s);
    case 2: return tiles<float, 128, 128, 2, 2, 2>(p, plan.parts, s);
    case 3: return tiles<float, 128, 64, 2, 2, 2>(p, plan.parts, s);
    default: return tiles<float, 64, 64, 2, 2, 2>(p, plan.parts, s);
  }
}

ProductPlan plan_of(int64_t M, int64_t N, int64_t K, int bf) {
  static thread_local PlanMemo<4, ProductPlan> memo;      // a call asks twice, and the estimates take a microsecond
  return *memo.of({(int)M, (int)N, (int)K, bf}, [&](ProductPlan& q) {
    q = choose_product_plan(M, N, K, bf);
    return true;
  });
}

}  // namespace

size_t product_workspace(int64_t M, int64_t N, int64_t K, int bf) {
  const ProductPlan plan = plan_of(M, N, K, bf);
  return plan.parts > 1 ? (size_t)plan.parts * (size_t)M * (size_t)N * sizeof(float) : 0;
}

hipError_t product_launch(const ProductParams& given, hipStream_t s) {
  ProductParams p = given;
  p.wide_stores = rows_aligned(p.y, p.y_stride, p.bf16 ? 2 : 4);
  return launch_plan(plan_of(p.M, p.N, p.K, p.bf16), p, s);
}

}  // namespace tac
