// Norm of every head of queries and keys and the rotation by position, and the backward pass.
//
// Memory-bound: every head is read once into registers and written from them.  A lane holds four pairs of features, both features of each, so that a pair is turned
// without another lane; 8 to 64 lanes share a head, whose sum of squares is three to six exchanges.
// An angle is position * base^(-i / n) in turns: formed in 64 bits and brought to the nearest turn there, sine and cosine are float32 from then on.  That costs
// some fifty instructions a pair, so a lane turns several heads of a row by the angles it has, and the next heads are read meanwhile (before: 177 us for the first case).
// 16384 rows of 24 heads of 128 bf16: 44 us (201 MB, 4.6 TB/s), backwards 58 (302 MB, 5.2 TB/s) and 4.6 for the gains' sums.  65536 rows of 18 heads, a quarter rotated:
// 141 us (604 MB, 4.3 TB/s).  16 rows of 24 heads: 5.1, of which the launch is some 3 and the rest the way from a position to its angle, 64-bit operations one after the other.
#include "tac_delta_common.h"

namespace tac {

namespace {

constexpr int kPairs = 4;            // of a lane
constexpr int kAtOnce = 4;           // heads whose loads are on their way together

// The two features of pair p: rotated pairs first, then what is left, paired half a remainder apart.
__device__ __forceinline__ int feature_of(const HeadNormParams& p, int pair, int second) {
  if (p.interleaved) return 2 * pair + second;
  const int rest = p.D / 2 - p.rotated;
  return pair < p.rotated ? pair + second * p.rotated : 2 * p.rotated + (pair - p.rotated) + second * rest;
}

// The first pair of a lane, and how many it has.
__device__ __forceinline__ int pairs_of(const HeadNormParams& p, int lane, int& count) {
  const int begin = p.apart ? (p.rotated + kPairs - 1) / kPairs : 0;      // lanes before the others' first
  const bool rotated = !p.apart || lane < begin;
  const int pair = rotated ? kPairs * lane : p.rotated + kPairs * (lane - begin), end = p.apart && rotated ? p.rotated : p.D / 2;
  count = min(max(end - pair, 0), kPairs);
  return pair;
}

// How a lane's eight features are read and written, in pieces at any address:
//   QUADS  the first and the second ones of its pairs are four neighbours each, all there or none     LOOSE_QUADS  some lanes have fewer than four pairs
//   ROW    all eight are neighbours, all there or none (interleaved)                                   LOOSE_ROW    the last lane has fewer
//   EACH   feature by feature: heads too short for a piece, and those of both kinds of pairs on a lane
// A loose piece is read so that it lies within the head, its features moved to their places; of a lane with fewer pairs each feature is written by itself.
enum { EACH, QUADS, ROW, LOOSE_QUADS, LOOSE_ROW };

template <int MODE>
struct Lane {
  static constexpr bool row = MODE == ROW || MODE == LOOSE_ROW, loose = MODE == LOOSE_QUADS || MODE == LOOSE_ROW;
  int at[2 * kPairs];                // features: the pairs' first ones, then their second ones (row: in their order); what is not there: 0
  int count;                         // pairs that there are
  double turns[kPairs];              // per unit of position
  int axis[kPairs];                  // -1: not rotated

  __device__ Lane(const HeadNormParams& p, int lane) {
    const int first_pair = pairs_of(p, lane, count);
    double part[kPairs];             // of the axis's pairs, those before this one
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
      const int pair = first_pair + j;
#pragma unroll
      for (int second = 0; second < 2; ++second) at[row ? 2 * j + second : j + kPairs * second] = j < count ? feature_of(p, pair, second) : 0;
      axis[j] = -1;
      part[j] = 0.0;
      int begin = 0;
#pragma unroll
      for (int a = 0; a < TAC_ROTATION_AXES; ++a) {
        if (a < p.axes && j < count && pair >= begin && pair < begin + p.pairs[a]) {
          axis[j] = a;
          part[j] = (double)(pair - begin) * p.log2_step[a];
        }
        begin += p.pairs[a];
      }
    }
#pragma unroll
    for (int j = 0; j < kPairs; ++j) turns[j] = exp2(-part[j]) * 0.15915494309189533577;      // 1 / (2 pi); four at once, not one in each branch
  }
  __device__ __forceinline__ int first(int j) const { return row ? 2 * j : j; }
  __device__ __forceinline__ int second(int j) const { return row ? 2 * j + 1 : j + kPairs; }

  __device__ __forceinline__ void angles(const HeadNormParams& p, int64_t row, float (&c)[kPairs], float (&s)[kPairs]) const {
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
      c[j] = 1.0f;
      s[j] = 0.0f;
      if (axis[j] >= 0) {
        const double t = (double)p.positions[row * p.axes + axis[j]] * turns[j];
        sincospif(2.0f * (float)(t - rint(t)), &s[j], &c[j]);
      }
    }
  }
  // without branches: a lane behind the last pair reads the head's first ones, and has zeros in their place
  template <typename T>
  __device__ __forceinline__ void load(const T* x, Piece<T, 8>& v, int D) const {
    if constexpr (row) {
      __builtin_memcpy(v.w, x + (loose ? min(at[0], D - 8) : at[0]), 8 * sizeof(T));
    } else if constexpr (MODE != EACH) {
      __builtin_memcpy(v.w, x + (loose ? min(at[0], D - 4) : at[0]), 4 * sizeof(T));
      __builtin_memcpy(&v.w[sizeof(v.w) / sizeof(v.w[0]) / 2], x + (loose ? min(at[4], D - 4) : at[4]), 4 * sizeof(T));
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v.set(e, x[at[e]]);
    }
  }
  template <typename T>
  __device__ __forceinline__ void values(const Piece<T, 8>& x, float (&v)[2 * kPairs], int D) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = value_of(x, e);
    if constexpr (loose) {
      // towards the front by what the piece was read too early: 0 .. 3 of four, 0 .. 7 of eight features
      constexpr int N = row ? 8 : 4;
#pragma unroll
      for (int q = 0; q < 8; q += N) {
        const int by = at[q] - min(at[q], D - N);
#pragma unroll
        for (int step = 1; step < N; step *= 2) {
#pragma unroll
          for (int e = 0; e < N; ++e) v[q + e] = by & step ? (e + step < N ? v[q + e + step] : 0.0f) : v[q + e];
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = count > (row ? e / 2 : e % kPairs) ? v[e] : 0.0f;
  }
  template <bool PAST, typename T>
  __device__ __forceinline__ void store(T* y, const float (&v)[2 * kPairs]) const {
    if (MODE != EACH && count == kPairs) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        T* const to = row ? y + at[0] + 4 * half : y + at[4 * half];
        const float* const w = v + 4 * half;
        if constexpr (sizeof(T) == 4) {
          const f32x4_t x = {w[0], w[1], w[2], w[3]};
          if constexpr (PAST) __builtin_nontemporal_store(x, reinterpret_cast<f32x4_t*>(to));
          else __builtin_memcpy(to, &x, 16);
        } else {
          const u32x2_t x = {pack_bf16(w[0], w[1]), pack_bf16(w[2], w[3])};
          if constexpr (PAST) __builtin_nontemporal_store(x, reinterpret_cast<u32x2_t*>(to));
          else __builtin_memcpy(to, &x, 8);
        }
      }
    } else if (MODE == EACH || loose) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (count > (row ? e / 2 : e % kPairs)) y[at[e]] = (T)v[e];
    }
  }
  __device__ __forceinline__ void gains(const float* gain, float (&v)[2 * kPairs]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = gain && count > (row ? e / 2 : e % kPairs) ? gain[at[e]] : 1.0f;
  }
};

// whatever the order that they are read in, features are summed in this one: results do not depend on addresses
template <int MODE>
__device__ __forceinline__ constexpr int in_order(int e) { return Lane<MODE>::row ? 2 * (e % kPairs) + e / kPairs : e; }

// Where a lane group is: slices of rows one after the other, of each the heads some at once.  The next ones are read while these are worked on.
template <int LANES, int AT_ONCE>
struct Walk {
  uint32_t unit, row;
  int slice, begin;
  __device__ __forceinline__ Walk() : unit(blockIdx.x * (256 / LANES) + threadIdx.x / LANES) {}
  __device__ __forceinline__ void enter(const HeadNormParams& p) {
    row = unit / (uint32_t)p.slices;
    slice = (int)(unit - row * (uint32_t)p.slices);
    begin = slice;
  }
  __device__ __forceinline__ bool more(const HeadNormParams& p) const { return unit < (uint32_t)p.rows * (uint32_t)p.slices; }
  __device__ __forceinline__ int head(const HeadNormParams& p, int i) const { return begin + i * p.slices; }
  __device__ __forceinline__ void next(const HeadNormParams& p, int heads) {
    begin += AT_ONCE * p.slices;
    if (begin < heads) return;
    unit += gridDim.x * (256 / LANES);
    enter(p);
  }
};

// where head h of a row stands, of queries and keys; F: which of the tensors
enum { X, GRAD_OUT, OUT };
template <int F, typename T>
__device__ __forceinline__ T* head_at(const HeadNormParams& p, uint32_t row, int h) {
  const bool key = h >= p.q.heads;
  const auto& s = F == X ? (key ? p.k.x_stride : p.q.x_stride) : F == GRAD_OUT ? (key ? p.k.grad_out_stride : p.q.grad_out_stride) : key ? p.k.out_stride : p.q.out_stride;
  const void* base = F == X ? (key ? p.k.x : p.q.x) : F == GRAD_OUT ? (key ? p.k.grad_out : p.q.grad_out) : key ? p.k.out : p.q.out;
  return (T*)base + (int64_t)row * s.row + (int64_t)(key ? h - p.q.heads : h) * s.head;
}

template <typename T, int LANES, int MODE, bool PAST>
__global__ __launch_bounds__(256) void head_norm_kernel(const HeadNormParams p) {
  const Lane<MODE> lane(p, threadIdx.x % LANES);
  float gain[2][8];
  lane.gains(p.q.gain, gain[0]);
  lane.gains(p.k.gain, gain[1]);
  const int heads = p.q.heads + p.k.heads;
  Walk<LANES, kAtOnce> here;
  if (!here.more(p)) return;
  Piece<T, 8> x[kAtOnce];
  const auto read = [&](const Walk<LANES, kAtOnce>& w) {
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) lane.load(head_at<X, const T>(p, w.row, min(w.head(p, i), heads - 1)), x[i], p.D);
  };
  here.enter(p);
  read(here);
  float c[kPairs], s[kPairs];
  while (true) {
    float v[kAtOnce][8];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) lane.values(x[i], v[i], p.D);
    if (here.begin == here.slice) lane.angles(p, here.row, c, s);
    Walk<LANES, kAtOnce> ahead = here;
    ahead.next(p, heads);
    const bool more = ahead.more(p);
    if (more) read(ahead);
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int h = here.head(p, i);
      if (h >= heads) break;
      float squares = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) squares = fmaf(v[i][in_order<MODE>(e)], v[i][in_order<MODE>(e)], squares);
      const float rstd = p.eps > 0.0f ? 1.0f / sqrtf(sum_over_lanes<LANES>(squares) / (float)p.D + p.eps) : 1.0f;
      const bool key = h >= p.q.heads;
      float y[8];
#pragma unroll
      for (int j = 0; j < kPairs; ++j) {
        const int f = lane.first(j), g = lane.second(j);
        const float a = v[i][f] * rstd * (key ? gain[1][f] : gain[0][f]), b = v[i][g] * rstd * (key ? gain[1][g] : gain[0][g]);
        y[f] = lane.axis[j] >= 0 ? fmaf(a, c[j], -(b * s[j])) : a;       // a NaN beside a feature that is not turned stays where it is
        y[g] = lane.axis[j] >= 0 ? fmaf(b, c[j], a * s[j]) : b;
      }
      lane.template store<PAST>(head_at<OUT, T>(p, here.row, h), y);
    }
    if (!more) return;
    here = ahead;
  }
}

// The gains' gradients stay in a lane's registers over all heads that it takes, are added up over the workgroup in LDS and leave as a row of the
// workspace [workgroup][queries, keys][8 LANES]; head_gain_kernel adds those up in their order.
template <typename T, int LANES, int MODE, bool PAST>
__global__ __launch_bounds__(256) void head_norm_backward_kernel(const HeadNormParams p) {
  constexpr int AT_ONCE = kAtOnce / 2;
  __shared__ float room[256 * 8];
  const Lane<MODE> lane(p, threadIdx.x % LANES);
  float gain[2][8], sums[2][8];
  lane.gains(p.q.gain, gain[0]);
  lane.gains(p.k.gain, gain[1]);
#pragma unroll
  for (int e = 0; e < 8; ++e) sums[0][e] = sums[1][e] = 0.0f;
  const int heads = p.q.heads + p.k.heads;
  Walk<LANES, AT_ONCE> here;
  Piece<T, 8> x[AT_ONCE], dy[AT_ONCE];
  const auto read = [&](const Walk<LANES, AT_ONCE>& w) {
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const int h = min(w.head(p, i), heads - 1);
      lane.load(head_at<X, const T>(p, w.row, h), x[i], p.D);
      lane.load(head_at<GRAD_OUT, const T>(p, w.row, h), dy[i], p.D);
    }
  };
  bool more = here.more(p);
  if (more) {
    here.enter(p);
    read(here);
  }
  float c[kPairs], s[kPairs];
  while (more) {
    float v[AT_ONCE][8], d[AT_ONCE][8];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      lane.values(x[i], v[i], p.D);
      lane.values(dy[i], d[i], p.D);
    }
    if (here.begin == here.slice) lane.angles(p, here.row, c, s);
    Walk<LANES, AT_ONCE> ahead = here;
    ahead.next(p, heads);
    more = ahead.more(p);
    if (more) read(ahead);
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const int h = here.head(p, i);
      if (h >= heads) break;
      const bool key = h >= p.q.heads;
      float rstd = 1.0f;
      if (p.eps > 0.0f) {
        float squares = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) squares = fmaf(v[i][in_order<MODE>(e)], v[i][in_order<MODE>(e)], squares);
        rstd = 1.0f / sqrtf(sum_over_lanes<LANES>(squares) / (float)p.D + p.eps);
      }
      float w[8], dot = 0.0f;
#pragma unroll
      for (int j = 0; j < kPairs; ++j) {
        const int f = lane.first(j), g = lane.second(j);
        w[f] = lane.axis[j] >= 0 ? fmaf(d[i][f], c[j], d[i][g] * s[j]) : d[i][f];
        w[g] = lane.axis[j] >= 0 ? fmaf(d[i][g], c[j], -(d[i][f] * s[j])) : d[i][g];
      }
#pragma unroll
      for (int m = 0; m < 8; ++m) {
        const int e = in_order<MODE>(m);
        v[i][e] *= rstd;
        const float one = w[e] * v[i][e];
        if (key) sums[1][e] += one;
        else sums[0][e] += one;
        w[e] *= key ? gain[1][e] : gain[0][e];
        dot = fmaf(w[e], v[i][e], dot);
      }
      if (p.eps > 0.0f) {
        const float mean = sum_over_lanes<LANES>(dot) / (float)p.D;
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = rstd * (w[e] - v[i][e] * mean);
      }
      lane.template store<PAST>(head_at<OUT, T>(p, here.row, h), w);
    }
    here = ahead;
  }
  if (!p.partial) return;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    __syncthreads();                        // the tensor before has been read
#pragma unroll
    for (int e = 0; e < 8; ++e) room[e * 256 + threadIdx.x] = sums[t][e];
    __syncthreads();
    for (int slot = threadIdx.x; slot < 8 * LANES; slot += 256) {
      const int e = slot / LANES, l = slot % LANES;
      float total = 0.0f;
#pragma unroll
      for (int g = 0; g < 256 / LANES; ++g) total += room[e * 256 + g * LANES + l];
      p.partial[((int64_t)blockIdx.x * 2 + t) * (8 * LANES) + slot] = total;
    }
  }
}

// Sums of partial [groups][2][8 LANES]: 16 slots and 16 slices of the groups a workgroup, then the slices in their order.
template <int MODE>
__global__ __launch_bounds__(256) void head_gain_kernel(const HeadNormParams p, int groups, int lanes) {
  __shared__ float room[16][16];
  const int slot = blockIdx.x * 16 + threadIdx.x % 16, slice = threadIdx.x / 16, t = blockIdx.y, slots = 8 * lanes;
  float total = 0.0f;
#pragma unroll 8
  for (int g = slice; g < groups; g += 16) total += p.partial[((int64_t)g * 2 + t) * slots + slot];
  room[slice][threadIdx.x % 16] = total;
  __syncthreads();
  if (slice) return;
#pragma unroll
  for (int s = 1; s < 16; ++s) total += room[s][threadIdx.x % 16];
  constexpr bool row = Lane<MODE>::row;
  int count;
  const int e = slot / lanes, j = row ? e / 2 : e % kPairs, pair = pairs_of(p, slot % lanes, count) + j, second = row ? e % 2 : e / kPairs;
  float* to = t ? p.grad_gain_k : p.grad_gain_q;
  if (to && j < count) to[feature_of(p, pair, second)] = total;
}

bool pieces_aligned(const void* at, const tac_head_strides_t& s, size_t piece, size_t el) {
  return !at || (((uintptr_t)at | (uintptr_t)(s.row * (int64_t)el) | (uintptr_t)(s.head * (int64_t)el)) & (piece - 1)) == 0;
}

int mode_of(const HeadNormParams& p) {
  if (p.interleaved) return p.D % 8 == 0 ? ROW : p.D > 8 ? LOOSE_ROW : EACH;
  if (!p.apart || p.D < 4) return EACH;
  return p.rotated % kPairs == 0 && (p.D / 2 - p.rotated) % kPairs == 0 ? QUADS : LOOSE_QUADS;
}

// lanes, slices and the way past the caches: large results whose pieces start where stores of their size may
void lay_out(HeadNormParams& p, int& lanes, bool& past) {
  const HeadLanes l = head_lanes(p.D, p.interleaved ? p.D / 2 : p.rotated);
  const size_t el = p.bf16 ? 2 : 4;
  lanes = l.lanes;
  p.apart = l.apart && !p.interleaved;
  p.slices = head_slices(p.rows, p.q.heads + p.k.heads, lanes);
  past = streamed(p.rows * (p.q.heads + p.k.heads) * p.D * (int64_t)el) && pieces_aligned(p.q.out, p.q.out_stride, 4 * el, el) &&
         (!p.k.heads || pieces_aligned(p.k.out, p.k.out_stride, 4 * el, el));
  const int mode = mode_of(p);
  past &= mode == QUADS || mode == ROW;
}

// f(lanes, mode, past) with all as constants
template <typename F>
hipError_t by_shape(const HeadNormParams& p, int lanes, bool past, F f) {
  using std::integral_constant;
  const auto with = [&](auto l) {
    const std::false_type here;
    const std::true_type beyond;
    switch (mode_of(p)) {
      case QUADS: return past ? f(l, integral_constant<int, QUADS>(), beyond) : f(l, integral_constant<int, QUADS>(), here);
      case ROW: return past ? f(l, integral_constant<int, ROW>(), beyond) : f(l, integral_constant<int, ROW>(), here);
      case LOOSE_QUADS: return f(l, integral_constant<int, LOOSE_QUADS>(), here);
      case LOOSE_ROW: return f(l, integral_constant<int, LOOSE_ROW>(), here);
      default: return f(l, integral_constant<int, EACH>(), here);
    }
  };
  switch (lanes) {
    case 8: return with(integral_constant<int, 8>());
    case 16: return with(integral_constant<int, 16>());
    case 32: return with(integral_constant<int, 32>());
    default: return with(integral_constant<int, 64>());
  }
}

}  // namespace

hipError_t head_norm_launch(const HeadNormParams& given, hipStream_t s) {
  HeadNormParams p = given;
  int lanes;
  bool past;
  lay_out(p, lanes, past);
  const unsigned groups = (unsigned)head_groups(p.rows, p.slices, lanes, kHeadGroups);
  return by_shape(p, lanes, past, [&](auto l, auto m, auto beyond) {
    constexpr int L = decltype(l)::value, M = decltype(m)::value;
    constexpr bool PAST = decltype(beyond)::value;
    if (p.bf16) hipLaunchKernelGGL((head_norm_kernel<bf16, L, M, PAST>), dim3(groups), dim3(256), 0, s, p);
    else hipLaunchKernelGGL((head_norm_kernel<float, L, M, PAST>), dim3(groups), dim3(256), 0, s, p);
    return hipGetLastError();
  });
}

size_t head_norm_workspace(const HeadNormParams& given) {
  HeadNormParams p = given;
  int lanes;
  bool past;
  lay_out(p, lanes, past);
  return (size_t)head_groups(p.rows, p.slices, lanes, kHeadBackwardGroups) * 2 * 8 * (size_t)lanes * sizeof(float);
}

hipError_t head_norm_backward_launch(const HeadNormParams& given, hipStream_t s) {
  HeadNormParams p = given;
  int lanes;
  bool past;
  lay_out(p, lanes, past);
  const unsigned groups = (unsigned)head_groups(p.rows, p.slices, lanes, kHeadBackwardGroups);
  if (!p.grad_gain_q && !p.grad_gain_k) p.partial = nullptr;
  return by_shape(p, lanes, past, [&](auto l, auto m, auto beyond) {
    constexpr int L = decltype(l)::value, M = decltype(m)::value;
    constexpr bool PAST = decltype(beyond)::value;
    if (p.bf16) hipLaunchKernelGGL((head_norm_backward_kernel<bf16, L, M, PAST>), dim3(groups), dim3(256), 0, s, p);
    else hipLaunchKernelGGL((head_norm_backward_kernel<float, L, M, PAST>), dim3(groups), dim3(256), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !p.partial) return e;
    hipLaunchKernelGGL((head_gain_kernel<M>), dim3(L / 2, p.k.heads ? 2 : 1), dim3(256), 0, s, p, (int)groups, L);
    return hipGetLastError();
  });
}

}  // namespace tac
