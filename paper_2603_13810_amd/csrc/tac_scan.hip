// Gated linear recurrence h_t = a_t h_{t-1} + (1 - a_t) value_t with a_t = 1 / (1 + exp(-gate_t)), its backward pass, and one step of it
// on a pool of states.
//
// Memory-bound: six bytes a channel and step forwards in bfloat16, ten backwards, against some 25 vector instructions.  Steps in a row are
// an affine map h -> A h + H, and two such maps in a row are one, so time is cut as the hardware wants it: a wave takes kChunk steps of 64 lanes'
// channels into registers, forms its map, the waves of a workgroup pass theirs through LDS, and each goes over its steps once
// more, in registers, from the state that it now knows.  Inputs are read once and outputs written once.  Where the channels are too few for
// the chip, workgroups share the length as well: a launch that only forms the maps of the parts, then one that starts every part from those before it.
#include "tac_head_common.h"
#include "tac_scan_plan.h"

namespace tac {

namespace {

constexpr int kChunk = TAC_SCAN_CHUNK;       // steps of a wave
constexpr int kWaves = kScanWaves;

// w = min(a, 1 - a) = 1 / (1 + exp(|gate|)), negative (as -0 too) where a is the smaller.  Updates are written around the nearer of the two ends,
//   a >= 1/2:  h' = h + w (value - h)        a < 1/2:  h' = value - w (value - h)
// so that a leak of nearly 1 does not lose the digits of 1 - a: a itself rounded to float32 leaves 1e-6 in states that remember a thousand steps.
__device__ __forceinline__ float leak(float gate) {
  const float e = __expf(-fabsf(gate));
  const float w = e * __builtin_amdgcn_rcpf(1.0f + e);
  return gate < 0.0f ? -w : w;               // a NaN stays one
}
__device__ __forceinline__ bool forgets(float s) { return (int)float_bits(s) < 0; }
__device__ __forceinline__ float step_state(float s, float h, float u) { return fmaf(s, u - h, forgets(s) ? u : h); }
__device__ __forceinline__ float times_a(float s, float x) { return fmaf(-s, x, forgets(s) ? 0.0f : x); }

// Those forms turn an infinity into inf - inf, and the difference of two values near float32's largest into an infinity; maps multiply infinities
// by factors that have become 0.  What is infinite or NaN stays one of the two in them, step by step and map by map, so that a look at the end of every
// chunk finds it.  The steps of such a channel are then taken again one after the other by the formula as it stands wherever the form above is not
// finite: an infinity goes on as a h + (1 - a) value says, NaN where float32 has its factor as 0.  (Not where outputs have taken the inputs' place.)
__device__ __forceinline__ bool finite(float v) { return fabsf(v) < __builtin_inff(); }
__device__ __forceinline__ float a_of(float s) { return forgets(s) ? fabsf(s) : 1.0f - fabsf(s); }
__device__ __forceinline__ float rest_of(float s) { return forgets(s) ? 1.0f - fabsf(s) : fabsf(s); }
__device__ __forceinline__ float careful_state(float s, float h, float u) {
  const float r = step_state(s, h, u);
  return finite(r) ? r : fmaf(a_of(s), h, rest_of(s) * u);
}
__device__ __forceinline__ float careful_times(float s, float x) {
  const float r = times_a(s, x);
  return finite(r) ? r : a_of(s) * x;
}

__device__ __forceinline__ int64_t length_of(const int32_t* lengths, int b, int64_t T) {
  return lengths ? min(max((int64_t)lengths[b], (int64_t)0), T) : T;
}

// V channels of a lane: one load of 4 bytes (two bfloat16 or one float32) or of 2
template <typename T, int V>
struct Lane {
  static_assert(sizeof(T) * V <= 4);
  using Raw = std::conditional_t<sizeof(T) * V == 4, uint32_t, uint16_t>;
  static __device__ __forceinline__ Raw load(const T* p) { return *reinterpret_cast<const Raw*>(p); }
  static __device__ __forceinline__ float value(Raw r, int e) {
    if constexpr (sizeof(T) == 4) return bits_float(r);
    else return bits_float(e ? (uint32_t)r & 0xffff0000u : (uint32_t)r << 16);
  }
  static __device__ __forceinline__ Raw pack(const float (&v)[V]) {
    if constexpr (sizeof(T) == 4) return float_bits(v[0]);
    else return (Raw)pack_bf16(v[0], v[V - 1]);
  }
  template <bool PAST>
  static __device__ __forceinline__ void store(T* p, Raw r) { store_past<PAST>(reinterpret_cast<Raw*>(p), r); }
  // a gate of +infinity: the step leaves the state as it is
  static constexpr Raw kKeep = (Raw)(sizeof(T) == 4 ? 0x7f800000u : 0x7f807f80u);
};

// Which channels and which part of the length a workgroup has.
struct Place {
  int b, d, tiles, first, last;      // sequence, the lane's first channel, tiles of the whole length, the part's tiles [first, last)
  bool on;
};
// first tile of a part, tiles part / parts in 32 bits (there are at most 512 parts)
__device__ __forceinline__ int part_from(int tiles, int part, int parts) { return tiles / parts * part + tiles % parts * part / parts; }
template <int V>
__device__ __forceinline__ Place place_of(int64_t T, int D) {
  const int per_b = (D + 64 * V - 1) / (64 * V), steps = (blockDim.x >> 6) * kChunk;
  Place q;
  q.b = blockIdx.x / per_b;
  q.d = ((blockIdx.x - q.b * per_b) * 64 + (threadIdx.x & 63)) * V;
  q.on = q.d < D;
  if (!q.on) q.d = 0;                // reads what is there, writes nothing
  q.tiles = (int)((T + steps - 1) / steps);
  q.first = part_from(q.tiles, blockIdx.y, gridDim.y);
  q.last = part_from(q.tiles, blockIdx.y + 1, gridDim.y);
  return q;
}

template <int V>
struct Map {                         // x -> a x + b
  float a[V], b[V];
};

// MAPS: only the map of the part, into workspace [part][2][B][D], from its last tile to its first (the tiles that the second launch starts with are
// then those that the caches have seen last).  The last part's is not needed: its place takes h0, from where every part of the second launch starts,
// since that launch writes h_last, which may be h0, in no order with its parts' reads.
// At most 128 registers, so that two workgroups share a compute unit (the walk behind the loop would let the compiler take 160).
template <typename T, int V, bool MAPS, bool PAST = false>
__global__ __launch_bounds__(64 * kWaves, 4) void scan_kernel(const ScanParams p) {
  using L = Lane<T, V>;
  __shared__ Map<V> maps[2][kWaves][64];
  __shared__ float starts[kWaves][V][64];      // what carry starts from, where it is asked for again: in memory the last state (gradient) may have its place
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const Place q = place_of<V>(p.T, p.D);
  const int64_t len = length_of(p.lengths, q.b, p.T), channels = (int64_t)p.B * p.D, n = (int64_t)q.b * p.D + q.d;
  const float* h0 = p.h0 && gridDim.y > 1 ? p.workspace + 2 * (gridDim.y - 1) * channels : p.h0;
  if (MAPS && blockIdx.y == gridDim.y - 1) {
    if (p.h0 && !wave && q.on) {
#pragma unroll
      for (int e = 0; e < V; ++e) p.workspace[2 * (gridDim.y - 1) * channels + n + e] = p.h0[n + e];
    }
    return;
  }
  const T *gate = (const T*)p.gate + q.b * p.in_b, *value = (const T*)p.value + q.b * p.in_b;
  T* out = (T*)p.out + q.b * p.out_b;
  typename L::Raw g[kChunk] = {}, u[kChunk] = {};
  auto load = [&](int tile) {
    const int64_t t0 = ((int64_t)tile * waves + wave) * kChunk;
    if (t0 >= len) return;
#pragma unroll
    for (int i = 0; i < kChunk; ++i) {         // behind the end the last step again; what it brings is replaced below
      const int64_t t = min(t0 + i, len - 1);
      g[i] = L::load(gate + t * p.in_t + q.d);
      u[i] = L::load(value + t * p.in_t + q.d);
    }
  };
  float carry[V], total[V];          // MAPS: the map of the tiles behind, else the state before the tile
  bool good[V];                      // nothing that is not finite so far
#pragma unroll
  for (int e = 0; e < V; ++e) {
    total[e] = 1.0f;
    good[e] = true;
    carry[e] = MAPS || !h0 ? 0.0f : h0[n + e];
    if constexpr (!MAPS) starts[wave][e][lane] = carry[e];
    if constexpr (!MAPS)
      for (int k = 0; k < (int)blockIdx.y; ++k)
        carry[e] = fmaf(p.workspace[2 * k * channels + n + e], carry[e], p.workspace[(2 * k + 1) * channels + n + e]);
  }
  load(MAPS ? q.last - 1 : q.first);
  for (int k = 0; k < q.last - q.first; ++k) {
    const int tile = MAPS ? q.last - 1 - k : q.first + k;
    const int64_t t0 = ((int64_t)tile * waves + wave) * kChunk;
    float s[kChunk][V];
    typename L::Raw x[kChunk];
    Map<V> mine;
    if (t0 + kChunk > len) {                   // steps behind the length keep the state
#pragma unroll
      for (int i = 0; i < kChunk; ++i)
        if (t0 + i >= len) {
          g[i] = L::kKeep;
          u[i] = 0;
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
      mine.a[e] = 1.0f;
      mine.b[e] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < kChunk; ++i) {
      x[i] = u[i];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        s[i][e] = leak(L::value(g[i], e));
        mine.b[e] = step_state(s[i][e], mine.b[e], L::value(x[i], e));
        mine.a[e] = times_a(s[i][e], mine.a[e]);
      }
    }
    maps[k & 1][wave][lane] = mine;
    if (k + 1 < q.last - q.first) load(MAPS ? tile - 1 : tile + 1);
    __syncthreads();                 // one a tile: what is written next is the other half, read before the barrier in between
    float h[V];
    if constexpr (MAPS) {
      for (int w = waves - 1; w >= 0; --w) {
        const Map<V> m = maps[k & 1][w][lane];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          carry[e] = fmaf(total[e], m.b[e], carry[e]);
          total[e] *= m.a[e];
        }
      }
    } else {
      for (int w = 0; w < waves; ++w) {
        const Map<V> m = maps[k & 1][w][lane];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          if (w == wave) h[e] = carry[e];
          carry[e] = fmaf(m.a[e], carry[e], m.b[e]);
        }
      }
      if (p.states && t0 < p.T && q.on) {
#pragma unroll
        for (int e = 0; e < V; ++e) p.states[t0 / kChunk * channels + n + e] = h[e];
      }
#pragma unroll
      for (int i = 0; i < kChunk; ++i) {
        float o[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          h[e] = step_state(s[i][e], h[e], L::value(x[i], e));
          o[e] = h[e];
        }
        x[i] = L::pack(o);
      }
#pragma unroll
      for (int e = 0; e < V; ++e) good[e] = good[e] && finite(h[e]);
      if (t0 + kChunk <= len) {
        if (q.on) {
#pragma unroll
          for (int i = 0; i < kChunk; ++i) L::template store<PAST>(out + (t0 + i) * p.out_t + q.d, x[i]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < kChunk; ++i)
          if (t0 + i < p.T && q.on) L::template store<PAST>(out + (t0 + i) * p.out_t + q.d, t0 + i < len ? x[i] : (typename L::Raw)0);
      }
    }
  }
  if constexpr (!MAPS) {             // channels that are not finite: every wave takes all steps and writes its own again
    const int64_t steps = (int64_t)waves * kChunk;
#pragma unroll 1
    for (int e = 0; e < V; ++e) {
      if (!q.on || !p.apart || ((e ? good[V - 1] : good[0]) && finite(e ? carry[V - 1] : carry[0]))) continue;
      float h = starts[wave][e][lane];
      int from = 0;                  // the first part that ends with something else than a number, or this one
      for (; from < (int)blockIdx.y; ++from) {
        const float next = fmaf(p.workspace[2 * from * channels + n + e], h, p.workspace[(2 * from + 1) * channels + n + e]);
        if (!finite(next)) break;
        h = next;
      }
      // a NaN makes all behind it NaN, and the steps have written that
      const int64_t first = q.first * steps, end = min(q.last * steps, len);
#pragma unroll 1
      for (int64_t t = part_from(q.tiles, from, gridDim.y) * steps; t < end && h == h; ++t) {
        const bool mine = t >= first && t / kChunk % waves == wave;
        if (mine && p.states && t % kChunk == 0) p.states[t / kChunk * channels + n + e] = h;
        h = careful_state(leak((float)gate[t * p.in_t + q.d + e]), h, (float)value[t * p.in_t + q.d + e]);
        if (mine) out[t * p.out_t + q.d + e] = (T)h;
      }
      // chunks behind the length
      if (p.states)
        for (int64_t c = max(q.first * (int64_t)waves, (len + kChunk - 1) / kChunk); c < min(q.last * (int64_t)waves, (p.T + kChunk - 1) / kChunk); ++c)
          if (c % waves == wave) p.states[c * channels + n + e] = h;
      (e ? carry[V - 1] : carry[0]) = h;
    }
  }
  if (wave || !q.on) return;
#pragma unroll
  for (int e = 0; e < V; ++e) {
    if constexpr (MAPS) {
      p.workspace[2 * blockIdx.y * channels + n + e] = total[e];
      p.workspace[(2 * blockIdx.y + 1) * channels + n + e] = carry[e];
    } else if (p.h_last && blockIdx.y == gridDim.y - 1) {
      p.h_last[n + e] = carry[e];
    }
  }
}

// The same backwards: the gradient c that arrives at a step's state obeys c <- a (c + grad_out).  With w = min(a, 1 - a) the gate's
// gradient is c w (1 - w) (h_{t-1} - value).  The states before the steps are formed again from the chunk's first, which the forward pass kept.
// Here the first part's map is not needed, and its place takes grad_h_last (which grad_h0 may be).
template <typename T, int V, bool MAPS, bool PAST = false>
__global__ __launch_bounds__(64 * kWaves) void scan_backward_kernel(const ScanBackwardParams p) {
  using L = Lane<T, V>;
  __shared__ Map<V> maps[2][kWaves][64];
  __shared__ float starts[kWaves][V][64];      // what carry starts from, where it is asked for again: in memory the last state (gradient) may have its place
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const Place q = place_of<V>(p.T, p.D);
  const int64_t len = length_of(p.lengths, q.b, p.T), channels = (int64_t)p.B * p.D, n = (int64_t)q.b * p.D + q.d;
  const float* last = p.grad_h_last && gridDim.y > 1 ? p.workspace : p.grad_h_last;
  if (MAPS && blockIdx.y == 0) {
    if (p.grad_h_last && !wave && q.on) {
#pragma unroll
      for (int e = 0; e < V; ++e) p.workspace[n + e] = p.grad_h_last[n + e];
    }
    return;
  }
  const T *gate = (const T*)p.gate + q.b * p.in_b, *value = (const T*)p.value + q.b * p.in_b, *grad_out = (const T*)p.grad_out + q.b * p.out_b;
  T *grad_gate = (T*)p.grad_gate + q.b * p.grad_b, *grad_value = (T*)p.grad_value + q.b * p.grad_b;
  typename L::Raw g[kChunk] = {}, u[kChunk] = {}, go[kChunk] = {};
  float first[V];                    // the state before the chunk
  auto load = [&](int tile) {
    const int64_t t0 = ((int64_t)tile * waves + wave) * kChunk;
#pragma unroll
    for (int e = 0; e < V; ++e) first[e] = !MAPS && t0 < p.T ? p.states[t0 / kChunk * channels + n + e] : 0.0f;
    if (t0 >= len) return;
#pragma unroll
    for (int i = 0; i < kChunk; ++i) {
      const int64_t t = min(t0 + i, len - 1);
      g[i] = L::load(gate + t * p.in_t + q.d);
      if constexpr (!MAPS) u[i] = L::load(value + t * p.in_t + q.d);
      go[i] = L::load(grad_out + t * p.out_t + q.d);
    }
  };
  float carry[V], total[V];
  bool good[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    total[e] = 1.0f;
    good[e] = true;
    carry[e] = MAPS || !last ? 0.0f : last[n + e];
    if constexpr (!MAPS) starts[wave][e][lane] = carry[e];
    if constexpr (!MAPS)
      for (int k = gridDim.y - 1; k > (int)blockIdx.y; --k)
        carry[e] = fmaf(p.workspace[2 * k * channels + n + e], carry[e], p.workspace[(2 * k + 1) * channels + n + e]);
  }
  load(MAPS ? q.first : q.last - 1);
  for (int k = 0; k < q.last - q.first; ++k) {
    const int tile = MAPS ? q.first + k : q.last - 1 - k;
    const int64_t t0 = ((int64_t)tile * waves + wave) * kChunk;
    float s[kChunk][V], before[kChunk][V];
    typename L::Raw x[kChunk], y[kChunk];
    Map<V> mine;
    if (t0 + kChunk > len) {
#pragma unroll
      for (int i = 0; i < kChunk; ++i)
        if (t0 + i >= len) {
          g[i] = L::kKeep;
          u[i] = go[i] = 0;
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
      mine.a[e] = 1.0f;
      mine.b[e] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < kChunk; ++i) {
      x[i] = u[i];
      y[i] = go[i];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        s[i][e] = leak(L::value(g[i], e));
        if constexpr (!MAPS) before[i][e] = i ? step_state(s[i - 1][e], before[i - 1][e], L::value(x[i - 1], e)) : first[e];
      }
    }
#pragma unroll
    for (int i = kChunk - 1; i >= 0; --i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        mine.b[e] = times_a(s[i][e], mine.b[e] + L::value(y[i], e));
        mine.a[e] = times_a(s[i][e], mine.a[e]);
      }
    maps[k & 1][wave][lane] = mine;
    if constexpr (!MAPS) {
#pragma unroll
      for (int e = 0; e < V; ++e) good[e] = good[e] && finite(before[kChunk - 1][e]);
    }
    if (k + 1 < q.last - q.first) load(MAPS ? tile + 1 : tile - 1);
    __syncthreads();
    float c[V];
    if constexpr (MAPS) {
      for (int w = 0; w < waves; ++w) {
        const Map<V> m = maps[k & 1][w][lane];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          carry[e] = fmaf(total[e], m.b[e], carry[e]);
          total[e] *= m.a[e];
        }
      }
    } else {
      for (int w = waves - 1; w >= 0; --w) {
        const Map<V> m = maps[k & 1][w][lane];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          if (w == wave) c[e] = carry[e];
          carry[e] = fmaf(m.a[e], carry[e], m.b[e]);
        }
      }
#pragma unroll
      for (int i = kChunk - 1; i >= 0; --i) {
        float dg[V], dv[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float w = fabsf(s[i][e]), now = c[e] + L::value(y[i], e);
          dv[e] = now * rest_of(s[i][e]);
          dg[e] = now * (w * (1.0f - w)) * (before[i][e] - L::value(x[i], e));
          c[e] = times_a(s[i][e], now);
        }
        x[i] = L::pack(dg);
        y[i] = L::pack(dv);
      }
#pragma unroll
      for (int e = 0; e < V; ++e) good[e] = good[e] && finite(c[e]);
      if (t0 + kChunk <= len) {
        if (q.on) {
#pragma unroll
          for (int i = 0; i < kChunk; ++i) {
            L::template store<PAST>(grad_gate + (t0 + i) * p.grad_t + q.d, x[i]);
            L::template store<PAST>(grad_value + (t0 + i) * p.grad_t + q.d, y[i]);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < kChunk; ++i)
          if (t0 + i < p.T && q.on) {
            const bool live = t0 + i < len;
            L::template store<PAST>(grad_gate + (t0 + i) * p.grad_t + q.d, live ? x[i] : (typename L::Raw)0);
            L::template store<PAST>(grad_value + (t0 + i) * p.grad_t + q.d, live ? y[i] : (typename L::Raw)0);
          }
      }
    }
  }
  if constexpr (!MAPS) {             // as forwards
    const int64_t steps = (int64_t)waves * kChunk;
#pragma unroll 1
    for (int e = 0; e < V; ++e) {
      if (!q.on || !p.apart || ((e ? good[V - 1] : good[0]) && finite(e ? carry[V - 1] : carry[0]))) continue;
      float c = starts[wave][e][lane];
      int from = gridDim.y - 1;
      for (; from > (int)blockIdx.y; --from) {
        const float next = fmaf(p.workspace[2 * from * channels + n + e], c, p.workspace[(2 * from + 1) * channels + n + e]);
        if (!finite(next)) break;
        c = next;
      }
      const int64_t first = q.first * steps, end = q.last * steps;
#pragma unroll 1
      for (int64_t t = min(part_from(q.tiles, from + 1, gridDim.y) * steps, len) - 1; t >= first && c == c; --t) {
        const float s = leak((float)gate[t * p.in_t + q.d + e]), now = c + (float)grad_out[t * p.out_t + q.d + e];
        if (t < end && t / kChunk % waves == wave) {
          const int64_t t0 = t / kChunk * kChunk;
          float h = p.states[t / kChunk * channels + n + e];
          for (int64_t j = t0; j < t; ++j) h = careful_state(leak((float)gate[j * p.in_t + q.d + e]), h, (float)value[j * p.in_t + q.d + e]);
          const float w = fabsf(s);
          grad_gate[t * p.grad_t + q.d + e] = (T)(now * (w * (1.0f - w)) * (h - (float)value[t * p.in_t + q.d + e]));
          grad_value[t * p.grad_t + q.d + e] = (T)(now * rest_of(s));
        }
        c = careful_times(s, now);
      }
      (e ? carry[V - 1] : carry[0]) = c;
    }
  }
  if (wave || !q.on) return;
#pragma unroll
  for (int e = 0; e < V; ++e) {
    if constexpr (MAPS) {
      p.workspace[2 * blockIdx.y * channels + n + e] = total[e];
      p.workspace[(2 * blockIdx.y + 1) * channels + n + e] = carry[e];
    } else if (p.grad_h0 && blockIdx.y == 0) {
      p.grad_h0[n + e] = carry[e];
    }
  }
}

// a thread per channel of a row
template <typename T>
__global__ __launch_bounds__(256) void step_kernel(const StepParams p) {
  const int d = blockIdx.x * 256 + threadIdx.x, b = blockIdx.y;
  if (d >= p.D) return;
  const int64_t slot = p.slots ? p.slots[b] : b;
  float h = 0.0f;
  if (slot >= 0 && slot < p.n_slots) {
    float* state = p.pool + slot * p.D + d;
    h = careful_state(leak((float)((const T*)p.gate)[b * p.in_b + d]), *state, (float)((const T*)p.value)[b * p.in_b + d]);
    *state = h;
  }
  ((T*)p.out)[b * p.out_b + d] = (T)h;
}

int64_t channel_groups(int B, int D, int v) { return (int64_t)B * ((D + 64 * v - 1) / (64 * v)); }

// Parts of the length: one where the channels alone give three workgroups to every four compute units, else enough for two to each.
int length_parts(int64_t T, int B, int D, int bf) {
  const int64_t groups = channel_groups(B, D, bf ? 2 : 1), tiles = (T + kWaves * kChunk - 1) / (kWaves * kChunk);
  if (groups >= kFittedUnits * 3 / 4) return 1;
  const int64_t want = (2 * kFittedUnits + groups - 1) / groups;
  return (int)(want < tiles ? want : tiles);
}

// two bfloat16 at once: an even number of channels, and rows that start at multiples of 4 bytes
bool pairs(int D, int64_t a, int64_t b, const void* p, const void* q) {
  return D % 2 == 0 && ((a | b) & 1) == 0 && (((uintptr_t)p | (uintptr_t)q) & 3u) == 0;
}

// Past the caches: 32768 x 2048 bfloat16 backwards 212 -> 188 us, 2048 x 16 x 2048 forwards 82 -> 73. Rows that end inside a memory line
// are left to them (30000 x 3 x 301 float32 backwards 217 us, past them 224).
bool streamed_rows(int64_t steps, int D, int bf) { return D % (bf ? 8 : 4) == 0 && streamed(steps * D * (bf ? 2 : 4)); }

template <typename T, int V>
hipError_t scan_typed(const ScanParams& p, hipStream_t s) {
  const unsigned groups = (unsigned)channel_groups(p.B, p.D, V);
  const int parts = length_parts(p.T, p.B, p.D, p.bf16), threads = 64 * scan_waves(p.T, groups);
  if (parts > 1) {
    hipLaunchKernelGGL((scan_kernel<T, V, true>), dim3(groups, parts), dim3(threads), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (streamed_rows(p.T * p.B, p.D, p.bf16)) hipLaunchKernelGGL((scan_kernel<T, V, false, true>), dim3(groups, parts), dim3(threads), 0, s, p);
  else hipLaunchKernelGGL((scan_kernel<T, V, false>), dim3(groups, parts), dim3(threads), 0, s, p);
  return hipGetLastError();
}

template <typename T, int V>
hipError_t scan_backward_typed(const ScanBackwardParams& p, hipStream_t s) {
  const unsigned groups = (unsigned)channel_groups(p.B, p.D, V);
  const int parts = length_parts(p.T, p.B, p.D, p.bf16), threads = 64 * scan_waves(p.T, groups);
  if (parts > 1) {
    hipLaunchKernelGGL((scan_backward_kernel<T, V, true>), dim3(groups, parts), dim3(threads), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (streamed_rows(2 * p.T * p.B, p.D, p.bf16)) hipLaunchKernelGGL((scan_backward_kernel<T, V, false, true>), dim3(groups, parts), dim3(threads), 0, s, p);
  else hipLaunchKernelGGL((scan_backward_kernel<T, V, false>), dim3(groups, parts), dim3(threads), 0, s, p);
  return hipGetLastError();
}

}  // namespace

size_t scan_workspace(int64_t T, int B, int D, int bf) {
  const int parts = length_parts(T, B, D, bf);
  return parts > 1 ? (size_t)parts * 2 * (size_t)B * (size_t)D * sizeof(float) : 0;
}

hipError_t scan_launch(const ScanParams& given, hipStream_t s) {
  ScanParams p = given;
  const Rows out = {p.out, p.out_t, p.out_b};
  p.apart = true;
  for (const void* in : {p.gate, p.value}) p.apart &= !rows_overlap({in, p.in_t, p.in_b}, out, p.T, p.B, p.D, p.bf16 ? 2 : 4);
  if (!p.bf16) return scan_typed<float, 1>(p, s);
  const bool two = pairs(p.D, p.in_t, p.in_b, p.gate, p.value) && pairs(p.D, p.out_t, p.out_b, p.out, nullptr);
  return two ? scan_typed<bf16, 2>(p, s) : scan_typed<bf16, 1>(p, s);
}

hipError_t scan_backward_launch(const ScanBackwardParams& given, hipStream_t s) {
  ScanBackwardParams p = given;
  p.apart = true;
  for (const Rows& in : {Rows{p.gate, p.in_t, p.in_b}, Rows{p.value, p.in_t, p.in_b}, Rows{p.grad_out, p.out_t, p.out_b}})
    for (const void* out : {p.grad_gate, p.grad_value}) p.apart &= !rows_overlap(in, {out, p.grad_t, p.grad_b}, p.T, p.B, p.D, p.bf16 ? 2 : 4);
  if (!p.bf16) return scan_backward_typed<float, 1>(p, s);
  const bool two = pairs(p.D, p.in_t, p.in_b, p.gate, p.value) && pairs(p.D, p.out_t, p.out_b, p.grad_out, nullptr) &&
                   pairs(p.D, p.grad_t, p.grad_b, p.grad_gate, p.grad_value);
  return two ? scan_backward_typed<bf16, 2>(p, s) : scan_backward_typed<bf16, 1>(p, s);
}

hipError_t step_launch(const StepParams& p, hipStream_t s) {
  const dim3 grid((unsigned)((p.D + 255) / 256), (unsigned)p.B);
  if (p.bf16) hipLaunchKernelGGL(step_kernel<bf16>, grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL(step_kernel<float>, grid, dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace tac
