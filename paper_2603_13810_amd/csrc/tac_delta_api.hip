// Host side of the head norm's and the gated delta rule's C ABI: argument checks and launch parameters.  Nothing is launched before all of them hold.
#include <cmath>

#include "tac_delta_chunk.h"

namespace {

constexpr int64_t kMost = (1ll << 31) - 1;

bool float_type(int32_t dtype) { return dtype == TAC_FP32 || dtype == TAC_BF16; }
size_t bytes_of(int32_t dtype) { return dtype == TAC_BF16 ? 2 : 4; }
bool misaligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) != 0; }
int finish(hipError_t e, const char* where) { return e == hipSuccess ? TAC_OK : tac::hip_fail(e, where); }

// `count` pieces of `width` elements, `stride` apart: not on top of each other, and within 2^62 bytes
bool bad_stride(int64_t count, int64_t stride, int64_t width) { return count > 1 && (stride < width || stride > (1ll << 60) / count); }

int check_heads(const tac_head_norm_desc_t* d) {
  if (!d) return TAC_ERR_NULL;
  if (d->rows < 1 || d->rows > kMost || d->query_heads < 1 || d->key_heads < 0 || d->D < 2 || d->D % 2) return TAC_ERR_BAD_SHAPE;
  if ((int64_t)d->query_heads + d->key_heads > 65535) return TAC_ERR_BAD_SHAPE;
  if (!float_type(d->dtype)) return TAC_ERR_BAD_PARAM;
  if (!(d->eps >= 0.0f) || !std::isfinite(d->eps)) return TAC_ERR_BAD_PARAM;
  if (d->axes < 0 || d->axes > TAC_ROTATION_AXES) return TAC_ERR_BAD_PARAM;
  int64_t pairs = 0;
  for (int a = 0; a < d->axes; ++a) {
    if (d->pairs[a] < 1) return TAC_ERR_BAD_PARAM;
    pairs += d->pairs[a];
  }
  if (pairs > d->D / 2) return TAC_ERR_BAD_PARAM;
  if (d->axes && (!(d->base > 0.0) || !std::isfinite(d->base))) return TAC_ERR_BAD_PARAM;
  if (d->D > TAC_HEAD_MAX_FEATURES) return TAC_ERR_UNSUPPORTED;
  return TAC_OK;
}

bool bad_heads(const tac_head_norm_desc_t* d, int heads, const tac_head_strides_t& s) {
  return heads && (bad_stride(heads, s.head, d->D) || bad_stride(d->rows, s.row, d->D));
}

tac::HeadNormParams head_params(const tac_head_norm_desc_t* d) {
  tac::HeadNormParams p = {};
  p.rows = d->rows;
  p.D = d->D;
  p.axes = d->axes;
  for (int a = 0; a < d->axes; ++a) p.rotated += p.pairs[a] = d->pairs[a];
  p.interleaved = d->interleaved != 0;
  p.bf16 = d->dtype == TAC_BF16;
  p.eps = d->eps;
  for (int a = 0; a < d->axes; ++a) p.log2_step[a] = std::log2(d->base) / d->pairs[a];
  return p;
}

int check_delta(const tac_delta_desc_t* d) {
  if (!d) return TAC_ERR_NULL;
  if (d->T < 1 || d->T > kMost || d->B < 1 || d->k_heads < 1 || d->v_heads < 1 || d->v_heads % d->k_heads || d->Dk < 1 || d->Dv < 1) return TAC_ERR_BAD_SHAPE;
  if (!float_type(d->dtype)) return TAC_ERR_BAD_PARAM;
  if (d->Dk > TAC_DELTA_MAX_KEY || d->Dv > TAC_DELTA_MAX_VALUE) return TAC_ERR_UNSUPPORTED;
  if (!tac::delta_fits(d->T, d->B, d->v_heads, d->Dv)) return TAC_ERR_BAD_SHAPE;
  return TAC_OK;
}

bool bad_steps(const tac_delta_desc_t* d, const tac_delta_strides_t& s, int heads, int width) {
  return bad_stride(heads, s.head, width) || bad_stride(d->T, s.t, width) || bad_stride(d->B, s.b, width);
}
// single numbers per head, next to each other
bool bad_gates(const tac_delta_desc_t* d, const tac_delta_strides_t& s) {
  return (d->v_heads > 1 && s.head != 1) || bad_stride(d->T, s.t, d->v_heads) || bad_stride(d->B, s.b, d->v_heads);
}

bool bad_inputs(const tac_delta_desc_t* d) {
  return bad_steps(d, d->query, d->k_heads, d->Dk) || bad_steps(d, d->key, d->k_heads, d->Dk) || bad_steps(d, d->value, d->v_heads, d->Dv) ||
         bad_gates(d, d->gate) || bad_gates(d, d->write) || bad_steps(d, d->out, d->v_heads, d->Dv);
}

tac::DeltaParams delta_params(const tac_delta_desc_t* d) {
  tac::DeltaParams p = {};
  p.T = d->T;
  p.B = d->B;
  p.k_heads = d->k_heads;
  p.v_heads = d->v_heads;
  p.Dk = d->Dk;
  p.Dv = d->Dv;
  p.bf16 = d->dtype == TAC_BF16;
  p.chunks = (int)tac::delta_chunks(d->T);
  p.q_at = d->query;
  p.k_at = d->key;
  p.v_at = d->value;
  p.gate_at = d->gate;
  p.write_at = d->write;
  p.out_at = d->out;
  p.grad_q_at = d->grad_query;
  p.grad_k_at = d->grad_key;
  p.grad_v_at = d->grad_value;
  p.grad_gate_at = d->grad_gate;
  p.grad_write_at = d->grad_write;
  return p;
}

bool any_misaligned(std::initializer_list<const void*> list, size_t to) {
  for (const void* p : list)
    if (misaligned(p, to)) return true;
  return false;
}

// Outputs that begin where an input or another output does; what is not there (NULL) is on nothing.  (Tensors that overlap in other ways are the caller's to keep apart: slices of the same rows lie between each other.)
bool on_each_other(std::initializer_list<const void*> written, std::initializer_list<const void*> read) {
  for (auto w = written.begin(); w != written.end(); ++w) {
    if (!*w) continue;
    for (const void* r : read)
      if (*w == r) return true;
    for (auto other = written.begin(); other != w; ++other)
      if (*w == *other) return true;
  }
  return false;
}
// in place, but not head by head
bool moved(const tac_head_norm_desc_t* d, int heads, const void* from, const tac_head_strides_t& a, const void* to, const tac_head_strides_t& b) {
  return from == to && ((d->rows > 1 && a.row != b.row) || (heads > 1 && a.head != b.head));
}

}  // namespace

extern "C" {

int tac_head_norm(const tac_head_norm_desc_t* d, const void* query, const void* key, const float* gain_query, const float* gain_key,
                  const int32_t* positions, void* out_query, void* out_key, void* stream) {
  const int rc = check_heads(d);
  if (rc) return rc;
  if (!query || !out_query || (d->key_heads && (!key || !out_key)) || (d->axes && !positions)) return TAC_ERR_NULL;
  if (!d->key_heads) key = out_key = nullptr, gain_key = nullptr;      // what is ignored may be anywhere, and no kernel reads it
  if (!d->axes) positions = nullptr;
  if (bad_heads(d, d->query_heads, d->query) || bad_heads(d, d->query_heads, d->out_query) || bad_heads(d, d->key_heads, d->key) ||
      bad_heads(d, d->key_heads, d->out_key))
    return TAC_ERR_BAD_SHAPE;
  const size_t el = bytes_of(d->dtype);
  if (any_misaligned({query, key, out_query, out_key}, el) || any_misaligned({gain_query, gain_key, positions}, 4)) return TAC_ERR_ALIGN;
  if (moved(d, d->query_heads, query, d->query, out_query, d->out_query) || (key && moved(d, d->key_heads, key, d->key, out_key, d->out_key)) ||
      on_each_other({out_query}, {key, out_key, gain_query, gain_key, positions}) || on_each_other({out_key}, {query, gain_query, gain_key, positions}))
    return TAC_ERR_BAD_PARAM;
  tac::HeadNormParams p = head_params(d);
  p.q = {query, nullptr, out_query, gain_query, d->query, {}, d->out_query, d->query_heads};
  p.k = {key, nullptr, out_key, gain_key, d->key, {}, d->out_key, d->key_heads};
  p.positions = positions;
  return finish(tac::head_norm_launch(p, (hipStream_t)stream), "tac_head_norm");
}

size_t tac_head_norm_workspace_bytes(const tac_head_norm_desc_t* d) {
  if (check_heads(d)) return 0;
  tac::HeadNormParams p = head_params(d);
  p.q.heads = d->query_heads;
  p.k.heads = d->key_heads;
  return tac::head_norm_workspace(p);
}

int tac_head_norm_backward(const tac_head_norm_desc_t* d, const void* query, const void* key, const float* gain_query, const float* gain_key,
                           const int32_t* positions, const void* grad_out_query, const void* grad_out_key, void* grad_query, void* grad_key,
                           float* grad_gain_query, float* grad_gain_key, void* workspace, void* stream) {
  const int rc = check_heads(d);
  if (rc) return rc;
  if (!query || !grad_out_query || !grad_query || (d->key_heads && (!key || !grad_out_key || !grad_key)) || (d->axes && !positions)) return TAC_ERR_NULL;
  if (!d->key_heads) key = grad_out_key = grad_key = nullptr, gain_key = grad_gain_key = nullptr;      // what is ignored may be anywhere, and no kernel reads it
  if (!d->axes) positions = nullptr;
  if (!grad_gain_query && !grad_gain_key) workspace = nullptr;
  else if (!workspace) return TAC_ERR_NULL;
  if (bad_heads(d, d->query_heads, d->query) || bad_heads(d, d->query_heads, d->out_query) || bad_heads(d, d->query_heads, d->grad_query) ||
      bad_heads(d, d->key_heads, d->key) || bad_heads(d, d->key_heads, d->out_key) || bad_heads(d, d->key_heads, d->grad_key))
    return TAC_ERR_BAD_SHAPE;
  const size_t el = bytes_of(d->dtype);
  if (any_misaligned({query, key, grad_out_query, grad_out_key, grad_query, grad_key}, el) ||
      any_misaligned({gain_query, gain_key, grad_gain_query, grad_gain_key, positions}, 4) || misaligned(workspace, 16))
    return TAC_ERR_ALIGN;
  if (moved(d, d->query_heads, grad_out_query, d->out_query, grad_query, d->grad_query) || (key && moved(d, d->key_heads, grad_out_key, d->out_key, grad_key, d->grad_key)) ||
      on_each_other({grad_query}, {query, key, grad_out_key, grad_key, gain_query, gain_key, positions}) ||
      on_each_other({grad_key}, {query, key, grad_out_query, gain_query, gain_key, positions}) ||
      on_each_other({grad_gain_query, grad_gain_key, workspace}, {query, key, gain_query, gain_key, positions, grad_out_query, grad_out_key, grad_query, grad_key}))
    return TAC_ERR_BAD_PARAM;
  tac::HeadNormParams p = head_params(d);
  p.q = {query, grad_out_query, grad_query, gain_query, d->query, d->out_query, d->grad_query, d->query_heads};
  p.k = {key, grad_out_key, grad_key, gain_key, d->key, d->out_key, d->grad_key, d->key_heads};
  p.positions = positions;
  p.partial = (float*)workspace;
  p.grad_gain_q = grad_gain_query;
  p.grad_gain_k = grad_gain_key;
  return finish(tac::head_norm_backward_launch(p, (hipStream_t)stream), "tac_head_norm_backward");
}

size_t tac_delta_scan_workspace_bytes(const tac_delta_desc_t* d) { return check_delta(d) ? 0 : tac::delta_workspace(delta_params(d)); }
size_t tac_delta_scan_backward_workspace_bytes(const tac_delta_desc_t* d) { return check_delta(d) ? 0 : tac::delta_backward_workspace(delta_params(d)); }

int tac_delta_scan(const tac_delta_desc_t* d, const void* query, const void* key, const void* value, const void* gate, const void* write,
                   const int32_t* lengths, const float* h0, void* out, float* h_last, float* states, float* updates, void* workspace, void* stream) {
  const int rc = check_delta(d);
  if (rc) return rc;
  if (!query || !key || !value || !gate || !write || !out || !workspace || !states != !updates) return TAC_ERR_NULL;
  if (bad_inputs(d)) return TAC_ERR_BAD_SHAPE;
  if (any_misaligned({query, key, value, gate, write, out}, bytes_of(d->dtype)) || any_misaligned({lengths, h0, h_last, states, updates}, 4) ||
      misaligned(workspace, 16))
    return TAC_ERR_ALIGN;
  if (on_each_other({out, h_last, states, updates, workspace}, {query, key, value, gate, write, lengths}) || on_each_other({out, states, updates, workspace}, {h0})) return TAC_ERR_BAD_PARAM;
  tac::DeltaParams p = delta_params(d);
  p.q = query;
  p.k = key;
  p.v = value;
  p.gate = gate;
  p.write = write;
  p.lengths = lengths;
  p.h0 = h0;
  p.out = out;
  p.h_last = h_last;
  p.states = states;
  p.updates = updates;
  return finish(tac::delta_scan_launch(p, (uint8_t*)workspace, (hipStream_t)stream), "tac_delta_scan");
}

int tac_delta_scan_backward(const tac_delta_desc_t* d, const void* query, const void* key, const void* value, const void* gate, const void* write,
                            const int32_t* lengths, const float* states, const float* updates, const void* grad_out, const float* grad_h_last,
                            void* grad_query, void* grad_key, void* grad_value, void* grad_gate, void* grad_write, float* grad_h0,
                            void* workspace, void* stream) {
  const int rc = check_delta(d);
  if (rc) return rc;
  if (!query || !key || !value || !gate || !write || !states || !updates || !grad_out || !grad_query || !grad_key || !grad_value || !grad_gate || !grad_write ||
      !workspace)
    return TAC_ERR_NULL;
  if (bad_inputs(d) || bad_steps(d, d->grad_query, d->k_heads, d->Dk) || bad_steps(d, d->grad_key, d->k_heads, d->Dk) || bad_steps(d, d->grad_value, d->v_heads, d->Dv) ||
      bad_gates(d, d->grad_gate) || bad_gates(d, d->grad_write))
    return TAC_ERR_BAD_SHAPE;
  if (any_misaligned({query, key, value, gate, write, grad_out, grad_query, grad_key, grad_value, grad_gate, grad_write}, bytes_of(d->dtype)) ||
      any_misaligned({lengths, states, updates, grad_h_last, grad_h0}, 4) || misaligned(workspace, 16))
    return TAC_ERR_ALIGN;
  if (on_each_other({grad_query, grad_key, grad_value, grad_gate, grad_write, grad_h0, workspace}, {query, key, value, gate, write, lengths, states, updates, grad_out}) ||
      on_each_other({grad_query, grad_key, grad_value, grad_gate, grad_write, workspace}, {grad_h_last}))
    return TAC_ERR_BAD_PARAM;
  tac::DeltaParams p = delta_params(d);
  p.q = query;
  p.k = key;
  p.v = value;
  p.gate = gate;
  p.write = write;
  p.lengths = lengths;
  p.states = const_cast<float*>(states);
  p.updates = const_cast<float*>(updates);
  p.grad_out = grad_out;
  p.grad_h_last = grad_h_last;
  p.grad_q = grad_query;
  p.grad_k = grad_key;
  p.grad_v = grad_value;
  p.grad_gate = grad_gate;
  p.grad_write = grad_write;
  p.grad_h0 = grad_h0;
  return finish(tac::delta_backward_launch(p, (uint8_t*)workspace, (hipStream_t)stream), "tac_delta_scan_backward");
}

int tac_delta_step(const tac_delta_desc_t* d, const void* query, const void* key, const void* value, const void* gate, const void* write,
                   float* pool, int64_t n_slots, const int32_t* slots, void* out, void* stream) {
  const int rc = check_delta(d);
  if (rc) return rc;
  if (!query || !key || !value || !gate || !write || !pool || !out) return TAC_ERR_NULL;
  if (d->T != 1 || n_slots < 1 || n_slots > kMost || (!slots && n_slots < d->B) || bad_inputs(d)) return TAC_ERR_BAD_SHAPE;
  if (any_misaligned({query, key, value, gate, write, out}, bytes_of(d->dtype)) || any_misaligned({pool, slots}, 4)) return TAC_ERR_ALIGN;
  if (on_each_other({out, pool}, {query, key, value, gate, write, slots})) return TAC_ERR_BAD_PARAM;
  const tac::DeltaStepParams p = {query, key, value, gate, write, pool, slots, out, n_slots, d->query, d->key, d->value, d->gate, d->write, d->out,
                                  d->B, d->k_heads, d->v_heads, d->Dk, d->Dv, d->dtype == TAC_BF16};
  return finish(tac::delta_step_launch(p, (hipStream_t)stream), "tac_delta_step");
}

}  // extern "C"
