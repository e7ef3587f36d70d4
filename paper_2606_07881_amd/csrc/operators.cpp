// The operator calls of include/paci_stage.h: argument checks and the launches.
// A negative status other than PACI_E_HIP means that nothing was enqueued.
#include <hip/hip_runtime.h>

#include <cmath>
#include <initializer_list>

#include "kernels.hpp"
#include "paci_stage.h"

namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Rows of `cols` elements with stride ld (elements): 16-byte aligned, not overlapping.
bool rows_ok(const void* p, int64_t ld, int64_t cols, int64_t rows, int dtype) {
  const int64_t vec = dtype == PACI_BF16 ? 8 : 4;
  return p && aligned(p, 16) && ld % vec == 0 && (ld >= cols || (rows <= 1 && ld >= 0)) && ld <= (1LL << 46) / rows;
}
bool floats_ok(const float* p) { return p && aligned(p, 4); }
// Whether a[na] and b[nb] share an element (null: no).
bool overlap(const float* a, int64_t na, const float* b, int64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && x < y + 4 * (uintptr_t)nb && y < x + 4 * (uintptr_t)na;
}

int done(hipError_t e) {
  if (e == hipSuccess) return PACI_OK;
  paci::note_hip_error(e);
  return PACI_E_HIP;
}

// ---- norms and rotation -----------------------------------------------------------------
int check_qk(const paci_qk_shapes* s) {
  if (!s || s->tokens < 0 || s->seq < 1 || s->q_heads < 0 || s->k_heads < 0 || s->rope_dims < 0 || s->head_dim < 1) return PACI_E_INVAL;
  if ((int64_t)s->q_heads + s->k_heads < 1) return PACI_E_INVAL;
  if ((s->norm != 0 && s->norm != 1) || (s->rope_pairs != PACI_ROPE_HALF && s->rope_pairs != PACI_ROPE_ADJACENT))
    return PACI_E_INVAL;
  if (!s->norm && s->rope_dims == 0) return PACI_E_INVAL;   // nothing to do
  if (s->norm && !(s->eps >= 0.f && std::isfinite(s->eps))) return PACI_E_INVAL;
  if (s->rope_dims > s->head_dim) return PACI_E_INVAL;
  if (s->dtype != PACI_FP32 && s->dtype != PACI_BF16) return PACI_E_UNSUPPORTED;
  if (s->head_dim % 16 || s->head_dim > 256 || s->rope_dims % 16) return PACI_E_UNSUPPORTED;
  if ((int64_t)s->q_heads + s->k_heads > 16384 || s->tokens > (1 << 30)) return PACI_E_UNSUPPORTED;
  return PACI_OK;
}
paci::RotArgs rot_args(const paci_qk_shapes& s) {
  paci::RotArgs r;
  r.dt = s.dtype == PACI_BF16 ? paci::DT_BF16 : paci::DT_F32;
  r.T = s.tokens;
  r.seq = s.seq;
  r.q_heads = s.q_heads;
  r.k_heads = s.k_heads;
  r.dh = s.head_dim;
  r.rope_dims = s.rope_dims;
  r.norm = s.norm != 0;
  r.adjacent = s.rope_pairs == PACI_ROPE_ADJACENT;
  r.eps = s.eps;
  return r;
}
// The parameters both directions read.
bool qk_params_ok(const paci_qk_shapes& s, const float* q_gain, const float* k_gain, const int32_t* pos, const double* freq) {
  if (s.norm && ((s.q_heads && !floats_ok(q_gain)) || (s.k_heads && !floats_ok(k_gain)))) return false;
  if (s.rope_dims && (!freq || !aligned(freq, 8))) return false;
  return aligned(pos, 4);
}

// ---- attention --------------------------------------------------------------------------
int check_attn(const paci_attn_shapes* s) {
  if (!s || s->batch < 0 || s->seq < 0 || s->n_heads < 1 || s->head_dim < 1 || s->n_buckets < 0) return PACI_E_INVAL;
  if (s->n_buckets > 0 && (s->n_buckets < 2 || s->max_distance < 1)) return PACI_E_INVAL;
  if (s->dtype != PACI_FP32 && s->dtype != PACI_BF16) return PACI_E_UNSUPPORTED;
  const int dh = s->head_dim;
  if ((dh != 32 && dh != 64 && dh != 128) || (s->dtype == PACI_FP32 && dh == 128)) return PACI_E_UNSUPPORTED;
  if (s->n_buckets > paci::MAX_BUCKETS || (s->n_buckets && s->max_distance > paci::MAX_DISTANCE)) return PACI_E_UNSUPPORTED;
  // launch grids: one workgroup column per (sequence, head), rows of at least 64 queries
  if ((int64_t)s->batch * s->n_heads > 65535 || s->seq > (1 << 20) || (int64_t)s->batch * s->seq > (1 << 30) ||
      (int64_t)s->batch * s->n_heads * s->seq * dh > (1LL << 33))
    return PACI_E_UNSUPPORTED;
  return PACI_OK;
}
paci::AttnArgs attn_shape_args(const paci_attn_shapes& s) {
  paci::AttnArgs a;
  a.dt = s.dtype == PACI_BF16 ? paci::DT_BF16 : paci::DT_F32;
  a.mu = s.batch;
  a.S = s.seq;
  a.H = s.n_heads;
  a.dh = s.head_dim;
  a.n_buckets = s.n_buckets;
  a.max_distance = s.n_buckets ? s.max_distance : 0;
  return a;
}
int64_t attn_ws_floats(const paci_attn_shapes& s) {
  if (!s.batch || !s.seq) return 0;
  const paci::AttnArgs a = attn_shape_args(s);
  return paci::attn_bwd_workspace_floats(a.dt, a.mu, a.S, a.H) + (s.n_buckets ? paci::attn_bias_workspace_floats(a) : 0);
}

}  // namespace

extern "C" int paci_rope_freqs(double theta, int rope_dims, double* host_freq) {
  if (!(theta > 0.0) || !std::isfinite(theta) || rope_dims < 2 || rope_dims % 2 || !host_freq) return PACI_E_INVAL;
  for (int i = 0; i < rope_dims / 2; ++i) host_freq[i] = std::pow(theta, -2.0 * i / rope_dims);
  return PACI_OK;
}

extern "C" int paci_qk_norm_rope_forward(const paci_qk_shapes* s, const void* dev_x, int64_t ld_x, const float* dev_q_gain,
                                         const float* dev_k_gain, const int32_t* dev_pos, const double* dev_freq,
                                         void* dev_y, int64_t ld_y, void* hip_stream) {
  const int v = check_qk(s);
  if (v) return v;
  if (s->tokens == 0) return PACI_OK;
  const int64_t cols = ((int64_t)s->q_heads + s->k_heads) * s->head_dim;
  if (!rows_ok(dev_x, ld_x, cols, s->tokens, s->dtype) || !rows_ok(dev_y, ld_y, cols, s->tokens, s->dtype) ||
      !qk_params_ok(*s, dev_q_gain, dev_k_gain, dev_pos, dev_freq) || (dev_x == dev_y && ld_x != ld_y))
    return PACI_E_INVAL;
  paci::RotArgs r = rot_args(*s);
  r.x = dev_x;
  r.ldx = ld_x;
  r.out = dev_y;
  r.ldout = ld_y;
  r.gain_q = dev_q_gain;
  r.gain_k = dev_k_gain;
  r.pos = dev_pos;
  r.freq = dev_freq;
  return done(paci::rotary(r, false, reinterpret_cast<hipStream_t>(hip_stream)));
}

extern "C" int paci_qk_norm_rope_workspace(const paci_qk_shapes* s, size_t* bytes) {
  if (!bytes) return PACI_E_INVAL;
  const int v = check_qk(s);
  if (v) return v;
  *bytes = sizeof(float) * (size_t)paci::rotary_workspace_floats(rot_args(*s));
  return PACI_OK;
}

extern "C" int paci_qk_norm_rope_backward(const paci_qk_shapes* s, const void* dev_x, int64_t ld_x, const void* dev_dy,
                                          int64_t ld_dy, const float* dev_q_gain, const float* dev_k_gain,
                                          const int32_t* dev_pos, const double* dev_freq, void* dev_dx, int64_t ld_dx,
                                          float* dev_g_q_gain, float* dev_g_k_gain, float* dev_g_bias, void* dev_ws,
                                          size_t ws_bytes, void* hip_stream) {
  const int v = check_qk(s);
  if (v) return v;
  if (s->tokens == 0) return PACI_OK;
  const int64_t cols = ((int64_t)s->q_heads + s->k_heads) * s->head_dim;
  if ((s->norm && !rows_ok(dev_x, ld_x, cols, s->tokens, s->dtype)) ||
      !rows_ok(dev_dy, ld_dy, cols, s->tokens, s->dtype) || !rows_ok(dev_dx, ld_dx, cols, s->tokens, s->dtype) ||
      !qk_params_ok(*s, dev_q_gain, dev_k_gain, dev_pos, dev_freq) || (dev_dx == dev_dy && ld_dx != ld_dy) ||
      (s->norm && dev_dx == dev_x))
    return PACI_E_INVAL;
  if (!s->norm && (dev_g_q_gain || dev_g_k_gain)) return PACI_E_INVAL;
  if (!aligned(dev_g_q_gain, 4) || !aligned(dev_g_k_gain, 4) || !aligned(dev_g_bias, 4)) return PACI_E_INVAL;
  // different workgroups add to them at once
  const int64_t dh = s->head_dim;
  if (overlap(dev_g_q_gain, dh, dev_g_k_gain, dh) || overlap(dev_g_q_gain, dh, dev_g_bias, cols) ||
      overlap(dev_g_k_gain, dh, dev_g_bias, cols))
    return PACI_E_INVAL;
  paci::RotArgs r = rot_args(*s);
  if (s->norm || dev_g_bias) {
    if (!dev_ws || !aligned(dev_ws, 16)) return PACI_E_INVAL;
    if (ws_bytes < sizeof(float) * (size_t)paci::rotary_workspace_floats(r)) return PACI_E_NOMEM;
  }
  r.x = dev_x;
  r.ldx = ld_x;
  r.dy = dev_dy;
  r.lddy = ld_dy;
  r.out = dev_dx;
  r.ldout = ld_dx;
  r.gain_q = dev_q_gain;
  r.gain_k = dev_k_gain;
  r.pos = dev_pos;
  r.freq = dev_freq;
  r.g_gain_q = dev_g_q_gain;
  r.g_gain_k = dev_g_k_gain;
  r.g_bias = dev_g_bias;
  r.ws = reinterpret_cast<float*>(dev_ws);
  return done(paci::rotary(r, true, reinterpret_cast<hipStream_t>(hip_stream)));
}

extern "C" int paci_rel_bounds(int n_buckets, int max_distance, int32_t* host_bounds) {
  const int e = n_buckets / 2, m = n_buckets - e;
  if (n_buckets < 2 || max_distance <= e || !host_bounds) return PACI_E_INVAL;
  if (n_buckets > paci::MAX_BUCKETS || max_distance > paci::MAX_DISTANCE) return PACI_E_UNSUPPORTED;
  for (int i = 0; i < e; ++i) host_bounds[i] = i;
  // bucket e + k starts at the first whole distance at or above e (max_distance / e)^(k / m).
  // Where that is a whole number, floating point can miss it either way: a value within
  // 1e-12 of one is taken for it (it is at most 512, and long double holds 19 digits).
  for (int k = 0; k < m; ++k) {
    const long double v = e * std::pow((long double)max_distance / e, (long double)k / m);
    const long double n = std::round(v);
    host_bounds[e + k] = (int32_t)(std::fabs(v - n) < 1e-12L ? n : std::ceil(v));
  }
  return PACI_OK;
}

extern "C" int paci_attn_forward(const paci_attn_shapes* s, const void* dev_q, int64_t ld_q, const void* dev_k,
                                 int64_t ld_k, const void* dev_v, int64_t ld_v, const float* dev_table,
                                 const int32_t* dev_bounds, void* dev_o, float* dev_lse2, void* hip_stream) {
  const int c = check_attn(s);
  if (c) return c;
  if (s->batch == 0 || s->seq == 0) return PACI_OK;
  const int64_t d = (int64_t)s->n_heads * s->head_dim, T = (int64_t)s->batch * s->seq;
  if (!rows_ok(dev_q, ld_q, d, T, s->dtype) || !rows_ok(dev_k, ld_k, d, T, s->dtype) ||
      !rows_ok(dev_v, ld_v, d, T, s->dtype) || !rows_ok(dev_o, d, d, T, s->dtype) || !floats_ok(dev_lse2))
    return PACI_E_INVAL;
  if (dev_o == dev_q || dev_o == dev_k || dev_o == dev_v) return PACI_E_INVAL;   // other workgroups still read them
  if (s->n_buckets ? !floats_ok(dev_table) || !dev_bounds || !aligned(dev_bounds, 4) : dev_table || dev_bounds)
    return PACI_E_INVAL;
  paci::AttnArgs a = attn_shape_args(*s);
  a.q = dev_q;
  a.ldq = ld_q;
  a.k = dev_k;
  a.ldk = ld_k;
  a.v = dev_v;
  a.ldv = ld_v;
  a.table = dev_table;
  a.bounds = dev_bounds;
  return done(paci::attn_fwd(a, dev_o, dev_lse2, reinterpret_cast<hipStream_t>(hip_stream)));
}

extern "C" int paci_attn_workspace(const paci_attn_shapes* s, size_t* bytes) {
  if (!bytes) return PACI_E_INVAL;
  const int c = check_attn(s);
  if (c) return c;
  *bytes = sizeof(float) * (size_t)attn_ws_floats(*s);
  return PACI_OK;
}

extern "C" int paci_attn_backward(const paci_attn_shapes* s, const void* dev_q, int64_t ld_q, const void* dev_k,
                                  int64_t ld_k, const void* dev_v, int64_t ld_v, const float* dev_table,
                                  const int32_t* dev_bounds, const void* dev_o, const float* dev_lse2,
                                  const void* dev_do, void* dev_dq, int64_t ld_dq, void* dev_dk, int64_t ld_dk,
                                  void* dev_dv, int64_t ld_dv, float* dev_g_table, void* dev_ws, size_t ws_bytes,
                                  void* hip_stream) {
  const int c = check_attn(s);
  if (c) return c;
  if (s->batch == 0 || s->seq == 0) return PACI_OK;
  const int64_t d = (int64_t)s->n_heads * s->head_dim, T = (int64_t)s->batch * s->seq;
  if (!rows_ok(dev_q, ld_q, d, T, s->dtype) || !rows_ok(dev_k, ld_k, d, T, s->dtype) ||
      !rows_ok(dev_v, ld_v, d, T, s->dtype) || !rows_ok(dev_o, d, d, T, s->dtype) || !rows_ok(dev_do, d, d, T, s->dtype) ||
      !floats_ok(dev_lse2))
    return PACI_E_INVAL;
  if (!rows_ok(dev_dq, ld_dq, d, T, s->dtype) || !rows_ok(dev_dk, ld_dk, d, T, s->dtype) ||
      !rows_ok(dev_dv, ld_dv, d, T, s->dtype))
    return PACI_E_INVAL;
  // other workgroups still read an operand when a gradient is written
  for (const void* out : {(const void*)dev_dq, (const void*)dev_dk, (const void*)dev_dv})
    for (const void* in : {dev_q, dev_k, dev_v, dev_o, dev_do})
      if (out == in) return PACI_E_INVAL;
  if (dev_dq == dev_dk || dev_dq == dev_dv || dev_dk == dev_dv) return PACI_E_INVAL;
  if (s->n_buckets ? !floats_ok(dev_table) || !dev_bounds || !aligned(dev_bounds, 4) : dev_table || dev_bounds || dev_g_table)
    return PACI_E_INVAL;
  if (!aligned(dev_g_table, 4) || !dev_ws || !aligned(dev_ws, 16)) return PACI_E_INVAL;
  if (ws_bytes < sizeof(float) * (size_t)attn_ws_floats(*s)) return PACI_E_NOMEM;
  paci::AttnArgs a = attn_shape_args(*s);
  a.q = dev_q;
  a.ldq = ld_q;
  a.k = dev_k;
  a.ldk = ld_k;
  a.v = dev_v;
  a.ldv = ld_v;
  a.table = dev_table;
  a.bounds = dev_bounds;
  paci::AttnGrads g;
  g.dq = dev_dq;
  g.ldq = ld_dq;
  g.dk = dev_dk;
  g.ldk = ld_dk;
  g.dv = dev_dv;
  g.ldv = ld_dv;
  g.g_table = dev_g_table;
  float* ws = reinterpret_cast<float*>(dev_ws);
  return done(paci::attn_bwd(a, g, dev_o, dev_do, dev_lse2, ws, ws + paci::attn_bwd_workspace_floats(a.dt, a.mu, a.S, a.H),
                             reinterpret_cast<hipStream_t>(hip_stream)));
}
