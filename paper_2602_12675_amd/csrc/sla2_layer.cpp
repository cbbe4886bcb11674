// Host side of the entry points around the attention (sla2_rope_*, sla2_norm_*): argument validation and launches.
// Declarations and their contracts are in include/sla2.h.
#include <float.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>

#include "host_checks.h"
#include "rows.h"

namespace sla2 {

static bool eps_ok(float eps) { return eps >= FLT_MIN && eps <= FLT_MAX; }      // not NaN, nothing that the root would take for 0
static bool vector_ok(const float* p) { return !misaligned16(p); }        // null too

static int make_rope(const sla2_rope_params* p, bool backward, int tensors, RopeArgs* a) {
  if (!p) return SLA2_EINVAL;
  if (p->B < 1 || p->H < 1 || p->N < 1) return SLA2_EINVAL;
  if (p->dtype != SLA2_F32 && p->dtype != SLA2_BF16) return SLA2_EINVAL;
  if (p->pairing != SLA2_ROPE_INTERLEAVED && p->pairing != SLA2_ROPE_HALVES) return SLA2_EINVAL;
  if (p->norm != SLA2_ROPE_NORM_NONE && p->norm != SLA2_ROPE_NORM_HEAD && p->norm != SLA2_ROPE_NORM_TOKEN) return SLA2_EINVAL;
  if (p->norm != SLA2_ROPE_NORM_NONE && !eps_ok(p->eps)) return SLA2_EINVAL;
  if (p->positions_per_batch != 0 && p->positions_per_batch != 1) return SLA2_EINVAL;
  if (p->d != 64 && p->d != 128) return SLA2_EUNSUPPORTED;
  if ((long long)p->B * p->H > 65535) return SLA2_EUNSUPPORTED;
  if (p->norm == SLA2_ROPE_NORM_TOKEN && (long long)p->H * p->d > kMaxRow) return SLA2_EUNSUPPORTED;
  *a = RopeArgs{};
  long long pairs = 0, cells = 1;
  const bool grid = p->grid[0] != 0 || p->grid[1] != 0 || p->grid[2] != 0;
  for (int i = 0; i < 3; i++) {
    if (p->axis_pairs[i] < 0) return SLA2_EINVAL;
    pairs += p->axis_pairs[i];
    if (pairs > p->d / 2) return SLA2_EINVAL;
    a->pairs_end[i] = (int)pairs;
    if (grid && p->grid[i] < 1) return SLA2_EINVAL;
    if (!grid && p->origin[i] != 0) return SLA2_EINVAL;
    if ((long long)p->origin[i] + p->grid[i] - 1 > INT_MAX) return SLA2_EINVAL;
    cells *= grid ? p->grid[i] : 1;
    if (cells > INT_MAX) return SLA2_EUNSUPPORTED;
    a->grid[i] = p->grid[i];
    a->origin[i] = p->origin[i];
  }
  const long long esz = p->dtype == SLA2_BF16 ? 2 : 4, count[3] = {p->B, p->H, p->N};
  HeadStrides* dst[2] = {&a->sin, &a->sout};
  const long long* src[2] = {p->in_stride, p->out_stride};
  for (int x = 0; x < 2; x++) {
    long long s[3] = {src[x][0], src[x][1], src[x][2]};
    if (s[0] == 0 && s[1] == 0 && s[2] == 0) {
      s[0] = (long long)p->H * p->N * p->d;
      s[1] = (long long)p->N * p->d;
      s[2] = p->d;
    }
    if (s[0] <= 0 || s[1] <= 0 || s[2] <= 0) return SLA2_EINVAL;
    if (s[2] < p->d) return SLA2_EUNSUPPORTED;
    for (long long st : s)
      if (st * esz % 16) return SLA2_EUNSUPPORTED;
    if (!extent_ok(3, count, s, p->d)) return SLA2_EUNSUPPORTED;
    *dst[x] = HeadStrides{s[0], s[1], s[2]};
  }
  a->tensors = tensors;
  a->B = p->B; a->H = p->H; a->N = p->N; a->d = p->d;
  a->eps = p->eps;
  a->norm = p->norm;
  a->bf16 = p->dtype == SLA2_BF16;
  a->halves = p->pairing == SLA2_ROPE_HALVES;
  a->sign = 1.0;
  a->positions_stride = p->positions_per_batch ? 3ll * p->N : 0;
  plan_rope(a, backward);
  return SLA2_OK;
}

static View head_view(const RopeArgs& a, const HeadStrides& s, const void* p) {
  return View{p, a.bf16 ? 2 : 4, 3, a.d, {a.B, a.H, a.N}, {s.b, s.h, s.n}};
}
// what both directions check of freq, positions and weights
static bool rope_inputs_ok(const RopeArgs& a, const double* freq, const int32_t* positions, const float* qw, const float* kw) {
  if (!freq || ((uintptr_t)freq & 7) || ((uintptr_t)positions & 3)) return false;
  if ((positions != nullptr) == (a.grid[0] != 0)) return false;
  if (a.norm == SLA2_ROPE_NORM_NONE && (qw || kw)) return false;
  return vector_ok(qw) && vector_ok(kw);
}
static long long weight_count(const RopeArgs& a) { return a.norm == SLA2_ROPE_NORM_TOKEN ? (long long)a.H * a.d : a.d; }

static int make_norm(const sla2_norm_params* p, NormArgs* a) {
  if (!p) return SLA2_EINVAL;
  if (p->B < 1 || p->N < 1 || p->C < 1) return SLA2_EINVAL;
  if ((p->dtype_x != SLA2_F32 && p->dtype_x != SLA2_BF16) || (p->dtype_h != SLA2_F32 && p->dtype_h != SLA2_BF16)) return SLA2_EINVAL;
  for (int k : {p->norm_in, p->norm_out})
    if (k != SLA2_NORM_NONE && k != SLA2_NORM_RMS && k != SLA2_NORM_LAYER) return SLA2_EINVAL;
  if ((p->norm_in != SLA2_NORM_NONE || p->norm_out != SLA2_NORM_NONE) && !eps_ok(p->eps)) return SLA2_EINVAL;
  if (!isfinite(p->residual_scale)) return SLA2_EINVAL;
  if (p->mod_layout != SLA2_MOD_BATCH && p->mod_layout != SLA2_MOD_TOKEN && p->mod_layout != SLA2_MOD_SHARED) return SLA2_EINVAL;
  if (p->C % kChunk || p->C > kMaxRow || p->B > 65535) return SLA2_EUNSUPPORTED;
  if (p->dtype_x == SLA2_BF16 && p->dtype_h == SLA2_F32) return SLA2_EUNSUPPORTED;
  *a = NormArgs{};
  const long long count[2] = {p->B, p->N}, dflt[2] = {(long long)p->N * p->C, p->C};
  long long *dst[2][2] = {{&a->x_b, &a->x_n}, {&a->h_b, &a->h_n}};
  const long long* src[2] = {p->x_stride, p->h_stride};
  const long long esz[2] = {p->dtype_x == SLA2_BF16 ? 2 : 4, p->dtype_h == SLA2_BF16 ? 2 : 4};
  for (int t = 0; t < 2; t++) {
    const bool unset = src[t][0] == 0 && src[t][1] == 0;
    const long long s[2] = {unset ? dflt[0] : src[t][0], unset ? dflt[1] : src[t][1]};
    if (s[0] <= 0 || s[1] <= 0) return SLA2_EINVAL;
    if (s[1] < p->C || s[0] * esz[t] % 16 || s[1] * esz[t] % 16) return SLA2_EUNSUPPORTED;
    if (!extent_ok(2, count, s, p->C)) return SLA2_EUNSUPPORTED;
    *dst[t][0] = s[0];
    *dst[t][1] = s[1];
  }
  const bool unset = p->mod_stride[0] == 0 && p->mod_stride[1] == 0;
  if (p->mod_layout == SLA2_MOD_SHARED) {
    if (!unset) return SLA2_EINVAL;
  } else {
    const bool token = p->mod_layout == SLA2_MOD_TOKEN;
    const long long s[2] = {unset ? (token ? dflt[0] : p->C) : p->mod_stride[0], unset ? (token ? p->C : 0) : p->mod_stride[1]};
    if (s[0] <= 0 || (token ? s[1] <= 0 : s[1] != 0)) return SLA2_EINVAL;
    if (s[0] % 4 || s[1] % 4 || s[0] < p->C || (token && s[1] < p->C)) return SLA2_EUNSUPPORTED;
    if (!extent_ok(2, count, s, p->C)) return SLA2_EUNSUPPORTED;
    a->mod_b = s[0];
    a->mod_n = s[1];
  }
  a->B = p->B; a->N = p->N; a->C = p->C;
  a->norm_in = p->norm_in; a->norm_out = p->norm_out; a->mods = p->mod_layout;
  a->eps = p->eps; a->rho = p->residual_scale;
  a->x_bf16 = p->dtype_x == SLA2_BF16;
  a->h_bf16 = p->dtype_h == SLA2_BF16;
  return SLA2_OK;
}
static View x_view(const NormArgs& a, const void* p) { return View{p, a.x_bf16 ? 2 : 4, 2, a.C, {a.B, a.N}, {a.x_b, a.x_n}}; }
static View h_view(const NormArgs& a, const void* p) { return View{p, a.h_bf16 ? 2 : 4, 2, a.C, {a.B, a.N}, {a.h_b, a.h_n}}; }
static View mod_view(const NormArgs& a, const void* p) {
  if (a.mods == SLA2_MOD_SHARED) return flat(p, 4, a.C);
  return View{p, 4, 2, a.C, {a.B, a.mods == SLA2_MOD_TOKEN ? a.N : 1}, {a.mod_b, a.mod_n}};
}
static size_t norm_partial_bytes(const NormArgs& a) { return (size_t)3 * a.B * a.walkers * a.C * sizeof(float); }

}  // namespace sla2

using namespace sla2;

extern "C" {

size_t sla2_rope_workspace_bytes(const sla2_rope_params* params) {
  RopeArgs a;
  if (make_rope(params, true, 2, &a) != SLA2_OK) return 0;
  const size_t n = align256(rope_partial_floats(a) * sizeof(float));
  return n ? n : 256;
}

int sla2_rope_frequencies(const sla2_rope_params* params, double theta, double* freq) {
  RopeArgs a;
  const int rc = make_rope(params, false, 2, &a);
  if (rc != SLA2_OK) return rc;
  if (!freq || !(theta > 0.0 && theta < INFINITY)) return SLA2_EINVAL;
  for (int j = 0, first = 0, axis = 0; j < a.d / 2; j++) {
    while (axis < 3 && j >= a.pairs_end[axis]) first = a.pairs_end[axis++];
    freq[j] = axis == 3 ? 0.0 : pow(theta, -(double)(j - first) / (a.pairs_end[axis] - first));
  }
  return SLA2_OK;
}

int sla2_rope_forward(const sla2_rope_params* params, const void* q, const void* k, const double* freq, const int32_t* positions,
                      const float* q_weight, const float* k_weight, void* q_out, void* k_out, void* hip_stream) {
  RopeArgs a;
  const int rc = make_rope(params, false, k ? 2 : 1, &a);
  if (rc != SLA2_OK) return rc;
  if (!q || !q_out || !k != !k_out || (!k && k_weight)) return SLA2_EINVAL;
  if (misaligned16(q) || misaligned16(k) || misaligned16(q_out) || misaligned16(k_out)) return SLA2_EINVAL;
  if (!rope_inputs_ok(a, freq, positions, q_weight, k_weight)) return SLA2_EINVAL;
  const View in[6] = {head_view(a, a.sin, q), head_view(a, a.sin, k), flat(freq, 8, a.d / 2),
                      flat(positions, 4, 3ll * a.N * (a.positions_stride ? a.B : 1)), flat(q_weight, 4, weight_count(a)),
                      flat(k_weight, 4, weight_count(a))};
  const Output out[2] = {{head_view(a, a.sout, q_out), {q, nullptr}}, {head_view(a, a.sout, k_out), {k, nullptr}}};
  if (aliased(out, 2, in, 6)) return SLA2_EALIAS;
  a.x[0] = q; a.x[1] = k;
  a.y[0] = q_out; a.y[1] = k_out;
  a.weight[0] = q_weight; a.weight[1] = k_weight;
  a.freq = freq;
  a.positions = positions;
  return launch_rope(a, (hipStream_t)hip_stream) == hipSuccess ? SLA2_OK : SLA2_EHIP;
}

int sla2_rope_backward(const sla2_rope_params* params, const void* q, const void* k, const double* freq, const int32_t* positions,
                       const float* q_weight, const float* k_weight, const void* dq_out, const void* dk_out, void* dq, void* dk,
                       float* dq_weight, float* dk_weight, void* workspace, size_t workspace_bytes, void* hip_stream) {
  RopeArgs a;
  int rc = make_rope(params, true, dk ? 2 : 1, &a);
  if (rc != SLA2_OK) return rc;
  const bool normed = a.norm != SLA2_ROPE_NORM_NONE;
  if (!dq_out || !dq || !dk_out != !dk) return SLA2_EINVAL;
  if (normed && (!q || !k != !dk)) return SLA2_EINVAL;
  if ((!normed && (dq_weight || dk_weight)) || (!dk && (k_weight || dk_weight))) return SLA2_EINVAL;
  if (!normed) q = k = nullptr;
  if (misaligned16(q) || misaligned16(k) || misaligned16(dq_out) || misaligned16(dk_out) || misaligned16(dq) || misaligned16(dk))
    return SLA2_EINVAL;
  if (!vector_ok(dq_weight) || !vector_ok(dk_weight) || !rope_inputs_ok(a, freq, positions, q_weight, k_weight)) return SLA2_EINVAL;
  const View in[8] = {head_view(a, a.sin, q), head_view(a, a.sin, k), head_view(a, a.sout, dq_out), head_view(a, a.sout, dk_out),
                      flat(freq, 8, a.d / 2), flat(positions, 4, 3ll * a.N * (a.positions_stride ? a.B : 1)),
                      flat(q_weight, 4, weight_count(a)), flat(k_weight, 4, weight_count(a))};
  const bool sums = dq_weight || dk_weight;
  const size_t need = rope_partial_floats(a) * sizeof(float);
  const Output out[5] = {{head_view(a, a.sin, dq), {q, dq_out}}, {head_view(a, a.sin, dk), {k, dk_out}},
                         {flat(dq_weight, 4, weight_count(a)), {}}, {flat(dk_weight, 4, weight_count(a)), {}},
                         {flat(sums ? workspace : nullptr, 1, (long long)need), {}}};
  if (aliased(out, 5, in, 8)) return SLA2_EALIAS;
  if (sums) {
    if ((rc = check_workspace(need, workspace, workspace_bytes)) != SLA2_OK) return rc;
    a.partial = (float*)workspace;
  }
  a.x[0] = q; a.x[1] = k;
  a.dy[0] = dq_out; a.dy[1] = dk_out;
  a.y[0] = dq; a.y[1] = dk;
  a.weight[0] = q_weight; a.weight[1] = k_weight;
  a.dweight[0] = dq_weight; a.dweight[1] = dk_weight;
  a.freq = freq;
  a.positions = positions;
  return launch_rope_bwd(a, (hipStream_t)hip_stream) == hipSuccess ? SLA2_OK : SLA2_EHIP;
}

size_t sla2_norm_workspace_bytes(const sla2_norm_params* params) {
  NormArgs a;
  if (make_norm(params, &a) != SLA2_OK) return 0;
  plan_norm(&a, true);
  return align256(norm_partial_bytes(a));
}

int sla2_norm_forward(const sla2_norm_params* params, const void* x, const void* y, const float* gate, const float* out_weight,
                      void* x_out, const float* in_weight, const float* scale, const float* shift, void* h, void* hip_stream) {
  NormArgs a;
  const int rc = make_norm(params, &a);
  if (rc != SLA2_OK) return rc;
  if (!x || !y != !x_out || (!y && !h)) return SLA2_EINVAL;
  if ((!y && (gate || out_weight)) || (!h && (in_weight || scale || shift))) return SLA2_EINVAL;
  if (misaligned16(x) || misaligned16(y) || misaligned16(x_out) || misaligned16(h)) return SLA2_EINVAL;
  for (const float* v : {gate, out_weight, in_weight, scale, shift})
    if (!vector_ok(v)) return SLA2_EINVAL;
  const View in[7] = {x_view(a, x), h_view(a, y), mod_view(a, gate), flat(out_weight, 4, a.C), flat(in_weight, 4, a.C),
                      mod_view(a, scale), mod_view(a, shift)};
  const Output out[2] = {{x_view(a, x_out), {x, nullptr}}, {h_view(a, h), {y, nullptr}}};
  if (aliased(out, 2, in, 7)) return SLA2_EALIAS;
  a.x = x; a.y = y; a.gate = gate; a.out_weight = out_weight; a.x_out = x_out;
  a.in_weight = in_weight; a.scale = scale; a.shift = shift; a.h = h;
  plan_norm(&a, false);
  return launch_norm(a, (hipStream_t)hip_stream) == hipSuccess ? SLA2_OK : SLA2_EHIP;
}

int sla2_norm_backward(const sla2_norm_params* params, const void* x, const void* y, const float* gate, const float* out_weight,
                       const float* in_weight, const float* scale, const void* dh, const void* dx_out, void* dx, void* dy,
                       float* dgate, float* dout_weight, float* din_weight, float* dscale, float* dshift, void* workspace,
                       size_t workspace_bytes, void* hip_stream) {
  NormArgs a;
  int rc = make_norm(params, &a);
  if (rc != SLA2_OK) return rc;
  if (!dx || !y != !dy || (!dh && !(y && dx_out)) || (dh && !x)) return SLA2_EINVAL;
  if ((!y && (gate || out_weight)) || (!dh && (in_weight || scale || dshift))) return SLA2_EINVAL;
  if ((dgate && !gate) || (dout_weight && !out_weight) || (din_weight && !in_weight) || (dscale && !scale)) return SLA2_EINVAL;
  if (!dh) x = nullptr;
  for (const void* p : {x, y, dh, dx_out, (const void*)dx, (const void*)dy})
    if (misaligned16(p)) return SLA2_EINVAL;
  for (const float* v : {gate, out_weight, in_weight, scale, (const float*)dgate, (const float*)dout_weight, (const float*)din_weight,
                         (const float*)dscale, (const float*)dshift})
    if (!vector_ok(v)) return SLA2_EINVAL;
  const View in[8] = {x_view(a, x), h_view(a, y), mod_view(a, gate), flat(out_weight, 4, a.C), flat(in_weight, 4, a.C),
                      mod_view(a, scale), h_view(a, dh), x_view(a, dx_out)};
  plan_norm(&a, true);
  const bool sums = dgate || dout_weight || din_weight || dscale || dshift;
  const size_t need = norm_partial_bytes(a);
  const Output out[8] = {{x_view(a, dx), {x, dx_out}}, {h_view(a, dy), {y, dh}}, {mod_view(a, dgate), {}}, {flat(dout_weight, 4, a.C), {}},
                         {flat(din_weight, 4, a.C), {}}, {mod_view(a, dscale), {}}, {mod_view(a, dshift), {}},
                         {flat(sums ? workspace : nullptr, 1, (long long)need), {}}};
  if (aliased(out, 8, in, 8)) return SLA2_EALIAS;
  if (sums) {
    if ((rc = check_workspace(need, workspace, workspace_bytes)) != SLA2_OK) return rc;
    a.partial = (float*)workspace;
  }
  a.x = x; a.y = y; a.gate = gate; a.out_weight = out_weight; a.in_weight = in_weight; a.scale = scale;
  a.dh = dh; a.dx_out = dx_out; a.dx = dx; a.dy = dy;
  a.dgate = dgate; a.dout_weight = dout_weight; a.din_weight = din_weight; a.dscale = dscale; a.dshift = dshift;
  return launch_norm_bwd(a, (hipStream_t)hip_stream) == hipSuccess ? SLA2_OK : SLA2_EHIP;
}

}  // extern "C"
