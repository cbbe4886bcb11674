// Host side of attention over packed sequences and of the paged cache (sla2_packed_*, sla2_cache_*): argument validation and launches.
// Declarations and their contracts are in include/sla2.h.
#include <limits.h>
#include <math.h>

#include "cache.h"
#include "host_checks.h"
#include "packed.h"

namespace sla2 {

static bool misaligned4(const void* p) { return ((uintptr_t)p & 3u) != 0; }
static bool rate_ok(float s) { return s >= 0.f && s < INFINITY; }
static float rate_or_default(float s, int d) { return s > 0.f ? s : 1.f / sqrtf((float)d); }

static int heads_ok(int H, int H_kv, int d, int dtype, float scale) {
  if (H < 1 || H_kv < 1 || H % H_kv || !rate_ok(scale)) return SLA2_EINVAL;
  if (dtype != SLA2_F32 && dtype != SLA2_BF16) return SLA2_EINVAL;
  if ((d != 64 && d != 128) || dtype != SLA2_BF16 || H > 65535) return SLA2_EUNSUPPORTED;
  return SLA2_OK;
}

// (head, row) strides of a [rows, heads, d] tensor of bf16
static int row_strides(const long long* src, int rows, int heads, int d, long long* h, long long* t) {
  const bool unset = src[0] == 0 && src[1] == 0;
  *h = unset ? d : src[0];
  *t = unset ? (long long)heads * d : src[1];
  if (*h <= 0 || *t <= 0) return SLA2_EINVAL;
  if (*h % 8 || *t % 8 || *t < d || *t >= 1 << 24) return SLA2_EUNSUPPORTED;
  const long long count[2] = {heads, rows > 0 ? rows : 1}, stride[2] = {*h, *t};
  return extent_ok(2, count, stride, d) ? SLA2_OK : SLA2_EUNSUPPORTED;
}
static View rows_view(const void* p, int rows, int heads, int d, long long h, long long t) {
  return View{rows ? p : nullptr, 2, 2, d, {heads, rows}, {h, t}};
}

// The workspace of a call, and where its parts lie
static size_t packed_layout(PackedArgs* a, bool backward, void* ws) {
  size_t off = 0;
  auto take = [&](size_t floats) {
    float* p = ws ? (float*)((char*)ws + off) : nullptr;
    off = align256(off + floats * sizeof(float));
    return p;
  };
  const size_t rows = (size_t)a->Tq * a->H;
  plan_packed(a, backward);
  if (backward) {
    a->lse2 = take(stat_rows(*a) * a->Hkv + 64);       // a step's 64 are read whole
    a->delta = take(stat_rows(*a) * a->Hkv + 64);
    if (a->k_parts > 1) a->part_kv = take(2 * (size_t)a->k_parts * a->Tk * a->Hkv * a->d);
  }
  if (a->q_parts > 1) {
    a->part_o = take(a->q_parts * rows * a->d);
    if (!backward) a->part_ml = take(2 * a->q_parts * rows);
  }
  return off ? off : 256;
}

static int make_packed(const sla2_packed_params* p, PackedArgs* a) {
  if (!p) return SLA2_EINVAL;
  if (p->sequences < 1 || p->tokens_q < 0 || p->tokens_k < 0 || (p->causal != 0 && p->causal != 1)) return SLA2_EINVAL;
  int rc = heads_ok(p->H, p->H_kv, p->d, p->dtype, p->scale);
  if (rc != SLA2_OK) return rc;
  if (p->sequences > 65535) return SLA2_EUNSUPPORTED;
  *a = PackedArgs{};
  long long t[4];
  if ((rc = row_strides(p->q_stride, p->tokens_q, p->H, p->d, &a->sq.h, &t[0])) != SLA2_OK) return rc;
  if ((rc = row_strides(p->kv_stride, p->tokens_k, p->H_kv, p->d, &a->skv.h, &t[1])) != SLA2_OK) return rc;
  if ((rc = row_strides(p->out_stride, p->tokens_q, p->H, p->d, &a->so.h, &t[2])) != SLA2_OK) return rc;
  a->sq.t = (int)t[0];
  a->skv.t = (int)t[1];
  a->so.t = (int)t[2];
  a->sg = a->so;
  if (p->dout_stride[0] || p->dout_stride[1]) {
    if ((rc = row_strides(p->dout_stride, p->tokens_q, p->H, p->d, &a->sg.h, &t[3])) != SLA2_OK) return rc;
    a->sg.t = (int)t[3];
  }
  a->S = p->sequences;
  a->Tq = p->tokens_q;
  a->Tk = p->tokens_k;
  a->H = p->H;
  a->Hkv = p->H_kv;
  a->group = p->H / p->H_kv;
  a->d = p->d;
  a->causal = p->causal != 0;
  a->scale = rate_or_default(p->scale, p->d);
  // Rows (queries of all heads, the backward pass's blocks of 16 filled up) are counted in 31 bits, and a launch has less than 2^24
  // workgroups of 256: tiles of 128 rows or keys, and for each sequence one that is not full.
  const long long last = 128ll * a->S;
  if ((a->Tq + last) * a->H > INT_MAX - 1024 || (a->Tk + last) * a->H > INT_MAX - 1024) return SLA2_EUNSUPPORTED;
  return SLA2_OK;
}
static View q_view(const PackedArgs& a, const void* p) { return rows_view(p, a.Tq, a.H, a.d, a.sq.h, a.sq.t); }
static View kv_view(const PackedArgs& a, const void* p) { return rows_view(p, a.Tk, a.Hkv, a.d, a.skv.h, a.skv.t); }
static View out_view(const PackedArgs& a, const void* p) { return rows_view(p, a.Tq, a.H, a.d, a.so.h, a.so.t); }
static View dout_view(const PackedArgs& a, const void* p) { return rows_view(p, a.Tq, a.H, a.d, a.sg.h, a.sg.t); }
static View starts_view(const PackedArgs& a, const int32_t* p) { return flat(p, 4, (long long)a.S + 1); }
static View lse_view(const PackedArgs& a, const float* p) { return flat(a.Tq ? p : nullptr, 4, (long long)a.H * a.Tq); }

static int make_cache(const sla2_cache_params* p, CacheArgs* a) {
  if (!p) return SLA2_EINVAL;
  if (p->B < 1 || p->pages < 1 || p->max_pages < 1 || p->tokens < 0 || p->table_stride < 0) return SLA2_EINVAL;
  if (p->quant_mode < SLA2_QUANT_NONE || p->quant_mode > SLA2_QUANT_FP8_V) return SLA2_EINVAL;
  int rc = heads_ok(p->H, p->H_kv, p->d, p->dtype, p->scale);
  if (rc != SLA2_OK) return rc;
  int shift = 0;
  while (shift < 9 && 1 << shift != p->page_size) shift++;
  if (shift < 4 || shift > 8) return SLA2_EUNSUPPORTED;
  if (p->tokens > kMostCacheTokens || p->quant_mode == SLA2_QUANT_FP8_V || p->B > 65535 || (long long)p->max_pages << shift > INT_MAX) return SLA2_EUNSUPPORTED;
  *a = CacheArgs{};
  a->table_stride = p->table_stride ? p->table_stride : p->max_pages;
  if (a->table_stride < p->max_pages) return SLA2_EINVAL;
  const long long rows = 1ll << shift, dflt[3] = {(long long)p->H_kv * rows * p->d, rows * p->d, p->d};
  const long long* src = p->cache_stride;
  const bool unset = src[0] == 0 && src[1] == 0 && src[2] == 0;
  const long long s[3] = {unset ? dflt[0] : src[0], unset ? dflt[1] : src[1], unset ? dflt[2] : src[2]};
  const int esz = p->quant_mode == SLA2_QUANT_NONE ? 2 : 1;
  for (long long st : s)
    if (st <= 0) return SLA2_EINVAL;
  for (long long st : s)
    if (st >= 1ll << 40 || st * esz % 16) return SLA2_EUNSUPPORTED;
  if (s[2] < p->d || s[2] >= 1 << 24) return SLA2_EUNSUPPORTED;
  const long long count[3] = {p->pages, p->H_kv, rows};
  if (!extent_ok(3, count, s, p->d)) return SLA2_EUNSUPPORTED;
  const long long table[1] = {p->B}, table_s[1] = {a->table_stride};
  if (!extent_ok(1, table, table_s, p->max_pages)) return SLA2_EUNSUPPORTED;
  if ((rc = row_strides(p->kv_stride, p->tokens, p->H_kv, p->d, &a->kv_h, &a->kv_t)) != SLA2_OK) return rc;
  if ((rc = row_strides(p->q_stride, p->B, p->H, p->d, &a->q_h, &a->q_b)) != SLA2_OK) return rc;
  if ((rc = row_strides(p->out_stride, p->B, p->H, p->d, &a->out_h, &a->out_b)) != SLA2_OK) return rc;
  a->page_stride = s[0];
  a->head_stride = s[1];
  a->token_stride = s[2];
  a->B = p->B;
  a->H = p->H;
  a->Hkv = p->H_kv;
  a->group = p->H / p->H_kv;
  a->d = p->d;
  a->pages = p->pages;
  a->page_shift = shift;
  a->max_pages = p->max_pages;
  a->tokens = p->tokens;
  a->quant = p->quant_mode;
  a->scale = rate_or_default(p->scale, p->d);
  plan_cache_attention(a);
  return SLA2_OK;
}
static View cache_view(const CacheArgs& a, const void* p) {
  return View{p, a.quant == SLA2_QUANT_NONE ? 2 : 1, 3, a.d, {a.pages, a.Hkv, 1ll << a.page_shift}, {a.page_stride, a.head_stride, a.token_stride}};
}
static View scale_view(const CacheArgs& a, const float* p) { return flat(p, 4, (long long)a.pages * a.Hkv << a.page_shift); }
static View table_view(const CacheArgs& a, const int32_t* p) { return flat(p, 4, (a.B - 1) * a.table_stride + a.max_pages); }
static View cache_rows(const CacheArgs& a, const void* p) { return rows_view(p, a.tokens, a.Hkv, a.d, a.kv_h, a.kv_t); }

// what every entry point checks of the cache itself
static bool cache_ok(const CacheArgs& a, const void* kc, const void* vc, const float* ks, const float* vs, const int32_t* table) {
  if (!kc || !vc || !table || misaligned16(kc) || misaligned16(vc) || misaligned4(table)) return false;
  if (a.quant == SLA2_QUANT_NONE) return !ks && !vs;
  return ks && vs && !misaligned16(ks) && !misaligned16(vs);
}

static int move_rows(const sla2_cache_params* params, bool write, const void* k, const void* v, const int32_t* start, const int32_t* first,
                     const int32_t* table, const void* kc, const void* vc, const float* ks, const float* vs, void* stream) {
  CacheArgs a;
  const int rc = make_cache(params, &a);
  if (rc != SLA2_OK) return rc;
  if (!cache_ok(a, kc, vc, ks, vs, table) || misaligned4(start) || misaligned4(first)) return SLA2_EINVAL;
  if ((a.tokens && (!k || !v)) || (!start && a.tokens > a.B)) return SLA2_EINVAL;
  if (misaligned16(k) || misaligned16(v)) return SLA2_EINVAL;
  const View rows[2] = {cache_rows(a, k), cache_rows(a, v)};
  const View cache[4] = {cache_view(a, kc), cache_view(a, vc), scale_view(a, ks), scale_view(a, vs)};
  const View plan[3] = {flat(start, 4, a.B + 1ll), flat(first, 4, a.B), table_view(a, table)};
  if (write) {
    const Output out[4] = {{cache[0], {}}, {cache[1], {}}, {cache[2], {}}, {cache[3], {}}};
    const View in[5] = {rows[0], rows[1], plan[0], plan[1], plan[2]};
    if (aliased(out, 4, in, 5)) return SLA2_EALIAS;
  } else {
    const Output out[2] = {{rows[0], {}}, {rows[1], {}}};
    const View in[7] = {cache[0], cache[1], cache[2], cache[3], plan[0], plan[1], plan[2]};
    if (aliased(out, 2, in, 7)) return SLA2_EALIAS;
  }
  a.k = (uint16_t*)k;
  a.v = (uint16_t*)v;
  a.kc = (void*)kc;
  a.vc = (void*)vc;
  a.ks = (float*)ks;
  a.vs = (float*)vs;
  a.start = start;
  a.first = first;
  a.table = table;
  return (write ? launch_cache_write(a, (hipStream_t)stream) : launch_cache_read(a, (hipStream_t)stream)) == hipSuccess ? SLA2_OK : SLA2_EHIP;
}

}  // namespace sla2

using namespace sla2;

extern "C" {

size_t sla2_packed_workspace_bytes(const sla2_packed_params* params, int backward) {
  PackedArgs a;
  if ((backward != 0 && backward != 1) || make_packed(params, &a) != SLA2_OK) return 0;
  const size_t fwd = packed_layout(&a, false, nullptr), bwd = backward ? packed_layout(&a, true, nullptr) : 0;
  return fwd > bwd ? fwd : bwd;
}

int sla2_packed_forward(const sla2_packed_params* params, const void* q, const void* k, const void* v, const int32_t* q_start,
                        const int32_t* k_start, void* out, float* lse_or_null, void* workspace, size_t workspace_bytes, void* hip_stream) {
  PackedArgs a;
  int rc = make_packed(params, &a);
  if (rc != SLA2_OK) return rc;
  if ((a.Tq && (!q || !out)) || (a.Tk && (!k || !v)) || !q_start || !k_start) return SLA2_EINVAL;
  if (misaligned16(q) || misaligned16(k) || misaligned16(v) || misaligned16(out)) return SLA2_EINVAL;
  if (misaligned4(q_start) || misaligned4(k_start) || misaligned4(lse_or_null)) return SLA2_EINVAL;
  const size_t need = packed_layout(&a, false, workspace);
  const View in[5] = {q_view(a, q), kv_view(a, k), kv_view(a, v), starts_view(a, q_start), starts_view(a, k_start)};
  const Output outs[3] = {{out_view(a, out), {}}, {lse_view(a, lse_or_null), {}}, {flat(workspace, 1, (long long)need), {}}};
  if (aliased(outs, 3, in, 5)) return SLA2_EALIAS;
  if ((rc = check_workspace(need, workspace, workspace_bytes)) != SLA2_OK) return rc;
  a.q = (const uint16_t*)q;
  a.k = (const uint16_t*)k;
  a.v = (const uint16_t*)v;
  a.q_start = q_start;
  a.k_start = k_start;
  a.o = (uint16_t*)out;
  a.lse_out = lse_or_null;
  return launch_packed_fwd(a, (hipStream_t)hip_stream) == hipSuccess ? SLA2_OK : SLA2_EHIP;
}

int sla2_packed_backward(const sla2_packed_params* params, const void* q, const void* k, const void* v, const int32_t* q_start,
                         const int32_t* k_start, const void* out, const float* lse, const void* dout, void* dq, void* dk, void* dv,
                         void* workspace, size_t workspace_bytes, void* hip_stream) {
  PackedArgs a;
  int rc = make_packed(params, &a);
  if (rc != SLA2_OK) return rc;
  if ((a.Tq && (!q || !out || !lse || !dout || !dq)) || (a.Tk && (!k || !v || !dk || !dv)) || !q_start || !k_start) return SLA2_EINVAL;
  for (const void* p : {q, k, v, out, dout, (const void*)dq, (const void*)dk, (const void*)dv})
    if (misaligned16(p)) return SLA2_EINVAL;
  if (misaligned4(q_start) || misaligned4(k_start) || misaligned4(lse)) return SLA2_EINVAL;
  const size_t need = packed_layout(&a, true, workspace);
  const View in[8] = {q_view(a, q), kv_view(a, k), kv_view(a, v), out_view(a, out), dout_view(a, dout), lse_view(a, lse),
                      starts_view(a, q_start), starts_view(a, k_start)};
  const Output outs[4] = {{q_view(a, dq), {}}, {kv_view(a, dk), {}}, {kv_view(a, dv), {}}, {flat(workspace, 1, (long long)need), {}}};
  if (aliased(outs, 4, in, 8)) return SLA2_EALIAS;
  if ((rc = check_workspace(need, workspace, workspace_bytes)) != SLA2_OK) return rc;
  a.q = (const uint16_t*)q;
  a.k = (const uint16_t*)k;
  a.v = (const uint16_t*)v;
  a.q_start = q_start;
  a.k_start = k_start;
  a.out = (const uint16_t*)out;
  a.lse = lse;
  a.dout = (const uint16_t*)dout;
  a.dq = (uint16_t*)dq;
  a.dk = (uint16_t*)dk;
  a.dv = (uint16_t*)dv;
  return launch_packed_bwd(a, (hipStream_t)hip_stream) == hipSuccess ? SLA2_OK : SLA2_EHIP;
}

int sla2_cache_write(const sla2_cache_params* params, const void* k, const void* v, const int32_t* start, const int32_t* first,
                     const int32_t* page_table, void* k_cache, void* v_cache, float* k_scale, float* v_scale, void* hip_stream) {
  return move_rows(params, true, k, v, start, first, page_table, k_cache, v_cache, k_scale, v_scale, hip_stream);
}

int sla2_cache_read(const sla2_cache_params* params, const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale,
                    const int32_t* start, const int32_t* first, const int32_t* page_table, void* k, void* v, void* hip_stream) {
  return move_rows(params, false, k, v, start, first, page_table, k_cache, v_cache, k_scale, v_scale, hip_stream);
}

size_t sla2_cache_workspace_bytes(const sla2_cache_params* params) {
  CacheArgs a;
  if (make_cache(params, &a) != SLA2_OK) return 0;
  const size_t n = align256(cache_part_floats(a) * sizeof(float));
  return n ? n : 256;
}

int sla2_cache_attention(const sla2_cache_params* params, const void* q, const void* k_cache, const void* v_cache, const float* k_scale,
                         const float* v_scale, const int32_t* length, const int32_t* page_table, void* out, float* lse_or_null,
                         void* workspace, size_t workspace_bytes, void* hip_stream) {
  CacheArgs a;
  int rc = make_cache(params, &a);
  if (rc != SLA2_OK) return rc;
  if (!q || !out || !length || !cache_ok(a, k_cache, v_cache, k_scale, v_scale, page_table)) return SLA2_EINVAL;
  if (misaligned16(q) || misaligned16(out) || misaligned4(length) || misaligned4(lse_or_null)) return SLA2_EINVAL;
  const size_t need = sla2_cache_workspace_bytes(params);
  const View in[7] = {rows_view(q, a.B, a.H, a.d, a.q_h, a.q_b), cache_view(a, k_cache), cache_view(a, v_cache), scale_view(a, k_scale),
                      scale_view(a, v_scale), flat(length, 4, a.B), table_view(a, page_table)};
  const Output outs[3] = {{rows_view(out, a.B, a.H, a.d, a.out_h, a.out_b), {q, nullptr}}, {flat(lse_or_null, 4, (long long)a.B * a.H), {}},
                          {flat(workspace, 1, (long long)need), {}}};
  if (aliased(outs, 3, in, 7)) return SLA2_EALIAS;
  if ((rc = check_workspace(need, workspace, workspace_bytes)) != SLA2_OK) return rc;
  a.q = (const uint16_t*)q;
  a.kc = (void*)k_cache;
  a.vc = (void*)v_cache;
  a.ks = (float*)k_scale;
  a.vs = (float*)v_scale;
  a.length = length;
  a.table = page_table;
  a.out = (uint16_t*)out;
  a.lse = lse_or_null;
  a.part_o = (float*)workspace;
  a.part_ml = a.part_o + (size_t)a.parts * 2 * a.H * a.d;
  return launch_cache_attention(a, (hipStream_t)hip_stream) == hipSuccess ? SLA2_OK : SLA2_EHIP;
}

}  // extern "C"
