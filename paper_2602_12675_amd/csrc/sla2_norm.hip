// Norms before and after a block, with the block's modulation, gate and residual:
//   x' = rho x + g (.) norm_out(y) w_out          h = norm_in(x') w_in (.) (1 + s) + b
// and the gradients of all of them.  norm(v) = (v - mu) r with mu = mean(v) (layer) or 0 (rms), r = 1 / sqrt(mean((v - mu)^2) + eps).
//
// Forward: a row of x and y is read once and x' and h are written once; what is the same for all rows of a batch (g w_out, w_in (1 + s), b)
// stays in registers while a workgroup goes through its rows.  h is taken of x' as it is stored, so the one call gives the bits of two.
//
// Backward, per row, with n = norm_in(x'), a = w_in (1 + s), t = dh a, m = norm_out(y):
//   u = dx' + r (t - mean(t) [layer] - n mean(t n)),   dx = rho u
//   t2 = u g w_out,   dy = r2 (t2 - mean(t2) [layer] - m mean(t2 m))
// and, over the rows of a batch, P = sum dh n, S = sum dh, Q = sum u m: ds = w_in P, db = S, dw_in = sum over batches of (1 + s) P,
// dg = w_out Q, dw_out = sum over batches of g Q.  Statistics are formed again from the row, which is in registers anyhow.  A
// workgroup adds up P, S, Q of its rows in registers, its teams theirs in a fixed order, and a second launch adds up the workgroups'.
// A modulation of every token needs no sums but those of the weights.
#include "rows.h"

namespace sla2 {

constexpr int kBefore = 1, kAfter = 2;       // parts of a call: h; x'

struct Moments {
  float mu, r;
};

// mu and r of the team's row x; places without a channel hold 0.  Several waves: the second moments of the waves around their own means
// are joined by M2 = sum of M2_w + n_w (mu_w - mu)^2, so that nothing is lost to a mean that is large beside the spread.
template <int V>
__device__ __forceinline__ Moments moments(Team& tm, int kind, const float (&x)[V][8], const bool (&has)[V], int chunks, float eps) {
  if (kind == SLA2_NORM_NONE) return {0.f, 1.f};
  const float count = (float)(chunks * kChunk);
  float s[1] = {0.f};
  if (kind == SLA2_NORM_RMS) {
#pragma unroll
    for (int v = 0; v < V; v++)
#pragma unroll
      for (int i = 0; i < 8; i++) s[0] += x[v][i] * x[v][i];
    tm.sum(s);
    return {0.f, 1.f / sqrtf(s[0] / count + eps)};
  }
#pragma unroll
  for (int v = 0; v < V; v++)
#pragma unroll
    for (int i = 0; i < 8; i++) s[0] += x[v][i];
  s[0] = lanes_sum(s[0], tm.t.lanes);
  const int wave = tm.lane / kWave;
  const float mine = tm.t.waves == 1 ? count : tm.channels(wave, chunks);
  float mu = mine > 0.f ? s[0] / mine : 0.f, m2 = 0.f;
#pragma unroll
  for (int v = 0; v < V; v++)
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const float c = has[v] ? x[v][i] - mu : 0.f;
      m2 += c * c;
    }
  m2 = lanes_sum(m2, tm.t.lanes);
  if (tm.t.waves > 1) {
    const float mean_of[2] = {s[0], m2};
    float all = 0.f, spread = 0.f, square = 0.f;
    tm.exchange(mean_of, [&](int, const float* o) { all += o[0]; });
    all /= count;
    const float* first = tm.last<2>();
    for (int w = 0; w < tm.t.waves; w++) {
      const float n = tm.channels(w, chunks), d = n > 0.f ? first[2 * w] / n - all : 0.f;
      spread += first[2 * w + 1];
      square += n * d * d;
    }
    mu = all;
    m2 = spread + square;
  }
  return {mu, 1.f / sqrtf(m2 / count + eps)};
}

// The same with mean(t) and mean(t n), n = (x - mu) r, for the gradient t behind the norm (kind is not none): all sums in one exchange.
struct BackMoments {
  float mu, r, t, tn;
};
template <int V>
__device__ __forceinline__ BackMoments back_moments(Team& tm, int kind, const float (&x)[V][8], const float (&t)[V][8], const bool (&has)[V],
                                                    int chunks, float eps) {
  if (kind == SLA2_NORM_NONE) return {0.f, 1.f, 0.f, 0.f};
  const float count = (float)(chunks * kChunk);
  if (kind == SLA2_NORM_RMS) {
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int v = 0; v < V; v++)
#pragma unroll
      for (int i = 0; i < 8; i++) {
        s[0] += x[v][i] * x[v][i];
        s[1] += t[v][i] * x[v][i];
      }
    tm.sum(s);
    const float r = 1.f / sqrtf(s[0] / count + eps);
    return {0.f, r, 0.f, s[1] * r / count};
  }
  float s = 0.f;
#pragma unroll
  for (int v = 0; v < V; v++)
#pragma unroll
    for (int i = 0; i < 8; i++) s += x[v][i];
  s = lanes_sum(s, tm.t.lanes);
  const float mine = tm.t.waves == 1 ? count : tm.channels(tm.lane / kWave, chunks);
  float mu = mine > 0.f ? s / mine : 0.f, m2 = 0.f, st = 0.f, stx = 0.f;
#pragma unroll
  for (int v = 0; v < V; v++)
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const float c = has[v] ? x[v][i] - mu : 0.f;
      m2 += c * c;
      st += t[v][i];
      stx += t[v][i] * c;
    }
  m2 = lanes_sum(m2, tm.t.lanes);
  st = lanes_sum(st, tm.t.lanes);
  stx = lanes_sum(stx, tm.t.lanes);
  if (tm.t.waves > 1) {
    const float own[4] = {s, m2, st, stx};
    float all = 0.f;
    tm.exchange(own, [&](int, const float* o) { all += o[0]; });
    all /= count;
    const float* first = tm.last<4>();
    m2 = st = stx = 0.f;
    for (int w = 0; w < tm.t.waves; w++) {
      const float n = tm.channels(w, chunks), d = n > 0.f ? first[4 * w] / n - all : 0.f;
      m2 += first[4 * w + 1] + n * d * d;
      st += first[4 * w + 2];
      stx += first[4 * w + 3] + d * first[4 * w + 2];
    }
    mu = all;
  }
  const float r = 1.f / sqrtf(m2 / count + eps);
  return {mu, r, st / count, stx * r / count};
}

// x' and h of the rows of a workgroup: of one batch, every walkers-th step.
template <int V, bool XB, bool HB, int PART, bool TOKEN>
__global__ __launch_bounds__(kTeamThreads) void norm_kernel(NormArgs a) {
  __shared__ float lds[kExchangeFloats];
  Team tm(a.team, lds);
  const int b = (int)blockIdx.x / a.walkers, walker = (int)blockIdx.x % a.walkers, chunks = a.C / kChunk;
  const bool own = tm.team < a.teams;
  bool has[V];
  int col[V];
  float g[V][8], w[V][8], sh[V][8], wo[V][8], wi[V][8];   // g w_out; w_in (1 + s); b.  TOKEN: w_out, w_in alone, the rest row by row
  const size_t mod = (size_t)b * a.mod_b;
#pragma unroll
  for (int v = 0; v < V; v++) {
    const int c = tm.lane + v * a.team.threads();
    has[v] = own && c < chunks;
    col[v] = has[v] ? c * kChunk : 0;
    if (PART & kAfter) load_vector8(a.out_weight, col[v], 1.f, wo[v]);
    if (PART & kBefore) load_vector8(a.in_weight, col[v], 1.f, wi[v]);
    if (!TOKEN) {
      if (PART & kAfter) {
        load_vector8(a.gate, mod + col[v], 1.f, g[v]);
#pragma unroll
        for (int i = 0; i < 8; i++) g[v][i] *= wo[v][i];
      }
      if (PART & kBefore) {
        load_vector8(a.scale, mod + col[v], 0.f, w[v]);
        load_vector8(a.shift, mod + col[v], 0.f, sh[v]);
#pragma unroll
        for (int i = 0; i < 8; i++) w[v][i] = wi[v][i] * (1.f + w[v][i]);
      }
    }
  }
  for (long long n0 = (long long)walker * a.teams; n0 < a.N; n0 += (long long)a.walkers * a.teams) {
    const long long n = n0 + tm.team;
    const bool row = own && n < a.N;
    const size_t xo = (size_t)b * a.x_b + (row ? n : 0) * a.x_n, ho = (size_t)b * a.h_b + (row ? n : 0) * a.h_n;
    Raw<XB> rx[V];
    Raw<HB> ry[V];
#pragma unroll
    for (int v = 0; v < V; v++) {
      const bool on = row && has[v];
      rx[v] = on ? load8<XB>(a.x, xo + col[v]) : zero8<XB>();
      if (PART & kAfter) ry[v] = on ? load8<HB>(a.y, ho + col[v]) : zero8<HB>();
    }
    if (TOKEN) {
      const size_t m = mod + (row ? n : 0) * a.mod_n;
#pragma unroll
      for (int v = 0; v < V; v++) {
        if (PART & kAfter) {
          load_vector8(a.gate, m + col[v], 1.f, g[v]);
#pragma unroll
          for (int i = 0; i < 8; i++) g[v][i] *= wo[v][i];
        }
        if (PART & kBefore) {
          load_vector8(a.scale, m + col[v], 0.f, w[v]);
          load_vector8(a.shift, m + col[v], 0.f, sh[v]);
#pragma unroll
          for (int i = 0; i < 8; i++) w[v][i] = wi[v][i] * (1.f + w[v][i]);
        }
      }
    }
    float x[V][8];
#pragma unroll
    for (int v = 0; v < V; v++) unpack8<XB>(rx[v], x[v]);
    if (PART & kAfter) {
      float y[V][8];
#pragma unroll
      for (int v = 0; v < V; v++) unpack8<HB>(ry[v], y[v]);
      const Moments m = moments<V>(tm, a.norm_out, y, has, chunks, a.eps);
#pragma unroll
      for (int v = 0; v < V; v++) {
#pragma unroll
        for (int i = 0; i < 8; i++) x[v][i] = a.rho * x[v][i] + g[v][i] * ((y[v][i] - m.mu) * m.r);
        rx[v] = pack8<XB>(x[v]);
        if (row && has[v]) store8<XB>(a.x_out, xo + col[v], rx[v]);
        else rx[v] = zero8<XB>();
        unpack8<XB>(rx[v], x[v]);
      }
    }
    if (PART & kBefore) {
      const Moments m = moments<V>(tm, a.norm_in, x, has, chunks, a.eps);
#pragma unroll
      for (int v = 0; v < V; v++) {
#pragma unroll
        for (int i = 0; i < 8; i++) x[v][i] = ((x[v][i] - m.mu) * m.r) * w[v][i] + sh[v][i];
        if (row && has[v]) store8<HB>(a.h, ho + col[v], pack8<HB>(x[v]));
      }
    }
  }
}

// One of the sums of a workgroup: its teams' in order, through LDS, into row `at` of the partial sums.
template <int V>
__device__ __forceinline__ void store_partial(const Team& tm, int teams, float* lds, const float (&acc)[V][8], const bool (&has)[V],
                                              const int (&col)[V], int C, float* to) {
  if (teams > 1) {
    __syncthreads();
    if (tm.team > 0 && tm.team < teams) {
#pragma unroll
      for (int v = 0; v < V; v++)
        if (has[v]) {
          float* p = lds + (size_t)(tm.team - 1) * C + col[v];
          *(f32x4*)p = f32x4{acc[v][0], acc[v][1], acc[v][2], acc[v][3]};
          *(f32x4*)(p + 4) = f32x4{acc[v][4], acc[v][5], acc[v][6], acc[v][7]};
        }
    }
    __syncthreads();
  }
  if (tm.team == 0) {
#pragma unroll
    for (int v = 0; v < V; v++)
      if (has[v]) {
        float s[8];
#pragma unroll
        for (int i = 0; i < 8; i++) s[i] = acc[v][i];
        for (int t = 1; t < teams; t++) {
          const float* p = lds + (size_t)(t - 1) * C + col[v];
#pragma unroll
          for (int i = 0; i < 8; i++) s[i] += p[i];
        }
        store8<false>(to, col[v], pack8<false>(s));
      }
  }
}

template <int V, bool XB, bool HB, int PART, bool TOKEN>
__global__ __launch_bounds__(kTeamThreads) void norm_bwd_kernel(NormArgs a) {
  __shared__ float lds[kExchangeFloats];
  extern __shared__ float teams_lds[];       // [teams - 1][C]
  Team tm(a.team, lds);
  const int b = (int)blockIdx.x / a.walkers, walker = (int)blockIdx.x % a.walkers, chunks = a.C / kChunk;
  const bool own = tm.team < a.teams;
  bool has[V];
  int col[V];
  float g[V][8], w[V][8], wo[V][8], wi[V][8];
  float p_sum[V][8], s_sum[V][8], q_sum[V][8];            // TOKEN: of d w_in, nothing, of d w_out
  const size_t mod = (size_t)b * a.mod_b;
#pragma unroll
  for (int v = 0; v < V; v++) {
    const int c = tm.lane + v * a.team.threads();
    has[v] = own && c < chunks;
    col[v] = has[v] ? c * kChunk : 0;
#pragma unroll
    for (int i = 0; i < 8; i++) p_sum[v][i] = s_sum[v][i] = q_sum[v][i] = 0.f;
    if (PART & kAfter) load_vector8(a.out_weight, col[v], 1.f, wo[v]);
    if (PART & kBefore) load_vector8(a.in_weight, col[v], 1.f, wi[v]);
    if (!TOKEN) {
      if (PART & kAfter) {
        load_vector8(a.gate, mod + col[v], 1.f, g[v]);
#pragma unroll
        for (int i = 0; i < 8; i++) g[v][i] *= wo[v][i];
      }
      if (PART & kBefore) {
        load_vector8(a.scale, mod + col[v], 0.f, w[v]);
#pragma unroll
        for (int i = 0; i < 8; i++) w[v][i] = wi[v][i] * (1.f + w[v][i]);
      }
    }
  }
  for (long long n0 = (long long)walker * a.teams; n0 < a.N; n0 += (long long)a.walkers * a.teams) {
    const long long n = n0 + tm.team;
    const bool row = own && n < a.N;
    const size_t xo = (size_t)b * a.x_b + (row ? n : 0) * a.x_n, ho = (size_t)b * a.h_b + (row ? n : 0) * a.h_n;
    const size_t mo = mod + (TOKEN && row ? n : 0) * a.mod_n;
    Raw<XB> rx[V], ru[V];
    Raw<HB> ry[V], rh[V];
#pragma unroll
    for (int v = 0; v < V; v++) {
      const bool on = row && has[v];
      if (PART & kBefore) {
        rx[v] = on && a.x ? load8<XB>(a.x, xo + col[v]) : zero8<XB>();
        rh[v] = on ? load8<HB>(a.dh, ho + col[v]) : zero8<HB>();
      }
      ru[v] = on && a.dx_out ? load8<XB>(a.dx_out, xo + col[v]) : zero8<XB>();
      if (PART & kAfter) ry[v] = on ? load8<HB>(a.y, ho + col[v]) : zero8<HB>();
    }
    float u[V][8];
#pragma unroll
    for (int v = 0; v < V; v++) unpack8<XB>(ru[v], u[v]);
    if (PART & kBefore) {
      float x[V][8], t[V][8], dh[V][8], s1[V][8];
#pragma unroll
      for (int v = 0; v < V; v++) {
        unpack8<XB>(rx[v], x[v]);
        unpack8<HB>(rh[v], dh[v]);
        if (TOKEN) load_vector8(a.scale, mo + col[v], 0.f, s1[v]);
#pragma unroll
        for (int i = 0; i < 8; i++) {
          if (TOKEN) s1[v][i] += 1.f;
          t[v][i] = TOKEN ? dh[v][i] * (wi[v][i] * s1[v][i]) : dh[v][i] * w[v][i];
        }
      }
      const BackMoments m = back_moments<V>(tm, a.norm_in, x, t, has, chunks, a.eps);
#pragma unroll
      for (int v = 0; v < V; v++) {
        const bool on = row && has[v];
        float ds[8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
          const float nv = on ? (x[v][i] - m.mu) * m.r : 0.f, pn = dh[v][i] * nv;
          u[v][i] += m.r * (t[v][i] - m.t - nv * m.tn);
          p_sum[v][i] += TOKEN ? pn * s1[v][i] : pn;
          if (!TOKEN) s_sum[v][i] += dh[v][i];
          ds[i] = pn * wi[v][i];
        }
        if (TOKEN && on && a.dscale) store8<false>(a.dscale, mo + col[v], pack8<false>(ds));
        if (TOKEN && on && a.dshift) store8<false>(a.dshift, mo + col[v], pack8<false>(dh[v]));
      }
    }
    if (PART & kAfter) {
      float y[V][8], t[V][8], gt[V][8];
#pragma unroll
      for (int v = 0; v < V; v++) {
        unpack8<HB>(ry[v], y[v]);
        if (TOKEN) load_vector8(a.gate, mo + col[v], 1.f, gt[v]);
#pragma unroll
        for (int i = 0; i < 8; i++) {
          if (!(row && has[v])) u[v][i] = 0.f;
          t[v][i] = TOKEN ? u[v][i] * (wo[v][i] * gt[v][i]) : u[v][i] * g[v][i];
        }
      }
      const BackMoments m = back_moments<V>(tm, a.norm_out, y, t, has, chunks, a.eps);
#pragma unroll
      for (int v = 0; v < V; v++) {
        const bool on = row && has[v];
        float dg[8], dy[8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
          const float mv = on ? (y[v][i] - m.mu) * m.r : 0.f, qn = u[v][i] * mv;
          q_sum[v][i] += TOKEN ? qn * gt[v][i] : qn;
          dg[i] = qn * wo[v][i];
          dy[i] = m.r * (t[v][i] - m.t - mv * m.tn);
          u[v][i] *= a.rho;
        }
        if (TOKEN && on && a.dgate) store8<false>(a.dgate, mo + col[v], pack8<false>(dg));
        if (on) store8<HB>(a.dy, ho + col[v], pack8<HB>(dy));
      }
    }
#pragma unroll
    for (int v = 0; v < V; v++)
      if (row && has[v]) store8<XB>(a.dx, xo + col[v], pack8<XB>(u[v]));
  }
  const size_t rows = (size_t)a.B * a.walkers, at = (size_t)blockIdx.x * a.C;
  if (PART & kBefore) {
    if (a.dscale || a.din_weight) store_partial<V>(tm, a.teams, teams_lds, p_sum, has, col, a.C, a.partial + at);
    if (!TOKEN && a.dshift) store_partial<V>(tm, a.teams, teams_lds, s_sum, has, col, a.C, a.partial + rows * a.C + at);
  }
  if ((PART & kAfter) && (a.dgate || a.dout_weight))
    store_partial<V>(tm, a.teams, teams_lds, q_sum, has, col, a.C, a.partial + 2 * rows * a.C + at);
}

// 32 columns (8 lanes of 4) by 64 rows at a time per workgroup; the 64 partial sums in order through LDS.
constexpr int kSumColumns = 32, kSumRows = 64;
__global__ __launch_bounds__(kSumRows * 8) void column_sums_kernel(ColumnJobs js) {
  __shared__ f32x4 lds[kSumRows][kSumColumns / 4];
  const int tiles = (js.columns + kSumColumns - 1) / kSumColumns, tile = (int)blockIdx.x % tiles;
  int y = (int)blockIdx.x / tiles, k = 0;
  while (y >= js.job[k].batches) y -= js.job[k++].batches;
  const ColumnJob& j = js.job[k];
  const int quad = (int)threadIdx.x % 8, r0 = (int)threadIdx.x / 8, c = tile * kSumColumns + 4 * quad;
  const bool on = c < js.columns;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if (on) {
    const float* p = j.rows + ((size_t)y * j.count) * js.columns + c;
    for (int r = r0; r < j.count; r += kSumRows) {
      f32x4 x = *(const f32x4*)(p + (size_t)r * js.columns);
      if (j.weight) x *= *(const f32x4*)(j.weight + (size_t)(r / j.per_weight) * j.weight_stride + c) + j.plus;
      s += x;
    }
  }
  lds[r0][quad] = s;
  for (int half = kSumRows / 2; half > 0; half /= 2) {
    __syncthreads();
    if (r0 < half) lds[r0][quad] += lds[r0 + half][quad];
  }
  if (r0 == 0 && on) {
    s = lds[0][quad];
    if (j.factor) s *= *(const f32x4*)(j.factor + c);
    *(f32x4*)(j.out + (size_t)y * j.out_stride + c) = s;
  }
}

hipError_t launch_column_sums(const ColumnJobs& j, hipStream_t stream) {
  int batches = 0;
  for (int k = 0; k < j.jobs; k++) batches += j.job[k].batches;
  if (batches == 0) return hipSuccess;
  column_sums_kernel<<<dim3((unsigned)((j.columns + kSumColumns - 1) / kSumColumns * batches)), kSumRows * 8, 0, stream>>>(j);
  return hipGetLastError();
}

void plan_norm(NormArgs* a, bool backward) {
  a->team = row_team(a->C / kChunk);
  a->teams = kTeamThreads / a->team.threads();
  if (a->teams > a->N) a->teams = a->N;
  const int resident = 512;                  // two workgroups of 8 waves a CU
  long long walkers = resident / a->B;
  const long long most = ((long long)a->N + a->teams - 1) / a->teams;
  if (walkers < 1) walkers = 1;
  a->walkers = (int)(walkers < most ? walkers : most);
  (void)backward;
}

template <int V, bool XB, bool HB, int PART>
static hipError_t launch_part(const NormArgs& a, bool backward, hipStream_t stream) {
  const dim3 grid((unsigned)(a.B * a.walkers)), block((a.teams * a.team.threads() + kWave - 1) / kWave * kWave);
  const size_t lds = backward ? (size_t)(a.teams - 1) * a.C * sizeof(float) : 0;
  const bool token = a.mods == SLA2_MOD_TOKEN;
  if (backward) {
    if (token) norm_bwd_kernel<V, XB, HB, PART, true><<<grid, block, lds, stream>>>(a);
    else norm_bwd_kernel<V, XB, HB, PART, false><<<grid, block, lds, stream>>>(a);
  } else {
    if (token) norm_kernel<V, XB, HB, PART, true><<<grid, block, 0, stream>>>(a);
    else norm_kernel<V, XB, HB, PART, false><<<grid, block, 0, stream>>>(a);
  }
  return hipGetLastError();
}
template <int V, bool XB, bool HB>
static hipError_t launch_types(const NormArgs& a, int part, bool backward, hipStream_t stream) {
  if (part == kBefore) return launch_part<V, XB, HB, kBefore>(a, backward, stream);
  if (part == kAfter) return launch_part<V, XB, HB, kAfter>(a, backward, stream);
  return launch_part<V, XB, HB, kBefore | kAfter>(a, backward, stream);
}
template <int V>
static hipError_t launch_vec(const NormArgs& a, int part, bool backward, hipStream_t stream) {
  if (a.x_bf16) return launch_types<V, true, true>(a, part, backward, stream);
  if (a.h_bf16) return launch_types<V, false, true>(a, part, backward, stream);
  return launch_types<V, false, false>(a, part, backward, stream);
}
static hipError_t launch_any(const NormArgs& a, int part, bool backward, hipStream_t stream) {
  return a.team.vec == 1 ? launch_vec<1>(a, part, backward, stream) : launch_vec<2>(a, part, backward, stream);
}

hipError_t launch_norm(const NormArgs& a, hipStream_t stream) {
  return launch_any(a, (a.h ? kBefore : 0) | (a.y ? kAfter : 0), false, stream);
}

hipError_t launch_norm_bwd(const NormArgs& a, hipStream_t stream) {
  if (hipError_t e = launch_any(a, (a.dh ? kBefore : 0) | (a.y ? kAfter : 0), true, stream); e != hipSuccess) return e;
  const int rows = a.B * a.walkers;
  const float *p = a.partial, *s = p + (size_t)rows * a.C, *q = s + (size_t)rows * a.C;
  const bool batch = a.mods == SLA2_MOD_BATCH, token = a.mods == SLA2_MOD_TOKEN;
  ColumnJobs js{};
  js.columns = a.C;
  // the sum over the rows of each batch, or of all
  auto add = [&](const float* from, const float* factor, float* out) {
    if (out) js.job[js.jobs++] = ColumnJob{from, batch ? a.B : 1, batch ? a.walkers : rows, factor, nullptr, 0.f, 1, 0, out, a.mod_b};
  };
  // a weight's: over all rows, each with the modulation of its batch (1 + s or g), which a token's own has in it already
  auto add_weight = [&](const float* from, const float* modulation, float plus, float* out) {
    if (out) js.job[js.jobs++] = ColumnJob{from, 1, rows, nullptr, token ? nullptr : modulation, plus, a.walkers, a.mod_b, out, 0};
  };
  if (a.dh) {
    if (!token) add(p, a.in_weight, a.dscale);
    if (!token) add(s, nullptr, a.dshift);
    add_weight(p, a.scale, 1.f, a.din_weight);
  }
  if (a.y) {
    if (!token) add(q, a.out_weight, a.dgate);
    add_weight(q, a.gate, 0.f, a.dout_weight);
  }
  return launch_column_sums(js, stream);
}

}  // namespace sla2
