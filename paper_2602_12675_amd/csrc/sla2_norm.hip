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
// rows of 3 chunks a thread with both parts, or with a modulation of every token
constexpr bool large_forward(int vec, int part, bool token) {
  const bool both = part == (kBefore | kAfter);
  return vec == 3 ? both || token : vec == 2 && both && token;
}

// What the statistics of a row need of the team: 1 / C, 1 / channels of this wave, and in LDS the channels of every wave.
struct Counts {
  float all, mine;
  const float* of;
  __device__ __forceinline__ Counts(const Team& tm, int chunks, float* lds) : of(lds) {
    all = 1.f / (float)(chunks * kChunk);
    mine = all;
    if (tm.t.waves == 1) return;
    const int own = tm.channels(tm.lane / kWave, chunks);
    mine = own ? 1.f / (float)own : 0.f;
    if ((int)threadIdx.x < tm.t.waves) lds[threadIdx.x] = (float)tm.channels((int)threadIdx.x, chunks);    // read behind an exchange's barrier
  }
};

struct Moments {
  float mu, r;
};

// mu and r of the team's row x; places without a channel hold 0.  The second moment is taken around the mean of the wave, and those of
// several waves are joined by M2 = sum of M2_w + n_w (mu_w - mu)^2: nothing is lost to a mean that is large beside the spread.
template <int V>
__device__ __forceinline__ Moments moments(Team& tm, const Counts& n, int kind, const float (&x)[V][8], const bool (&has)[V], float eps) {
  if (kind == SLA2_NORM_NONE) return {0.f, 1.f};
  float s[1] = {0.f};
  if (kind == SLA2_NORM_RMS) {
#pragma unroll
    for (int v = 0; v < V; v++)
#pragma unroll
      for (int i = 0; i < 8; i++) s[0] += x[v][i] * x[v][i];
    tm.sum(s);
    return {0.f, inv_sqrt(s[0] * n.all + eps)};
  }
#pragma unroll
  for (int v = 0; v < V; v++)
#pragma unroll
    for (int i = 0; i < 8; i++) s[0] += x[v][i];
  float mu = lanes_sum(s[0], tm.t.lanes) * n.mine, m2 = 0.f;
#pragma unroll
  for (int v = 0; v < V; v++) {
    const float m = has[v] ? mu : 0.f;
#pragma unroll
    for (int i = 0; i < 8; i++) m2 += (x[v][i] - m) * (x[v][i] - m);
  }
  m2 = lanes_sum(m2, tm.t.lanes);
  if (tm.t.waves > 1) {
    const float own[2] = {mu, m2};
    const float* o = tm.exchange(own);
    mu = m2 = 0.f;
    for (int w = 0; w < tm.t.waves; w++) mu += n.of[w] * o[2 * w];
    mu *= n.all;
    for (int w = 0; w < tm.t.waves; w++) m2 += o[2 * w + 1] + n.of[w] * (o[2 * w] - mu) * (o[2 * w] - mu);
  }
  return {mu, inv_sqrt(m2 * n.all + eps)};
}

// The same with mean(t) and mean(t n), n = (x - mu) r, for the gradient t behind the norm: all sums in one exchange.
struct BackMoments {
  float mu, r, t, tn;
};
template <int V>
__device__ __forceinline__ BackMoments back_moments(Team& tm, const Counts& n, int kind, const float (&x)[V][8], const float (&t)[V][8],
                                                    const bool (&has)[V], float eps) {
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
    const float r = inv_sqrt(s[0] * n.all + eps);
    return {0.f, r, 0.f, s[1] * n.all * r};
  }
  float mu = 0.f, m2 = 0.f, st = 0.f, stx = 0.f;
#pragma unroll
  for (int v = 0; v < V; v++)
#pragma unroll
    for (int i = 0; i < 8; i++) {
      mu += x[v][i];
      st += t[v][i];
    }
  mu = lanes_sum(mu, tm.t.lanes) * n.mine;
#pragma unroll
  for (int v = 0; v < V; v++) {
    const float m = has[v] ? mu : 0.f;
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const float c = x[v][i] - m;
      m2 += c * c;
      stx += t[v][i] * c;
    }
  }
  m2 = lanes_sum(m2, tm.t.lanes);
  st = lanes_sum(st, tm.t.lanes);
  stx = lanes_sum(stx, tm.t.lanes);
  if (tm.t.waves > 1) {
    const float own[4] = {mu, m2, st, stx};
    const float* o = tm.exchange(own);
    mu = m2 = st = stx = 0.f;
    for (int w = 0; w < tm.t.waves; w++) mu += n.of[w] * o[4 * w];
    mu *= n.all;
    for (int w = 0; w < tm.t.waves; w++) {
      const float d = o[4 * w] - mu;
      m2 += o[4 * w + 1] + n.of[w] * d * d;
      st += o[4 * w + 2];
      stx += o[4 * w + 3] + d * o[4 * w + 2];
    }
  }
  const float r = inv_sqrt(m2 * n.all + eps);
  return {mu, r, st * n.all, stx * n.all * r};
}

// A thread's chunks of the rows of a workgroup, which are of one batch and every walkers-th step of its.
template <int V> struct Columns {
  bool has[V];
  unsigned col[V], x[V], h[V], mod[V];       // channel; offsets from the first row of the wave
  __device__ __forceinline__ Columns(const NormArgs& a, const Team& tm) {
#pragma unroll
    for (int v = 0; v < V; v++) {
      const int c = tm.lane + v * a.team.threads();
      has[v] = tm.team < a.teams && c < a.C / kChunk;
      col[v] = has[v] ? c * kChunk : 0;
      x[v] = tm.sub * (unsigned)a.x_n + col[v];
      h[v] = tm.sub * (unsigned)a.h_n + col[v];
      mod[v] = tm.sub * (unsigned)a.mod_n + col[v];
    }
  }
};

// x' and h
template <int V, bool XB, bool HB, int PART, bool TOKEN>
__global__ __launch_bounds__(kTeamThreads, waves_of(large_forward(V, PART, TOKEN))) void norm_kernel(NormArgs a) {
  __shared__ float lds[kExchangeFloats], counts[kTeamThreads / kWave];
  Team tm(a.team, lds);
  const int b = (int)blockIdx.x / a.walkers, walker = (int)blockIdx.x % a.walkers;
  const Counts n_of(tm, a.C / kChunk, counts);
  const Columns<V> at(a, tm);
  float g[V][8], w[V][8], sh[V][8], wo[V][8], wi[V][8];   // g w_out; w_in (1 + s); b.  TOKEN: row by row, of w_out and w_in
  auto vectors = [&](long long mod, const unsigned (&off)[V]) {
#pragma unroll
    for (int v = 0; v < V; v++) {
      if (PART & kAfter) {
        load_vector8(a.gate ? a.gate + mod : nullptr, off[v], 1.f, g[v]);
#pragma unroll
        for (int i = 0; i < 8; i++) g[v][i] *= wo[v][i];
      }
      if (PART & kBefore) {
        load_vector8(a.scale ? a.scale + mod : nullptr, off[v], 0.f, w[v]);
        load_vector8(a.shift ? a.shift + mod : nullptr, off[v], 0.f, sh[v]);
#pragma unroll
        for (int i = 0; i < 8; i++) w[v][i] = wi[v][i] * (1.f + w[v][i]);
      }
    }
  };
#pragma unroll
  for (int v = 0; v < V; v++) {
    if (PART & kAfter) load_vector8(a.out_weight, at.col[v], 1.f, wo[v]);
    if (PART & kBefore) load_vector8(a.in_weight, at.col[v], 1.f, wi[v]);
#pragma unroll
    for (int i = 0; i < 8; i++) g[v][i] = w[v][i] = sh[v][i] = 0.f;
  }
  if (!TOKEN) vectors(b * a.mod_b, at.col);
  for (long long n0 = (long long)walker * a.teams; n0 < a.N; n0 += (long long)a.walkers * a.teams) {
    const long long n = n0 + tm.first;
    const bool row = n + tm.sub < a.N;
    const void *px = at_elem<XB>(a.x, b * a.x_b + n * a.x_n), *py = at_elem<HB>(a.y, b * a.h_b + n * a.h_n);
    Raw<XB> rx[V];
    Raw<HB> ry[V];
#pragma unroll
    for (int v = 0; v < V; v++) {
      const bool on = row && at.has[v];
      rx[v] = on ? load8<XB>(px, at.x[v]) : zero8<XB>();
      if (PART & kAfter) ry[v] = on ? load8<HB>(py, at.h[v]) : zero8<HB>();
    }
    if (TOKEN && row) vectors(b * a.mod_b + n * a.mod_n, at.mod);
    float x[V][8];
#pragma unroll
    for (int v = 0; v < V; v++) unpack8<XB>(rx[v], x[v]);
    if (PART & kAfter) {
      void* po = at_elem<XB>(a.x_out, b * a.x_b + n * a.x_n);
      float y[V][8];
#pragma unroll
      for (int v = 0; v < V; v++) unpack8<HB>(ry[v], y[v]);
      const Moments m = moments<V>(tm, n_of, a.norm_out, y, at.has, a.eps);
#pragma unroll
      for (int v = 0; v < V; v++) {
        const bool on = row && at.has[v];
#pragma unroll
        for (int i = 0; i < 8; i++) x[v][i] = a.rho * x[v][i] + g[v][i] * ((y[v][i] - m.mu) * m.r);
        rx[v] = pack8<XB>(x[v]);
        if (on) put8<XB>(po, at.x[v], rx[v]);
        else rx[v] = zero8<XB>();
        unpack8<XB>(rx[v], x[v]);
      }
    }
    if (PART & kBefore) {
      void* ph = at_elem<HB>(a.h, b * a.h_b + n * a.h_n);
      const Moments m = moments<V>(tm, n_of, a.norm_in, x, at.has, a.eps);
#pragma unroll
      for (int v = 0; v < V; v++) {
#pragma unroll
        for (int i = 0; i < 8; i++) x[v][i] = ((x[v][i] - m.mu) * m.r) * w[v][i] + sh[v][i];
        if (row && at.has[v]) put8<HB>(ph, at.h[v], pack8<HB>(x[v]));
      }
    }
  }
}

// One of the sums of a workgroup: its teams' in order, through LDS, into row `at` of the partial sums.
template <int V>
__device__ __forceinline__ void store_partial(const Team& tm, int teams, float* lds, const float (&acc)[V][8], const bool (&has)[V],
                                              const unsigned (&col)[V], int C, float* to) {
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
__global__ __launch_bounds__(kTeamThreads, waves_of(V > 1)) void norm_bwd_kernel(NormArgs a) {
  __shared__ float lds[kExchangeFloats], counts[kTeamThreads / kWave];
  extern __shared__ float teams_lds[];       // [teams - 1][C]
  Team tm(a.team, lds);
  const int b = (int)blockIdx.x / a.walkers, walker = (int)blockIdx.x % a.walkers;
  const Counts n_of(tm, a.C / kChunk, counts);
  const Columns<V> at(a, tm);
  float g[V][8], w[V][8], wo[V][8], wi[V][8];             // as in norm_kernel; TOKEN: g, 1 + s, w_out, w_in
  float p_sum[V][8], s_sum[V][8], q_sum[V][8];            // TOKEN: of d w_in, nothing, of d w_out
  auto vectors = [&](long long mod, const unsigned (&off)[V]) {
#pragma unroll
    for (int v = 0; v < V; v++) {
      if (PART & kAfter) load_vector8(a.gate ? a.gate + mod : nullptr, off[v], 1.f, g[v]);
      if (PART & kBefore) {
        load_vector8(a.scale ? a.scale + mod : nullptr, off[v], 0.f, w[v]);
#pragma unroll
        for (int i = 0; i < 8; i++) w[v][i] += 1.f;
      }
    }
  };
#pragma unroll
  for (int v = 0; v < V; v++) {
#pragma unroll
    for (int i = 0; i < 8; i++) g[v][i] = w[v][i] = p_sum[v][i] = s_sum[v][i] = q_sum[v][i] = 0.f;
    if (PART & kAfter) load_vector8(a.out_weight, at.col[v], 1.f, wo[v]);
    if (PART & kBefore) load_vector8(a.in_weight, at.col[v], 1.f, wi[v]);
  }
  if (!TOKEN) {
    vectors(b * a.mod_b, at.col);
#pragma unroll
    for (int v = 0; v < V; v++)
#pragma unroll
      for (int i = 0; i < 8; i++) {
        if (PART & kBefore) w[v][i] *= wi[v][i];
        if (PART & kAfter) g[v][i] = at.has[v] ? g[v][i] * wo[v][i] : 0.f;
      }
  }
  for (long long n0 = (long long)walker * a.teams; n0 < a.N; n0 += (long long)a.walkers * a.teams) {
    const long long n = n0 + tm.first;
    const bool row = n + tm.sub < a.N;
    const long long xo = b * a.x_b + n * a.x_n, ho = b * a.h_b + n * a.h_n, mo = b * a.mod_b + n * a.mod_n;
    const void *px = at_elem<XB>(a.x, xo), *pu = at_elem<XB>(a.dx_out, xo), *ph = at_elem<HB>(a.dh, ho), *py = at_elem<HB>(a.y, ho);
    Raw<XB> rx[V], ru[V];
    Raw<HB> ry[V], rh[V];
#pragma unroll
    for (int v = 0; v < V; v++) {
      const bool on = row && at.has[v];
      if (PART & kBefore) {
        rx[v] = on ? load8<XB>(px, at.x[v]) : zero8<XB>();
        rh[v] = on ? load8<HB>(ph, at.h[v]) : zero8<HB>();
      }
      ru[v] = on && a.dx_out ? load8<XB>(pu, at.x[v]) : zero8<XB>();
      if (PART & kAfter) ry[v] = on ? load8<HB>(py, at.h[v]) : zero8<HB>();
    }
    if (TOKEN && row) vectors(mo, at.mod);
    float u[V][8];
#pragma unroll
    for (int v = 0; v < V; v++) unpack8<XB>(ru[v], u[v]);
    // Behind a norm: grad[] += the gradient in front of it from t, of the value x; each(v, i, n) with the normalised value
    auto through = [&](int kind, const float (&x)[V][8], const float (&t)[V][8], float (&grad)[V][8], auto each) {
      if (kind == SLA2_NORM_NONE) {
#pragma unroll
        for (int v = 0; v < V; v++)
#pragma unroll
          for (int i = 0; i < 8; i++) {
            each(v, i, x[v][i]);
            grad[v][i] += t[v][i];
          }
        return;
      }
      const BackMoments m = back_moments<V>(tm, n_of, kind, x, t, at.has, a.eps);
      const float rt = -m.r * m.t, rtn = -m.r * m.tn;
#pragma unroll
      for (int v = 0; v < V; v++)
#pragma unroll
        for (int i = 0; i < 8; i++) {
          const float nv = (x[v][i] - m.mu) * m.r;
          each(v, i, nv);
          grad[v][i] += m.r * t[v][i] + (nv * rtn + rt);
        }
    };
    if (PART & kBefore) {
      float x[V][8], t[V][8], dh[V][8], ds[V][8];
#pragma unroll
      for (int v = 0; v < V; v++) {
        unpack8<XB>(rx[v], x[v]);
        unpack8<HB>(rh[v], dh[v]);
#pragma unroll
        for (int i = 0; i < 8; i++) t[v][i] = dh[v][i] * (TOKEN ? wi[v][i] * w[v][i] : w[v][i]);
      }
      through(a.norm_in, x, t, u, [&](int v, int i, float nv) {
        if (TOKEN) {
          ds[v][i] = dh[v][i] * nv;
          p_sum[v][i] += row ? ds[v][i] * w[v][i] : 0.f;
          ds[v][i] *= wi[v][i];
        } else {
          p_sum[v][i] += dh[v][i] * nv;
          s_sum[v][i] += dh[v][i];
        }
      });
      if (TOKEN) {
        float *pds = a.dscale + mo, *pdb = a.dshift + mo;
#pragma unroll
        for (int v = 0; v < V; v++) {
          if (row && at.has[v] && a.dscale) put8<false>(pds, at.mod[v], pack8<false>(ds[v]));
          if (row && at.has[v] && a.dshift) put8<false>(pdb, at.mod[v], pack8<false>(dh[v]));
        }
      }
    }
    if (PART & kAfter) {
      float y[V][8], t[V][8], dy[V][8], dg[V][8];
#pragma unroll
      for (int v = 0; v < V; v++) {
        unpack8<HB>(ry[v], y[v]);
#pragma unroll
        for (int i = 0; i < 8; i++) {
          if (TOKEN) t[v][i] = row && at.has[v] ? u[v][i] * (wo[v][i] * g[v][i]) : 0.f;
          else t[v][i] = u[v][i] * g[v][i];
          dy[v][i] = 0.f;
        }
      }
      through(a.norm_out, y, t, dy, [&](int v, int i, float nv) {
        if (TOKEN) {
          dg[v][i] = u[v][i] * nv;
          q_sum[v][i] += row ? dg[v][i] * g[v][i] : 0.f;
          dg[v][i] *= wo[v][i];
        } else {
          q_sum[v][i] += u[v][i] * nv;
        }
      });
      void* pdy = at_elem<HB>(a.dy, ho);
      float* pdg = a.dgate + mo;
#pragma unroll
      for (int v = 0; v < V; v++) {
        const bool on = row && at.has[v];
        if (on) put8<HB>(pdy, at.h[v], pack8<HB>(dy[v]));
        if (TOKEN && on && a.dgate) put8<false>(pdg, at.mod[v], pack8<false>(dg[v]));
#pragma unroll
        for (int i = 0; i < 8; i++) u[v][i] *= a.rho;
      }
    }
    void* pdx = at_elem<XB>(a.dx, xo);
#pragma unroll
    for (int v = 0; v < V; v++)
      if (row && at.has[v]) put8<XB>(pdx, at.x[v], pack8<XB>(u[v]));
  }
  const size_t rows = (size_t)a.B * a.walkers, first = (size_t)blockIdx.x * a.C;
  if (PART & kBefore) {
    if (a.dscale || a.din_weight) store_partial<V>(tm, a.teams, teams_lds, p_sum, at.has, at.col, a.C, a.partial + first);
    if (!TOKEN && a.dshift) store_partial<V>(tm, a.teams, teams_lds, s_sum, at.has, at.col, a.C, a.partial + rows * a.C + first);
  }
  if ((PART & kAfter) && (a.dgate || a.dout_weight))
    store_partial<V>(tm, a.teams, teams_lds, q_sum, at.has, at.col, a.C, a.partial + 2 * rows * a.C + first);
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
    const float* p = j.rows + (size_t)y * j.count * js.columns + c;
    // 8 rows on their way at a time: one after the other, 512 rows took as long as 8 trips to memory
    for (int r = r0; r < j.count; r += 8 * kSumRows) {
      f32x4 x[8];
#pragma unroll
      for (int k = 0; k < 8; k++) {
        const int at = r + k * kSumRows;
        x[k] = at < j.count ? *(const f32x4*)(p + (size_t)at * js.columns) : f32x4{0.f, 0.f, 0.f, 0.f};
        if (j.weight && at < j.count) x[k] *= *(const f32x4*)(j.weight + (size_t)(at / j.per_weight) * j.weight_stride + c) + j.weight_plus;
      }
#pragma unroll
      for (int k = 0; k < 8; k++) s += x[k];
    }
  }
  lds[r0][quad] = s;
  for (int half = kSumRows / 2; half > 0; half /= 2) {
    __syncthreads();
    if (r0 < half) lds[r0][quad] += lds[r0 + half][quad];
  }
  if (r0 == 0 && on) {
    s = lds[0][quad];
    if (j.factor) s *= *(const f32x4*)(j.factor + c) + j.factor_plus;
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

static int part_of(const NormArgs& a, bool backward) { return ((backward ? a.dh : a.h) ? kBefore : 0) | (a.y ? kAfter : 0); }

void plan_norm(NormArgs* a, bool backward) {
  a->team = row_team(a->C / kChunk, backward ? 1 : 3);
  // the rows of a wave lie within 2 GB of its first; where strides are longer than that it has one
  const long long x_n = a->x_n > a->h_n ? a->x_n : a->h_n, widest = x_n > a->mod_n ? x_n : a->mod_n;
  if (widest >= (1ll << 29) / (kWave / a->team.lanes)) a->team.lanes = kWave;
  a->teams = block_teams(a->team, a->N);
  const bool large = backward ? a->team.vec > 1 : large_forward(a->team.vec, part_of(*a, false), false);
  const int walkers = resident_workgroups(a->team, a->teams, threads_of(large)) / a->B, most = (int)(((long long)a->N + a->teams - 1) / a->teams);
  a->walkers = walkers < 1 ? 1 : walkers < most ? walkers : most;
}

template <int V, bool XB, bool HB, int PART>
static hipError_t launch_part(const NormArgs& a, bool backward, hipStream_t stream) {
  const dim3 grid((unsigned)(a.B * a.walkers)), block((a.teams * a.team.threads() + kWave - 1) / kWave * kWave);
  const size_t lds = backward ? (size_t)(a.teams - 1) * a.C * sizeof(float) : 0;
  const bool token = a.mods == SLA2_MOD_TOKEN;
  if (backward) {
    if constexpr (V <= 2) {
      if (token) norm_bwd_kernel<V, XB, HB, PART, true><<<grid, block, lds, stream>>>(a);
      else norm_bwd_kernel<V, XB, HB, PART, false><<<grid, block, lds, stream>>>(a);
    }
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
  return a.team.vec == 1 ? launch_vec<1>(a, part, backward, stream) : a.team.vec == 2 ? launch_vec<2>(a, part, backward, stream) : launch_vec<3>(a, part, backward, stream);
}

hipError_t launch_norm(const NormArgs& a, hipStream_t stream) {
  return launch_any(a, part_of(a, false), false, stream);
}

hipError_t launch_norm_bwd(const NormArgs& a, hipStream_t stream) {
  if (hipError_t e = launch_any(a, part_of(a, true), true, stream); e != hipSuccess) return e;
  const int rows = a.B * a.walkers;
  const float *p = a.partial, *s = p + (size_t)rows * a.C, *q = s + (size_t)rows * a.C;
  const bool batch = a.mods == SLA2_MOD_BATCH, token = a.mods == SLA2_MOD_TOKEN;
  ColumnJobs js{};
  js.columns = a.C;
  // the sum over the rows of each batch, or of all
  auto add = [&](const float* from, const float* factor, float* out) {
    if (out) js.job[js.jobs++] = ColumnJob{from, batch ? a.B : 1, batch ? a.walkers : rows, factor, 0.f, nullptr, 0.f, 1, 0, out, a.mod_b};
  };
  // a weight's: over all rows, each with the modulation of its batch (1 + s or g); one that is the same for all rows comes behind the sum,
  // and that of a token is in it already
  auto add_weight = [&](const float* from, const float* modulation, float plus, float* out) {
    const bool by_row = batch && a.B > 1;
    const float *factor = by_row || token ? nullptr : modulation, *weight = by_row ? modulation : nullptr;
    if (out) js.job[js.jobs++] = ColumnJob{from, 1, rows, factor, plus, weight, plus, a.walkers, a.mod_b, out, 0};
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
