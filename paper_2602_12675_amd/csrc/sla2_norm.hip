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
// workgroup adds up P, S, Q of its rows in registers, its teams theirs in a fixed order, and a second launch adds up the workgroups',
// unless there is but one.
// A modulation of every token needs no sums but those of the weights.
#include "rows.h"

namespace sla2 {

// What the statistics of a row need of the team: 1 / C, 1 / channels of this wave, and the channels of wave l % 16 on lane l.
struct Counts {
  float all, mine, other;
  __device__ __forceinline__ Counts(const Team& tm, int chunks) {
    all = 1.f / (float)(chunks * kChunk);
    mine = all;
    other = 0.f;
    if (tm.t.waves == 1) return;
    const int own = tm.channels(tm.lane / kWave, chunks), w = (int)threadIdx.x % 16;
    mine = own ? 1.f / (float)own : 0.f;
    other = w < tm.t.waves ? (float)tm.channels(w, chunks) : 0.f;
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
    float o[2] = {mu, m2};
    tm.exchange(o);
    mu = sum16(n.other * o[0]) * n.all;
    const float d = o[0] - mu;
    m2 = sum16(o[1] + n.other * d * d);
  }
  return {mu, inv_sqrt(m2 * n.all + eps)};
}

// The same with mean(t) and mean(t n), n = (x - mu) r, for the gradient t behind the norm: all sums in one exchange.  value(x) and
// gradient(t) give a thread's chunk of either.
struct BackMoments {
  float mu, r, t, tn;
};
template <class Value, class Gradient>
__device__ __forceinline__ BackMoments back_moments(Team& tm, const Counts& n, int kind, Value value, Gradient gradient, bool has, float eps) {
  float x[8], t[8];
  value(x);
  if (kind == SLA2_NORM_RMS) {
    float s[2] = {0.f, 0.f};
    gradient(t);
#pragma unroll
    for (int i = 0; i < 8; i++) {
      s[0] += x[i] * x[i];
      s[1] += t[i] * x[i];
    }
    tm.sum(s);
    const float r = inv_sqrt(s[0] * n.all + eps);
    return {0.f, r, 0.f, s[1] * n.all * r};
  }
  float mu = 0.f, m2 = 0.f, st = 0.f, stx = 0.f;
#pragma unroll
  for (int i = 0; i < 8; i++) mu += x[i];
  mu = lanes_sum(mu, tm.t.lanes) * n.mine;
  const float m = has ? mu : 0.f;
  gradient(t);
#pragma unroll
  for (int i = 0; i < 8; i++) {
    const float c = x[i] - m;
    m2 += c * c;
    st += t[i];
    stx += t[i] * c;
  }
  m2 = lanes_sum(m2, tm.t.lanes);
  st = lanes_sum(st, tm.t.lanes);
  stx = lanes_sum(stx, tm.t.lanes);
  if (tm.t.waves > 1) {
    float o[4] = {mu, m2, st, stx};
    tm.exchange(o);
    mu = sum16(n.other * o[0]) * n.all;
    const float d = o[0] - mu;
    m2 = sum16(o[1] + n.other * d * d);
    st = sum16(o[2]);
    stx = sum16(o[3] + d * o[2]);
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
__global__ __launch_bounds__(kTeamThreads, waves_of(large_norm(V, PART, TOKEN))) void norm_kernel(NormArgs a) {
  __shared__ float lds[kExchangeFloats];
  Team tm(a.team, lds);
  const int b = (int)blockIdx.x / a.walkers, walker = (int)blockIdx.x % a.walkers;
  const Counts n_of(tm, a.C / kChunk);
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

// out = (plus + factor) (.) sum, where out is wanted; factor null: sum
__device__ __forceinline__ void store_scaled(float* out, const float* factor, float plus, const float (&sum)[8], unsigned col) {
  if (!out) return;
  float f[8];
  load_vector8(factor, col, 1.f - plus, f);
#pragma unroll
  for (int i = 0; i < 8; i++) f[i] = (plus + f[i]) * sum[i];
  store8<false>(out, col, pack8<false>(f));
}

// A thread has one chunk, and nothing is kept in fp32 across the sums of a row: the values are unpacked again behind them, and the vectors of
// the batch are read from LDS.  What stays from row to row are the sums for the column gradients.  The time hangs on the waves that
// registers leave room for: with the vectors in registers, two chunks a thread from 4,096 channels on (its second workgroup finding no place
// on the CU) 7,180 rows of 4,976 bf16 channels took 205 us, layer norms on both sides, and 20,000 of 5,120 with an fp32 stream 411 us;
// so 140 and 344 us.  The next row fetched ahead cost more in registers than it gave.
template <bool XB, bool HB, int PART, bool TOKEN>
__global__ __launch_bounds__(kMaxThreads, 4) void norm_bwd_kernel(NormArgs a) {
  __shared__ float lds[kExchangeFloats];
  // g w_out and w_in (1 + s) of the batch, [2][C + 8], the last 8 being 0 for threads without a channel; at the end the sums of the teams,
  // [teams - 1][C]
  extern __shared__ float shared[];
  Team tm(a.team, lds);
  const int b = (int)blockIdx.x / a.walkers, walker = (int)blockIdx.x % a.walkers;
  const Counts n_of(tm, a.C / kChunk);
  const Columns<1> columns(a, tm);
  const bool has = columns.has[0];
  const unsigned col = columns.col[0], at_x = columns.x[0], at_h = columns.h[0], at_mod = columns.mod[0], place = has ? col : (unsigned)a.C;
  float p_sum[8], s_sum[8], q_sum[8];                     // TOKEN: of d w_in, nothing, of d w_out
#pragma unroll
  for (int i = 0; i < 8; i++) p_sum[i] = s_sum[i] = q_sum[i] = 0.f;
  float* const scales_lds = shared + a.C + kChunk;
  if (!TOKEN) {
    if ((int)threadIdx.x < kChunk) shared[a.C + threadIdx.x] = scales_lds[a.C + threadIdx.x] = 0.f;
    for (int c = (int)threadIdx.x * 4; c < a.C; c += (int)blockDim.x * 4) {
      const f32x4 one = {1.f, 1.f, 1.f, 1.f};
      const long long mod = b * a.mod_b + c;
      if (PART & kAfter) *(f32x4*)(shared + c) = (a.gate ? *(const f32x4*)(a.gate + mod) : one) * (a.out_weight ? *(const f32x4*)(a.out_weight + c) : one);
      if (PART & kBefore) *(f32x4*)(scales_lds + c) = (a.scale ? *(const f32x4*)(a.scale + mod) + one : one) * (a.in_weight ? *(const f32x4*)(a.in_weight + c) : one);
    }
    __syncthreads();
  }
  for (long long n0 = (long long)walker * a.teams; n0 < a.N; n0 += (long long)a.walkers * a.teams) {
    const long long n = n0 + tm.first;
    const bool row = n + tm.sub < a.N, on = row && has;
    const long long xo = b * a.x_b + n * a.x_n, ho = b * a.h_b + n * a.h_n, mo = b * a.mod_b + n * a.mod_n;
    Raw<XB> rx, ru = on && a.dx_out ? load8<XB>(at_elem<XB>(a.dx_out, xo), at_x) : zero8<XB>();
    Raw<HB> ry, rh;
    if (PART & kBefore) {
      rx = on ? load8<XB>(at_elem<XB>(a.x, xo), at_x) : zero8<XB>();
      rh = on ? load8<HB>(at_elem<HB>(a.dh, ho), at_h) : zero8<HB>();
    }
    if (PART & kAfter) ry = on ? load8<HB>(at_elem<HB>(a.y, ho), at_h) : zero8<HB>();
    // the gate and 1 + s: with their weights, or of a token without them; 0 where there is no value
    auto gates = [&](float (&g)[8]) {
      if (TOKEN) {
        load_vector8(a.gate && row ? a.gate + mo : nullptr, at_mod, 1.f, g);
#pragma unroll
        for (int i = 0; i < 8; i++) g[i] = on ? g[i] : 0.f;
      } else {
        load_vector8(shared, place, 0.f, g);
      }
    };
    auto scales = [&](float (&w)[8]) {
      if (TOKEN) {
        load_vector8(a.scale && row ? a.scale + mo : nullptr, at_mod, 0.f, w);
#pragma unroll
        for (int i = 0; i < 8; i++) w[i] = on ? w[i] + 1.f : 0.f;
      } else {
        load_vector8(scales_lds, place, 0.f, w);
      }
    };
    // Behind a norm of the value with the gradient: each(n, g) with the normalised values and the gradient in front of it
    auto through = [&](int kind, auto value, auto gradient, auto again, auto each) {
      float x[8], t[8];
      if (kind == SLA2_NORM_NONE) {
        value(x);
        gradient(t);
        each(x, t);
        return;
      }
      const BackMoments m = back_moments(tm, n_of, kind, value, gradient, has, a.eps);
      const float rt = -m.r * m.t, rtn = -m.r * m.tn;
      again();
      value(x);
      gradient(t);
#pragma unroll
      for (int i = 0; i < 8; i++) {
        x[i] = (x[i] - m.mu) * m.r;
        t[i] = m.r * t[i] + (x[i] * rtn + rt);
      }
      each(x, t);
    };
    float u[8];
    if (!(PART & kBefore)) {
      unpack8<XB>(ru, u);
    } else {
      auto value = [&](float (&x)[8]) { unpack8<XB>(rx, x); };
      auto gradient = [&](float (&t)[8]) {
        float w[8];
        unpack8<HB>(rh, t);
        scales(w);
        if (TOKEN) {
          float wi[8];
          load_vector8(a.in_weight, col, 1.f, wi);
#pragma unroll
          for (int i = 0; i < 8; i++) w[i] *= wi[i];
        }
#pragma unroll
        for (int i = 0; i < 8; i++) t[i] *= w[i];
      };
      auto again = [&]() {
        unpack_again(rx);
        unpack_again(rh);
      };
      through(a.norm_in, value, gradient, again, [&](const float (&nv)[8], const float (&grad)[8]) {
        float dh[8];
        unpack8<HB>(rh, dh);
        unpack8<XB>(ru, u);
        if (TOKEN) {
          float w[8], wi[8], ds[8];
          scales(w);
          load_vector8(a.in_weight, col, 1.f, wi);
#pragma unroll
          for (int i = 0; i < 8; i++) {
            ds[i] = dh[i] * nv[i];
            p_sum[i] += ds[i] * w[i];
            ds[i] *= wi[i];
          }
          if (on && a.dscale) put8<false>(a.dscale + mo, at_mod, pack8<false>(ds));
          if (on && a.dshift) put8<false>(a.dshift + mo, at_mod, pack8<false>(dh));
        }
#pragma unroll
        for (int i = 0; i < 8; i++) {
          if (!TOKEN) {
            p_sum[i] += dh[i] * nv[i];
            s_sum[i] += dh[i];
          }
          u[i] += grad[i];
        }
      });
    }
    if (PART & kAfter) {
      auto value = [&](float (&x)[8]) { unpack8<HB>(ry, x); };
      auto gradient = [&](float (&t)[8]) {
        gates(t);
        if (TOKEN) {
          float wo[8];
          load_vector8(a.out_weight, col, 1.f, wo);
#pragma unroll
          for (int i = 0; i < 8; i++) t[i] *= wo[i];
        }
#pragma unroll
        for (int i = 0; i < 8; i++) t[i] *= u[i];
      };
      auto again = [&]() { unpack_again(ry); };
      through(a.norm_out, value, gradient, again, [&](const float (&nv)[8], const float (&grad)[8]) {
        if (TOKEN) {
          float g[8], wo[8], dg[8];
          gates(g);
          load_vector8(a.out_weight, col, 1.f, wo);
#pragma unroll
          for (int i = 0; i < 8; i++) {
            dg[i] = u[i] * nv[i];
            q_sum[i] += dg[i] * g[i];
            dg[i] *= wo[i];
          }
          if (on && a.dgate) put8<false>(a.dgate + mo, at_mod, pack8<false>(dg));
        } else {
#pragma unroll
          for (int i = 0; i < 8; i++) q_sum[i] += u[i] * nv[i];
        }
        if (on) put8<HB>(at_elem<HB>(a.dy, ho), at_h, pack8<HB>(grad));
#pragma unroll
        for (int i = 0; i < 8; i++) u[i] *= a.rho;
      });
    }
    if (on) put8<XB>(at_elem<XB>(a.dx, xo), at_x, pack8<XB>(u));
  }
  auto sum_of = [&](float (&acc)[8]) {       // of the workgroup; whether this thread has some of it
    join_parts(shared, tm.team, a.teams, a.C, col, has, acc);
    return tm.team == 0 && has;
  };
  // into a row of the partial sums; where this workgroup had all rows, into the results
  const size_t rows = (size_t)a.B * a.walkers, first = (size_t)blockIdx.x * a.C;
  const long long mod = b * a.mod_b;
  const float *scale = TOKEN || !a.scale ? nullptr : a.scale + mod, *gate = TOKEN || !a.gate ? nullptr : a.gate + mod;
  if (PART & kBefore) {
    if (((!TOKEN && a.dscale) || a.din_weight) && sum_of(p_sum)) {
      if (a.direct) {
        if (!TOKEN && a.dscale) store_scaled(a.dscale + mod, a.in_weight, 0.f, p_sum, col);
        store_scaled(a.din_weight, scale, 1.f, p_sum, col);
      } else {
        store8<false>(a.partial + first, col, pack8<false>(p_sum));
      }
    }
    if (!TOKEN && a.dshift && sum_of(s_sum))
      store8<false>(a.direct ? a.dshift + mod : a.partial + rows * a.C + first, col, pack8<false>(s_sum));
  }
  if ((PART & kAfter) && ((!TOKEN && a.dgate) || a.dout_weight) && sum_of(q_sum)) {
    if (a.direct) {
      if (!TOKEN && a.dgate) store_scaled(a.dgate + mod, a.out_weight, 0.f, q_sum, col);
      store_scaled(a.dout_weight, gate, 0.f, q_sum, col);
    } else {
      store8<false>(a.partial + 2 * rows * a.C + first, col, pack8<false>(q_sum));
    }
  }
}

// 32 columns (8 lanes of 4) by 64 rows at a time per workgroup; the 64 partial sums in order through LDS.  A dimension of a launch holds less than
// 2^32 threads (one of more is dropped without an error): beyond 2^31 of them, with 8,192 channels from 5,461 sequences on, they go on in y.
constexpr int kSumColumns = 32, kSumRows = 64, kSumGroups = (1u << 31) / (kSumRows * 8);
__global__ __launch_bounds__(kSumRows * 8) void column_sums_kernel(ColumnJobs js) {
  __shared__ f32x4 lds[kSumRows][kSumColumns / 4];
  const int item = (int)blockIdx.x + kSumGroups * (int)blockIdx.y;
  if (item >= js.items) return;
  const int tiles = (js.columns + kSumColumns - 1) / kSumColumns, tile = item % tiles;
  int y = item / tiles, k = 0;
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

hipError_t launch_column_sums(const ColumnJobs& jobs, hipStream_t stream) {
  ColumnJobs j = jobs;
  int batches = 0;
  for (int k = 0; k < j.jobs; k++) batches += j.job[k].batches;
  if (batches == 0) return hipSuccess;
  j.items = (j.columns + kSumColumns - 1) / kSumColumns * batches;               // at most 256 (3 x 65,535 + 2)
  const dim3 grid((unsigned)(j.items < kSumGroups ? j.items : kSumGroups), (unsigned)((j.items - 1) / kSumGroups + 1));
  column_sums_kernel<<<grid, kSumRows * 8, 0, stream>>>(j);
  return hipGetLastError();
}

// f(types, part, modulation of every token) with the constants of a call
template <class F> static void with_types(const NormArgs& a, int part, F f) {
  auto with_part = [&](auto xb, auto hb) {
    auto with_token = [&](auto p) {
      if (a.mods == SLA2_MOD_TOKEN) f(xb, hb, p, std::true_type());
      else f(xb, hb, p, std::false_type());
    };
    if (part == kBefore) with_token(std::integral_constant<int, kBefore>());
    else if (part == kAfter) with_token(std::integral_constant<int, kAfter>());
    else with_token(std::integral_constant<int, kBefore | kAfter>());
  };
  if (a.x_bf16) with_part(std::true_type(), std::true_type());
  else if (a.h_bf16) with_part(std::false_type(), std::true_type());
  else with_part(std::false_type(), std::false_type());
}
static dim3 norm_block(const NormArgs& a) { return dim3((a.teams * a.team.threads() + kWave - 1) / kWave * kWave); }

hipError_t launch_norm(const NormArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)(a.B * a.walkers)), block = norm_block(a);
  with_types(a, part_of(a, false), [&](auto xb, auto hb, auto part, auto token) {
    constexpr bool XB = decltype(xb)::value, HB = decltype(hb)::value, TOKEN = decltype(token)::value;
    constexpr int PART = decltype(part)::value;
    if (a.team.vec == 1) norm_kernel<1, XB, HB, PART, TOKEN><<<grid, block, 0, stream>>>(a);
    else if (a.team.vec == 2) norm_kernel<2, XB, HB, PART, TOKEN><<<grid, block, 0, stream>>>(a);
    else norm_kernel<3, XB, HB, PART, TOKEN><<<grid, block, 0, stream>>>(a);
  });
  return hipGetLastError();
}

hipError_t launch_norm_bwd(const NormArgs& args, hipStream_t stream) {
  NormArgs a = args;
  plan_norm_direct(&a);
  const dim3 grid((unsigned)(a.B * a.walkers)), block = norm_block(a);
  const int vectors = 2 * (a.C + kChunk), sums = (a.teams - 1) * a.C;
  const size_t lds = (size_t)(vectors > sums ? vectors : sums) * sizeof(float);
  hipError_t e = hipSuccess;
  with_types(a, part_of(a, true), [&](auto xb, auto hb, auto part, auto token) {
    constexpr auto kernel = norm_bwd_kernel<decltype(xb)::value, decltype(hb)::value, decltype(part)::value, decltype(token)::value>;
    static OncePerDevice once;
    e = allow_dynamic_lds(once, (const void*)kernel, 2 * (kMaxRow + kChunk) * (int)sizeof(float));
    if (e == hipSuccess) kernel<<<grid, block, lds, stream>>>(a);
  });
  if (e == hipSuccess) e = hipGetLastError();
  if (e != hipSuccess || a.direct) return e;
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
