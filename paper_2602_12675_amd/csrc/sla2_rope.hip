// q and k on their way into the attention: RMS norm over a head or over all heads of a token, then rotary positions of up to three axes.
//   m = x r w,  r = 1 / sqrt(mean(x^2) + eps);   pair j of a head, of axis a(j):  angle = p_a(j)(token) f_j,
//   (m_1, m_2) -> (m_1 cos - m_2 sin, m_1 sin + m_2 cos)
// and backward, with g = the gradient turned back by the angle, n = x r, t = g w:  dw = sum g n,  dx = r (t - n mean(t n)).
//
// A row is a token with all its heads (as many as kMaxRow channels hold, where no sum goes over them), of q and of k: one reading of
// each, one writing, and the angles are formed once for all heads of both.  A thread's chunks all lie at the same channels of their
// heads, so it needs 4 angles (pairs of neighbours) or 8 (halves: the partner's channels come from a lane 4 or 8 further, by vector
// instructions).  Angles are products in fp64, with the whole turns off before the rounding to fp32: a position of 2^31 is as exact as fp64
// has it.  What ends in fp32, the gradients of the weights among it, takes sines and cosines that are good to its last places, bf16 results
// the hardware's.
#include "rows.h"

namespace sla2 {

// x of the lane that holds the other channel of each pair of a head of LANES lanes
template <int LANES> __device__ __forceinline__ float half_head_away(float x) {
  if constexpr (LANES == 16) return rotate16<8>(x);
  else return dpp_move<0x1B>(dpp_move<0x141>(x));           // row_half_mirror (l ^ 7), quad_perm 3 2 1 0 (l ^ 3)
}

// Where the tokens of a thread's rows are, one step of the workgroup after the other.
struct Position {
  unsigned t, y, x;                          // of the grid
  unsigned dt, dy, dx;                       // a step
  __device__ __forceinline__ Position(const RopeArgs& a, long long first, long long step) : t(0), y(0), x(0), dt(0), dy(0), dx(0) {
    if (a.positions) return;
    const unsigned cols = (unsigned)a.grid[2], rows = (unsigned)a.grid[1], n = (unsigned)first, s = (unsigned)step;
    x = n % cols; y = n / cols % rows; t = n / cols / rows;
    dx = s % cols; dy = s / cols % rows; dt = s / cols / rows;
  }
  __device__ __forceinline__ void advance(const RopeArgs& a) {
    x += dx; y += dy; t += dt;
    if (x >= (unsigned)a.grid[2]) { x -= (unsigned)a.grid[2]; y++; }
    if (y >= (unsigned)a.grid[1]) { y -= (unsigned)a.grid[1]; t++; }
  }
  // of token n of batch b, which is where the steps are
  __device__ __forceinline__ void at(const RopeArgs& a, int b, long long n, bool row, int& p0, int& p1, int& p2) const {
    if (a.positions) {
      const int32_t* q = a.positions + b * a.positions_stride + (row ? 3 * n : 0);
      p0 = q[0]; p1 = q[1]; p2 = q[2];
    } else {
      const bool in = t < (unsigned)a.grid[0];
      p0 = in ? a.origin[0] + (int)t : 0;
      p1 = in ? a.origin[1] + (int)y : 0;
      p2 = in ? a.origin[2] + (int)x : 0;
    }
  }
};

// t less the whole number next to it.  Of t as it is rounded: contracted with the product that t is, the difference holds that product's own
// rounding, which past 2^53 is large.
__device__ __forceinline__ double off_whole(double t) {
#pragma clang fp contract(off)
  return t - rint(t);
}

// Sine and cosine of t quarters of a turn, within 3 units of 2^-24 of themselves.  Whole quarters go off in fp64, before the rounding to fp32: the
// last place of a fraction of a turn in fp32 is 9.4e-8 in either result, however close to zero that is.  1.5 x 2^52 has its last place at 1:
// added, it leaves the number of quarters there (past 2^51 of them t has no fraction that means anything, and the result is a point of the
// circle still).  Taylor's series over +-pi/4 (what is left out: 2.5e-9 of the sine, 1.5e-10 of the cosine).
__device__ __forceinline__ void sin_cos_of_quarters(double t, float& s, float& c) {
  const unsigned q = (unsigned)__builtin_bit_cast(unsigned long long, rint(t) + 6755399441055744.0);
  const float x = (float)(off_whole(t) * 1.5707963267948966), z = x * x;
  const float s0 = x + x * (z * (-1.f / 6 + z * (1.f / 120 + z * (-1.f / 5040 + z * (1.f / 362880)))));
  const float c0 = 1.f + z * (-0.5f + z * (1.f / 24 + z * (-1.f / 720 + z * (1.f / 40320 + z * (-1.f / 3628800)))));
  s = q & 1 ? c0 : s0;
  c = q & 1 ? s0 : c0;
  if (q & 2) s = -s;
  if ((q + 1) & 2) c = -c;
}

// The cosines and sines of the pairs of a thread's channels.  A token has d / 2 angles in all: each lane of a wave forms those of one
// pair, or as many as there are tokens in the wave more, and all take theirs from LDS, where a wave has a place of its own.  Each lane
// forming its own 4 or 8, most of them again in other lanes, was up to half of the instructions of a row.
constexpr int kAngleFloats = 512;            // of a wave: 8 tokens of 64 channels, 4 of 128: cosines, then sines, of the pairs of each
struct AngleLds {
  double turns[64];                          // of a pair per position; or quarters of a turn
  float of[kMaxThreads / kWave * kAngleFloats];            // at the end of the backward kernel: the sums of all threads but the first part's
};
static_assert(kAngleFloats >= kWave * kChunk, "");
template <bool HARDWARE, bool HALVES> struct Angles {
  static constexpr int kPairs = HALVES ? 8 : 4;
  const double* turns;
  int end0, end1, lanes, pair, half;         // of the axes; lanes of a token in the wave; the first pair that this one forms; d / 2
  float *token, *from;
  float other;                               // halves: which way the other channel of a pair goes into this one
  float c[kPairs], s[kPairs];
  __device__ __forceinline__ Angles(const RopeArgs& a, const Team& tm, AngleLds& lds) : turns(lds.turns), end0(a.pairs_end[0]), end1(a.pairs_end[1]) {
    lanes = tm.t.lanes;
    half = a.d / 2;
    pair = tm.lane % lanes;
    for (int j = (int)threadIdx.x; j < half; j += (int)blockDim.x)
      lds.turns[j] = j < a.pairs_end[2] ? a.freq[j] * (a.sign * (HARDWARE ? 1 : 4) * 0.15915494309189533577) : 0.0;     // 1 / (2 pi); backward: the other way round
    __syncthreads();
    token = lds.of + (int)threadIdx.x / kWave * kAngleFloats + (int)threadIdx.x % kWave / lanes * a.d;
    other = HALVES && tm.lane % (a.d / kChunk) < a.d / kChunk / 2 ? -1.f : 1.f;
    from = token + (HALVES ? tm.lane * kChunk % half : tm.lane % (a.d / kChunk) * 4);
  }
  // HARDWARE, for bf16 results: the hardware's sine and cosine of a fraction of a turn, whose error is far below half a step of bf16 (over all
  // fp32 fractions 1.25e-7 at most, with the rounding of the fraction 2.2e-7; half a step at 1 is 3.9e-3)
  __device__ __forceinline__ void at(int p0, int p1, int p2) {
    wave_lds_fence();
    for (int j = pair; j < half; j += lanes) {
      const double t = (double)(j < end0 ? p0 : j < end1 ? p1 : p2) * turns[j];
      float si, co;
      if constexpr (HARDWARE) {
        const float f = (float)off_whole(t);
        si = __builtin_amdgcn_sinf(f);
        co = __builtin_amdgcn_cosf(f);
      } else {
        sin_cos_of_quarters(t, si, co);
      }
      token[j] = co;
      token[half + j] = si;
    }
    wave_lds_fence();
#pragma unroll
    for (int i = 0; i < kPairs; i += 4) {
      const f32x4 co = *(const f32x4*)(from + i), si = *(const f32x4*)(from + half + i);
#pragma unroll
      for (int k = 0; k < 4; k++) {
        c[i + k] = co[k];
        s[i + k] = HALVES ? other * si[k] : si[k];
      }
    }
  }
};

template <bool HARDWARE, bool HALVES>
__device__ __forceinline__ void turn(const RopeArgs& a, const Angles<HARDWARE, HALVES>& an, float (&x)[8]) {
  if constexpr (HALVES) {
    float o[8];
    if (a.d == 128) {
#pragma unroll
      for (int i = 0; i < 8; i++) o[i] = half_head_away<16>(x[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++) o[i] = half_head_away<8>(x[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] = x[i] * an.c[i] + o[i] * an.s[i];
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const float p = x[2 * i], q = x[2 * i + 1];
      x[2 * i] = p * an.c[i] - q * an.s[i];
      x[2 * i + 1] = p * an.s[i] + q * an.c[i];
    }
  }
}

__device__ __forceinline__ float head_sum(float x, int d) { return d == 128 ? sum16(x) : sum8(x); }

// What a thread holds of its rows: V chunks of heads.
template <int V> struct Place {
  bool has[V];
  size_t in[V], out[V];                      // offsets from the first token of the wave
  int col[V];                                // channel among all heads
  int channel;                               // of its chunks in their heads
  __device__ __forceinline__ Place(const RopeArgs& a, const Team& tm, int group) {
    const int per_head = a.d / kChunk;
    channel = tm.lane % per_head * kChunk;
#pragma unroll
    for (int v = 0; v < V; v++) {
      const int c = tm.lane + v * a.team.threads(), head = group * a.heads + c / per_head;
      has[v] = tm.team < a.teams && c < a.heads * per_head && head < a.H;
      const int h = has[v] ? head : 0;
      in[v] = (size_t)tm.sub * a.sin.n + (size_t)h * a.sin.h + channel;
      out[v] = (size_t)tm.sub * a.sout.n + (size_t)h * a.sout.h + channel;
      col[v] = has[v] ? h * a.d + channel : 0;
    }
  }
};

template <int V, bool BF16, bool HALVES, int NORM>
__global__ __launch_bounds__(kTeamThreads, waves_of(large_rope(V, NORM))) void rope_kernel(RopeArgs a) {
  __shared__ float lds[kExchangeFloats];
  __shared__ AngleLds angles;
  constexpr int W = NORM == SLA2_ROPE_NORM_TOKEN ? V : 1;
  Team tm(a.team, lds);
  const int part = (int)blockIdx.x / a.walkers, walker = (int)blockIdx.x % a.walkers, b = part / a.groups;
  const Place<V> at(a, tm, part % a.groups);
  Angles<BF16, HALVES> an(a, tm, angles);
  const float share = 1.f / (float)(NORM == SLA2_ROPE_NORM_TOKEN ? a.H * a.d : a.d);
  float w[2][W][8];
  if (NORM != SLA2_ROPE_NORM_NONE) {
#pragma unroll
    for (int t = 0; t < 2; t++)
#pragma unroll
      for (int v = 0; v < W; v++) load_vector8(a.weight[t], NORM == SLA2_ROPE_NORM_TOKEN ? at.col[v] : at.channel, 1.f, w[t][v]);
  }
  const long long step = (long long)a.walkers * a.teams;
  Position where(a, (long long)walker * a.teams + tm.team, step);
  struct Row {
    Raw<BF16> x[2][V];
    int p0, p1, p2;
  };
  auto load = [&](long long n0) {
    const long long n = n0 + tm.first;
    const bool row = n + tm.sub < a.N;
    Row r;
#pragma unroll
    for (int t = 0; t < 2; t++) {
      const void* px = at_elem<BF16>(a.x[t], b * a.sin.b + n * a.sin.n);
#pragma unroll
      for (int v = 0; v < V; v++) r.x[t][v] = row && at.has[v] && t < a.tensors ? load8<BF16>(px, at.in[v]) : zero8<BF16>();
    }
    where.at(a, b, n + tm.sub, row, r.p0, r.p1, r.p2);
    return r;
  };
  for (long long n0 = (long long)walker * a.teams; n0 < a.N; n0 += step) {
    const long long n = n0 + tm.first;
    const bool row = n + tm.sub < a.N;
    const long long yo = b * a.sout.b + n * a.sout.n;
    Row cur = load(n0);
    Raw<BF16> (&raw)[2][V] = cur.x;
    where.advance(a);
    an.at(cur.p0, cur.p1, cur.p2);
    float s[2] = {0.f, 0.f};
    if (NORM == SLA2_ROPE_NORM_TOKEN) {
#pragma unroll
      for (int t = 0; t < 2; t++)
#pragma unroll
        for (int v = 0; v < V; v++) {
          float x[8];
          unpack8<BF16>(raw[t][v], x);
#pragma unroll
          for (int i = 0; i < 8; i++) s[t] += x[i] * x[i];
        }
      tm.sum(s);
#pragma unroll
      for (int t = 0; t < 2; t++) s[t] = inv_sqrt(s[t] * share + a.eps);
    }
#pragma unroll
    for (int t = 0; t < 2; t++) {
      if (t >= a.tensors) break;
#pragma unroll
      for (int v = 0; v < V; v++) {
        float x[8];
        unpack8<BF16>(raw[t][v], x);
        if (NORM == SLA2_ROPE_NORM_HEAD) {
          float q = 0.f;
#pragma unroll
          for (int i = 0; i < 8; i++) q += x[i] * x[i];
          s[t] = inv_sqrt(head_sum(q, a.d) * share + a.eps);
        }
        if (NORM != SLA2_ROPE_NORM_NONE) {
#pragma unroll
          for (int i = 0; i < 8; i++) x[i] = x[i] * s[t] * w[t][v % W][i];
        }
        turn(a, an, x);
        if (row && at.has[v]) {
          if (a.cached) store8<BF16>(at_elem<BF16>(a.y[t], yo), at.out[v], pack8<BF16>(x));
          else put8<BF16>(at_elem<BF16>(a.y[t], yo), at.out[v], pack8<BF16>(x));
        }
      }
    }
  }
}

// Gradients of x and, where there are partial sums, of the weights, which are fp32 whatever x is: its sines and cosines are the exact ones
// (2 x 20 heads of 4,429 tokens in bf16 35.4 us, with the hardware's 35.0).  A thread has one chunk of q and of k; with two it would need more
// registers than leave a CU 16 waves (12 heads of 32,760 tokens 139 us, with one 117).
template <bool BF16, bool HALVES, bool TOKEN>
__global__ __launch_bounds__(kMaxThreads, 4) void rope_bwd_kernel(RopeArgs a) {
  __shared__ float lds[kExchangeFloats];
  __shared__ AngleLds angles;
  Team tm(a.team, lds);
  const int part = (int)blockIdx.x / a.walkers, walker = (int)blockIdx.x % a.walkers, b = part / a.groups;
  const Place<1> at(a, tm, part % a.groups);
  Angles<false, HALVES> an(a, tm, angles);
  const float share = 1.f / (float)(TOKEN ? a.H * a.d : a.d);
  float w[2][8], acc[2][8];
#pragma unroll
  for (int t = 0; t < 2; t++) {
    load_vector8(a.weight[t], TOKEN ? at.col[0] : at.channel, 1.f, w[t]);
#pragma unroll
    for (int i = 0; i < 8; i++) acc[t][i] = 0.f;
  }
  const long long step = (long long)a.walkers * a.teams;
  Position where(a, (long long)walker * a.teams + tm.team, step);
  for (long long n0 = (long long)walker * a.teams; n0 < a.N; n0 += step) {
    const long long n = n0 + tm.first, xo = b * a.sin.b + n * a.sin.n, yo = b * a.sout.b + n * a.sout.n;
    const bool row = n + tm.sub < a.N, on = row && at.has[0];
    Raw<BF16> rx[2], rg[2];
#pragma unroll
    for (int t = 0; t < 2; t++) {
      rx[t] = on && t < a.tensors ? load8<BF16>(at_elem<BF16>(a.x[t], xo), at.in[0]) : zero8<BF16>();
      rg[t] = on && t < a.tensors ? load8<BF16>(at_elem<BF16>(a.dy[t], yo), at.out[0]) : zero8<BF16>();
    }
    int p0, p1, p2;
    where.at(a, b, n + tm.sub, row, p0, p1, p2);
    where.advance(a);
    an.at(p0, p1, p2);
    float g[2][8], s[4];                     // sum x^2, sum t x: of q, of k
    auto sums = [&](int t) {
      float x[8];
      unpack8<BF16>(rx[t], x);
      unpack8<BF16>(rg[t], g[t]);
      turn(a, an, g[t]);
      s[2 * t] = s[2 * t + 1] = 0.f;
#pragma unroll
      for (int i = 0; i < 8; i++) {
        s[2 * t] += x[i] * x[i];
        s[2 * t + 1] += g[t][i] * w[t][i] * x[i];
      }
    };
    auto finish = [&](int t) {
      float x[8];
      unpack8<BF16>(rx[t], x);
      const float r = inv_sqrt(s[2 * t] * share + a.eps), mean = s[2 * t + 1] * share * r;
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const float nx = x[i] * r;
        acc[t][i] += g[t][i] * nx;
        x[i] = r * (g[t][i] * w[t][i] - nx * mean);
      }
      if (on) put8<BF16>(at_elem<BF16>(a.y[t], xo), at.in[0], pack8<BF16>(x));
    };
    if constexpr (TOKEN) {                   // both in one exchange
      sums(0);
      sums(1);
      tm.sum(s);
      finish(0);
      if (a.tensors > 1) finish(1);
    } else {
#pragma unroll
      for (int t = 0; t < 2; t++) {
        if (t >= a.tensors) break;
        sums(t);
        s[2 * t] = head_sum(s[2 * t], a.d);
        s[2 * t + 1] = head_sum(s[2 * t + 1], a.d);
        finish(t);
      }
    }
  }
  if (!a.dweight[0] && !a.dweight[1]) return;
  // parts: the teams, or the places of a head in a row of any team, which are a head's lanes apart
  const int cols = TOKEN ? a.H * a.d : a.d, lanes = TOKEN ? a.team.threads() : a.d / kChunk;
  const int me = (int)threadIdx.x, part_of = me / lanes, parts = TOKEN ? a.teams : (int)blockDim.x / lanes;
#pragma unroll
  for (int t = 0; t < 2; t++) {
    if (!a.dweight[t]) continue;
    join_parts(angles.of, part_of, parts, lanes * kChunk, (unsigned)(me % lanes * kChunk), true, acc[t]);
    if (part_of != 0 || (TOKEN && !at.has[0])) continue;
    float* to = a.direct ? a.dweight[t] : a.partial + ((size_t)t * gridDim.x + blockIdx.x) * cols;
    store8<false>(to, (unsigned)(TOKEN ? at.col[0] : at.channel), pack8<false>(acc[t]));
  }
}

// f(element type, pairing) with the constants of a call
template <class F> static void with_types(const RopeArgs& a, F f) {
  auto with_pairs = [&](auto bf16) {
    if (a.halves) f(bf16, std::true_type());
    else f(bf16, std::false_type());
  };
  if (a.bf16) with_pairs(std::true_type());
  else with_pairs(std::false_type());
}
static int whole_waves(const RopeArgs& a) { return (a.teams * a.team.threads() + kWave - 1) / kWave * kWave; }

template <int V, bool BF16, bool HALVES> static void launch_forward(const RopeArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)workgroups(a)), block(whole_waves(a));
  if (a.norm == SLA2_ROPE_NORM_TOKEN) rope_kernel<V, BF16, HALVES, SLA2_ROPE_NORM_TOKEN><<<grid, block, 0, stream>>>(a);
  else if (a.norm == SLA2_ROPE_NORM_HEAD) rope_kernel<V, BF16, HALVES, SLA2_ROPE_NORM_HEAD><<<grid, block, 0, stream>>>(a);
  else rope_kernel<V, BF16, HALVES, SLA2_ROPE_NORM_NONE><<<grid, block, 0, stream>>>(a);
}
hipError_t launch_rope(const RopeArgs& a, hipStream_t stream) {
  with_types(a, [&](auto bf16, auto halves) {
    constexpr bool BF16 = decltype(bf16)::value, HALVES = decltype(halves)::value;
    if (a.team.vec == 1) launch_forward<1, BF16, HALVES>(a, stream);
    else if (a.team.vec == 2) launch_forward<2, BF16, HALVES>(a, stream);
    else launch_forward<3, BF16, HALVES>(a, stream);
  });
  return hipGetLastError();
}

hipError_t launch_rope_bwd(const RopeArgs& args, hipStream_t stream) {
  RopeArgs a = args;
  a.sign = -1.0;
  if (a.norm == SLA2_ROPE_NORM_NONE) {       // the rotation back, from the layout of the results to that of x
    for (int t = 0; t < 2; t++) a.x[t] = a.dy[t];
    const HeadStrides s = a.sin;
    a.sin = a.sout;
    a.sout = s;
    plan_rope(&a, false);
    a.cached = false;
    return launch_rope(a, stream);
  }
  plan_rope_direct(&a);
  with_types(a, [&](auto bf16, auto halves) {
    constexpr bool BF16 = decltype(bf16)::value, HALVES = decltype(halves)::value;
    const dim3 grid((unsigned)workgroups(a)), block(whole_waves(a));
    if (a.norm == SLA2_ROPE_NORM_TOKEN) rope_bwd_kernel<BF16, HALVES, true><<<grid, block, 0, stream>>>(a);
    else rope_bwd_kernel<BF16, HALVES, false><<<grid, block, 0, stream>>>(a);
  });
  if (hipError_t e = hipGetLastError(); e != hipSuccess || a.direct) return e;
  ColumnJobs js{};
  js.columns = a.norm == SLA2_ROPE_NORM_TOKEN ? a.H * a.d : a.d;
  const int rows = workgroups(a);
  for (int t = 0; t < 2; t++)
    if (a.dweight[t])
      js.job[js.jobs++] = ColumnJob{a.partial + (size_t)t * rows * js.columns, 1, rows, nullptr, 0.f, nullptr, 0.f, 1, 0, a.dweight[t], 0};
  return launch_column_sums(js, stream);
}

}  // namespace sla2
