// How the kernels around the attention (sla2_rope.hip, sla2_norm.hip) spread rows over threads, teams and workgroups: host arithmetic on the
// sizes of a call alone, which a test on the CPU compiles as it is.
#pragma once
#include "common.h"

namespace sla2 {

constexpr int kChunk = 8;                    // channels: 16 bytes of bf16
constexpr int kMaxRow = 8192;                // channels of a row: 16 waves of a chunk a lane
constexpr int kTeamThreads = 512;            // threads of a workgroup
constexpr int kMaxThreads = 1024;
constexpr int kCus = 256;
// Waves of a SIMD that a kernel leaves registers for: 4 (two workgroups a CU), or 2 where a row takes more than 128 registers a thread.
constexpr int waves_of(bool many_registers) { return many_registers ? 2 : 4; }
constexpr int threads_of(bool many_registers) { return 4 * kWave * waves_of(many_registers); }

// How a row of `chunks` chunks is spread over threads.
struct RowTeam {
  int lanes, waves, vec;                     // lanes of a wave, whole waves (1 where lanes < 64), chunks a thread
  __host__ __device__ int threads() const { return lanes * waves; }
};
// The fewest waves with at most `most` chunks a thread (with more where a workgroup of `threads` threads has not that many waves), and then the
// fewest chunks.
inline RowTeam row_team(int chunks, int most, int threads = kTeamThreads) {
  RowTeam t{64, 1, 1};
  if (chunks <= 64) {
    while (t.lanes > 8 && t.lanes / 2 >= chunks) t.lanes /= 2;
    return t;
  }
  const int rounds = (chunks + 63) / 64, waves = (rounds + most - 1) / most;      // rounds: of a whole wave
  t.waves = waves < threads / kWave ? waves : threads / kWave;
  t.vec = (rounds + t.waves - 1) / t.waves;
  t.waves = (rounds + t.vec - 1) / t.vec;
  return t;
}
// Teams of a workgroup of `threads` threads, where there are rows enough.
inline int block_teams(const RowTeam& t, int rows, int threads = kTeamThreads) {
  const int n = t.threads() < threads ? threads / t.threads() : 1;
  return n < rows ? n : rows;
}
// Workgroups of a launch: those that are resident at once, with `threads` threads a CU.  Each goes through its rows side by side with the
// others, so that all read and write one stretch of memory.  Two and four times as many take 2 % less to 5 % more time forward, 14 to 57 %
// more backward (12 heads of 32,760 tokens 78.1 us, 79.5 and 79.0; backward 117, 147 and 142; 2 x 4,096 rows of 1,152 backward 56.8, 64.8, 69.3).
inline int resident_workgroups(const RowTeam& t, int teams, int threads) {
  const int block = (teams * t.threads() + kWave - 1) / kWave * kWave, n = threads / block;
  return kCus * (n < 1 ? 1 : n);
}

// ---- q and k: RMS norm and rotation ----
struct HeadStrides {
  long long b, h, n;
};
struct RopeArgs {
  const void* x[2];                          // q, k (k: null where there is none)
  const void* dy[2];                         // backward: gradients of the results
  void* y[2];                                // results; backward: gradients of x
  const float* weight[2];                    // [d] or [H, d], or null
  const double* freq;                        // [d / 2]
  const int32_t* positions;                  // [N, 3] or [B, N, 3], or null: the grid
  float* partial;                            // backward with a norm: [2][workgroups][d or H d], or null: no gradient of the weights
  float* dweight[2];
  int tensors, B, H, N, d;
  int pairs_end[3];                          // of the axes, one behind the last pair of each
  int grid[3], origin[3];
  long long positions_stride;                // of a batch
  HeadStrides sin, sout;                     // of x (and its gradient); of the results (and their gradients)
  float eps;
  int norm;                                  // sla2_rope_norm
  bool bf16, halves;
  bool cached;                               // the results stay in the caches
  double sign;                               // of the angles
  // launch
  RowTeam team;
  int teams, heads, groups, walkers;         // teams of a workgroup; heads of a row, rows of a token; workgroups of a (batch, group)
  bool direct;                               // backward: one workgroup has all rows and writes the results
};

// Whether a row takes more than 128 registers a thread: 3 chunks of q and of k behind a sum over all heads (40 heads of 75,601 tokens 566 us as
// 256 workgroups, 580 as 512).
constexpr bool large_rope(int vec, int norm) { return vec == 3 && norm == SLA2_ROPE_NORM_TOKEN; }

// Results - of q and k, or of the one that the call has - that fit the 256 MB memory-side cache are left there for the attention, which reads
// them next: 12 heads of 32,760 tokens (201 MB) with sla2_forward behind them 473 us, past the caches 489 us, though the call alone takes
// 80.7 and 75.8 us; 2 x 20 heads of 4,096 at d = 64 90.1 / 92.3 us; 40 heads of 75,600 (1.5 GB) 6,347 / 6,300 us; q alone of 146 and 191 MB
// the same to 1 %.
constexpr long long kCacheBytes = 256ll << 20;

// The sizes, types and number of tensors are there.  That number changes nothing but `cached`: a workspace is of the size for both.
inline void plan_rope(RopeArgs* a, bool backward) {
  const int most = kMaxRow / a->d;           // heads of a row
  a->groups = (a->H + most - 1) / most;
  a->heads = (a->H + a->groups - 1) / a->groups;
  const int chunks = a->heads * a->d / kChunk;
  a->cached = !backward && (long long)a->tensors * a->B * a->H * a->N * a->d * (a->bf16 ? 2 : 4) <= kCacheBytes;
  a->team = backward ? row_team(chunks, 1, kMaxThreads) : row_team(chunks, 3, kTeamThreads);
  // backward: one large workgroup a CU where a team has 5 waves or more (plan_norm)
  a->teams = block_teams(a->team, a->N, backward && a->team.waves > 4 ? kMaxThreads : kTeamThreads);
  const int threads = threads_of(!backward && large_rope(a->team.vec, a->norm));
  const int walkers = resident_workgroups(a->team, a->teams, threads) / (a->B * a->groups);
  const int needed = (int)(((long long)a->N + a->teams - 1) / a->teams);
  a->walkers = walkers < 1 ? 1 : walkers < needed ? walkers : needed;
}

inline int workgroups(const RopeArgs& a) { return a.B * a.groups * a.walkers; }
inline size_t rope_partial_floats(const RopeArgs& a) {
  return a.norm == SLA2_ROPE_NORM_NONE ? 0 : (size_t)2 * workgroups(a) * (a.norm == SLA2_ROPE_NORM_TOKEN ? a.H * a.d : a.d);
}

// Few rows: one workgroup takes them all and writes the gradients of the weights itself (plan_norm_direct); one token of 12 heads 3.9 us (two
// launches 7.0), 8 tokens with two rows a team 8.7 (7.8).
inline void plan_rope_direct(RopeArgs* a) {
  const int teams = block_teams(a->team, a->N, kMaxThreads);
  if (a->B * a->groups > 1 || a->N > teams) return;
  a->teams = teams;
  a->walkers = 1;
  a->direct = true;
}

// ---- norms around a block ----
struct NormArgs {
  const void *x, *y;                         // backward: x is what norm_in was taken of
  const float *gate, *out_weight, *in_weight, *scale, *shift;
  void *x_out, *h;
  // backward
  const void *dh, *dx_out;
  void *dx, *dy;
  float *dgate, *dout_weight, *din_weight, *dscale, *dshift;
  float* partial;                            // [3][B * walkers][C]: sums for scale, shift, gate of the rows of a workgroup
  int B, N, C;
  long long x_b, x_n, h_b, h_n, mod_b, mod_n;
  int norm_in, norm_out, mods;               // sla2_norm_kind, sla2_mod_layout
  float eps, rho;
  bool x_bf16, h_bf16;
  RowTeam team;
  int teams, walkers;                        // teams of a workgroup; workgroups of a batch
  bool direct;                               // backward: one workgroup has all rows and writes the results
};

constexpr int kBefore = 1, kAfter = 2;       // parts of a call: h; x'
// Whether a row takes more than 128 registers a thread, so that one workgroup of 8 waves fills a CU: 3 chunks with both parts (75,600 rows of
// 5,120 channels 868 us as 256 workgroups, 884 as 512, of which half wait), or with a modulation of every token.  A token's own modulation does
// not count for the number of workgroups, although half of 512 wait: both parts with 2 chunks, 2 x 12,481 rows of 2,048, 185 us as 256, 180 as
// 512; one part with 3 chunks 124.9 / 124.3 (32,760 rows of 1,536), 84.4 / 82.4 (2 x 12,481 of 1,536, bf16), 265.8 / 262.1 (20,000 of 5,120), and
// the other way round where there are few rows: 82.7 / 83.8 (7,000 of 5,120, bf16), 14.9 / 15.7 (3,000 of 1,536, fp32 throughout).
constexpr bool large_norm(int vec, int part, bool token) {
  const bool both = part == (kBefore | kAfter);
  return vec == 3 ? both || token : vec == 2 && both && token;
}

inline int part_of(const NormArgs& a, bool backward) { return ((backward ? a.dh : a.h) ? kBefore : 0) | (a.y ? kAfter : 0); }

inline void plan_norm(NormArgs* a, bool backward) {
  a->team = backward ? row_team(a->C / kChunk, 1, kMaxThreads) : row_team(a->C / kChunk, 3, kTeamThreads);
  // the rows of a wave lie within 2 GB of its first; where strides are longer than that it has one
  const long long x_n = a->x_n > a->h_n ? a->x_n : a->h_n, widest = x_n > a->mod_n ? x_n : a->mod_n;
  if (widest >= (1ll << 29) / (kWave / a->team.lanes)) a->team.lanes = kWave;
  const bool large = !backward && large_norm(a->team.vec, part_of(*a, false), false);
  // backward: one workgroup of up to 16 waves a CU where a team has 5 waves or more - of two with an odd number of waves the second often
  // finds no place (4 x 3,478 rows of 2,520 channels, 5 waves: 107 us as two, 78 as one) - else two, one of which works while the other waits
  // (31,201 rows of 1,536: 164 us as two of 6 waves, 172 as one of 15)
  a->teams = block_teams(a->team, a->N, backward && a->team.waves > 4 ? kMaxThreads : kTeamThreads);
  const int walkers = resident_workgroups(a->team, a->teams, threads_of(large)) / a->B, most = (int)(((long long)a->N + a->teams - 1) / a->teams);
  a->walkers = walkers < 1 ? 1 : walkers < most ? walkers : most;
}

// No more rows than one workgroup has teams: it takes them all and writes the gradients of the vectors itself, and the second launch is left
// out.  LayerNorm with scale and shift, one token of 1,536 channels 4.2 us (two launches 7.0), of 5,120 5.7 (8.4); with two rows a team it is
// even (8 tokens of 1,536: 7.9, 7.7) or worse (4 of 5,120: 10.2, 8.4).
inline void plan_norm_direct(NormArgs* a) {
  const int teams = block_teams(a->team, a->N, kMaxThreads);
  if (a->B > 1 || a->N > teams) return;
  a->teams = teams;
  a->walkers = 1;
  a->direct = true;
}

}  // namespace sla2
