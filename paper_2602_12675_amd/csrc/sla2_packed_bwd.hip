// Backward pass of attention over packed sequences.  With P = exp(scale Q K^T - lse) and D = rowsum(dO . O):
//   dV = P^T dO,   dS = P . (dO V^T - D),   dQ = scale dS K,   dK = scale dS^T Q.
//
// Two kernels, so that every sum has one owner and a fixed order: one for each tile of rows (D and dQ), one for each tile of keys (dK
// and dV, over the rows of all heads of the group).  Both form P and dO V^T themselves: 7 products in all for 5 that are needed, where
// a sum of dQ over workgroups would take a d-wide row of fp32 written and read back for each tile of keys.
#include "packed.h"

namespace sla2 {

template <int D> struct PackedBwdSmem {
  static constexpr int kTile = PackedTile<D>::kTileBytes;
  static constexpr int kLd = D + 8;
  static constexpr int kStatOff = 4 * kTile;                   // float [2][2][64]: lse log2(e) and D of a step's rows (key side)
  static constexpr int kBytes = kStatOff + 4 * 64 * 4;
  static_assert(4 * 32 * kLd * 2 <= kStatOff, "32 result rows of a wave in the place of the tiles");
};

// 32 rows of a wave from accumulators (channels x rows) through LDS to memory, times `by`; row_ptr(r): where row r goes, null: nowhere
template <int D, class Row>
__device__ __forceinline__ void store_rows(const f32x16 (&acc)[D / 32], float by, uint16_t* os /* [32][D + 8], of this wave */, int lane, Row row_ptr) {
  constexpr int LD = D + 8;
#pragma unroll
  for (int et = 0; et < D / 32; et++)
#pragma unroll
    for (int v4 = 0; v4 < 4; v4++) {
      bf16x4 pk;
#pragma unroll
      for (int r = 0; r < 4; r++) pk[r] = (__bf16)(by * acc[et][4 * v4 + r]);
      *reinterpret_cast<bf16x4*>(os + lane % 32 * LD + 32 * et + 8 * v4 + 4 * (lane / 32)) = pk;
    }
  wave_lds_fence();
#pragma unroll
  for (int i = 0; i < 32 * (D / 8) / kWave; i++) {
    const int idx = lane + kWave * i, r = idx / (D / 8), ch = idx % (D / 8);
    uint16_t* dst = row_ptr(r);
    if (dst) *reinterpret_cast<u32x4*>(dst + 8 * ch) = *reinterpret_cast<const u32x4*>(os + r * LD + 8 * ch);
  }
  wave_lds_fence();
}
template <int D>
__device__ __forceinline__ void store_part(const f32x16 (&acc)[D / 32], float* dst, int g) {
#pragma unroll
  for (int et = 0; et < D / 32; et++)
#pragma unroll
    for (int v4 = 0; v4 < 4; v4++)
      *reinterpret_cast<f32x4*>(dst + 32 * et + 8 * v4 + 4 * g) =
          f32x4{acc[et][4 * v4], acc[et][4 * v4 + 1], acc[et][4 * v4 + 2], acc[et][4 * v4 + 3]};
}
__device__ __forceinline__ void pin(bf16x8& f) {       // converted here: eight registers less than the fp32 values
  u32x4 u = __builtin_bit_cast(u32x4, f);
  settle(u);
  f = __builtin_bit_cast(bf16x8, u);
}

// acc[et] += A^T f: the 32 rows of a tile at `lo` / `hi` (tr_read_offset) contracted, as two 16-row steps, into all channels
template <int D>
__device__ __forceinline__ void contract32(f32x16 (&acc)[D / 32], const bf16x8* f, unsigned lo_at, unsigned hi_at) {
  constexpr int ET = D / 32, kFrags = 2 * ET, kAhead = 3, kSlots = kAhead + 1;
  u32x2 lo[kSlots], hi[kSlots];
  auto issue = [&](int n) {
    lo[n % kSlots] = lds_read_tr_untracked_at<32 * D>(lo_at ^ (64u * (n % ET)), n / ET);
    hi[n % kSlots] = lds_read_tr_untracked_at<32 * D>(hi_at ^ (64u * (n % ET)), n / ET);
  };
#pragma unroll
  for (int n = 0; n < kAhead; n++) issue(n);
#pragma unroll
  for (int n = 0; n < kFrags; n++) {
    if (n + kAhead < kFrags) issue(n + kAhead);
    wait_lgkmcnt(2 * (n + kAhead < kFrags ? kAhead : kFrags - 1 - n));
    settle(lo[n % kSlots]);
    settle(hi[n % kSlots]);
    const u32x4 v4 = {lo[n % kSlots][0], lo[n % kSlots][1], hi[n % kSlots][0], hi[n % kSlots][1]};
    acc[n % ET] = mfma_bf16(__builtin_bit_cast(bf16x8, v4), f[n / ET], acc[n % ET]);
  }
}

// D and dQ of 128 rows: S^T = K Q^T and dP^T = V dO^T (keys x rows), dQ^T += K^T dS^T, as in the forward pass with K in the place of V.
template <int D, bool PARTS>
__global__ __launch_bounds__(256, 2) void packed_dq_kernel(PackedArgs a) {
  constexpr int NW = 4, KS = D / 16, ET = D / 32;
  typedef PackedBwdSmem<D> SM;
  typedef PackedTile<D> SL;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid % kWave, g = lane / 32;
  const int w = __builtin_amdgcn_readfirstlane(tid / kWave);
  const TileHead th = tile_head(blockIdx.x, a.Hkv);
  const int hk = th.head;
  TilePlace at = find_tile<false>(a, kRowTile, th.tile, lane);
  if (at.tile < 0) return;
  if (a.causal) at.tile = at.tiles - 1 - at.tile;      // the longest first
  const int nr = at.nq * a.group, nk = at.nk, row0 = at.tile * kRowTile, row = row0 + 32 * w + lane % 32;
  const uint16_t* kh = a.k + (size_t)hk * a.skv.h + (size_t)at.k0 * a.skv.t;
  const uint16_t* vh = a.v + (size_t)hk * a.skv.h + (size_t)at.k0 * a.skv.t;
  const int past = nk - at.nq;
  const int2 my = query_of(a, min(row, nr - 1));
  const int mine = a.causal ? min(nk, my.x + past + 1) : nk;
  const int keys = a.causal ? min(nk, max(0, query_of(a, min(row0 + kRowTile, nr) - 1).x + past + 1)) : nk;
  const int w_row = row0 + 32 * w;
  const int w_keys = w_row >= nr ? 0 : __builtin_amdgcn_readlane(mine, 31), w_full = __builtin_amdgcn_readfirstlane(mine);
  int t_begin = 0, t_end = (keys + kTileTokens - 1) / kTileTokens;
  if (PARTS) {
    const int n = t_end;
    t_begin = (int)((long long)n * blockIdx.y / a.q_parts);
    t_end = (int)((long long)n * (blockIdx.y + 1) / a.q_parts);
  }
  auto kbuf = [&](int t) { return lds_address(smem) + (t & 1) * 2 * SM::kTile; };
  auto dma = [&](int t) {
    const int t0 = t * kTileTokens, valid = min(kTileTokens, nk - t0), ln = (int)lane_again();
    dma_tile<D, NW, SL>(kh + (size_t)t0 * a.skv.t, a.skv.t, valid, kbuf(t), w, ln);
    dma_tile<D, NW, SL>(vh + (size_t)t0 * a.skv.t, a.skv.t, valid, kbuf(t) + SM::kTile, w, ln);
  };
  if (t_begin < t_end) dma(t_begin);
  bf16x8 qf[KS], gf[KS];
  float delta = 0.f;
  const size_t row_at = (size_t)hk * a.Tq * a.group + (size_t)at.q0 * a.group + row;       // among the rows of all key heads
  const int h = hk * a.group + my.y, token = at.q0 + my.x;
  {
    const uint16_t* src = a.q + (size_t)h * a.sq.h + (size_t)token * a.sq.t + 8 * g;
    const uint16_t* gsrc = a.dout + (size_t)h * a.so.h + (size_t)token * a.so.t + 8 * g;
    const uint16_t* osrc = a.out + (size_t)h * a.so.h + (size_t)token * a.so.t + 8 * g;
#pragma unroll
    for (int ks = 0; ks < KS; ks++) {
      qf[ks] = *reinterpret_cast<const bf16x8*>(src + 16 * ks);
      gf[ks] = *reinterpret_cast<const bf16x8*>(gsrc + 16 * ks);
      const bf16x8 o = *reinterpret_cast<const bf16x8*>(osrc + 16 * ks);
#pragma unroll
      for (int e = 0; e < 8; e++) delta += (float)gf[ks][e] * (float)o[e];
    }
  }
  delta = swap_halves_sum(delta);
  const float lse = a.lse[(size_t)h * a.Tq + token];
  const float l2 = lse == -INFINITY ? INFINITY : lse * kLog2e;   // a row that reads no key: P = 0
  if (row < nr && g == 0 && (!PARTS || blockIdx.y == 0)) {
    a.delta[row_at] = delta;
    a.lse2[row_at] = l2;
  }
  const float c1 = kLog2e * a.scale;
  f32x16 acc[ET];
#pragma unroll
  for (int et = 0; et < ET; et++)
#pragma unroll
    for (int e = 0; e < 16; e++) acc[et][e] = 0.f;
  const unsigned k_off = row_read_offset<D>(lane), t_lo = tr_read_offset<D>(lane, 0), t_hi = tr_read_offset<D>(lane, 1);
  wait_vmcnt<0>();
#pragma unroll
  for (int ks = 0; ks < KS; ks++) { settle(qf[ks]); settle(gf[ks]); }
  phase_barrier();
  for (int t = t_begin; t < t_end; t++) {
    if (t + 1 < t_end) dma(t + 1);
    const int t0 = t * kTileTokens;
    if (t0 < w_keys) {
#pragma unroll
      for (int mt = 0; mt < 2; mt++) {
        const unsigned ka = kbuf(t) + 64 * D * mt;
        f32x16 s, dp;
#pragma unroll
        for (int e = 0; e < 16; e++) s[e] = dp[e] = 0.f;
        bf16x8 df[2];
        const bool edge = t0 + 32 * mt + 32 > w_full;
        constexpr int kItems = 2 * KS, kAhead = 4, kSlots = kAhead + 1;
        u32x4 ring[kSlots];
        auto issue = [&](int n) {
          ring[n % kSlots] = lds_read16_untracked<0>((ka + (n < KS ? 0 : SM::kTile) + k_off) ^ (32u * (n % KS)));
        };
#pragma unroll
        for (int n = 0; n < kAhead; n++) issue(n);
#pragma unroll
        for (int n = 0; n < kItems; n++) {
          if (n + kAhead < kItems) issue(n + kAhead);
          wait_lgkmcnt(n + kAhead < kItems ? kAhead : kItems - 1 - n);
          settle(ring[n % kSlots]);
          const bf16x8 f = __builtin_bit_cast(bf16x8, ring[n % kSlots]);
          if (n < KS) {
            s = mfma_bf16(f, qf[n], s);
          } else {
            dp = mfma_bf16(f, gf[n - KS], dp);
            constexpr int kStep = KS / 4;              // behind every quarter of the products of dP four exponentials
            if ((n - KS) % kStep == kStep - 1) {
              const int v4 = (n - KS) / kStep;
#pragma unroll
              for (int r = 0; r < 4; r++) {
                float p = fast_exp2(s[4 * v4 + r] * c1 - l2);
                settle(p);
                s[4 * v4 + r] = p;
              }
            }
          }
        }
        if (edge) {
#pragma unroll
          for (int e = 0; e < 16; e++)
            if (t0 + 32 * mt + 8 * (e / 4) + 4 * g + e % 4 >= mine) s[e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < 16; e++) df[e / 8][e % 8] = (__bf16)(s[e] * (dp[e] - delta));
        pin(df[0]);
        pin(df[1]);
        contract32<D>(acc, df, ka + t_lo, ka + t_hi);
      }
    }
    wait_vmcnt<0>();
    phase_barrier();
  }
  if (PARTS) {
    if (row < nr) store_part<D>(acc, a.part_o + ((size_t)blockIdx.y * a.Tq * a.H + row_at) * D, g);
    return;
  }
  store_rows<D>(acc, a.scale, reinterpret_cast<uint16_t*>(smem) + w * 32 * SM::kLd, lane, [&](int r) -> uint16_t* {
    if (w_row + r >= nr) return nullptr;
    const int2 x = query_of(a, w_row + r);
    return a.dq + (size_t)(hk * a.group + x.y) * a.sq.h + (size_t)(at.q0 + x.x) * a.sq.t;
  });
}

// dK and dV of 128 keys: S = Q K^T and dP = dO V^T (rows x keys), a key on lanes l and l + 32 with its row of K and V in registers;
// dV^T += dO^T P and dK^T += Q^T dS, 64 rows a step, which arrive in LDS one step ahead.
template <int D, bool PARTS>
__global__ __launch_bounds__(256, 2) void packed_dkv_kernel(PackedArgs a) {
  constexpr int NW = 4, KS = D / 16, ET = D / 32;
  typedef PackedBwdSmem<D> SM;
  typedef PackedTile<D> SL;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  float* stat = reinterpret_cast<float*>(smem + SM::kStatOff);
  const int tid = threadIdx.x, lane = tid % kWave, g = lane / 32;
  const int w = __builtin_amdgcn_readfirstlane(tid / kWave);
  const TileHead th = tile_head(blockIdx.x, a.Hkv);
  const int hk = th.head;
  const TilePlace at = find_tile<true>(a, kKeyTile, th.tile, lane);
  if (at.tile < 0) return;
  const int nr = at.nq * a.group, nk = at.nk, key0 = at.tile * kKeyTile, key = key0 + 32 * w + lane % 32;
  const size_t token = (size_t)at.k0 + min(key, nk - 1);
  const int past = nk - at.nq;
  const uint16_t* qh = a.q + (size_t)hk * a.group * a.sq.h + (size_t)at.q0 * a.sq.t;
  const uint16_t* gh = a.dout + (size_t)hk * a.group * a.so.h + (size_t)at.q0 * a.so.t;
  const float* lh = a.lse2 + (size_t)hk * a.Tq * a.group + (size_t)at.q0 * a.group;
  const float* dh = a.delta + (size_t)hk * a.Tq * a.group + (size_t)at.q0 * a.group;
  // the rows that read a key: from this one on (causal)
  auto from_of = [&](int j) { return a.causal ? max(0, j - past) * a.group : 0; };
  const int from = from_of(key), w_from = from_of(key0 + 32 * w), w_last = from_of(key0 + 32 * w + 31);
  int t_begin = from_of(key0) / kTileTokens, t_end = max(t_begin, (nr + kTileTokens - 1) / kTileTokens);
  const bool parts = PARTS && t_end - t_begin > a.k_chunk;
  if (PARTS) {
    t_begin += (int)blockIdx.y * a.k_chunk;
    if (t_begin >= t_end && blockIdx.y) return;
    t_end = min(t_end, t_begin + a.k_chunk);
  }
  auto qbuf = [&](int t) { return lds_address(smem) + (t & 1) * 2 * SM::kTile; };
  // Step t: rows [64 t, + 64) of Q and dO and their lse log2(e) and D; rows past the end repeat the last one, see no_rows
  auto request = [&](int t) {
    constexpr int kRowsPerInstr = 1024 / (D * 2), kInstrs = kTileTokens / kRowsPerInstr / NW;
    const int ln = (int)lane_again(), r0 = t * kTileTokens, valid = min(kTileTokens, nr - r0);
    const int2 q0 = query_of(a, r0);
    const int row_w = w * kRowsPerInstr + ln / SL::kChunks;
    const unsigned col = 16u * (unsigned)((ln % SL::kChunks) ^ SL::swz(row_w));
    const char *qb = (const char*)(qh + (size_t)q0.x * a.sq.t), *gb = (const char*)(gh + (size_t)q0.x * a.so.t);
#pragma unroll
    for (int i = 0; i < kInstrs; i++) {
      const int2 x = near_query_of(a, (unsigned)(q0.y + min(row_w + i * NW * kRowsPerInstr, valid - 1)));
      dma_lane16(qb, ((unsigned)x.x * (unsigned)a.sq.t + (unsigned)x.y * (unsigned)a.sq.h) * 2 + col, qbuf(t) + (i * NW + w) * 1024);
      dma_lane16(gb, ((unsigned)x.x * (unsigned)a.so.t + (unsigned)x.y * (unsigned)a.so.h) * 2 + col, qbuf(t) + SM::kTile + (i * NW + w) * 1024);
    }
    const unsigned so = 4u * (unsigned)min(ln, valid - 1);
    if (w == 0) dma_lane4(lh + r0, so, lds_address(stat + (t & 1) * 128));
    if (w == 1) dma_lane4(dh + r0, so, lds_address(stat + (t & 1) * 128 + 64));
  };
  // behind the arrival of step t: lse = +inf for rows past the end, their P is 0
  auto no_rows = [&](int t) {
    if (w == 0 && (t + 1) * kTileTokens > nr) {
      if (t * kTileTokens + lane >= nr) stat[(t & 1) * 128 + lane] = INFINITY;
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
  };
  if (t_begin < t_end) request(t_begin);
  bf16x8 kf[KS], vf[KS];
  {
    const uint16_t* src = a.k + (size_t)hk * a.skv.h + token * a.skv.t + 8 * g;
    const uint16_t* vsrc = a.v + (size_t)hk * a.skv.h + token * a.skv.t + 8 * g;
#pragma unroll
    for (int ks = 0; ks < KS; ks++) {
      kf[ks] = *reinterpret_cast<const bf16x8*>(src + 16 * ks);
      vf[ks] = *reinterpret_cast<const bf16x8*>(vsrc + 16 * ks);
    }
  }
  const float c1 = kLog2e * a.scale;
  f32x16 dk[ET], dv[ET];
#pragma unroll
  for (int et = 0; et < ET; et++)
#pragma unroll
    for (int e = 0; e < 16; e++) dk[et][e] = dv[et][e] = 0.f;
  const unsigned r_off = row_read_offset<D>(lane), t_lo = tr_read_offset<D>(lane, 0), t_hi = tr_read_offset<D>(lane, 1);
  wait_vmcnt<0>();
#pragma unroll
  for (int ks = 0; ks < KS; ks++) { settle(kf[ks]); settle(vf[ks]); }
  if (t_begin < t_end) no_rows(t_begin);
  phase_barrier();
  for (int t = t_begin; t < t_end; t++) {
    if (t + 1 < t_end) request(t + 1);
#pragma unroll
    for (int rh = 0; rh < 2; rh++) {
      const int r0 = t * kTileTokens + 32 * rh;
      if (r0 + 32 <= w_from || r0 >= nr) continue;
      const unsigned qa = qbuf(t) + 64 * D * rh, ga = qa + SM::kTile;
      const unsigned st = lds_address(stat + (t & 1) * 128 + 32 * rh + 4 * g);
      f32x16 s, dp;
      bf16x8 pf[2], df[2];
#pragma unroll
      for (int e = 0; e < 16; e++) s[e] = dp[e] = 0.f;
      // One stream of LDS reads, kAhead of them in flight: the rows of Q for S; four groups of a quarter of the rows of dO for dP and lse
      // of four rows, whose exponentials then run beside the products; D of the rows.
      constexpr int kGroup = KS / 4 + 1, kItems = KS + 4 * kGroup + 4, kAhead = 4, kSlots = kAhead + 1;
      u32x4 ring[kSlots];
      auto issue = [&](int n) {
        const int m = n - KS, v4 = m / kGroup;
        if (n < KS) ring[n % kSlots] = lds_read16_untracked<0>((qa + r_off) ^ (32u * n));
        else if (m >= 4 * kGroup) ring[n % kSlots] = lds_read16_untracked<0>(st + 256 + 32 * (m - 4 * kGroup));
        else if (m % kGroup == kGroup - 1) ring[n % kSlots] = lds_read16_untracked<0>(st + 32 * v4);
        else ring[n % kSlots] = lds_read16_untracked<0>((ga + r_off) ^ (32u * (v4 * (kGroup - 1) + m % kGroup)));
      };
      const bool edge = r0 < w_last;
#pragma unroll
      for (int n = 0; n < kAhead; n++) issue(n);
#pragma unroll
      for (int n = 0; n < kItems; n++) {
        if (n + kAhead < kItems) issue(n + kAhead);
        wait_lgkmcnt(n + kAhead < kItems ? kAhead : kItems - 1 - n);
        settle(ring[n % kSlots]);
        const int m = n - KS, v4 = m / kGroup;
        if (n < KS) {
          s = mfma_bf16(__builtin_bit_cast(bf16x8, ring[n % kSlots]), kf[n], s);
        } else if (m >= 4 * kGroup) {
          const int x = m - 4 * kGroup;
          const f32x4 d4 = __builtin_bit_cast(f32x4, ring[n % kSlots]);
#pragma unroll
          for (int r = 0; r < 4; r++) {
            const int e = 4 * x + r;
            pf[x / 2][e % 8] = (__bf16)s[e];
            df[x / 2][e % 8] = (__bf16)(s[e] * (dp[e] - d4[r]));
          }
          if (x % 2 == 1) {
            pin(pf[x / 2]);
            pin(df[x / 2]);
          }
        } else if (m % kGroup == kGroup - 1) {
          const f32x4 l4 = __builtin_bit_cast(f32x4, ring[n % kSlots]);
#pragma unroll
          for (int r = 0; r < 4; r++) {
            const int e = 4 * v4 + r;
            float p = fast_exp2(s[e] * c1 - l4[r]);
            if (edge) p = r0 + 8 * v4 + 4 * g + r >= from ? p : 0.f;
            settle(p);                                 // here, not where the compiler would gather them
            s[e] = p;
          }
        } else {
          dp = mfma_bf16(__builtin_bit_cast(bf16x8, ring[n % kSlots]), vf[v4 * (kGroup - 1) + m % kGroup], dp);
        }
      }
      contract32<D>(dv, pf, ga + t_lo, ga + t_hi);
      contract32<D>(dk, df, qa + t_lo, qa + t_hi);
    }
    wait_vmcnt<0>();                                   // the next step's rows have landed ...
    if (t + 1 < t_end) no_rows(t + 1);
    phase_barrier();                                   // ... for everyone; this step's tiles are free
  }
  if (parts) {
    if (key >= nk) return;
    const size_t part = ((size_t)blockIdx.y * a.Tk + token) * a.Hkv + hk;
    store_part<D>(dk, a.part_kv + part * D, g);
    store_part<D>(dv, a.part_kv + ((size_t)a.k_parts * a.Tk * a.Hkv + part) * D, g);
    return;
  }
  uint16_t* os = reinterpret_cast<uint16_t*>(smem) + w * 32 * SM::kLd;
  auto to = [&](uint16_t* p) {
    return [=](int r) -> uint16_t* {
      return key0 + 32 * w + r < nk ? p + (size_t)hk * a.skv.h + (size_t)(at.k0 + key0 + 32 * w + r) * a.skv.t : nullptr;
    };
  };
  store_rows<D>(dk, a.scale, os, lane, to(a.dk));
  store_rows<D>(dv, 1.f, os, lane, to(a.dv));
}

// Sums of the parts, four channels a thread: dQ (rows of all key heads), dK and dV.
template <int D>
__global__ __launch_bounds__(256) void packed_sum_q_kernel(PackedArgs a) {
  const long long idx = (long long)blockIdx.x * 256 + threadIdx.x, row = idx / (D / 4), rows = (long long)a.Tq * a.H;
  const int c = (int)(idx % (D / 4)) * 4;
  if (row >= rows) return;
  const int hk = (int)(row / ((long long)a.Tq * a.group));
  const int2 x = query_of(a, (int)(row - (long long)hk * a.Tq * a.group));
  if (x.x < a.q_start[0] || x.x >= a.q_start[a.S]) return;       // of no sequence
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int i = 0; i < a.q_parts; i++) sum += *reinterpret_cast<const f32x4*>(a.part_o + (i * rows + row) * D + c);
  bf16x4 r;
#pragma unroll
  for (int e = 0; e < 4; e++) r[e] = (__bf16)(a.scale * sum[e]);
  *reinterpret_cast<bf16x4*>(a.dq + (size_t)(hk * a.group + x.y) * a.sq.h + (size_t)x.x * a.sq.t + c) = r;
}
template <int D>
__global__ __launch_bounds__(256) void packed_sum_kv_kernel(PackedArgs a) {
  const TileHead th = tile_head(blockIdx.x, a.Hkv);
  const TilePlace at = find_tile<true>(a, kKeyTile, th.tile, threadIdx.x % kWave);
  if (at.tile < 0) return;
  // as packed_dkv_kernel has it
  const int key0 = at.tile * kKeyTile, from = a.causal ? max(0, key0 - (at.nk - at.nq)) * a.group : 0, t_begin = from / kTileTokens;
  const int steps = (at.nq * a.group + kTileTokens - 1) / kTileTokens - t_begin;
  if (steps <= a.k_chunk) return;
  const int n = (steps + a.k_chunk - 1) / a.k_chunk;
  const size_t rows = (size_t)a.Tk * a.Hkv;
  const float* src = a.part_kv + (blockIdx.y ? a.k_parts * rows * D : 0);
  const float by = blockIdx.y ? 1.f : a.scale;
  uint16_t* dst = (blockIdx.y ? a.dv : a.dk) + (size_t)th.head * a.skv.h;
  for (int idx = threadIdx.x + 256 * blockIdx.z; idx < min(kKeyTile, at.nk - key0) * (D / 4); idx += 256 * gridDim.z) {
    const int token = at.k0 + key0 + idx / (D / 4), c = idx % (D / 4) * 4;
    const float* p = src + ((size_t)token * a.Hkv + th.head) * D + c;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < n; i++) sum += *reinterpret_cast<const f32x4*>(p + i * rows * D);
    bf16x4 r;
#pragma unroll
    for (int e = 0; e < 4; e++) r[e] = (__bf16)(by * sum[e]);
    *reinterpret_cast<bf16x4*>(dst + (size_t)token * a.skv.t + c) = r;
  }
}

template <int D> static hipError_t launch_bwd(const PackedArgs& a, hipStream_t stream) {
  constexpr int smem = PackedBwdSmem<D>::kBytes;
  static OncePerDevice once[4];
  const void* kernels[4] = {(const void*)packed_dq_kernel<D, false>, (const void*)packed_dq_kernel<D, true>,
                            (const void*)packed_dkv_kernel<D, false>, (const void*)packed_dkv_kernel<D, true>};
  const long long q_tiles = most_tiles((long long)a.Tq * a.group, a.S, kRowTile) * a.Hkv, k_tiles = most_tiles(a.Tk, a.S, kKeyTile) * a.Hkv;
  const int q = a.q_parts > 1, k = a.k_parts > 1;
  if (hipError_t e = allow_dynamic_lds(once[q], kernels[q], smem); e != hipSuccess) return e;
  if (hipError_t e = allow_dynamic_lds(once[2 + k], kernels[2 + k], smem); e != hipSuccess) return e;
  if (q_tiles) {
    if (q) packed_dq_kernel<D, true><<<dim3((unsigned)q_tiles, a.q_parts), 256, smem, stream>>>(a);
    else packed_dq_kernel<D, false><<<(unsigned)q_tiles, 256, smem, stream>>>(a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (q) {
      packed_sum_q_kernel<D><<<(unsigned)(((long long)a.Tq * a.H * (D / 4) + 255) / 256), 256, 0, stream>>>(a);
      if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
  }
  if (k_tiles) {
    if (k) packed_dkv_kernel<D, true><<<dim3((unsigned)k_tiles, a.k_parts), 256, smem, stream>>>(a);
    else packed_dkv_kernel<D, false><<<(unsigned)k_tiles, 256, smem, stream>>>(a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (k) packed_sum_kv_kernel<D><<<dim3((unsigned)k_tiles, 2, 4), 256, 0, stream>>>(a);
  }
  return hipGetLastError();
}
hipError_t launch_packed_bwd(const PackedArgs& a, hipStream_t stream) { return a.d == 128 ? launch_bwd<128>(a, stream) : launch_bwd<64>(a, stream); }

}  // namespace sla2
