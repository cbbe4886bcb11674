// Backward pass of attention over packed sequences.  With P = exp(scale Q K^T - lse) and D = rowsum(dO . O):
//   dV = P^T dO,   dS = P . (dO V^T - D),   dQ = scale dS K,   dK = scale dS^T Q.
//
// Two sides, so that every sum has one owner and a fixed order: a workgroup for each tile of rows (dQ), one for each tile of keys (dK
// and dV, over the rows of all heads of the group).  Both form P and dO V^T themselves: 7 products in all for 5 that are needed, where
// a sum of dQ over workgroups would take a d-wide row of fp32 written and read back for each tile of keys.
//
// Where the tiles of rows fill the GPU each side is a launch, and the rows' one, which comes first, forms D for the keys'.  Where they do not,
// a small kernel forms D and both sides are in one launch; tiles of either side may then be dealt to several workgroups (tiles of keys in
// both forms), whose sums one more kernel for each side joins.
//
// On both a wave asks LDS for the operands of all products of 32 rows (keys) in one stream, some reads ahead of the products, and the
// exponentials run beside the products of dP.  Causal, 40 heads on 8, 8,192 tokens in sequences of 4,096, 2,048, 1,026, 1,021 and 1
// (118 GFLOP a product): rows 345 us = 1.0 PFLOP/s, keys 475 us = 1.0, sums of parts 37.  Bound by the matrix cores' and the vector
// unit's work one behind the other (49 to 53 and 32 to 41 % busy; two waves a SIMD, their registers full) and, on the key side, by moving Q and
// dO for every tile of keys (10 % of the two together without it).  d = 64, causal, 48 heads on 3, 1,767 tokens: 130 us, 142 with a
// stream for each product.  Not faster: one wave a SIMD with 64 keys, half the reads of LDS (results of products in the second half of the
// register file, copied out for every exponential: 1,001 us for 880), transfers spread between the products (904 for 834: spills).
#include "packed.h"

namespace sla2 {

template <int D> struct PackedBwdSmem {
  static constexpr int kTile = PackedTile<D>::kTileBytes;
  static constexpr int kStatOff = 4 * kTile;                   // float [2][2][64]: lse log2(e) and D of a step's rows (key side)
  static constexpr int kBytes = kStatOff + 4 * 64 * 4;
};

__device__ __forceinline__ void pin(bf16x8& f) {       // converted here: eight registers less than the fp32 values
  u32x4 u = __builtin_bit_cast(u32x4, f);
  settle(u);
  f = __builtin_bit_cast(bf16x8, u);
}

__device__ __forceinline__ long long kept(long long x) {   // a scalar that is held in registers and not worked out where it is used
  asm("" : "+s"(x));
  return x;
}

// 16 bytes of a step's row quantities, 32 bytes apart: lse at n = 0 .. 3 and D, 256 bytes on, at 4 .. 7
__device__ __forceinline__ u32x4 stat_read(unsigned base, int n) {
  switch (n) {
    case 0: return lds_read16_untracked<0>(base);
    case 1: return lds_read16_untracked<32>(base);
    case 2: return lds_read16_untracked<64>(base);
    case 3: return lds_read16_untracked<96>(base);
    case 4: return lds_read16_untracked<256>(base);
    case 5: return lds_read16_untracked<288>(base);
    case 6: return lds_read16_untracked<320>(base);
    default: return lds_read16_untracked<352>(base);
  }
}

// D and dQ of 128 rows: S^T = K Q^T and dP^T = V dO^T (keys x rows), dQ^T += K^T dS^T, as in the forward pass with K in the place of V.
template <int D, bool PARTS>
__device__ __forceinline__ void packed_dq(const PackedArgs& a, int bx, int by) {
  constexpr int NW = 4, KS = D / 16, ET = D / 32;
  typedef PackedBwdSmem<D> SM;
  typedef PackedTile<D> SL;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid % kWave, g = lane / 32;
  const int w = __builtin_amdgcn_readfirstlane(tid / kWave);
  const TileHead th = tile_head(bx, a.Hkv);
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
    t_begin = (int)((long long)n * by / a.q_parts);
    t_end = (int)((long long)n * (by + 1) / a.q_parts);
  }
  auto kbuf = [&](int t) { return lds_address(smem) + (t & 1) * 2 * SM::kTile; };
  const unsigned lane_off = tile_lane_off<D, NW, SL>(a.skv.t, w, lane);
  auto dma = [&](int t) {
    packed_dma<D, NW>(kh, a.skv.t, t * kTileTokens, nk, kbuf(t), w, lane_off);
    packed_dma<D, NW>(vh, a.skv.t, t * kTileTokens, nk, kbuf(t) + SM::kTile, w, lane_off);
  };
  if (t_begin < t_end) dma(t_begin);
  bf16x8 qf[KS], gf[KS];
  float delta = 0.f;
  const int h = hk * a.group + my.y, token = at.q0 + my.x;
  {
    const uint16_t* src = a.q + (size_t)h * a.sq.h + (size_t)token * a.sq.t + 8 * g;
    const uint16_t* gsrc = a.dout + (size_t)h * a.sg.h + (size_t)token * a.sg.t + 8 * g;
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
  if (!PARTS && row < nr && g == 0) {                  // PARTS: packed_stats_kernel has them
    const size_t st = stat_first(a, hk, at.s, at.q0) + stat_at(a, my.x, my.y);
    a.delta[st] = delta;
    a.lse2[st] = l2;
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
        // one stream of LDS reads, kAhead items of it in flight: K for S, V for dP, K again, transposed, for dQ
        constexpr int kItems = 2 * KS + 2 * ET, kAhead = 6, kSlots = kAhead + 1;
        u32x4 ring[kSlots];
        u32x2 lo[kSlots], hi[kSlots];
        auto issue = [&](int n) {
          const unsigned x = (ka + k_off) ^ (32u * (n % KS));
          if (n < KS) ring[n % kSlots] = lds_read16_untracked<0>(x);
          else if (n < 2 * KS) ring[n % kSlots] = lds_read16_untracked<SM::kTile>(x);
          else {
            const int f = n - 2 * KS;
            const unsigned at_lo = (ka + t_lo) ^ (64u * (f % ET)), at_hi = (ka + t_hi) ^ (64u * (f % ET));
            lo[n % kSlots] = f < ET ? lds_read_tr_untracked<0>(at_lo) : lds_read_tr_untracked<32 * D>(at_lo);
            hi[n % kSlots] = f < ET ? lds_read_tr_untracked<0>(at_hi) : lds_read_tr_untracked<32 * D>(at_hi);
          }
        };
#pragma unroll
        for (int n = 0; n < kAhead; n++) issue(n);
        unrolled<kItems>([&](auto at_n) {
          constexpr int n = decltype(at_n)::value, f = n - 2 * KS;
          if (n + kAhead < kItems) issue(n + kAhead);
          int behind = 0;                              // reads asked for behind this item's
#pragma unroll
          for (int y = 1; y <= kAhead; y++) behind += n + y < kItems ? (n + y < 2 * KS ? 1 : 2) : 0;
          wait_lgkmcnt(behind);
          if constexpr (n < 2 * KS) {
            settle(ring[n % kSlots]);
            const bf16x8 x = __builtin_bit_cast(bf16x8, ring[n % kSlots]);
            if constexpr (n < KS) {
              s = mfma_bf16(x, qf[n], s);
            } else {
              dp = mfma_bf16(x, gf[n - KS], dp);
              constexpr int kStep = KS / 4;            // behind every quarter of the products of dP four exponentials
              if constexpr ((n - KS) % kStep == kStep - 1) {
                constexpr int v4 = (n - KS) / kStep;
#pragma unroll
                for (int r = 0; r < 4; r++) {
                  float p = fast_exp2(s[4 * v4 + r] * c1 - l2);
                  settle(p);
                  s[4 * v4 + r] = p;
                }
              }
            }
            if constexpr (n == 2 * KS - 1) {
              if (edge) {
#pragma unroll
                for (int e = 0; e < 16; e++)
                  if (t0 + 32 * mt + 8 * (e / 4) + 4 * g + e % 4 >= mine) s[e] = 0.f;
              }
#pragma unroll
              for (int e = 0; e < 16; e++) df[e / 8][e % 8] = (__bf16)(s[e] * (dp[e] - delta));
              pin(df[0]);
              pin(df[1]);
            }
          } else {
            settle(lo[n % kSlots]);
            settle(hi[n % kSlots]);
            const u32x4 u = {lo[n % kSlots][0], lo[n % kSlots][1], hi[n % kSlots][0], hi[n % kSlots][1]};
            acc[f % ET] = mfma_bf16(__builtin_bit_cast(bf16x8, u), df[f / ET], acc[f % ET]);
          }
        });
      }
    }
    wait_vmcnt<0>();
    phase_barrier();
  }
  const int ln = (int)lane_again(), last_row = w_row + ln % 32;    // what is made of the lane's place is not kept through the loop
  if (PARTS && a.q_parts > 1) {
    const size_t part = (size_t)by * a.Tq * a.H + (size_t)hk * a.Tq * a.group + (size_t)at.q0 * a.group + last_row;   // among the rows of all key heads
    if (last_row < nr) store_part<D>(acc, a.part_o + part * D, ln / 32);
    return;
  }
  const int2 x = query_of(a, min(last_row, nr - 1));
  store_row<D>(acc, a.scale, a.dq + (size_t)(hk * a.group + x.y) * a.sq.h + (size_t)(at.q0 + x.x) * a.sq.t, ln / 32, last_row < nr);
}

// dK and dV of 128 keys: S = Q K^T and dP = dO V^T (rows x keys), a key on lanes l and l + 32 with its row of K and V in registers;
// dV^T += dO^T P and dK^T += Q^T dS, 64 rows a step, which arrive in LDS one step ahead.
template <int D, bool PARTS>
__device__ __forceinline__ void packed_dkv(const PackedArgs& a, int bx, int by) {
  constexpr int NW = 4, KS = D / 16, ET = D / 32;
  typedef PackedBwdSmem<D> SM;
  typedef PackedTile<D> SL;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  float* stat = reinterpret_cast<float*>(smem + SM::kStatOff);
  const int lane = threadIdx.x % kWave;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const TileHead th = tile_head(bx, a.Hkv);
  const int hk = th.head;
  const TilePlace at = find_tile<true>(a, kKeyTile, th.tile, lane);
  if (at.tile < 0) return;
  const int nk = at.nk, nq = at.nq, past = nk - nq, key0 = at.tile * kKeyTile, w_key = key0 + 32 * w;
  // The rows in blocks of 16 queries of one head (packed.h), four blocks a step: within a block a transfer's addresses are a lane's place
  // beside a scalar.  A key is read by the queries from this one on (causal):
  auto from_of = [&](int j) { return a.causal ? max(0, j - past) : 0; };
  const int w_from = from_of(w_key), w_last = from_of(w_key + 31), q_blocks = (nq + kQueryBlock - 1) / kQueryBlock;
  int t_begin = from_of(key0) / kQueryBlock * a.group / 4, t_end = max(t_begin, (q_blocks * a.group + 3) / 4);
  bool parts = false;
  if (PARTS) {
    // chunks from the sequence's first row on, the same for all of its tiles: those at work at a time read the same rows
    const int first = t_begin / a.k_chunk, last = max(first, (t_end - 1) / a.k_chunk), part = by;
    if (part < first || part > last) return;
    parts = first < last;
    t_begin = max(t_begin, part * a.k_chunk);
    t_end = min(t_end, (part + 1) * a.k_chunk);
  }
  const size_t st0 = stat_first(a, hk, at.s, at.q0);
  // A block: its query block and head, and where it begins in Q and dO.  Counted along, not worked out: the scalar unit's multiplications
  // and divisions, 320 instructions a step, took a quarter of the kernel's time.
  struct Block {
    int q, h;
    const uint16_t *qp, *gp;
  };
  // How far a step of one block, and of four, goes on in the same queries and to later ones (elements; kept, not made again)
  const long long q_row = (long long)kQueryBlock * a.sq.t, g_row = (long long)kQueryBlock * a.sg.t;
  const int four_q = 4 / a.group, four_h = 4 % a.group;
  const long long q_one = a.sq.h, g_one = a.sg.h, q_wrap = kept(q_row - (a.group - 1) * a.sq.h), g_wrap = kept(g_row - (a.group - 1) * a.sg.h);
  const long long q_four = kept(four_q * q_row + four_h * a.sq.h), g_four = kept(four_q * g_row + four_h * a.sg.h);
  const long long q_four_wrap = kept(q_four + q_row - a.group * a.sq.h), g_four_wrap = kept(g_four + g_row - a.group * a.sg.h);
  auto next = [&](Block b) {
    const bool wrap = b.h + 1 == a.group;
    return Block{b.q + wrap, wrap ? 0 : b.h + 1, b.qp + (wrap ? q_wrap : q_one), b.gp + (wrap ? g_wrap : g_one)};
  };
  auto after4 = [&](Block b) {
    const bool wrap = b.h + four_h >= a.group;
    return Block{b.q + four_q + wrap, b.h + four_h - (wrap ? a.group : 0), b.qp + (wrap ? q_four_wrap : q_four), b.gp + (wrap ? g_four_wrap : g_four)};
  };
  // whether all queries of the four blocks from b on exist, told from the first one's: the fourth's are at most so many blocks further
  const int further = 1 + 2 / a.group, whole_below = nq / kQueryBlock - further;
  auto whole = [&](Block b) { return b.q < whole_below; };
  auto qbuf = [&](int t) { return lds_address(smem) + (t & 1) * 2 * SM::kTile; };
  // Step t, whose first block is b: the rows of four blocks of Q and dO and their lse log2(e) and D.  Queries past the end repeat the
  // last one, blocks past the end the one in front of them, see no_rows.
  auto request = [&](int t, Block b) {
    constexpr int kRows = 1024 / (D * 2), kInstrs = kTileTokens / kRows / NW;          // of a transfer; a wave's transfers
    const int ln = (int)lane_again(), row = w * kRows % kQueryBlock + ln / SL::kChunks;
    const unsigned col = 16u * (unsigned)((ln % SL::kChunks) ^ SL::swz(w * kRows + ln / SL::kChunks));
    const unsigned q_off = (unsigned)row * (unsigned)a.sq.t * 2 + col, g_off = (unsigned)row * (unsigned)a.sg.t * 2 + col;
    if (w < 2) dma_lane4((w == 0 ? a.lse2 : a.delta) + st0 + (size_t)t * kTileTokens, 4u * (unsigned)ln, lds_address(stat + (t & 1) * 128 + 64 * w));
    if (whole(b)) {
      if (kRows * NW > kQueryBlock && w * kRows >= kQueryBlock) b = next(b);
#pragma unroll
      for (int i = 0; i < kInstrs; i++) {
        dma_lane16(b.qp, q_off, qbuf(t) + (i * NW + w) * 1024);
        dma_lane16(b.gp, g_off, qbuf(t) + SM::kTile + (i * NW + w) * 1024);
        if (i + 1 < kInstrs) b = kRows * NW > kQueryBlock ? next(next(b)) : next(b);
      }
      return;
    }
    auto on = [&]() {
      const Block x = next(b);
      if (x.q < q_blocks) b = x;
    };
    if (kRows * NW > kQueryBlock && w * kRows >= kQueryBlock) on();                    // two blocks a transfer of all waves
#pragma unroll
    for (int i = 0; i < kInstrs; i++) {
      const int valid = nq - b.q * kQueryBlock;
      unsigned qo = q_off, go = g_off;
      if (valid < kQueryBlock) {
        const unsigned back = (unsigned)max(0, row - (valid - 1));
        qo -= back * (unsigned)a.sq.t * 2;
        go -= back * (unsigned)a.sg.t * 2;
      }
      dma_lane16(b.qp, qo, qbuf(t) + (i * NW + w) * 1024);
      dma_lane16(b.gp, go, qbuf(t) + SM::kTile + (i * NW + w) * 1024);
      on();
      if (kRows * NW > kQueryBlock) on();
    }
  };
  // Behind the arrival of step t, by the waves that asked for them: what was read for queries past the end has no meaning.  With
  // lse = +inf and D = 0 their P and dS are 0.
  auto no_rows = [&](int t, Block b) {
    if (w > 1 || whole(b)) return;
    const Block b1 = next(b), b2 = next(b1), b3 = next(b2);
    const int ln = (int)lane_again(), q = ln < 32 ? ln < 16 ? b.q : b1.q : ln < 48 ? b2.q : b3.q;
    if (q * kQueryBlock + ln % kQueryBlock >= nq) stat[(t & 1) * 128 + 64 * w + ln] = w == 0 ? INFINITY : 0.f;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  };
  Block cur{t_begin * 4 / a.group, t_begin * 4 % a.group, nullptr, nullptr};
  cur.qp = a.q + (size_t)(hk * a.group + cur.h) * a.sq.h + ((size_t)at.q0 + cur.q * kQueryBlock) * a.sq.t;
  cur.gp = a.dout + (size_t)(hk * a.group + cur.h) * a.sg.h + ((size_t)at.q0 + cur.q * kQueryBlock) * a.sg.t;
  if (t_begin < t_end) request(t_begin, cur);
  bf16x8 kf[KS], vf[KS];
  {
    const size_t token = (size_t)at.k0 + min(w_key + lane % 32, nk - 1);
    const uint16_t* src = a.k + (size_t)hk * a.skv.h + token * a.skv.t + 8 * (lane / 32);
    const uint16_t* vsrc = a.v + (size_t)hk * a.skv.h + token * a.skv.t + 8 * (lane / 32);
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
  if (t_begin < t_end) no_rows(t_begin, cur);
  phase_barrier();
  for (int t = t_begin; t < t_end; t++) {
    const Block following = after4(cur);
    if (t + 1 < t_end) request(t + 1, following);
#pragma unroll
    for (int rh = 0; rh < 2; rh++) {
      const Block b0 = rh ? next(next(cur)) : cur, b1 = next(b0);
      if (b0.q >= q_blocks || b1.q * kQueryBlock + kQueryBlock <= w_from) continue;
      const unsigned qa = qbuf(t) + 64 * D * rh, ra = qa + r_off;
      const unsigned st = lds_address(stat + (t & 1) * 128 + 32 * rh) + lane_again() / 32 * 16;
      f32x16 s, dp;
      bf16x8 pf[2], df[2];
#pragma unroll
      for (int e = 0; e < 16; e++) s[e] = dp[e] = 0.f;
      // One stream of LDS reads, kAhead items of it in flight: the rows of Q for S; four groups of a quarter of the rows of dO for dP and
      // lse of four rows, whose exponentials then run beside the products; dO for dV, behind the first of which D of the rows; Q for dK.
      constexpr int kGroup = KS / 4 + 1, kV = KS + 4 * kGroup, kK = kV + 4 + 2 * ET, kItems = kK + 2 * ET;
      constexpr int kAhead = D == 64 ? 6 : 2 /* the registers: with 3 they spill */, kSlots = kAhead + 1;
      u32x4 ring[kSlots];
      u32x2 lo[kSlots], hi[kSlots];
      auto is_d = [](int n) { return n > kV && n <= kV + 4; };
      auto fragment = [](int n) { return n >= kK ? n - kK : n == kV ? 0 : n - kV - 4; };           // of dO or Q, transposed
      auto reads = [&](int n) { return n < kV || is_d(n) ? 1 : 2; };
      auto issue = [&](int n) {
        const int m = n - KS, v4 = m / kGroup, f = fragment(n);
        if (n < KS) ring[n % kSlots] = lds_read16_untracked<0>(ra ^ (32u * n));
        else if (is_d(n)) ring[n % kSlots] = stat_read(st, 4 + n - kV - 1);
        else if (n >= kV) {
          const unsigned at_lo = (qa + t_lo) ^ (64u * (f % ET)), at_hi = (qa + t_hi) ^ (64u * (f % ET));
          if (n < kK) {
            lo[n % kSlots] = f < ET ? lds_read_tr_untracked<SM::kTile>(at_lo) : lds_read_tr_untracked<SM::kTile + 32 * D>(at_lo);
            hi[n % kSlots] = f < ET ? lds_read_tr_untracked<SM::kTile>(at_hi) : lds_read_tr_untracked<SM::kTile + 32 * D>(at_hi);
          } else {
            lo[n % kSlots] = f < ET ? lds_read_tr_untracked<0>(at_lo) : lds_read_tr_untracked<32 * D>(at_lo);
            hi[n % kSlots] = f < ET ? lds_read_tr_untracked<0>(at_hi) : lds_read_tr_untracked<32 * D>(at_hi);
          }
        }
        else if (m % kGroup == kGroup - 1) ring[n % kSlots] = stat_read(st, v4);
        else ring[n % kSlots] = lds_read16_untracked<SM::kTile>(ra ^ (32u * (v4 * (kGroup - 1) + m % kGroup)));
      };
#pragma unroll
      for (int n = 0; n < kAhead; n++) issue(n);
      unrolled<kItems>([&](auto at_n) {
        constexpr int n = decltype(at_n)::value, m = n - KS, v4 = m / kGroup;
        constexpr bool d_item = n > kV && n <= kV + 4;
        if (n + kAhead < kItems) issue(n + kAhead);
        int behind = 0;                                // reads asked for behind this item's
#pragma unroll
        for (int y = 1; y <= kAhead; y++) behind += n + y < kItems ? reads(n + y) : 0;
        wait_lgkmcnt(behind);
        if constexpr (n < kV || d_item) {
          settle(ring[n % kSlots]);
        } else {
          settle(lo[n % kSlots]);
          settle(hi[n % kSlots]);
        }
        if constexpr (n < KS) {
          s = mfma_bf16(__builtin_bit_cast(bf16x8, ring[n % kSlots]), kf[n], s);
          if (n == KS - 1 && b0.q * kQueryBlock < w_last) {            // some rows do not read some of the keys
            const int ln = (int)lane_again(), from = from_of(w_key + ln % 32) - 4 * (ln / 32);
#pragma unroll
            for (int e = 0; e < 16; e++)
              if ((e < 8 ? b0.q : b1.q) * kQueryBlock + e % 8 / 4 * 8 + e % 4 < from) s[e] = -INFINITY;
          }
        } else if constexpr (d_item) {
          constexpr int x = n - kV - 1;
          const f32x4 d4 = __builtin_bit_cast(f32x4, ring[n % kSlots]);
#pragma unroll
          for (int r = 0; r < 4; r++) df[x / 2][(4 * x + r) % 8] = (__bf16)(s[4 * x + r] * (dp[4 * x + r] - d4[r]));
          if (x % 2 == 1) pin(df[x / 2]);
        } else if constexpr (n >= kV) {
          constexpr int f = n >= kK ? n - kK : n == kV ? 0 : n - kV - 4;
          const u32x4 u = {lo[n % kSlots][0], lo[n % kSlots][1], hi[n % kSlots][0], hi[n % kSlots][1]};
          if constexpr (n < kK) dv[f % ET] = mfma_bf16(__builtin_bit_cast(bf16x8, u), pf[f / ET], dv[f % ET]);
          else dk[f % ET] = mfma_bf16(__builtin_bit_cast(bf16x8, u), df[f / ET], dk[f % ET]);
        } else if constexpr (m % kGroup == kGroup - 1) {
          const f32x4 l4 = __builtin_bit_cast(f32x4, ring[n % kSlots]);
#pragma unroll
          for (int r = 0; r < 4; r++) {
            float p = fast_exp2(s[4 * v4 + r] * c1 - l4[r]);
            settle(p);                                 // here, not where the compiler would gather them
            s[4 * v4 + r] = p;
            pf[v4 / 2][(4 * v4 + r) % 8] = (__bf16)p;
          }
          if (v4 % 2 == 1) pin(pf[v4 / 2]);
        } else {
          dp = mfma_bf16(__builtin_bit_cast(bf16x8, ring[n % kSlots]), vf[v4 * (kGroup - 1) + m % kGroup], dp);
        }
      });
    }
    wait_vmcnt<0>();                                   // the next step's rows have landed ...
    if (t + 1 < t_end) no_rows(t + 1, following);
    phase_barrier();                                   // ... for everyone; this step's tiles are free
    cur = following;
  }
  const int ln = (int)lane_again(), key = w_key + ln % 32, g = ln / 32;      // what is made of the lane's place is not kept through the loop
  if (parts) {
    if (key >= nk) return;
    const size_t part = ((size_t)by * a.Tk + at.k0 + key) * a.Hkv + hk;
    store_part<D>(dk, a.part_kv + part * D, g);
    store_part<D>(dv, a.part_kv + ((size_t)a.k_parts * a.Tk * a.Hkv + part) * D, g);
    return;
  }
  const size_t to = (size_t)hk * a.skv.h + (size_t)(at.k0 + key) * a.skv.t;
  store_row<D>(dk, a.scale, a.dk + to, g, key < nk);
  store_row<D>(dv, 1.f, a.dv + to, g, key < nk);
}

template <int D>
__global__ __launch_bounds__(256, 2) void packed_dq_kernel(PackedArgs a) {
  packed_dq<D, false>(a, blockIdx.x, 0);
}
template <int D, bool PARTS>
__global__ __launch_bounds__(256, 2) void packed_dkv_kernel(PackedArgs a) {
  packed_dkv<D, PARTS>(a, blockIdx.x, blockIdx.y);
}
// Both in one launch, where the tiles of rows do not fill the GPU: those whose workgroups take longer first (plan_packed).  Five heads of sequences
// of 171 to 2,991 tokens 128 us, one launch after the other 146; 5,966 and 4,062 296, 324; tens of queries of 16 heads on 12,832 keys 40, 48.  (Where
// the rows fill it, reading out and dout once more would cost what it saves.)
template <int D>
__global__ __launch_bounds__(256, 2) void packed_both_kernel(PackedArgs a, int k_tiles, int q_tiles) {
  const int keys = k_tiles * a.k_parts, rows = q_tiles * a.q_parts, n = blockIdx.x, rows_first = a.rows_first ? rows : 0;
  const int r = rows_first ? n : n - keys;               // the number among the rows' workgroups
  if (r >= 0 && r < rows) packed_dq<D, true>(a, r % q_tiles, r / q_tiles);
  else packed_dkv<D, true>(a, (n - rows_first) % k_tiles, (n - rows_first) / k_tiles);
}
// .. what the keys' side needs of every row before: D and lse log2(e), D / 8 lanes a row.
template <int D>
__global__ __launch_bounds__(256) void packed_stats_kernel(PackedArgs a) {
  constexpr int LANES = D / 8;
  const TileHead th = tile_head(blockIdx.x, a.Hkv);
  const TilePlace at = find_tile<false>(a, kRowTile, th.tile, threadIdx.x % kWave);
  if (at.tile < 0) return;
  const int row0 = at.tile * kRowTile + threadIdx.x / LANES, col = threadIdx.x % LANES * 8, nr = at.nq * a.group;
#pragma unroll
  for (int i = 0; i < kRowTile * LANES / 256; i++) {
    const int row = row0 + i * (256 / LANES);
    const int2 x = query_of(a, min(row, nr - 1));
    const int h = th.head * a.group + x.y, token = at.q0 + x.x;
    const bf16x8 o = *reinterpret_cast<const bf16x8*>(a.out + (size_t)h * a.so.h + (size_t)token * a.so.t + col);
    const bf16x8 g = *reinterpret_cast<const bf16x8*>(a.dout + (size_t)h * a.sg.h + (size_t)token * a.sg.t + col);
    float d = 0.f;
#pragma unroll
    for (int e = 0; e < 8; e++) d += (float)o[e] * (float)g[e];
#pragma unroll
    for (int by = 1; by < LANES; by *= 2) d += __shfl_xor(d, by);
    if (row < nr && col == 0) {
      const float lse = a.lse[(size_t)h * a.Tq + token];
      const size_t st = stat_first(a, th.head, at.s, at.q0) + stat_at(a, x.x, x.y);
      a.delta[st] = d;
      a.lse2[st] = lse == -INFINITY ? INFINITY : lse * kLog2e;
    }
  }
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
  const int key0 = at.tile * kKeyTile, from = a.causal ? max(0, key0 - (at.nk - at.nq)) : 0, t_begin = from / kQueryBlock * a.group / 4;
  const int t_end = max(t_begin, ((at.nq + kQueryBlock - 1) / kQueryBlock * a.group + 3) / 4);
  const int p0 = t_begin / a.k_chunk, p1 = max(p0, (t_end - 1) / a.k_chunk);
  if (p0 == p1) return;
  const size_t rows = (size_t)a.Tk * a.Hkv;
  const float* src = a.part_kv + (blockIdx.y ? a.k_parts * rows * D : 0);
  const float by = blockIdx.y ? 1.f : a.scale;
  uint16_t* dst = (blockIdx.y ? a.dv : a.dk) + (size_t)th.head * a.skv.h;
  for (int idx = threadIdx.x + 256 * blockIdx.z; idx < min(kKeyTile, at.nk - key0) * (D / 4); idx += 256 * gridDim.z) {
    const int token = at.k0 + key0 + idx / (D / 4), c = idx % (D / 4) * 4;
    const float* p = src + ((size_t)token * a.Hkv + th.head) * D + c;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int i = p0; i <= p1; i++) sum += *reinterpret_cast<const f32x4*>(p + i * rows * D);
    bf16x4 r;
#pragma unroll
    for (int e = 0; e < 4; e++) r[e] = (__bf16)(by * sum[e]);
    *reinterpret_cast<bf16x4*>(dst + (size_t)token * a.skv.t + c) = r;
  }
}

template <int D> static hipError_t launch_bwd(const PackedArgs& a, hipStream_t stream) {
  constexpr int smem = PackedBwdSmem<D>::kBytes;
  static OncePerDevice once[4];
  const void* kernels[4] = {(const void*)packed_dkv_kernel<D, false>, (const void*)packed_dkv_kernel<D, true>, (const void*)packed_dq_kernel<D>,
                            (const void*)packed_both_kernel<D>};
  const long long q_tiles = most_tiles((long long)a.Tq * a.group, a.S, kRowTile) * a.Hkv, k_tiles = most_tiles(a.Tk, a.S, kKeyTile) * a.Hkv;
  const int q = a.q_parts > 1, k = a.k_parts > 1;
  if (q_tiles && k_tiles && q_tiles <= kPlaces && k_tiles < kMostOfKeys) {       // so it is wherever rows have parts
    if (hipError_t e = allow_dynamic_lds(once[3], kernels[3], smem); e != hipSuccess) return e;
    packed_stats_kernel<D><<<(unsigned)q_tiles, 256, 0, stream>>>(a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    packed_both_kernel<D><<<(unsigned)(q_tiles * a.q_parts + k_tiles * a.k_parts), 256, smem, stream>>>(a, (int)k_tiles, (int)q_tiles);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  } else {
    if (hipError_t e = allow_dynamic_lds(once[2], kernels[2], smem); e != hipSuccess) return e;
    if (hipError_t e = allow_dynamic_lds(once[k], kernels[k], smem); e != hipSuccess) return e;
    if (q_tiles) {
      packed_dq_kernel<D><<<(unsigned)q_tiles, 256, smem, stream>>>(a);
      if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    if (k_tiles) {
      if (k) packed_dkv_kernel<D, true><<<dim3((unsigned)k_tiles, a.k_parts), 256, smem, stream>>>(a);
      else packed_dkv_kernel<D, false><<<(unsigned)k_tiles, 256, smem, stream>>>(a);
      if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
  }
  if (q_tiles && q) {
    packed_sum_q_kernel<D><<<(unsigned)(((long long)a.Tq * a.H * (D / 4) + 255) / 256), 256, 0, stream>>>(a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  if (k_tiles && k) packed_sum_kv_kernel<D><<<dim3((unsigned)k_tiles, 2, k_tiles < 256 ? D / 8 : 4), 256, 0, stream>>>(a);   // few tiles: one sum a thread
  return hipGetLastError();
}
hipError_t launch_packed_bwd(const PackedArgs& a, hipStream_t stream) { return a.d == 128 ? launch_bwd<128>(a, stream) : launch_bwd<64>(a, stream); }

}  // namespace sla2
