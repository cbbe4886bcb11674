// Forward pass of attention over packed sequences: out = softmax(scale Q K^T) V, lse, with grouped heads and a causal mask.
//
// One workgroup = 4 waves = 128 rows of one key head and sequence (packed.h); a wave has 32 of them, one on lanes l and l + 32.  One
// pass over the keys, 64 at a time, with the running maximum and sum of the softmax: S^T = K Q^T (keys x rows), so that a lane holds
// scores of one row, P^T goes back into O^T += V^T P^T as it lies in the registers, and a row's maximum and sum are its lane's own and
// one exchange with the other half of the wave.  K and V tiles go from memory into LDS past the registers: V into one of two buffers,
// a tile ahead, K into its one buffer behind the scores.  Two workgroups (d = 64: four) are on a CU, as many as their registers allow, and one's
// products run beside another's exponentials, first reads and results.
//
// Bound by the vector unit beside the matrix cores: 32 keys x 32 rows take 512 cycles of products (d = 128) and some 350 of maximum,
// exponential, sum and rounding, which only overlap as far as two waves of a SIMD happen to be in different phases (busy 45 % and 48 % of the cycles).
// Causal, 40 heads on 8, sequences of 4,096, 2,777, 1,021, 1 and 297: 280 us for 262 GFLOP = 0.94 PFLOP/s; 12 heads of 2 x 32,760
// queries on 512 and 131 keys: 200 us for 129 GFLOP and 410 MB, 11 steps a tile between first reads and results that nothing of the
// same tile covers.
#include "packed.h"

namespace sla2 {

// S^T = K Q^T of 64 keys at `ka` (with row_read_offset) and a wave's 32 rows, two 32-key halves; reads run two steps ahead
template <int D>
__device__ __forceinline__ void packed_scores(unsigned ka, const bf16x8 (&qf)[D / 16], f32x16 (&sacc)[2]) {
  constexpr int KS = D / 16, KA = 2;
  u32x4 kr[KA + 1][2];
#pragma unroll
  for (int ks = 0; ks < KA; ks++) {
    kr[ks][0] = lds_read16_untracked<0>(ka ^ (32u * ks));
    kr[ks][1] = lds_read16_untracked<32 * D * 2>(ka ^ (32u * ks));
  }
#pragma unroll
  for (int mt = 0; mt < 2; mt++)
#pragma unroll
    for (int e = 0; e < 16; e++) sacc[mt][e] = 0.f;
#pragma unroll
  for (int ks = 0; ks < KS; ks++) {
    if (ks + KA < KS) {
      kr[(ks + KA) % (KA + 1)][0] = lds_read16_untracked<0>(ka ^ (32u * (ks + KA)));
      kr[(ks + KA) % (KA + 1)][1] = lds_read16_untracked<32 * D * 2>(ka ^ (32u * (ks + KA)));
    }
    const int ahead = KS - 1 - ks < KA ? KS - 1 - ks : KA;
#pragma unroll
    for (int mt = 0; mt < 2; mt++) {
      wait_lgkmcnt(2 * ahead + 1 - mt);
      settle(kr[ks % (KA + 1)][mt]);
      sacc[mt] = mfma_bf16(__builtin_bit_cast(bf16x8, kr[ks % (KA + 1)][mt]), qf[ks], sacc[mt]);
    }
  }
}

// What a wave keeps of its rows: O^T, the reference m of the exponentials (log2) and their sum l
template <int D> struct RowSums {
  f32x16 o[D / 32];
  float m, l;
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int et = 0; et < D / 32; et++)
#pragma unroll
      for (int e = 0; e < 16; e++) o[et][e] = 0.f;
    m = kNoScore;
    l = 0.f;
  }
};
// .. and what 64 more keys with scores sacc bring to it; V at va (with tr_read_offset)
template <int D>
__device__ __forceinline__ void packed_absorb(f32x16 (&sacc)[2], float c1, RowSums<D>& r, unsigned va_lo, unsigned va_hi) {
  constexpr int ET = D / 32;
  bf16x8 pf[4];
  float mx = -INFINITY;
#pragma unroll
  for (int mt = 0; mt < 2; mt++)
#pragma unroll
    for (int e = 0; e < 16; e++) mx = fmaxf(mx, sacc[mt][e]);
  mx = swap_halves_max(mx) * c1;
  // the reference is kept while the row maximum stays within 2^8 of it (decided for the whole wave)
  const bool rescale = __builtin_amdgcn_ballot_w64(mx > r.m + 8.f) != 0;
  const float m_new = rescale ? fmaxf(r.m, mx) : r.m;
  float rs = 0.f;
#pragma unroll
  for (int mt = 0; mt < 2; mt++)
#pragma unroll
    for (int e = 0; e < 16; e += 2) {
      const float p0 = fast_exp2(sacc[mt][e] * c1 - m_new), p1 = fast_exp2(sacc[mt][e + 1] * c1 - m_new);
      rs += p0 + p1;
      pf[2 * mt + e / 8][e % 8] = (__bf16)p0;
      pf[2 * mt + e / 8][e % 8 + 1] = (__bf16)p1;
    }
  if (rescale) {
    const float corr = fast_exp2(r.m - m_new);         // 0 on the first step
    r.l *= corr;
    r.m = m_new;
#pragma unroll
    for (int et = 0; et < ET; et++)
#pragma unroll
      for (int e = 0; e < 16; e++) r.o[et][e] *= corr;
  }
  r.l += swap_halves_sum(rs);
  // O^T += V^T P^T: fragment (ks, et) = two transposing reads, kept three fragments ahead of the products
  constexpr int kAhead = 3, kFrags = (kTileTokens / 16) * ET;
  u32x2 vlo[kAhead + 1], vhi[kAhead + 1];
  auto issue = [&](int f) {
    vlo[f % (kAhead + 1)] = lds_read_tr_untracked_at<16 * D * 2>(va_lo ^ (64u * (f % ET)), f / ET);
    vhi[f % (kAhead + 1)] = lds_read_tr_untracked_at<16 * D * 2>(va_hi ^ (64u * (f % ET)), f / ET);
  };
#pragma unroll
  for (int f = 0; f < kAhead; f++) issue(f);
#pragma unroll
  for (int f = 0; f < kFrags; f++) {
    if (f + kAhead < kFrags) issue(f + kAhead);
    const int left = kFrags - 1 - f;
    wait_lgkmcnt(2 * (left < kAhead ? left : kAhead));
    u32x2 &lo = vlo[f % (kAhead + 1)], &hi = vhi[f % (kAhead + 1)];
    settle(lo);
    settle(hi);
    const u32x4 v4 = {lo[0], lo[1], hi[0], hi[1]};
    r.o[f % ET] = mfma_bf16(__builtin_bit_cast(bf16x8, v4), pf[f / ET], r.o[f % ET]);
  }
}
// scores of the keys from `mine` on (counted from the first of the 64) out of the softmax
__device__ __forceinline__ void packed_mask(f32x16 (&sacc)[2], int mine, int g) {
#pragma unroll
  for (int mt = 0; mt < 2; mt++)
#pragma unroll
    for (int e = 0; e < 16; e++)
      if (32 * mt + 8 * (e / 4) + e % 4 >= mine - 4 * g) sacc[mt][e] = -INFINITY;
}
// Q as B operand: lane <- Q[row][16 ks + 8 g + 0..7]; a row past the end repeats the last one
template <int D>
__device__ __forceinline__ void packed_load_q(const PackedArgs& a, const TilePlace& at, int hk, int row, int lane, bf16x8 (&qf)[D / 16]) {
  const int2 x = query_of(a, min(row, at.nq * a.group - 1));
  const uint16_t* src = a.q + (size_t)(hk * a.group + x.y) * a.sq.h + (size_t)(at.q0 + x.x) * a.sq.t + 8 * (lane / 32);
#pragma unroll
  for (int ks = 0; ks < D / 16; ks++) qf[ks] = *reinterpret_cast<const bf16x8*>(src + 16 * ks);
}
// a lane's row of the result, and its lse
template <int D>
__device__ __forceinline__ void packed_result(const PackedArgs& a, const TilePlace& at, int hk, int row, int lane, RowSums<D>& r) {
  const bool any = r.l != 0.f, there = row < at.nq * a.group;      // NaN is some
  if (!any) r.clear();
  const int2 x = query_of(a, min(row, at.nq * a.group - 1));
  const int h = hk * a.group + x.y, token = at.q0 + x.x;
  store_row<D>(r.o, any ? 1.f / r.l : 0.f, a.o + (size_t)h * a.so.h + (size_t)token * a.so.t, lane / 32, there);
  if (a.lse_out && lane < 32 && there) a.lse_out[(size_t)h * a.Tq + token] = any ? (r.m + log2f(r.l)) * (1.f / kLog2e) : -INFINITY;
}

// LDS: K, two of V.
template <int D> constexpr int kPackedSmem = 3 * PackedTile<D>::kTileBytes;

template <int D, bool PARTS>
__global__ __launch_bounds__(256, D == 128 ? 2 : PARTS ? 3 : 4) void packed_fwd_kernel(PackedArgs a) {
  constexpr int NW = 4, KS = D / 16, kTile = PackedTile<D>::kTileBytes;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const int lane = threadIdx.x % kWave;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const TileHead th = tile_head(blockIdx.x, a.Hkv);
  const int hk = th.head;
  TilePlace at = find_tile<false>(a, kRowTile, th.tile, lane);
  if (at.tile < 0) return;
  if (a.causal) at.tile = at.tiles - 1 - at.tile;      // the longest first
  const int nr = at.nq * a.group, nk = at.nk, row0 = at.tile * kRowTile, w_row = row0 + 32 * w;
  const uint16_t* kh = a.k + (size_t)hk * a.skv.h + (size_t)at.k0 * a.skv.t;
  const uint16_t* vh = a.v + (size_t)hk * a.skv.h + (size_t)at.k0 * a.skv.t;
  const int past = nk - at.nq;                         // query i reads the keys below i + past + 1 (causal), all otherwise
  const int mine = a.causal ? min(nk, query_of(a, min(w_row + lane % 32, nr - 1)).x + past + 1) : nk;
  // the keys that the tile, and this wave, have to do with: below ..; and those that all rows of the wave read
  const int keys = a.causal ? min(nk, max(0, query_of(a, min(row0 + kRowTile, nr) - 1).x + past + 1)) : nk;
  const int w_keys = w_row >= nr ? 0 : __builtin_amdgcn_readlane(mine, 31), w_full = __builtin_amdgcn_readfirstlane(mine);
  int t_begin = 0, t_end = (keys + kTileTokens - 1) / kTileTokens;
  if (PARTS) {
    const int n = t_end;
    t_begin = (int)((long long)n * blockIdx.y / a.q_parts);
    t_end = (int)((long long)n * (blockIdx.y + 1) / a.q_parts);
  }
  const unsigned kbuf = lds_address(smem);
  auto vbuf = [&](int t) { return kbuf + (1 + (t & 1)) * kTile; };
  const unsigned lane_off = tile_lane_off<D, NW, PackedTile<D>>(a.skv.t, w, lane);
  auto dma = [&](const uint16_t* src, int t, unsigned to) { packed_dma<D, NW>(src, a.skv.t, t * kTileTokens, nk, to, w, lane_off); };
  if (t_begin < t_end) {
    dma(kh, t_begin, kbuf);
    dma(vh, t_begin, vbuf(t_begin));
  }
  bf16x8 qf[KS];
  packed_load_q<D>(a, at, hk, w_row + lane % 32, lane, qf);
  RowSums<D> sums;
  sums.clear();
  const float c1 = kLog2e * a.scale;
  const unsigned k_off = row_read_offset<D>(lane), v_lo = tr_read_offset<D>(lane, 0), v_hi = tr_read_offset<D>(lane, 1);
  wait_vmcnt<0>();
#pragma unroll
  for (int ks = 0; ks < KS; ks++) settle(qf[ks]);
  phase_barrier();
  for (int t = t_begin; t < t_end; t++) {
    if (t + 1 < t_end) dma(vh, t + 1, vbuf(t + 1));
    const int t0 = t * kTileTokens;
    const bool work = t0 < w_keys;
    f32x16 sacc[2];
    if (work) packed_scores<D>(kbuf + k_off, qf, sacc);
    phase_barrier();                                   // K has been read
    if (t + 1 < t_end) dma(kh, t + 1, kbuf);
    if (work) {
      if (t0 + kTileTokens > w_full) packed_mask(sacc, mine - t0, lane / 32);
      packed_absorb<D>(sacc, c1, sums, vbuf(t) + v_lo, vbuf(t) + v_hi);
    }
    wait_vmcnt<0>();                                   // the next step's K and V have landed, for everyone behind the barrier
    phase_barrier();
  }
  // from here on the lane's place is made again: it is not kept through the loop
  const int ln = (int)lane_again(), row = w_row + ln % 32;
  if (PARTS) {
    if (row >= nr) return;
    const size_t row_at = (size_t)blockIdx.y * a.Tq * a.H + (size_t)hk * a.Tq * a.group + (size_t)at.q0 * a.group + row;   // among the rows of all key heads
    store_part<D>(sums.o, a.part_o + row_at * D, ln / 32);
    if (ln < 32) *reinterpret_cast<float2*>(a.part_ml + 2 * row_at) = make_float2(sums.m, sums.l);
    return;
  }
  packed_result<D>(a, at, hk, row, ln, sums);
}

// The parts of one row: their O, weighted with 2^(m - the largest m), over their l, weighted alike.  A wave a row.
template <int D>
__global__ __launch_bounds__(256) void packed_join_kernel(PackedArgs a) {
  constexpr int E = D / kWave;
  const int lane = threadIdx.x % kWave;
  const long long row = (long long)blockIdx.x * 4 + threadIdx.x / kWave, rows = (long long)a.Tq * a.H;
  if (row >= rows) return;
  const int hk = (int)(row / ((long long)a.Tq * a.group));
  const int2 x = query_of(a, (int)(row - (long long)hk * a.Tq * a.group));       // x.x: token
  if (x.x < a.q_start[0] || x.x >= a.q_start[a.S]) return;                       // of no sequence
  const int h = hk * a.group + x.y;
  float m = -INFINITY;
  for (int i = 0; i < a.q_parts; i++) m = fmaxf(m, a.part_ml[2 * (i * rows + row)]);
  float l = 0.f, o[E] = {};
  for (int i = 0; i < a.q_parts; i++) {
    const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + 2 * (i * rows + row));
    const float by = fast_exp2(ml.x - m);
    l += by * ml.y;
#pragma unroll
    for (int e = 0; e < E; e++) o[e] += by * a.part_o[(i * rows + row) * D + E * lane + e];
  }
  const bool any = l != 0.f;
#pragma unroll
  for (int e = 0; e < E; e++)
    a.o[(size_t)h * a.so.h + (size_t)x.x * a.so.t + E * lane + e] = __builtin_bit_cast(uint16_t, (__bf16)(any ? o[e] / l : 0.f));
  if (a.lse_out && lane == 0) a.lse_out[(size_t)h * a.Tq + x.x] = any ? (m + log2f(l)) * (1.f / kLog2e) : -INFINITY;
}

// Parts of a tile of rows, where the tiles leave places for them (two workgroups a CU): as many as take the least time, by what was measured
// of each: a step 1.1 us (backward 1.5) for a workgroup on its own, the joining 6 us and 4 TB/s of parts written and read.  Not known here
// are the lengths; the longest sequence is taken to have twice its share of the keys.
// Parts of a tile of keys: so that no workgroup has much more than its share of all steps, which with a causal mask or sequences of
// different lengths the first tiles have.
// Backward with parts and without: 27,724 queries of 8 heads on 585 keys of one 270 us, 6.8 ms; 12 heads of 32,760 on 512 388, 1,157; causal, 40
// heads on 8, 8,192 tokens 826, 1,009; d = 64, 17 and 26 queries on 4,789 and 145 keys 32, 83.
constexpr long long kPartBytes = 1ll << 30;
void plan_packed(PackedArgs* a, bool backward) {
  a->q_parts = a->k_parts = 1;
  const long long rows = (long long)a->Tq * a->group, places = kPlaces;
  const long long q_tiles = most_tiles(rows, a->S, kRowTile) * a->Hkv, k_tiles = most_tiles(a->Tk, a->S, kKeyTile) * a->Hkv;
  const long long longest = a->S == 1 ? a->Tk : a->S == 2 ? a->Tk * 3ll / 4 : 2ll * a->Tk / a->S, steps = (longest + kTileTokens - 1) / kTileTokens;
  if (q_tiles && q_tiles <= places && steps && (!backward || k_tiles < kMostOfKeys)) {
    const double step = backward ? 1.5 : 1.1, bytes = (double)a->Tq * a->H * a->d * 8;
    double best = steps * step;
    for (int n = 2; n <= 64 && (n - 1) * q_tiles < 2 * places && n * 4 <= steps; n++) {
      const long long rounds = (n * q_tiles + places - 1) / places;      // a causal mask halves what they have on average
      const double time = (double)((steps + n - 1) / n) * (a->causal ? (rounds + 1) / 2.0 : (double)rounds) * step + 6 + n * bytes / 4e6;
      if (time < best) {
        best = time;
        a->q_parts = n;
      }
    }
  }
  if (!backward || !k_tiles || !rows) return;
  // Steps of 64 rows of all tiles of keys, were the sequences alike and their last tiles half full, over the places, and a little more,
  // so that the last round is not a few workgroups; at most 128 parts of the longest sequence that there can be, and kPartBytes of them
  // (where two parts take more, there are tiles for several rounds).
  const long long row_steps = ((a->Tq + 15ll) / 16 * a->group + 3) / 4, tiles = (a->Tk + (a->S - 1) * (kKeyTile / 2ll) + kKeyTile - 1) / kKeyTile;
  const long long all = tiles * a->Hkv * ((row_steps + a->S - 1) / a->S) / (a->causal ? 2 : 1);
  long long chunk = all / places + all / (places * 12) + 1;
  // A part has some 5 us of its own and is written and read: 8 steps at least for one sequence (16 heads of 6,410 queries on 339 keys 119 us,
  // with 16 127), 16 where the longest is not known (five of 171 to 2,991: 146, with 8 148 and with 5 163).
  const long long least = a->S == 1 ? 8 : 16;
  if (chunk < least) chunk = least;
  if (chunk < (row_steps + 127) / 128) chunk = (row_steps + 127) / 128;
  const long long part = 2ll * a->Tk * a->Hkv * a->d * 4, most = part > kPartBytes ? 1 : kPartBytes / part;    // bytes of one; as many as may be
  if (chunk < (row_steps + most - 1) / most) chunk = (row_steps + most - 1) / most;
  const long long places_for = k_tiles < kMostOfKeys ? kMostOfKeys / k_tiles : 1;
  if (chunk < (row_steps + places_for - 1) / places_for) chunk = (row_steps + places_for - 1) / places_for;
  a->k_chunk = (int)chunk;
  a->k_parts = (int)((row_steps + chunk - 1) / chunk);
  // rows dealt to several workgroups with more steps each than those of the keys have: 40 us for 54 (tens of queries on 12,832 keys), otherwise 67 for 76
  // (d = 64, 8 heads on 1, 298 and 1,984 tokens)
  const long long usual = 2 * row_steps / a->S;
  a->rows_first = a->q_parts > 1 && steps / a->q_parts >= (usual < chunk ? usual : chunk);
}

template <int D> static hipError_t launch_fwd(const PackedArgs& a, hipStream_t stream) {
  const long long grid = most_tiles((long long)a.Tq * a.group, a.S, kRowTile) * a.Hkv;
  if (!grid) return hipSuccess;
  if (a.q_parts == 1) {
    packed_fwd_kernel<D, false><<<(unsigned)grid, 256, kPackedSmem<D>, stream>>>(a);
    return hipGetLastError();
  }
  packed_fwd_kernel<D, true><<<dim3((unsigned)grid, a.q_parts), 256, kPackedSmem<D>, stream>>>(a);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  packed_join_kernel<D><<<(unsigned)(((long long)a.Tq * a.H + 3) / 4), 256, 0, stream>>>(a);
  return hipGetLastError();
}
hipError_t launch_packed_fwd(const PackedArgs& a, hipStream_t stream) { return a.d == 128 ? launch_fwd<128>(a, stream) : launch_fwd<64>(a, stream); }

}  // namespace sla2
