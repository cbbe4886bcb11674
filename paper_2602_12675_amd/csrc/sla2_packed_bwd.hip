// Backward pass of attention over packed sequences.  With P = exp(scale Q K^T - lse) and D = rowsum(dO . O):
//   dV = P^T dO,   dS = P . (dO V^T - D),   dQ = scale dS K,   dK = scale dS^T Q.
//
// Two kernels, so that every sum has one owner and a fixed order: one for each tile of queries (D and dQ), one for each tile of keys (dK
// and dV, over the queries of all heads of the group).  Both form P and dO V^T themselves: 7 products in all for 5 that are needed, where
// a sum of dQ over workgroups would take a d-wide row of fp32 written and read back for each tile of keys.
#include "packed.h"

namespace sla2 {

// D and dQ of 128 rows: S^T = K Q^T and dP^T = V dO^T (keys x rows), dQ^T += K^T dS^T, as in the forward pass with K in the place of V.
template <int D>
__global__ __launch_bounds__(256) void packed_dq_kernel(PackedArgs a) {
  constexpr int BQ = 128, NT = 256, KS = D / 16, ET = D / 32;
  typedef PaddedLayout<D> PL;
  __shared__ __attribute__((aligned(16))) uint16_t ks_[kTileTokens * PL::kRowElems], vs_[kTileTokens * PL::kRowElems];
  const int tid = threadIdx.x, lane = tid % kWave, w = tid / kWave, g = lane / 32;
  const int h = blockIdx.x % a.H;
  const TilePlace at = find_tile(a.q_start, a.S, a.Tq, BQ, blockIdx.x / a.H, lane);
  if (at.s < 0) return;
  const int2 qs = stretch_of(a.q_start, at.s, a.Tq), kx = stretch_of(a.k_start, at.s, a.Tk);
  const int nq = qs.y, nk = kx.y, row0 = at.tile * BQ, row = row0 + 32 * w + lane % 32;
  const size_t first = (size_t)qs.x + min(row, nq - 1);          // this lane's row, in range
  const uint16_t* kh = a.k + (size_t)(h / a.group) * a.skv.h + (size_t)kx.x * a.skv.t;
  const uint16_t* vh = a.v + (size_t)(h / a.group) * a.skv.h + (size_t)kx.x * a.skv.t;
  const int past = a.causal ? nk - nq : nk;
  const int last = min(row0 + BQ, nq);
  const int keys = a.causal ? min(nk, max(0, last + past)) : nk;
  const int mine = a.causal ? min(nk, row + past + 1) : nk;
  bf16x8 qf[KS], gf[KS];
  float delta = 0.f;
  {
    const uint16_t* src = a.q + (size_t)h * a.sq.h + first * a.sq.t + 8 * g;
    const uint16_t* gsrc = a.dout + (size_t)h * a.so.h + first * a.so.t + 8 * g;
    const uint16_t* osrc = a.out + (size_t)h * a.so.h + first * a.so.t + 8 * g;
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
  if (row < nq && g == 0) a.delta[(size_t)h * a.Tq + first] = delta;
  const float lse = a.lse[(size_t)h * a.Tq + first];
  const float l2 = lse == -INFINITY ? INFINITY : lse * kLog2e;   // a row that reads no key: P = 0
  const float c1 = kLog2e * a.scale;
  f32x16 acc[ET];
#pragma unroll
  for (int et = 0; et < ET; et++)
#pragma unroll
    for (int e = 0; e < 16; e++) acc[et][e] = 0.f;
  for (int t0 = 0; t0 < keys; t0 += kTileTokens) {
    u32x4 r[TileCopy<D, NT>::kLoads], rv[TileCopy<D, NT>::kLoads];
    TileCopy<D, NT>::load(r, kh + (size_t)t0 * a.skv.t, a.skv.t, min(kTileTokens, nk - t0), tid);
    TileCopy<D, NT>::load(rv, vh + (size_t)t0 * a.skv.t, a.skv.t, min(kTileTokens, nk - t0), tid);
    __syncthreads();
    TileCopy<D, NT>::store(r, ks_, tid);
    TileCopy<D, NT>::store(rv, vs_, tid);
    __syncthreads();
    bf16x8 df[4];
#pragma unroll
    for (int mt = 0; mt < 2; mt++) {
      f32x16 s, dp;
#pragma unroll
      for (int e = 0; e < 16; e++) s[e] = dp[e] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ks++) {
        s = mfma_bf16(row_fragment<PL>(ks_, 32 * mt + lane % 32, 16 * ks + 8 * g), qf[ks], s);
        dp = mfma_bf16(row_fragment<PL>(vs_, 32 * mt + lane % 32, 16 * ks + 8 * g), gf[ks], dp);
      }
#pragma unroll
      for (int e = 0; e < 16; e++) {
        const float p = fast_exp2(s[e] * c1 - l2);
        const float ds = t0 + 32 * mt + 8 * (e / 4) + 4 * g + e % 4 >= mine ? 0.f : p * (dp[e] - delta);
        df[2 * mt + e / 8][e % 8] = (__bf16)ds;
      }
    }
#pragma unroll
    for (int et = 0; et < ET; et++)
#pragma unroll
      for (int ks = 0; ks < 4; ks++) acc[et] = mfma_bf16(v_fragment<PL>(ks_, ks, 32 * et, lane), df[ks], acc[et]);
  }
  if (row >= nq) return;
  uint16_t* dst = a.dq + (size_t)h * a.sq.h + first * a.sq.t;
#pragma unroll
  for (int et = 0; et < ET; et++)
#pragma unroll
    for (int v4 = 0; v4 < 4; v4++) {
      bf16x4 pk;
#pragma unroll
      for (int r = 0; r < 4; r++) pk[r] = (__bf16)(a.scale * acc[et][4 * v4 + r]);
      *reinterpret_cast<bf16x4*>(dst + 32 * et + 8 * v4 + 4 * g) = pk;
    }
}

// dK and dV of 128 keys: S = Q K^T and dP = dO V^T (rows x keys), a key on lanes l and l + 32 with its row of K and V in registers;
// dV^T += dO^T P and dK^T += Q^T dS over the rows, 64 at a time, of every head of the group.
template <int D>
__global__ __launch_bounds__(256) void packed_dkv_kernel(PackedArgs a) {
  constexpr int BK = 128, NT = 256, KS = D / 16, ET = D / 32;
  typedef PaddedLayout<D> PL;
  __shared__ __attribute__((aligned(16))) uint16_t qs_[kTileTokens * PL::kRowElems], gs_[kTileTokens * PL::kRowElems];
  __shared__ __attribute__((aligned(16))) float ls_[kTileTokens], ds_[kTileTokens];
  const int tid = threadIdx.x, lane = tid % kWave, w = tid / kWave, g = lane / 32;
  const int hkv = a.H / a.group, hk = blockIdx.x % hkv;
  const TilePlace at = find_tile(a.k_start, a.S, a.Tk, BK, blockIdx.x / hkv, lane);
  if (at.s < 0) return;
  const int2 qx = stretch_of(a.q_start, at.s, a.Tq), kx = stretch_of(a.k_start, at.s, a.Tk);
  const int nq = qx.y, nk = kx.y, key0 = at.tile * BK, key = key0 + 32 * w + lane % 32;
  const size_t first = (size_t)kx.x + min(key, nk - 1);
  bf16x8 kf[KS], vf[KS];
  {
    const uint16_t* src = a.k + (size_t)hk * a.skv.h + first * a.skv.t + 8 * g;
    const uint16_t* vsrc = a.v + (size_t)hk * a.skv.h + first * a.skv.t + 8 * g;
#pragma unroll
    for (int ks = 0; ks < KS; ks++) {
      kf[ks] = *reinterpret_cast<const bf16x8*>(src + 16 * ks);
      vf[ks] = *reinterpret_cast<const bf16x8*>(vsrc + 16 * ks);
    }
  }
  const float c1 = kLog2e * a.scale;
  const int from = a.causal ? max(0, key - (nk - nq)) : 0;       // this lane's key is read by the rows from this one on
  const int start = a.causal ? max(0, key0 - (nk - nq)) / kTileTokens * kTileTokens : 0;
  f32x16 dk[ET], dv[ET];
#pragma unroll
  for (int et = 0; et < ET; et++)
#pragma unroll
    for (int e = 0; e < 16; e++) dk[et][e] = dv[et][e] = 0.f;
  for (int h = hk * a.group; h < (hk + 1) * a.group; h++) {
    const uint16_t* qh = a.q + (size_t)h * a.sq.h + (size_t)qx.x * a.sq.t;
    const uint16_t* gh = a.dout + (size_t)h * a.so.h + (size_t)qx.x * a.so.t;
    const float* lh = a.lse + (size_t)h * a.Tq + qx.x;
    const float* dh = a.delta + (size_t)h * a.Tq + qx.x;
    for (int r0 = start; r0 < nq; r0 += kTileTokens) {
      u32x4 r[TileCopy<D, NT>::kLoads], rg[TileCopy<D, NT>::kLoads];
      TileCopy<D, NT>::load(r, qh + (size_t)r0 * a.sq.t, a.sq.t, min(kTileTokens, nq - r0), tid);
      TileCopy<D, NT>::load(rg, gh + (size_t)r0 * a.so.t, a.so.t, min(kTileTokens, nq - r0), tid);
      float l = 0.f, d = 0.f;
      if (tid < kTileTokens) {
        const int i = min(r0 + tid, nq - 1);
        l = lh[i];
        l = l == -INFINITY ? INFINITY : l * kLog2e;
        d = dh[i];
      }
      __syncthreads();
      TileCopy<D, NT>::store(r, qs_, tid);
      TileCopy<D, NT>::store(rg, gs_, tid);
      if (tid < kTileTokens) {
        ls_[tid] = l;
        ds_[tid] = d;
      }
      __syncthreads();
      bf16x8 pf[4], df[4];
#pragma unroll
      for (int mt = 0; mt < 2; mt++) {
        f32x16 s, dp;
#pragma unroll
        for (int e = 0; e < 16; e++) s[e] = dp[e] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ks++) {
          s = mfma_bf16(row_fragment<PL>(qs_, 32 * mt + lane % 32, 16 * ks + 8 * g), kf[ks], s);
          dp = mfma_bf16(row_fragment<PL>(gs_, 32 * mt + lane % 32, 16 * ks + 8 * g), vf[ks], dp);
        }
#pragma unroll
        for (int e = 0; e < 16; e++) {
          const int i = 32 * mt + 8 * (e / 4) + 4 * g + e % 4;
          const bool reads = r0 + i >= from && r0 + i < nq;
          const float p = reads ? fast_exp2(s[e] * c1 - ls_[i]) : 0.f;
          pf[2 * mt + e / 8][e % 8] = (__bf16)p;
          df[2 * mt + e / 8][e % 8] = (__bf16)(reads ? p * (dp[e] - ds_[i]) : 0.f);
        }
      }
#pragma unroll
      for (int et = 0; et < ET; et++)
#pragma unroll
        for (int ks = 0; ks < 4; ks++) {
          dv[et] = mfma_bf16(v_fragment<PL>(gs_, ks, 32 * et, lane), pf[ks], dv[et]);
          dk[et] = mfma_bf16(v_fragment<PL>(qs_, ks, 32 * et, lane), df[ks], dk[et]);
        }
    }
  }
  if (key >= nk) return;
  uint16_t* dst = a.dk + (size_t)hk * a.skv.h + first * a.skv.t;
  uint16_t* vdst = a.dv + (size_t)hk * a.skv.h + first * a.skv.t;
#pragma unroll
  for (int et = 0; et < ET; et++)
#pragma unroll
    for (int v4 = 0; v4 < 4; v4++) {
      bf16x4 pk, pv;
#pragma unroll
      for (int r = 0; r < 4; r++) {
        pk[r] = (__bf16)(a.scale * dk[et][4 * v4 + r]);
        pv[r] = (__bf16)dv[et][4 * v4 + r];
      }
      *reinterpret_cast<bf16x4*>(dst + 32 * et + 8 * v4 + 4 * g) = pk;
      *reinterpret_cast<bf16x4*>(vdst + 32 * et + 8 * v4 + 4 * g) = pv;
    }
}

hipError_t launch_packed_bwd(const PackedArgs& a, hipStream_t stream) {
  const long long q_tiles = most_tiles(a.Tq, a.S, 128) * a.H, k_tiles = most_tiles(a.Tk, a.S, 128) * (a.H / a.group);
  if (q_tiles) {
    if (a.d == 128) packed_dq_kernel<128><<<(unsigned)q_tiles, 256, 0, stream>>>(a);
    else packed_dq_kernel<64><<<(unsigned)q_tiles, 256, 0, stream>>>(a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  if (k_tiles) {
    if (a.d == 128) packed_dkv_kernel<128><<<(unsigned)k_tiles, 256, 0, stream>>>(a);
    else packed_dkv_kernel<64><<<(unsigned)k_tiles, 256, 0, stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace sla2
