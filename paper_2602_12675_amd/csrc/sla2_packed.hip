// Forward pass of attention over packed sequences: out = softmax(scale Q K^T) V, lse, with grouped heads and a causal mask.
//
// One workgroup = 4 waves = 128 query rows of one head and sequence; a wave has 32 of them, one on lanes l and l + 32.  One pass over
// the keys, 64 at a time, with the running maximum and sum of the softmax: S^T = K Q^T (keys x rows), so that a lane holds scores of
// one row, P^T goes back into O^T += V^T P^T as it lies in the registers, and a row's maximum and sum are its lane's own and one
// exchange with the other half of the wave.
#include "packed.h"

namespace sla2 {

template <int D>
__global__ __launch_bounds__(256) void packed_fwd_kernel(PackedArgs a, int heads_first) {
  constexpr int BQ = 128, NT = 256, KS = D / 16, ET = D / 32;
  typedef PaddedLayout<D> PL;
  __shared__ __attribute__((aligned(16))) uint16_t ks_[kTileTokens * PL::kRowElems], vs_[kTileTokens * PL::kRowElems];
  const int tid = threadIdx.x, lane = tid % kWave, w = tid / kWave, g = lane / 32;
  const int h = blockIdx.x % a.H;
  const TilePlace at = find_tile(a.q_start, a.S, a.Tq, BQ, blockIdx.x / a.H, lane);
  if (at.s < 0) return;
  const int2 qs = stretch_of(a.q_start, at.s, a.Tq), kx = stretch_of(a.k_start, at.s, a.Tk);
  const int nq = qs.y, nk = kx.y, row0 = at.tile * BQ, row = row0 + 32 * w + lane % 32;
  const uint16_t* qh = a.q + (size_t)h * a.sq.h + (size_t)qs.x * a.sq.t;
  const uint16_t* kh = a.k + (size_t)(h / a.group) * a.skv.h + (size_t)kx.x * a.skv.t;
  const uint16_t* vh = a.v + (size_t)(h / a.group) * a.skv.h + (size_t)kx.x * a.skv.t;
  const int past = a.causal ? nk - nq : nk;            // row i reads keys below i + past + 1 (causal), all otherwise
  const int last = min(row0 + BQ, nq);                 // behind the tile's last row
  const int keys = a.causal ? min(nk, max(0, last + past)) : nk;
  const int mine = a.causal ? min(nk, row + past + 1) : nk;      // this lane's row: below this
  bf16x8 qf[KS];
  {
    const uint16_t* src = qh + (size_t)min(row, nq - 1) * a.sq.t + 8 * g;
#pragma unroll
    for (int ks = 0; ks < KS; ks++) qf[ks] = *reinterpret_cast<const bf16x8*>(src + 16 * ks);
  }
  f32x16 oacc[ET];
#pragma unroll
  for (int et = 0; et < ET; et++)
#pragma unroll
    for (int e = 0; e < 16; e++) oacc[et][e] = 0.f;
  float m_run = -1e30f, l_run = 0.f;
  const float c1 = kLog2e * a.scale;
  for (int t0 = 0; t0 < keys; t0 += kTileTokens) {
    u32x4 r[TileCopy<D, NT>::kLoads], rv[TileCopy<D, NT>::kLoads];
    TileCopy<D, NT>::load(r, kh + (size_t)t0 * a.skv.t, a.skv.t, min(kTileTokens, nk - t0), tid);
    TileCopy<D, NT>::load(rv, vh + (size_t)t0 * a.skv.t, a.skv.t, min(kTileTokens, nk - t0), tid);
    __syncthreads();
    TileCopy<D, NT>::store(r, ks_, tid);
    TileCopy<D, NT>::store(rv, vs_, tid);
    __syncthreads();
    f32x16 sacc[2];
#pragma unroll
    for (int mt = 0; mt < 2; mt++) {
#pragma unroll
      for (int e = 0; e < 16; e++) sacc[mt][e] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ks++)
        sacc[mt] = mfma_bf16(row_fragment<PL>(ks_, 32 * mt + lane % 32, 16 * ks + 8 * g), qf[ks], sacc[mt]);
    }
    float mx = -INFINITY;
#pragma unroll
    for (int mt = 0; mt < 2; mt++)
#pragma unroll
      for (int e = 0; e < 16; e++) {
        if (t0 + 32 * mt + 8 * (e / 4) + 4 * g + e % 4 >= mine) sacc[mt][e] = -INFINITY;
        mx = fmaxf(mx, sacc[mt][e]);
      }
    mx = swap_halves_max(mx) * c1;
    const float m_new = fmaxf(m_run, mx), corr = fast_exp2(m_run - m_new);
    m_run = m_new;
    float rs = 0.f;
    bf16x8 pf[4];
#pragma unroll
    for (int mt = 0; mt < 2; mt++)
#pragma unroll
      for (int e = 0; e < 16; e++) {
        const float p = fast_exp2(sacc[mt][e] * c1 - m_new);
        rs += p;
        pf[2 * mt + e / 8][e % 8] = (__bf16)p;
      }
    l_run = l_run * corr + swap_halves_sum(rs);
#pragma unroll
    for (int et = 0; et < ET; et++) {
#pragma unroll
      for (int e = 0; e < 16; e++) oacc[et][e] *= corr;
#pragma unroll
      for (int ks = 0; ks < 4; ks++) oacc[et] = mfma_bf16(v_fragment<PL>(vs_, ks, 32 * et, lane), pf[ks], oacc[et]);
    }
  }
  if (row >= nq) return;
  const bool any = l_run != 0.f;                       // NaN is some
  const float inv = any ? 1.f / l_run : 0.f;
  uint16_t* dst = a.o + (size_t)h * a.so.h + (size_t)(qs.x + row) * a.so.t;
#pragma unroll
  for (int et = 0; et < ET; et++)
#pragma unroll
    for (int v4 = 0; v4 < 4; v4++) {
      bf16x4 pk;
#pragma unroll
      for (int r = 0; r < 4; r++) pk[r] = (__bf16)(any ? inv * oacc[et][4 * v4 + r] : 0.f);
      *reinterpret_cast<bf16x4*>(dst + 32 * et + 8 * v4 + 4 * g) = pk;
    }
  if (a.lse_out && g == 0) a.lse_out[(size_t)h * a.Tq + qs.x + row] = any ? (m_run + log2f(l_run)) * (1.f / kLog2e) : -INFINITY;
}

hipError_t launch_packed_fwd(const PackedArgs& a, hipStream_t stream) {
  const long long grid = most_tiles(a.Tq, a.S, 128) * a.H;
  if (!grid) return hipSuccess;
  if (a.d == 128) packed_fwd_kernel<128><<<(unsigned)grid, 256, 0, stream>>>(a, 0);
  else packed_fwd_kernel<64><<<(unsigned)grid, 256, 0, stream>>>(a, 0);
  return hipGetLastError();
}

}  // namespace sla2
