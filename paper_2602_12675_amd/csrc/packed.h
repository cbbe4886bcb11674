// Attention over packed sequences: what its kernels (sla2_packed.hip, sla2_packed_bwd.hip) share.
#pragma once
#include "mfma_tiles.h"

namespace sla2 {

struct RowStrides {                          // elements; the channels of a head are neighbours
  long long h;
  int t;
};
struct PackedArgs {
  const uint16_t *q, *k, *v, *out, *dout;
  const int32_t *q_start, *k_start;
  const float* lse;
  uint16_t *o, *dq, *dk, *dv;
  float* lse_out;
  RowStrides sq, skv, so;
  int S, Tq, Tk, H, group, d;                // group: query heads of a key head
  bool causal;
  float scale;                               // of the scores
  // scratch
  float* delta;                              // backward: [H][Tq], sum of dO . O of a row
};

hipError_t launch_packed_fwd(const PackedArgs& a, hipStream_t stream);
hipError_t launch_packed_bwd(const PackedArgs& a, hipStream_t stream);

// Tiles of `rows` rows that sequences of `tokens` rows in all have at most.
inline long long most_tiles(int tokens, int sequences, int rows) {
  return tokens / rows + (long long)(sequences < tokens ? sequences : tokens);
}

#ifdef __HIPCC__
// A sequence: where its queries and keys lie, whatever the offsets hold inside the tensors.
struct Stretch {
  int q0, nq, k0, nk;
};
__device__ __forceinline__ int2 stretch_of(const int32_t* start, int s, int tokens) {
  const int a = min(max(start[s], 0), tokens), b = min(max(start[s + 1], a), tokens);
  return make_int2(a, b - a);
}

// The n-th tile, of `rows` rows, of the sequences one behind the other: its sequence, and its number in it.  A wave looks at 64
// sequences at a time; all lanes return the same.  s < 0: there are fewer tiles.
struct TilePlace {
  int s, tile;
};
__device__ __forceinline__ TilePlace find_tile(const int32_t* start, int S, int tokens, int rows, int n, int lane) {
  for (int s0 = 0; s0 < S; s0 += kWave) {
    const int s = s0 + lane;
    const int own = s < S ? (stretch_of(start, s, tokens).y + rows - 1) / rows : 0;
    int sum = own;                                     // of the lanes up to this one
#pragma unroll
    for (int by = 1; by < kWave; by *= 2) {
      const int x = __shfl_up(sum, by);
      sum += lane >= by ? x : 0;
    }
    const unsigned long long has = __builtin_amdgcn_ballot_w64(sum > n);
    if (has) {
      const int f = __builtin_ctzll(has);
      return TilePlace{s0 + f, __builtin_amdgcn_readfirstlane(n - __shfl(sum - own, f))};
    }
    n -= __builtin_amdgcn_readlane(sum, kWave - 1);
  }
  return TilePlace{-1, 0};
}
#endif

}  // namespace sla2
