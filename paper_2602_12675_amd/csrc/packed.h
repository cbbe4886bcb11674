// Attention over packed sequences: what its kernels (sla2_packed.hip, sla2_packed_bwd.hip) share.
//
// The queries of a sequence and of all heads of a key head's group are taken as the rows of one matrix, row r being query r / group of
// head r % group: they read the same keys and values, and with few queries of many heads a tile has no empty rows.
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
  RowStrides sq, skv, so, sg;                // of q and dq; k, v, dk and dv; out; dout
  int S, Tq, Tk, H, Hkv, group, d;           // group: query heads of a key head
  bool causal;
  float scale;                               // of the scores
  // The steps of a tile's inner loop are dealt to several workgroups, whose sums another kernel joins.  Of a tile of rows evenly to
  // q_parts; of a tile of keys k_chunk steps to each, k_parts at most.  1: none
  int q_parts, k_parts, k_chunk;
  bool rows_first;                           // backward, in one launch: the workgroups of the rows before those of the keys
  // scratch.  Sums of parts: O or dQ [q_parts][rows][d], (m, l) [q_parts][rows][2], the rows of all key heads being [Hkv][Tq group]; dK and
  // dV [2][k_parts][Tk][Hkv][d]
  float *lse2, *delta;                       // backward: lse log2(e) and D of every row, see stat_at
  float *part_o, *part_ml, *part_kv;
};

constexpr int kRowTile = 128, kKeyTile = 128;        // rows, and keys, of a workgroup: 32 a wave
constexpr int kPlaces = 512;                         // workgroups that are at work at a time: two a CU
constexpr int kMostOfKeys = 1 << 22;                 // workgroups of the keys, where those of the rows are in the same launch

void plan_packed(PackedArgs* a, bool backward);
hipError_t launch_packed_fwd(const PackedArgs& a, hipStream_t stream);
hipError_t launch_packed_bwd(const PackedArgs& a, hipStream_t stream);

// Tiles of `rows` rows that sequences of `tokens` rows in all have at most.
inline long long most_tiles(long long tokens, int sequences, int rows) {
  return tokens / rows + (sequences < tokens ? sequences : tokens);
}

#ifdef __HIPCC__
// The n-th tile, of `rows` rows (of `rows` keys), of the sequences one behind the other: its number in its sequence, how many that one
// has, and where its queries and keys lie, whatever the offsets hold inside the tensors.  A wave looks at 64 sequences at a time; all
// lanes return the same.  tile < 0: there are fewer tiles.
struct TilePlace {
  int tile, tiles, s, q0, nq, k0, nk;
};
template <bool KEYS> __device__ __forceinline__ TilePlace find_tile(const PackedArgs& a, int rows, int n, int lane) {
  for (int s0 = 0; s0 < a.S; s0 += kWave) {
    const int s = s0 + lane;
    int q0 = 0, q1 = 0, k0 = 0, k1 = 0;
    if (s < a.S) {
      q0 = a.q_start[s], q1 = a.q_start[s + 1], k0 = a.k_start[s], k1 = a.k_start[s + 1];
      q0 = min(max(q0, 0), a.Tq);
      q1 = min(max(q1, q0), a.Tq);
      k0 = min(max(k0, 0), a.Tk);
      k1 = min(max(k1, k0), a.Tk);
    }
    const int own = (int)(((unsigned)(KEYS ? k1 - k0 : (q1 - q0) * a.group) + rows - 1) / (unsigned)rows);
    int sum = own;                                     // of the lanes up to this one
    if (a.S > 1) {
#pragma unroll
      for (int by = 1; by < kWave; by *= 2) {
        const int x = __shfl_up(sum, by);
        sum += lane >= by ? x : 0;
      }
    }
    const unsigned long long has = __builtin_amdgcn_ballot_w64(sum > n);
    if (has) {
      const int f = __builtin_ctzll(has);
      auto of = [&](int x) { return __builtin_amdgcn_readlane(x, f); };
      return TilePlace{n - of(sum - own), of(own), s0 + f, of(q0), of(q1 - q0), of(k0), of(k1 - k0)};
    }
    n -= __builtin_amdgcn_readlane(sum, kWave - 1);
  }
  return TilePlace{-1, 0, 0, 0, 0, 0, 0};
}

// query and head (inside the group) of a row
__device__ __forceinline__ int2 query_of(const PackedArgs& a, int row) {
  if (a.group == 1) return make_int2(row, 0);
  const int i = row / a.group;
  return make_int2(i, row - i * a.group);
}
// Where the backward pass keeps what belongs to a row: for each key head the blocks of its sequences, 16 queries of one head each, the
// heads of the group one after the other.  Sequence s has room for 16 queries more than it has, from query q0 + 16 s of the key head on.
constexpr int kQueryBlock = 16;
__host__ __device__ __forceinline__ size_t stat_rows(const PackedArgs& a) { return ((size_t)a.Tq + (size_t)kQueryBlock * a.S) * a.group; }
__device__ __forceinline__ size_t stat_first(const PackedArgs& a, int hk, int s, int q0) {
  return (size_t)hk * stat_rows(a) + ((size_t)q0 + (size_t)kQueryBlock * s) * a.group;
}
__device__ __forceinline__ size_t stat_at(const PackedArgs& a, int query, int head) {
  return ((size_t)(query / kQueryBlock) * a.group + head) * kQueryBlock + query % kQueryBlock;
}

// Workgroup n of a launch over tiles x key heads: consecutive workgroups go to the XCDs in turn, so that where the heads are a multiple
// of the XCDs each of these has heads, and their keys and values, of its own.
struct TileHead {
  int tile, head;
};
__device__ __forceinline__ TileHead tile_head(int n, int heads) { return TileHead{n / heads, n % heads}; }

template <int D> using PackedTile = typename std::conditional<D == 128, SwizzledLayoutB<128>, SwizzledLayout<64>>::type;   // no bank conflicts

// A lane's row of accumulators (channels x rows) to memory: as fp32 ..
template <int D>
__device__ __forceinline__ void store_part(const f32x16 (&acc)[D / 32], float* dst, int g) {
#pragma unroll
  for (int et = 0; et < D / 32; et++)
#pragma unroll
    for (int v4 = 0; v4 < 4; v4++)
      *reinterpret_cast<f32x4*>(dst + 32 * et + 8 * v4 + 4 * g) =
          f32x4{acc[et][4 * v4], acc[et][4 * v4 + 1], acc[et][4 * v4 + 2], acc[et][4 * v4 + 3]};
}
// .. and times `by` as bf16: lanes l and l + 32 have four channels each of every eight, and exchange them for all eight of every other
// eight, 16 bytes a store.
template <int D>
__device__ __forceinline__ void store_row(const f32x16 (&acc)[D / 32], float by, uint16_t* dst, int g, bool there) {
#pragma unroll
  for (int et = 0; et < D / 32; et++)
#pragma unroll
    for (int v = 0; v < 2; v++) {
      u32x2 c[2];                                      // channels 16 v + 8 i + 4 g + 0..3
#pragma unroll
      for (int i = 0; i < 2; i++) {
        bf16x4 pk;
#pragma unroll
        for (int r = 0; r < 4; r++) pk[r] = (__bf16)(by * acc[et][8 * v + 4 * i + r]);
        c[i] = __builtin_bit_cast(u32x2, pk);
      }
      u32x4 out;                                       // channels 16 v + 8 g + 0..7
#pragma unroll
      for (int i = 0; i < 2; i++) {
        const auto r = __builtin_amdgcn_permlane32_swap(c[0][i], c[1][i], false, false);
        out[i] = r[0];
        out[2 + i] = r[1];
      }
      if (there) *reinterpret_cast<u32x4*>(dst + 32 * et + 16 * v + 8 * g) = out;
    }
}

// Rows t0 .. t0 + 63 of n into a tile; rows past the end repeat the last one.  lane_off: tile_lane_off.
template <int D, int NW>
__device__ __forceinline__ void packed_dma(const uint16_t* src, int stride, int t0, int n, unsigned to, int w, unsigned lane_off) {
  const uint16_t* first = src + (size_t)t0 * stride;
  if (t0 + kTileTokens <= n) dma_tile_full<D, NW, PackedTile<D>>(first, stride, to, w, lane_off);
  else dma_tile<D, NW, PackedTile<D>>(first, stride, n - t0, to, w, (int)lane_again());
}

// LDS byte offsets of a lane's operand reads inside a 64-row tile, both for the rows 32 h further by 64 h D bytes.
// Row-wise: row l % 32, channel step ks at (offset of step 0) ^ 32 ks.  Transposing (cf. read_tr4): rows 4 g + (l % 16) / 4 (lo) and 8
// further (hi), channel tile et at (offset of tile 0) ^ 64 et, 16-row step ks 32 D ks further.
template <int D> __device__ __forceinline__ unsigned row_read_offset(int lane) {
  return (unsigned)PackedTile<D>::offset(lane % 32, 8 * (lane / 32)) * 2;
}
template <int D> __device__ __forceinline__ unsigned tr_read_offset(int lane, int hi) {
  return (unsigned)PackedTile<D>::offset(8 * hi + 4 * (lane / 32) + (lane % 16) / 4, 16 * ((lane / 16) % 2) + 4 * (lane % 4)) * 2;
}
#endif

}  // namespace sla2
