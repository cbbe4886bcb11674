// How the attention over a paged cache (sla2_cache_attn.hip) spreads the tokens of all sequences over workgroups: the arithmetic that its
// two kernels have to agree on, which a test on the CPU compiles as it is.
//
// The blocks of all sequences lie one behind the other on a line, each sequence with kOverhead blocks' worth of time in front of its own (first
// reads, the joining of the waves; 3, 12 and 24 were slower).  The workgroups of a key head have equal stretches of it, whatever the lengths:
// whole sequences, and at its two ends parts of one, which go into slot 0 (a sequence that began before the stretch) or slot 1 (one that goes on
// behind it) of the workgroup.
#pragma once
#include "common.h"

namespace sla2 {

constexpr int kDecodeBlock = 32;             // tokens
constexpr int kHeadRows = 16;                // query heads of a workgroup
constexpr int kOverhead = 6;
// Places of a workgroup's stretch at least, where there are parts.  Workgroups that read at once are worth more than waves with several blocks:
// 2,000 tokens of 40 heads on 8 in INT8, room for 131,072: 11.3 us, with 1 11.9, 4 12.2, 8 13.9, 16 18.1; eight sequences of 300, bf16: 13.4, 13.5, 14.0,
// 17.2, 20.6.  40 tokens of 12 heads, with 2 no part but the whole: 6.7, with 1 8.0.
constexpr int kLeastStretch = 2;

// Workgroups of a key head (of each kHeadRows of its group) that a launch has, from the room of the page table: 0, one for each sequence of at most
// 1,024 tokens; otherwise as many as two to a CU are, with 4 blocks a wave at least where sequences are as long as the table.  (The line from 256
// tokens on: four sequences of up to 300 15 us for 11; from 4,096: 17 of up to 2,284 39 us for 21.)
inline int most_parts(int B, long long room, long long heads) {
  if (room <= 1024) return 0;
  const long long blocks = B * ((room + kDecodeBlock - 1) / kDecodeBlock);
  long long parts = 512 / heads;
  if (parts > blocks / 16) parts = blocks / 16;
  return parts < 1 ? 1 : (int)parts;
}
// .. and how many of them share a line of length `all`: lengths are known on the device alone, and may be far below the table's room.  No
// stretch is empty, so that every part that is joined has been written.
__host__ __device__ __forceinline__ int parts_of(int most, long long all) {
  const long long n = all / kLeastStretch;
  return n < 1 ? 1 : n < most ? (int)n : most;
}
__host__ __device__ __forceinline__ long long stretch_begin(long long all, int parts, int p) { return all * p / parts; }      // ends where p + 1 begins
// the workgroup that has place x: the last one whose stretch begins at or in front of it
__host__ __device__ __forceinline__ int part_at(long long all, int parts, long long x) { return (int)(((x + 1) * parts - 1) / all); }

// The blocks lo .. hi - 1 of a sequence of nb, whose first one is at place `first`, that stretch [x, y) has
struct BlockRange {
  int lo, hi;
};
__host__ __device__ __forceinline__ BlockRange blocks_in(long long x, long long y, long long first, int nb) {
  auto inside = [&](long long at) { return (int)(at < first ? 0 : at - first < nb ? at - first : nb); };
  return BlockRange{inside(x), inside(y)};
}
// Where workgroup p keeps its part of a sequence: of one that it began, or of one that another did
__host__ __device__ __forceinline__ size_t part_slot(int p, bool began) { return (size_t)p * 2 + (began ? 1 : 0); }

}  // namespace sla2
