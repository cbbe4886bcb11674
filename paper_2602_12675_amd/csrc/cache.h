// A paged cache of keys and values: what its kernels (sla2_cache.hip, sla2_cache_attn.hip) and their host side share.
#pragma once
#include "common.h"

namespace sla2 {

struct CacheArgs {
  // rows of k and v: read by a write, written by a read
  uint16_t *k, *v;
  void *kc, *vc;                             // the cache
  float *ks, *vs;                            // scales [pages, H_kv, page_size]
  const int32_t *start, *first, *table, *length;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  long long table_stride;
  long long page_stride, head_stride, token_stride;              // of the cache, elements
  long long kv_h, kv_t, q_h, q_b, out_h, out_b;
  int B, H, Hkv, group, d, pages, page_shift, max_pages, tokens, quant;
  float scale;
  // attention: the workgroups of a key head that share the tokens of all sequences, at most (0: one for each sequence; cache_line.h); with
  // more than one, parts of sequences are in scratch: O [parts][2][H][d] fp32 and (m, l) [parts][2][H][2]
  int parts;
  float *part_o, *part_ml;
};

// Rows of a workgroup that writes or reads, one for each lane of a wave while their places are looked up, and of a call: a launch has less
// than 2^24 workgroups of 256 threads.
constexpr int kCacheThreads = 256, kCacheRows = 64, kMostCacheTokens = ((1 << 24) - 1) * kCacheRows;

void plan_cache_attention(CacheArgs* a);
inline size_t cache_part_floats(const CacheArgs& a) { return a.parts > 1 ? (size_t)a.parts * 2 * a.H * (a.d + 2) : 0; }
hipError_t launch_cache_write(const CacheArgs& a, hipStream_t stream);
hipError_t launch_cache_read(const CacheArgs& a, hipStream_t stream);
hipError_t launch_cache_attention(const CacheArgs& a, hipStream_t stream);

}  // namespace sla2
