// A paged cache of keys and values: rows of bf16 into it, with one FP8 or INT8 scale for each token and head, and back.
//
// A row (the d channels of a token and head) is 8 channels on each of d / 8 neighbouring lanes, read once and written once; its largest
// magnitude is a maximum over those lanes, taken on the bits of |x|, which order finite numbers, infinities and NaNs alike.  A
// workgroup has neighbouring tokens of one head, whose codes and scales are neighbours in a page.
//
// Bound by memory: 74,655 tokens of 40 heads from INT8 461 us = 5.0 TB/s, a copy's rate; 32,760 tokens of 12 heads into FP8 57 us in the
// kernel, 5.3 TB/s (68 a call with the tensors out of the caches).  A row a thread, keys and values apart, took
// 822 and 92 us: every workgroup looks up its rows' places before it moves anything.
#include "cache.h"
#include "rows.h"

namespace sla2 {

// Where row i of k and v is in the cache: page and slot; page -1: nowhere, -2: the row is of no sequence.  A row a lane, the rows of a
// wave being neighbours.  Its sequence is the number of sequences that end at or in front of it, counted 64 at a time: for all rows at
// once where no sequence ends between them.  (Offsets that do not ascend give some sequence, whose pages bound the place.)
struct Place {
  int page, slot;
};
__device__ __forceinline__ Place place_of(const CacheArgs& a, int i, int lane) {
  int b = i;
  long long at = 0;
  if (a.start) {
    const int i0 = __builtin_amdgcn_readfirstlane(i), i1 = __builtin_amdgcn_readlane(i, kWave - 1);
    b = 0;
    for (int s0 = 0; s0 < a.B; s0 += kWave) {
      const int end = s0 + lane < a.B ? a.start[s0 + lane + 1] : INT32_MAX;
      const unsigned long long before = __builtin_amdgcn_ballot_w64(end <= i0);
      if (__builtin_amdgcn_ballot_w64(end <= i1) == before) {
        b += __builtin_popcountll(before);
        continue;
      }
      int n = 0;                                         // halving: the ends ascend
#pragma unroll
      for (int step = kWave / 2; step; step /= 2) n += __shfl(end, n + step - 1) <= i ? step : 0;
      b += n + (__shfl(end, n) <= i ? 1 : 0);
    }
  }
  if (i >= a.tokens || b >= a.B) return Place{-2, 0};
  if (a.start) {
    const int s = a.start[b];
    if (i < s) return Place{-2, 0};                      // in front of the first sequence
    at = i - (long long)s;
  }
  if (a.first) at += a.first[b];
  const long long column = at >> a.page_shift;
  if (at < 0 || column >= a.max_pages) return Place{-1, 0};
  const int page = a.table[b * a.table_stride + column];
  return Place{page >= 0 && page < a.pages ? page : -1, (int)(at & ((1 << a.page_shift) - 1))};
}

// |x| of the largest of a row, an infinity if one of them is not finite
template <int LANES> __device__ __forceinline__ float row_amax(const Raw<true>& r) {
  unsigned m = 0;
#pragma unroll
  for (int i = 0; i < 4; i++) m = max(m, max(r.a[0][i] & 0x7fffu, r.a[0][i] >> 16 & 0x7fffu));
  float x = __builtin_bit_cast(float, min(m, 0x7f80u) << 16);
  x = quad_max(x);
  x = fmaxf(x, dpp_move<0x141>(x));                      // row_half_mirror
  if (LANES > 8) x = fmaxf(x, dpp_move<0x140>(x));       // row_mirror
  return x;
}

// 8 codes of a row whose largest magnitude is amax, and its scale
template <int QUANT> __device__ __forceinline__ u32x2 codes_of(const Raw<true>& r, float amax, float* scale) {
  constexpr float top = QUANT == SLA2_QUANT_FP8 ? kE4M3Max : kInt8Max;
  const bool some = amax >= 0x1p-100f && amax < INFINITY;
  const float by = some ? top * (1.f / amax) : 0.f;
  *scale = some ? amax * (1.f / top) : amax < INFINITY ? 1.f : NAN;
  float x[8];
  unpack8<true>(r, x);
  u32x2 c;
#pragma unroll
  for (int i = 0; i < 2; i++) {
    if constexpr (QUANT == SLA2_QUANT_FP8) {
      int u = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i] * by, x[4 * i + 1] * by, 0, false);
      c[i] = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2] * by, x[4 * i + 3] * by, u, true);
    } else {
      unsigned u = 0;
#pragma unroll
      for (int e = 0; e < 4; e++) u |= ((unsigned)(int)rintf(x[4 * i + e] * by) & 255u) << 8 * e;
      c[i] = u;
    }
  }
  if (!some) c = u32x2{0, 0};                            // NaN x 0 is no code
  return c;
}

template <int QUANT> __device__ __forceinline__ Raw<true> values_of(u32x2 c, float scale) {
  float x[8];
#pragma unroll
  for (int i = 0; i < 2; i++) {
    if constexpr (QUANT == SLA2_QUANT_FP8) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i], true);
      x[4 * i] = lo[0], x[4 * i + 1] = lo[1], x[4 * i + 2] = hi[0], x[4 * i + 3] = hi[1];
    } else {
#pragma unroll
      for (int e = 0; e < 4; e++) x[4 * i + e] = (float)((int)(c[i] << (24 - 8 * e)) >> 24);
    }
  }
#pragma unroll
  for (int i = 0; i < 8; i++) x[i] *= scale;
  return pack8<true>(x);
}

// Keys and values of 64 neighbouring rows of a head, U of each on their way to a thread.
template <int D, int QUANT, bool WRITE>
__global__ __launch_bounds__(kCacheThreads) void cache_rows_kernel(CacheArgs a) {
  constexpr int LANES = D / 8, ROWS = kCacheThreads / LANES, U = kCacheRows / ROWS, ESZ = QUANT == SLA2_QUANT_NONE ? 2 : 1;
  const int tid = threadIdx.x, lane = tid % kWave, col = 8 * (tid % LANES), h = blockIdx.y, i0 = blockIdx.x * kCacheRows;
  Raw<true> r[2][U];
  const long long own = (long long)h * a.kv_h + col;
  if (WRITE) {
#pragma unroll
    for (int u = 0; u < U; u++) {
      const long long at = own + (long long)min(i0 + u * ROWS + tid / LANES, a.tokens - 1) * a.kv_t;
      r[0][u] = load8<true>(a.k, at);
      r[1][u] = load8<true>(a.v, at);
    }
  }
  const Place mine = place_of(a, i0 + lane, lane);
  Place p[U];
  long long slot[U];
#pragma unroll
  for (int u = 0; u < U; u++) {
    const int x = u * ROWS + tid / LANES;
    p[u] = Place{__shfl(mine.page, x), __shfl(mine.slot, x)};
    slot[u] = p[u].page * a.page_stride + h * a.head_stride + p[u].slot * a.token_stride + col;
  }
  auto scale_at = [&](int u) { return (((long long)p[u].page * a.Hkv + h) << a.page_shift) + p[u].slot; };
  if constexpr (WRITE) {
#pragma unroll
    for (int x = 0; x < 2; x++)
#pragma unroll
      for (int u = 0; u < U; u++) {
        char* cache = (char*)(x ? a.vc : a.kc) + slot[u] * ESZ;
        if constexpr (QUANT == SLA2_QUANT_NONE) {
          if (p[u].page >= 0) *(u32x4*)cache = r[x][u].a[0];
        } else {
          float s;
          const u32x2 c = codes_of<QUANT>(r[x][u], row_amax<LANES>(r[x][u]), &s);
          if (p[u].page >= 0) {
            *(u32x2*)cache = c;
            if (col == 0) (x ? a.vs : a.ks)[scale_at(u)] = s;
          }
        }
      }
  } else {
    u32x2 c[2][U];
    float s[2][U];
#pragma unroll
    for (int x = 0; x < 2; x++)
#pragma unroll
      for (int u = 0; u < U; u++) {
        const char* cache = (const char*)(x ? a.vc : a.kc) + slot[u] * ESZ;
        r[x][u] = zero8<true>();
        c[x][u] = u32x2{0, 0};
        s[x][u] = 0.f;
        if (p[u].page < 0) continue;
        if constexpr (QUANT == SLA2_QUANT_NONE) {
          r[x][u].a[0] = *(const u32x4*)cache;
        } else {
          c[x][u] = *(const u32x2*)cache;
          s[x][u] = (x ? a.vs : a.ks)[scale_at(u)];
        }
      }
#pragma unroll
    for (int x = 0; x < 2; x++)
#pragma unroll
      for (int u = 0; u < U; u++) {
        if (p[u].page < -1) continue;
        if constexpr (QUANT != SLA2_QUANT_NONE) r[x][u] = values_of<QUANT>(c[x][u], s[x][u]);
        store8<true>(x ? a.v : a.k, own + (long long)(i0 + u * ROWS + tid / LANES) * a.kv_t, r[x][u]);
      }
  }
}

template <bool WRITE> static hipError_t launch_rows(const CacheArgs& a, hipStream_t stream) {
  if (!a.tokens) return hipSuccess;
  const dim3 grid((a.tokens + kCacheRows - 1) / kCacheRows, a.Hkv);
#define SLA2_ROWS(D)                                                                                                          \
  (a.quant == SLA2_QUANT_NONE  ? cache_rows_kernel<D, SLA2_QUANT_NONE, WRITE><<<grid, kCacheThreads, 0, stream>>>(a)          \
   : a.quant == SLA2_QUANT_FP8 ? cache_rows_kernel<D, SLA2_QUANT_FP8, WRITE><<<grid, kCacheThreads, 0, stream>>>(a)           \
                               : cache_rows_kernel<D, SLA2_QUANT_INT8, WRITE><<<grid, kCacheThreads, 0, stream>>>(a))
  if (a.d == 128) SLA2_ROWS(128);
  else SLA2_ROWS(64);
#undef SLA2_ROWS
  return hipGetLastError();
}
hipError_t launch_cache_write(const CacheArgs& a, hipStream_t stream) { return launch_rows<true>(a, stream); }
hipError_t launch_cache_read(const CacheArgs& a, hipStream_t stream) { return launch_rows<false>(a, stream); }

}  // namespace sla2
