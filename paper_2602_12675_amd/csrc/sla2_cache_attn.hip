// Attention of one new token of each sequence over a paged cache of keys and values.
//
// Bound by the bytes of the cache, which are read once: a workgroup has tokens of a sequence and a key head, with up to 16 query heads of
// its group as the 16 rows of the matrix products, and each of its waves works on blocks of 32 tokens by itself, from registers alone:
// no operand passes through LDS, no barrier stands in the loop.
//   S^T = K Q^T (v_mfma_f32_16x16x32_bf16, 16 tokens a product): lane l feeds the token of row l % 16.  Row m of product t is token
//   8 (m / 4) + 4 t + m % 4 of the block, so that lane l ends with head l % 16 and the scores of the 8 tokens 8 (l / 16) + 0..7: what it
//   has to feed as P in O = P V.
//   V: a lane reads D / 16 neighbouring channels of each of the same 8 tokens, whole rows a quarter wave, and turns its 8 x (D / 16)
//   block in registers (v_perm_b32, two channels of two tokens at a time) into the operands of D / 16 products, the i-th of which has
//   the channels D / 16 (l % 16) + i.
// Codes become bf16 exactly; a token's scales multiply its scores and its probability.  Parts of a sequence are joined by a second kernel.
//
// 64 sequences of 17 to 8,192 tokens, 40 heads on 8, bf16: 76 us for 360 MB, of them 6 for the join = 5.1 TB/s in the loop; a workgroup for
// every chunk of 1,024 tokens instead of an equal stretch of all took 138.  One sequence of 32,761 in FP8, 12 heads: 25.5 us for 104 MB.
#include <limits.h>

#include "cache.h"
#include "cache_line.h"
#include "mfma_tiles.h"

namespace sla2 {

constexpr int kDecodeWaves = 4;
constexpr int kIdBlocks = 32;                // blocks whose pages a wave holds, one for 16 tokens a lane

__device__ __forceinline__ int tokens_of(const CacheArgs& a, int b) {
  return (int)min((long long)max(a.length[b], 0), (long long)a.max_pages << a.page_shift);
}
__device__ __forceinline__ int blocks_of(int tokens) { return (int)(((unsigned)tokens + kDecodeBlock - 1) / kDecodeBlock); }
__device__ __forceinline__ long long wave_total(long long x) {
#pragma unroll
  for (int by = 1; by < kWave; by *= 2) x += __shfl_xor(x, by);
  return x;
}
__device__ __forceinline__ long long uniform64(long long x) {
  const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)x), hi = __builtin_amdgcn_readfirstlane((unsigned)((unsigned long long)x >> 32));
  return (long long)((unsigned long long)hi << 32 | lo);
}
// the length of the line; all lanes of the wave take part
__device__ __forceinline__ long long line_length(const CacheArgs& a, int lane) {
  if (a.B == 1) return kOverhead + blocks_of(tokens_of(a, 0));
  long long n = 0;
  for (int b = lane; b < a.B; b += kWave) n += kOverhead + blocks_of(tokens_of(a, b));
  return wave_total(n);
}
// The sequence that place x of the line is in, and where on the line it begins; with `of` >= 0 where sequence `of` begins.
struct OnLine {
  int b;
  long long at;
};
__device__ __forceinline__ OnLine on_line(const CacheArgs& a, long long x, int of, int lane) {
  long long at = 0;
  if (a.B == 1) return OnLine{0, 0};
  for (int b0 = 0; b0 < a.B; b0 += kWave) {
    const int b = b0 + lane;
    const int own = b < a.B ? kOverhead + blocks_of(tokens_of(a, b)) : 0;
    long long sum = own;
#pragma unroll
    for (int by = 1; by < kWave; by *= 2) {
      const long long y = __shfl_up(sum, by);
      sum += lane >= by ? y : 0;
    }
    const unsigned long long has = of >= 0 ? (of < b0 + kWave ? 1ull << (of - b0) : 0) : __builtin_amdgcn_ballot_w64(at + sum > x);
    if (has) {
      const int f = __builtin_ctzll(has);
      return OnLine{b0 + f, at + __shfl(sum - own, f)};
    }
    at += __shfl(sum, kWave - 1);
  }
  return OnLine{a.B, at};
}

__device__ __forceinline__ float over_quarters_max(float x) {       // lanes l, l ^ 16, l ^ 32, l ^ 48
  const unsigned u = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return swap_halves_max(fmaxf(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1])));
}
__device__ __forceinline__ float over_quarters_sum(float x) {
  const unsigned u = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return swap_halves_sum(__builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]));
}

// N codes (a multiple of 4, N / 4 registers) as N / 2 registers of bf16 pairs
template <int QUANT, int N> __device__ __forceinline__ void widen(const unsigned (&c)[N / 4], unsigned (&y)[N / 2]) {
#pragma unroll
  for (int i = 0; i < N / 4; i++) {
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    bf16x2 lo, hi;
    if constexpr (QUANT == SLA2_QUANT_FP8) {
      const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i], true);
      lo = bf16x2{(__bf16)a[0], (__bf16)a[1]};
      hi = bf16x2{(__bf16)b[0], (__bf16)b[1]};
    } else {
      lo = bf16x2{(__bf16)(float)((int)(c[i] << 24) >> 24), (__bf16)(float)((int)(c[i] << 16) >> 24)};
      hi = bf16x2{(__bf16)(float)((int)(c[i] << 8) >> 24), (__bf16)(float)((int)c[i] >> 24)};
    }
    y[2 * i] = __builtin_bit_cast(unsigned, lo);
    y[2 * i + 1] = __builtin_bit_cast(unsigned, hi);
  }
}
template <int BYTES> __device__ __forceinline__ void load_words(const void* p, unsigned (&w)[BYTES / 4]) {
  if constexpr (BYTES == 16) {
    const u32x4 x = *(const u32x4*)p;
    w[0] = x[0], w[1] = x[1], w[2] = x[2], w[3] = x[3];
  } else if constexpr (BYTES == 8) {
    const u32x2 x = *(const u32x2*)p;
    w[0] = x[0], w[1] = x[1];
  } else {
    w[0] = *(const unsigned*)p;
  }
}

// What a wave keeps of 16 query heads: O (rows 4 (l / 16) + 0..3 of the i-th product's channels), the reference m of the exponentials and the
// sum l of this lane's tokens, of head l % 16.
template <int D> struct HeadSums {
  f32x4 o[D / 16];
  float m, l;
};

// The blocks lo + w, lo + w + 4, .. below hi of sequence b, of which it reads the tokens below `end`
template <int D, int QUANT>
__device__ __forceinline__ void attend_blocks(const CacheArgs& a, int b, int hk, int lo, int hi, int end, const bf16x8 (&qf)[D / 32], HeadSums<D>& sums,
                                              int w, int lane) {
  constexpr int ESZ = QUANT == SLA2_QUANT_NONE ? 2 : 1;
  constexpr int KE = QUANT == SLA2_QUANT_NONE ? 8 : 16;            // channels of a 16-byte read of a key
  constexpr int KL = D / (4 * KE);                                 // reads of a key row
  constexpr int C = D / 16;                                        // channels of a lane's read of a value row
  const int g = lane / 16, n = lane % 16, slot_mask = (1 << a.page_shift) - 1;
  const float c1 = kLog2e * a.scale;
  const char* kc = (const char*)a.kc + hk * a.head_stride * ESZ;
  const char* vc = (const char*)a.vc + hk * a.head_stride * ESZ;
  f32x4(&oacc)[C] = sums.o;
  int id = -1;                                                     // the pages of the next 32 blocks, 16 tokens a lane
  for (int block = lo + w, c0 = lo - kIdBlocks; block < hi; block += kDecodeWaves) {
    if (block >= c0 + kIdBlocks) {
      c0 += kIdBlocks;
      const unsigned t = (unsigned)c0 * kDecodeBlock + 16 * lane;
      id = t < (unsigned)end ? a.table[b * a.table_stride + (t >> a.page_shift)] : -1;
    }
    const int t0 = block * kDecodeBlock, i0 = 2 * (block - c0);
    int p0 = __builtin_amdgcn_readlane(id, i0), p1 = __builtin_amdgcn_readlane(id, i0 + 1);
    const bool ok0 = p0 >= 0 && p0 < a.pages, ok1 = p1 >= 0 && p1 < a.pages;
    const bool whole = ok0 && ok1 && end - t0 >= kDecodeBlock;
    p0 = ok0 ? p0 : 0;
    p1 = ok1 ? p1 : p0;
    const int s0 = t0 & slot_mask, s1 = (t0 + 16) & slot_mask;
    const long long at0 = p0 * a.page_stride + s0 * a.token_stride, at1 = p1 * a.page_stride + s1 * a.token_stride;
    // ---- requests ----
    unsigned kw[2][KL][4], vw[8][C * ESZ / 4];
    const char* krow = kc + (n < 8 ? at0 : at1) * ESZ + 16 * g;    // tokens 8 (n / 4) + .. of the block: 16 a page at least
#pragma unroll
    for (int t = 0; t < 2; t++)
#pragma unroll
      for (int x = 0; x < KL; x++)
        load_words<16>(krow + (8 * (n / 4 % 2) + 4 * t + n % 4) * a.token_stride * ESZ + 64 * x, kw[t][x]);
    const char* vrow = vc + (g < 2 ? at0 : at1) * ESZ + C * ESZ * n;
#pragma unroll
    for (int j = 0; j < 8; j++) load_words<C * ESZ>(vrow + (8 * (g % 2) + j) * a.token_stride * ESZ, vw[j]);
    float ks[8], vs[8];
    if constexpr (QUANT != SLA2_QUANT_NONE) {
      const long long at = ((((long long)(g < 2 ? p0 : p1) * a.Hkv + hk)) << a.page_shift) + (g < 2 ? s0 : s1) + 8 * (g % 2);
#pragma unroll
      for (int x = 0; x < 2; x++) {
        const f32x4 k4 = *(const f32x4*)(a.ks + at + 4 * x), v4 = *(const f32x4*)(a.vs + at + 4 * x);
#pragma unroll
        for (int e = 0; e < 4; e++) ks[4 * x + e] = k4[e], vs[4 * x + e] = v4[e];
      }
    }
    unsigned dead = 0;                                             // tokens of this lane that have no part
    if (!whole) {
#pragma unroll
      for (int j = 0; j < 8; j++)
        if (t0 + 8 * g + j >= end || !(g < 2 ? ok0 : ok1)) dead |= 1u << j;
    }
    // ---- scores ----
    f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int t = 0; t < 2; t++)
#pragma unroll
      for (int x = 0; x < KL; x++) {
        if constexpr (QUANT == SLA2_QUANT_NONE) {
          const u32x4 k4 = {kw[t][x][0], kw[t][x][1], kw[t][x][2], kw[t][x][3]};
          s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k4), qf[x], s[t], 0, 0, 0);
        } else {
          unsigned y[8];
          widen<QUANT, 16>(kw[t][x], y);
          const u32x4 lo = {y[0], y[1], y[2], y[3]}, hi = {y[4], y[5], y[6], y[7]};
          s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, lo), qf[2 * x], s[t], 0, 0, 0);
          s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, hi), qf[2 * x + 1], s[t], 0, 0, 0);
        }
      }
    float sc[8];
#pragma unroll
    for (int j = 0; j < 8; j++) {
      sc[j] = s[j / 4][j % 4];
      if constexpr (QUANT != SLA2_QUANT_NONE) sc[j] *= ks[j];
    }
    if (!whole) {
#pragma unroll
      for (int j = 0; j < 8; j++)
        if (dead >> j & 1) {
          sc[j] = -INFINITY;
          if constexpr (QUANT != SLA2_QUANT_NONE) vs[j] = 0.f;
#pragma unroll
          for (int x = 0; x < C * ESZ / 4; x++) vw[j][x] = 0;
        }
    }
    // ---- softmax ----
    float mx = sc[0];
#pragma unroll
    for (int j = 1; j < 8; j++) mx = fmaxf(mx, sc[j]);
    mx = over_quarters_max(mx) * c1;
    if (__builtin_amdgcn_ballot_w64(mx > sums.m + 8.f)) {           // the reference is kept while the maximum stays within 2^8 of it
      const float m_new = fmaxf(sums.m, mx), corr = fast_exp2(sums.m - m_new);
      sums.m = m_new;
      sums.l *= corr;
#pragma unroll
      for (int r = 0; r < 4; r++) {
        const float cr = __shfl(corr, 4 * g + r);                  // of the head of this accumulator row
#pragma unroll
        for (int i = 0; i < C; i++) oacc[i][r] *= cr;
      }
    }
    // P (times the value's scale) as two bf16 numbers, the second what the first leaves: rounded to one, P would add half as much again to the
    // error of rounding the result, and the second product is free beside the reads.
    bf16x8 pf, pr;
#pragma unroll
    for (int j = 0; j < 8; j++) {
      float p = fast_exp2(sc[j] * c1 - sums.m);
      sums.l += p;
      if constexpr (QUANT != SLA2_QUANT_NONE) p *= vs[j];
      pf[j] = (__bf16)p;
      pr[j] = (__bf16)(p - (float)pf[j]);
    }
    // ---- O += P V ----
    unsigned vb[8][C / 2];
#pragma unroll
    for (int j = 0; j < 8; j++) {
      if constexpr (QUANT == SLA2_QUANT_NONE) {
#pragma unroll
        for (int x = 0; x < C / 2; x++) vb[j][x] = vw[j][x];
      } else {
        widen<QUANT, C>(vw[j], vb[j]);
      }
    }
#pragma unroll
    for (int i = 0; i < C; i++) {
      u32x4 v4;
#pragma unroll
      for (int x = 0; x < 4; x++)
        v4[x] = __builtin_amdgcn_perm(vb[2 * x + 1][i / 2], vb[2 * x][i / 2], i % 2 ? 0x07060302u : 0x05040100u);
      oacc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pf, __builtin_bit_cast(bf16x8, v4), oacc[i], 0, 0, 0);
      oacc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pr, __builtin_bit_cast(bf16x8, v4), oacc[i], 0, 0, 0);
    }
  }
}

template <int D, int QUANT>
__global__ __launch_bounds__(kDecodeWaves * kWave, 2) void cache_attention_kernel(CacheArgs a) {
  constexpr int KE = QUANT == SLA2_QUANT_NONE ? 8 : 16;            // channels of a 16-byte read of a key
  constexpr int KS = D / 32;                                       // products of a key row
  constexpr int C = D / 16;                                        // channels of a lane's read of a value row
  __shared__ float part[kDecodeWaves][kHeadRows][D + 4];           // a wave's O, m and l
  const int tid = threadIdx.x, lane = tid % kWave, w = __builtin_amdgcn_readfirstlane(tid / kWave), g = lane / 16, n = lane % 16;
  const int tiles = (a.group + kHeadRows - 1) / kHeadRows;         // of query heads
  const int hk = blockIdx.y / tiles, row0 = blockIdx.y % tiles * kHeadRows, rows = min(kHeadRows, a.group - row0);
  const int h0 = hk * a.group + row0;                              // first query head
  // this workgroup's stretch [x, y) of the line; without parts: one sequence
  long long x = 0, y = LLONG_MAX, at = 0;
  int b = blockIdx.x;
  if (a.parts) {
    const long long all = uniform64(line_length(a, lane));
    const int parts = parts_of(a.parts, all), p = blockIdx.x;
    if (p >= parts) return;
    x = stretch_begin(all, parts, p);
    y = stretch_begin(all, parts, p + 1);
    const OnLine o = on_line(a, x, -1, lane);
    b = __builtin_amdgcn_readfirstlane(o.b);
    at = uniform64(o.at);
  }
  const int b_end = a.parts ? a.B : b + 1;
  for (; b < b_end && at < y; b++) {
    const int len = __builtin_amdgcn_readfirstlane(tokens_of(a, b)), nb = blocks_of(len);
    const long long first = at + kOverhead;                        // the place of its first block
    const bool begins = at >= x;
    at = first + nb;
    const BlockRange r = blocks_in(x, y, first, nb);
    const int lo = r.lo, hi = r.hi;
    if (lo >= hi && !(nb == 0 && begins)) continue;
    // Q as B operand: lane <- head l % 16, the channels that its reads of a key have
    bf16x8 qf[KS];
    const uint16_t* src = a.q + (size_t)b * a.q_b + (size_t)(h0 + min(n, rows - 1)) * a.q_h;
#pragma unroll
    for (int ks = 0; ks < KS; ks++)
      qf[ks] = *reinterpret_cast<const bf16x8*>(src + (KE == 8 ? 32 * ks + 8 * g : 64 * (ks / 2) + 16 * g + 8 * (ks % 2)));
    HeadSums<D> sums;
#pragma unroll
    for (int i = 0; i < C; i++) sums.o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    sums.m = kNoScore;
    sums.l = 0.f;
    attend_blocks<D, QUANT>(a, b, hk, lo, hi, (int)min((unsigned)len, (unsigned)hi * kDecodeBlock), qf, sums, w, lane);
    // ---- the waves' parts ----
    sums.l = over_quarters_sum(sums.l);
    if (g == 0) {
      part[w][n][D] = sums.m;
      part[w][n][D + 1] = sums.l;
    }
#pragma unroll
    for (int r = 0; r < 4; r++)
      if (4 * g + r < rows) {
#pragma unroll
        for (int i = 0; i < C; i++) part[w][4 * g + r][C * n + i] = sums.o[i][r];
      }
    __syncthreads();
    for (int idx = tid; idx < rows * (D / 2); idx += kDecodeWaves * kWave) {
      const int row = idx / (D / 2), c = idx % (D / 2) * 2, h = h0 + row;
      float m = part[0][row][D];
#pragma unroll
      for (int x = 1; x < kDecodeWaves; x++) m = fmaxf(m, part[x][row][D]);
      float l = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll
      for (int x = 0; x < kDecodeWaves; x++) {
        const float by = fast_exp2(part[x][row][D] - m);
        l += by * part[x][row][D + 1];
        o0 += by * part[x][row][c];
        o1 += by * part[x][row][c + 1];
      }
      if (lo > 0 || hi < nb) {
        const size_t slot = part_slot(blockIdx.x, lo == 0) * a.H + h;
        *(float2*)(a.part_o + slot * D + c) = make_float2(o0, o1);
        if (c == 0) *(float2*)(a.part_ml + 2 * slot) = make_float2(m, l);
      } else {
        const bool any = l != 0.f;
        const float inv = any ? 1.f / l : 0.f;
        typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
        *(bf16x2*)(a.out + (size_t)b * a.out_b + (size_t)h * a.out_h + c) = bf16x2{(__bf16)(any ? o0 * inv : 0.f), (__bf16)(any ? o1 * inv : 0.f)};
        if (a.lse && c == 0) a.lse[(size_t)b * a.H + h] = any ? (m + log2f(l)) * (1.f / kLog2e) : -INFINITY;
      }
    }
    __syncthreads();
  }
}

// A sequence and head whose blocks several workgroups had: their O, weighted with 2^(m - the largest m), over their l, weighted alike.
// W of a workgroup's 8 waves for each head.
constexpr int kJoinWaves = 8;
template <int D, int W>
__global__ __launch_bounds__(kJoinWaves * kWave) void cache_join_kernel(CacheArgs a) {
  constexpr int E = D / kWave;                                     // channels of a lane
  __shared__ float part[kJoinWaves][D + 1];
  const int lane = threadIdx.x % kWave, w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), b = blockIdx.y;
  const int h = blockIdx.x * (kJoinWaves / W) + w / W;
  const int nb = blocks_of(tokens_of(a, b));
  if (!nb) return;
  const long long all = line_length(a, lane), first = on_line(a, 0, b, lane).at + kOverhead;
  const int parts = parts_of(a.parts, all), p0 = part_at(all, parts, first), p1 = part_at(all, parts, first + nb - 1);
  if (p0 == p1) return;                                            // written by the one that had it
  auto slot = [&](int p) { return part_slot(p, p == p0) * a.H + h; };
  float m = -INFINITY, l = 0.f, o[E] = {};
  if (h < a.H) {
    for (int p = p0 + lane; p <= p1; p += kWave) m = fmaxf(m, a.part_ml[2 * slot(p)]);
    m = wave_max(m);
#pragma unroll 4
    for (int p = p0 + w % W; p <= p1; p += W) {
      const float2 ml = *(const float2*)(a.part_ml + 2 * slot(p));
      const float by = fast_exp2(ml.x - m);
      l += by * ml.y;
#pragma unroll
      for (int e = 0; e < E; e++) o[e] += by * a.part_o[slot(p) * D + E * lane + e];
    }
  }
  if (W > 1) {
#pragma unroll
    for (int e = 0; e < E; e++) part[w][E * lane + e] = o[e];
    if (lane == 0) part[w][D] = l;
    __syncthreads();
    if (w) return;
#pragma unroll
    for (int x = 1; x < W; x++) {
      l += part[x][D];
#pragma unroll
      for (int e = 0; e < E; e++) o[e] += part[x][E * lane + e];
    }
  }
  if (h >= a.H) return;
  const bool any = l != 0.f;
  uint16_t* dst = a.out + (size_t)b * a.out_b + (size_t)h * a.out_h + E * lane;
#pragma unroll
  for (int e = 0; e < E; e++) dst[e] = __builtin_bit_cast(uint16_t, (__bf16)(any ? o[e] / l : 0.f));
  if (a.lse && lane == 0) a.lse[(size_t)b * a.H + h] = any ? (m + log2f(l)) * (1.f / kLog2e) : -INFINITY;
}

void plan_cache_attention(CacheArgs* a) {
  a->parts = most_parts(a->B, (long long)a->max_pages << a->page_shift, (long long)a->Hkv * ((a->group + kHeadRows - 1) / kHeadRows));
}

hipError_t launch_cache_attention(const CacheArgs& a, hipStream_t stream) {
  const dim3 grid(a.parts ? a.parts : a.B, a.Hkv * ((a.group + kHeadRows - 1) / kHeadRows));
#define SLA2_DECODE(D)                                                                                                          \
  (a.quant == SLA2_QUANT_NONE  ? cache_attention_kernel<D, SLA2_QUANT_NONE><<<grid, kDecodeWaves * kWave, 0, stream>>>(a)       \
   : a.quant == SLA2_QUANT_FP8 ? cache_attention_kernel<D, SLA2_QUANT_FP8><<<grid, kDecodeWaves * kWave, 0, stream>>>(a)        \
                               : cache_attention_kernel<D, SLA2_QUANT_INT8><<<grid, kDecodeWaves * kWave, 0, stream>>>(a))
  if (a.d == 128) SLA2_DECODE(128);
  else SLA2_DECODE(64);
#undef SLA2_DECODE
  if (hipError_t e = hipGetLastError(); e != hipSuccess || a.parts <= 1) return e;
  // few sequences and heads: all waves of a workgroup for one, so that its parts are read at once
  const bool few = (long long)a.B * a.H < 1024;
  const dim3 join(few ? a.H : (a.H + kJoinWaves - 1) / kJoinWaves, a.B);
#define SLA2_JOIN(D)                                                                                    \
  (few ? cache_join_kernel<D, kJoinWaves><<<join, kJoinWaves * kWave, 0, stream>>>(a)                   \
       : cache_join_kernel<D, 1><<<join, kJoinWaves * kWave, 0, stream>>>(a))
  if (a.d == 128) SLA2_JOIN(128);
  else SLA2_JOIN(64);
#undef SLA2_JOIN
  return hipGetLastError();
}

}  // namespace sla2
