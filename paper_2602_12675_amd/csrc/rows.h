// Rows of channels in registers: what the kernels around the attention share (sla2_rope.hip, sla2_norm.hip).
//
// A row (the channels of a token, or of some of its heads) is read once, in chunks of 8 channels, by a team: `lanes` neighbouring lanes
// of a wave (8, 16, 32 or 64), or several whole waves, each thread holding V chunks, chunk l + v T being thread l's of T.  Everything
// these kernels do is bound by memory, so a row stays in registers from its load to the store of what is made of it, and a workgroup
// goes on with other rows of the same batch, whose modulation, gate or weights it then holds already, in registers or LDS.  What keeps
// memory busy is the bytes that a CU's waves have on their way: forward kernels hold up to 3 chunks a thread (32,760 rows of 1,536
// channels before a block: 92 us as one chunk in three waves, 56 us as three in one), backward kernels, whose sums for the column
// gradients stay in registers, one.  The sums of a row are kept in fp32; within a wave they are vector instructions only, and where a
// team has several waves these exchange all sums of a step through LDS at once, behind one barrier.
#pragma once
#include "row_plan.h"

namespace sla2 {

// 8 neighbouring elements as they are stored, and as fp32.
template <bool BF16> struct Raw {
  u32x4 a[BF16 ? 1 : 2];
};
typedef __attribute__((ext_vector_type(8))) float f32x8;
template <bool BF16> constexpr size_t elem_bytes() { return BF16 ? 2 : 4; }
// element `elem` of a tensor
template <bool BF16, class T> __device__ __forceinline__ T* at_elem(T* p, long long elem) {
  return (T*)((const char*)p + elem * (long long)elem_bytes<BF16>());
}
template <bool BF16, class Offset> __device__ __forceinline__ Raw<BF16> load8(const void* p, Offset elem) {     // unsigned: 32 bits beside a scalar address
  const u32x4* a = (const u32x4*)((const char*)p + elem * (Offset)elem_bytes<BF16>());
  Raw<BF16> r;
  r.a[0] = a[0];
  if constexpr (!BF16) r.a[1] = a[1];
  return r;
}
template <bool BF16> __device__ __forceinline__ Raw<BF16> zero8() {
  Raw<BF16> r;
  r.a[0] = u32x4{0, 0, 0, 0};
  if constexpr (!BF16) r.a[1] = u32x4{0, 0, 0, 0};
  return r;
}
template <bool BF16, class Offset> __device__ __forceinline__ void store8(void* p, Offset elem, const Raw<BF16>& r) {
  u32x4* a = (u32x4*)((char*)p + elem * (Offset)elem_bytes<BF16>());
  a[0] = r.a[0];
  if constexpr (!BF16) a[1] = r.a[1];
}
// Results.  bf16: past the caches, in whole cache lines a wave.  fp32: a wave's two stores share their lines, which the cache has to join.
template <bool BF16, class Offset> __device__ __forceinline__ void put8(void* p, Offset elem, const Raw<BF16>& r) {
  if constexpr (BF16) store_streamed((u32x4*)((char*)p + elem * (Offset)2), r.a[0]);
  else store8<false>(p, elem, r);
}
template <bool BF16> __device__ __forceinline__ void unpack8(const Raw<BF16>& r, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; i++) {
    const unsigned u = BF16 ? r.a[0][i / 2] : r.a[i / 4 % (BF16 ? 1 : 2)][i % 4];
    x[i] = __builtin_bit_cast(float, !BF16 ? u : i % 2 ? u & 0xffff0000u : u << 16);
  }
}
template <bool BF16> __device__ __forceinline__ Raw<BF16> pack8(const float (&x)[8]) {   // bf16: to the nearest, ties to even
  Raw<BF16> r;
  if constexpr (BF16) {
    const f32x8 f = {x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]};
    r.a[0] = __builtin_bit_cast(u32x4, __builtin_convertvector(f, bf16x8));
  } else {
    r.a[0] = __builtin_bit_cast(u32x4, f32x4{x[0], x[1], x[2], x[3]});
    r.a[1] = __builtin_bit_cast(u32x4, f32x4{x[4], x[5], x[6], x[7]});
  }
  return r;
}
// The compiler takes r to be another value from here on, so that what is unpacked from it is unpacked again rather than kept.
template <bool BF16> __device__ __forceinline__ void unpack_again(Raw<BF16>& r) {
  if constexpr (BF16) asm volatile("" : "+v"(r.a[0]));
}
// 8 fp32 values of a vector of channels that may be absent
__device__ __forceinline__ void load_vector8(const float* p, unsigned elem, float absent, float (&x)[8]) {
  if (p) {
    unpack8<false>(load8<false>(p, elem), x);
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] = absent;
  }
}

// x and that of another lane of its 16, added in one instruction: every lane of these patterns has a source, so what an absent one would
// give does not matter, and the compiler may put the move into the addition.
template <int CTRL> __device__ __forceinline__ float dpp_add(float x) {
  return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float sum8(float x) { return dpp_add<0x141>(dpp_add<0x4E>(dpp_add<0xB1>(x))); }      // quad_perm 1 0 3 2, 2 3 0 1, row_half_mirror
__device__ __forceinline__ float sum16(float x) { return dpp_add<0x140>(sum8(x)); }                               // row_mirror
// Sum over `lanes` neighbouring lanes (8, 16, 32, 64; the same for the whole launch), on all of them.
__device__ __forceinline__ float lanes_sum(float x, int lanes) {
  x = sum8(x);
  if (lanes > 8) x = dpp_add<0x140>(x);
  if (lanes > 16) {
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    x = __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
  }
  if (lanes > 32) x = swap_halves_sum(x);
  return x;
}

// 1 / sqrt(x) to a step of fp32; x is at least a normal number (eps is)
__device__ __forceinline__ float inv_sqrt(float x) { return __builtin_amdgcn_rsqf(x); }

// A thread's place in its team, and its team's among those of the workgroup.  Every thread of a workgroup takes part in every exchange, so
// all its teams make equally many steps.  What is the same for a wave is in scalar registers: the rows' addresses above all.
constexpr int kExchange = 4;                 // sums that a step exchanges at most
constexpr int kExchangeFloats = 2 * (kMaxThreads / kWave) * kExchange;
struct Team {
  RowTeam t;
  int team, lane;                            // team of the workgroup; thread of the team
  int first, sub;                            // the first team of the wave; how far behind it this thread's is
  float* lds;                                // kExchangeFloats floats
  int flip = 0;
  __device__ Team(const RowTeam& t_, float* lds_) : t(t_), lds(lds_) {
    team = (int)threadIdx.x / t.threads();
    lane = (int)threadIdx.x - team * t.threads();
    first = __builtin_amdgcn_readfirstlane(team);
    sub = team - first;
  }
  // x[k] of wave l % 16 of the team on lane l (0 where there is no such wave), behind a barrier: one read of LDS, and what is done with the
  // waves' values is done by 16 lanes side by side.  Two buffers in turn: the next exchange but one writes over this one's, behind the barrier
  // of the next, which every wave reaches after its reads.
  template <int K> __device__ __forceinline__ void exchange(float (&x)[K]) {
    static_assert(K <= kExchange, "");
    float* m = lds + flip;
    flip ^= kExchangeFloats / 2;
    const int wave = (int)threadIdx.x / kWave, other = (int)threadIdx.x % 16;
    if ((int)threadIdx.x % kWave == 0) {
#pragma unroll
      for (int k = 0; k < K; k++) m[wave * kExchange + k] = x[k];
    }
    __syncthreads();
    const float* o = m + (first * t.waves + (other < t.waves ? other : 0)) * kExchange;
#pragma unroll
    for (int k = 0; k < K; k++) x[k] = other < t.waves ? o[k] : 0.f;
  }
  // sums over the team
  template <int K> __device__ __forceinline__ void sum(float (&x)[K]) {
#pragma unroll
    for (int k = 0; k < K; k++) x[k] = lanes_sum(x[k], t.lanes);
    if (t.waves == 1) return;
    exchange(x);
#pragma unroll
    for (int k = 0; k < K; k++) x[k] = sum16(x[k]);
  }
  // channels that wave w of the team holds of a row of `chunks` chunks
  __device__ __forceinline__ int channels(int w, int chunks) const {
    int n = 0;
    for (int v = 0; v < t.vec; v++) {
      const int left = chunks - v * t.threads() - w * kWave;
      n += left < 0 ? 0 : left > kWave ? kWave : left;
    }
    return n * kChunk;
  }
};

// The sum of acc over the parts of a workgroup, one chunk of a part's `width` values a thread, left with part 0: halves of what remains are
// added through LDS, [parts - 1][width], in the same order every time.  All threads call it, and what was in LDS has been read behind it.
// 64 parts, two sums (the gradients of a norm of 64 tokens of 64 channels): 6.2 us, with one part after the other 9.5.
__device__ __forceinline__ void join_parts(float* lds, int part, int parts, int width, unsigned col, bool has, float (&acc)[8]) {
  if (parts < 2) return;
  __syncthreads();
  int half = 1;
  while (2 * half < parts) half *= 2;
  for (; half > 0; half /= 2) {
    if (has && part >= half && part < 2 * half && part < parts) store8<false>(lds, (unsigned)((part - 1) * width) + col, pack8<false>(acc));
    __syncthreads();
    if (has && part < half && part + half < parts) {
      float o[8];
      load_vector8(lds, (unsigned)((part + half - 1) * width) + col, 0.f, o);
#pragma unroll
      for (int i = 0; i < 8; i++) acc[i] += o[i];
    }
  }
}

// ---- sums of the columns of a matrix, as both backward passes end:
//      out[c] = (factor_plus + factor[c]) * sum over rows of (weight_plus + weight[row][c]) rows[row][c] ----
struct ColumnJob {
  const float* rows;                         // [batches][count][columns]
  int batches, count;
  const float* factor;                       // [columns], or null: 1
  float factor_plus;
  const float* weight;                       // a vector of channels for every `per_weight` rows, weight_stride apart; null: 1
  float weight_plus;
  int per_weight;
  long long weight_stride;
  float* out;                                // [batches], out_stride apart
  long long out_stride;
};
constexpr int kMaxJobs = 5;
struct ColumnJobs {
  int jobs, columns, items;                  // items: workgroups, filled in by the launch
  ColumnJob job[kMaxJobs];
};
hipError_t launch_column_sums(const ColumnJobs& j, hipStream_t stream);

// ---- q and k: RMS norm and rotation ----
hipError_t launch_rope(const RopeArgs& a, hipStream_t stream);
hipError_t launch_rope_bwd(const RopeArgs& a, hipStream_t stream);

// ---- norms around a block ----
hipError_t launch_norm(const NormArgs& a, hipStream_t stream);
hipError_t launch_norm_bwd(const NormArgs& a, hipStream_t stream);

}  // namespace sla2
