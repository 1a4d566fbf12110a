// What the attention kernels of several query tokens per sequence share: operand types, unpacking of codes into binary16, the staging of
// the query.
#pragma once
#include "kvq_internal.h"
#include "kvq_quantizer.h"

namespace kvq {
namespace {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNoMax = -1.0e30f;
constexpr int kRec = kHeadDim + 4;       // floats of a partial record: 128 sums, maximum, weight sum

__device__ __forceinline__ half2v as_half2(uint32_t x) { return __builtin_bit_cast(half2v, x); }
__device__ __forceinline__ uint32_t as_u32(half2v x) { return __builtin_bit_cast(uint32_t, x); }
// A binary32 value whose two binary16 parts are formed next.  Left to itself the compiler merges the operation that made it with the rounding
// of the first part (one rounding instead of two, the other side of a tie), but not with the difference that becomes the second.
__device__ __forceinline__ float as_rounded(float x) { asm("" : "+v"(x)); return x; }
__device__ __forceinline__ float other_half(float x) {           // lane ^ 32's value
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}
// Two whole numbers below 1024 in the halves of x (masked out of it) -> the same as binary16: the pattern of 1024 + x, less 1024.
// `one_k` is that pattern, 1024 in both halves, in a vector register of its own: mask and pattern together are then one instruction, which
// takes no two constants.
__device__ __forceinline__ uint32_t one_k_pattern() { uint32_t x = 0x64006400u; asm("" : "+v"(x)); return x; }
__device__ __forceinline__ half2v whole_to_half2(uint32_t x, uint32_t mask, uint32_t one_k) {
  return as_half2((x & mask) | one_k) - half2v{(_Float16)1024.0f, (_Float16)1024.0f};
}
// Two patterns of the unquantized type -> binary16 (bfloat16: exact in binary16's normal range)
__device__ __forceinline__ uint32_t raw_to_half2(uint32_t x, bool bf) {
  if (!bf) return x;
  half2v h;
  h[0] = (_Float16)__uint_as_float(x << 16);
  h[1] = (_Float16)__uint_as_float(x & 0xFFFF0000u);
  return as_u32(h);
}

// Channel order inside a 32-channel chunk of an unpacked key row: with P = 16 / (field width), field pair (p, p + P) of dword w is
// slots 2 (w P + p) and + 1.  The slot of channel x (0..31):
__device__ __forceinline__ int key_slot(int x, int per) {
  const int w = x / (2 * per), rem = x % (2 * per);
  return 2 * (w * per + rem % per) + rem / per;
}
__device__ __forceinline__ int key_fields(int bits) { return bits == 3 ? 8 : bits == 6 ? 4 : 16 / bits; }

// Query rows [row0, row0 + n) of a kv head (row = query token * heads_per_kv + head; rows behind the last repeat it) to LDS, by 16 lanes a
// row: binary16 in slot order, 256 bytes a row whose 16-byte pieces are permuted by the row's number (piece p at p ^ (r & 15)); the sums of
// ng equal parts of the row (4 at most), each as two binary16 parts (`parts`, may be null) or in binary32 (`sums`, may be null); and the factor of the row's scores (every row is scaled by a power of two).
template <int THREADS>
__device__ __forceinline__ void stage_query(const ChunkArgs& a, int b, int h, int row0, int rows, int n, int ng, uint8_t* dst, uint32_t (*parts)[4],
                                            float (*sums)[4], float* kappa) {
  const Geom& g = a.g;
  const int tid = threadIdx.x, lane = tid & 63, lane16 = tid & 15, d0 = 8 * lane16, R = a.heads_per_kv;
  const int fields = key_fields(g.bits_k);
  // (read out one by one: a choice among words of the argument block may become a table in private memory)
  uint32_t words[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) words[i] = __builtin_amdgcn_readfirstlane(g.signs_k[i]);
  const int w = lane16 >> 2;
  const uint32_t signs = ((w == 0 ? words[0] : w == 1 ? words[1] : w == 2 ? words[2] : words[3]) >> (8 * (lane16 & 3))) & 0xFFu;
  for (int r = tid >> 4; r < n; r += THREADS / 16) {
    const int row = min(row0 + r, rows - 1);
    const int i = row / R, hq = h * R + row % R;
    const uint4 raw = *reinterpret_cast<const uint4*>(a.q + (b * a.q_sb + i * a.q_st + hq * a.q_sh + d0));
    const uint32_t rw[4] = {raw.x, raw.y, raw.z, raw.w};
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = widen16((uint16_t)(rw[e >> 1] >> (16 * (e & 1))), a.q_bf16);
    if (g.rotate_k) rotate8(x, lane16, signs);
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) { x[e] = (float)(_Float16)x[e]; sum += x[e]; }
    sum += lane_xor<1>(sum);
    sum += lane_xor<2>(sum);
    if (ng <= 2) sum += lane_xor<4>(sum);
    if (ng == 1) sum += lane_xor<8>(sum);
    // Every row is scaled by a power of two that takes its largest element or sum to [2^13, 2^14): sums then fit binary16, and no element that
    // counts is a subnormal (next to codes that are, the matrix unit loses those).  Elements below 2^-27 of the largest lose bits.
    float most = fabsf(sum);
#pragma unroll
    for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(x[e]));
    most = fmaxf(most, lane_xor<1>(most));
    most = fmaxf(most, lane_xor<2>(most));
    most = fmaxf(most, lane_xor<4>(most));
    most = fmaxf(most, lane_xor<8>(most));
    const int up = 127 + 13 - max((int)(__float_as_uint(most) >> 23), 90);   // (rows of zeros: any factor will do)
    const float unit = __uint_as_float((uint32_t)(127 + up) << 23);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int slot = (d0 & ~31) + key_slot((d0 & 31) + e, fields);
      const int at = (((slot >> 3) ^ (r & 15)) << 4) + (slot & 7) * 2;
      *reinterpret_cast<_Float16*>(dst + r * 256 + at) = (_Float16)(x[e] * unit);
    }
    if (lane16 == 0) kappa[r] = a.softmax_scale * kLog2e * __uint_as_float((uint32_t)(127 - up) << 23);
    const int q = lane16 >> 2;                         // part q's sum: in lane 16 q / ng of the row (all lanes take part)
    const float group_sum = __shfl(sum, (lane & ~15) + (ng == 1 ? 0 : ng == 2 ? 8 * (q & 1) : 4 * q));
    if ((lane16 & 3) == 0) {
      const float mine = q < ng ? group_sum * unit : 0.0f;
      half2v p;
      p[0] = (_Float16)mine;
      p[1] = (_Float16)(mine - (float)p[0]);
      if (parts) parts[r][q] = as_u32(p);
      if (sums) sums[r][q] = mine;
    }
  }
}

// One output element group: four neighbouring channels at element o in the caller's type (16-bit types: rounded once).
__device__ __forceinline__ void store_out4(void* out, int out_dtype, int64_t o, const float (&y)[4]) {
  if (out_dtype == KVQ_F32) *reinterpret_cast<float4v*>((float*)out + o) = float4v{y[0], y[1], y[2], y[3]};
  else {
    uint2 w;
    if (out_dtype == KVQ_F16) {
      half2v u, t;
      u[0] = (_Float16)y[0]; u[1] = (_Float16)y[1]; t[0] = (_Float16)y[2]; t[1] = (_Float16)y[3];
      w = make_uint2(as_u32(u), as_u32(t));
    } else {
      w = make_uint2(f32_to_bf16_bits(y[0]) | (uint32_t)f32_to_bf16_bits(y[1]) << 16, f32_to_bf16_bits(y[2]) | (uint32_t)f32_to_bf16_bits(y[3]) << 16);
    }
    *reinterpret_cast<uint2*>((uint16_t*)out + o) = w;
  }
}

// ---- partial records: [row][split][kRec], a row's 128 sums, its maximum and its weight sum.  They travel between workgroups that may sit on
// different parts of the chip, so stores and loads are device-scope atomic accesses, two floats each.
__device__ __forceinline__ void store_record2(float* p, float x, float y) {
  const uint64_t w = (uint64_t)__float_as_uint(x) | (uint64_t)__float_as_uint(y) << 32;
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 load_record2(const float* p) {
  const uint64_t w = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((uint32_t)w), __uint_as_float((uint32_t)(w >> 32)));
}
// The rules of kvq_merge_count.h.  One thread calls merge_announce before its workgroup stores records; all threads call merge_arrive behind
// their stores: true (in all of them) in the workgroup that brings the count to `records`.
__device__ __forceinline__ void merge_announce(MergeWord* word, MergeWord tag) {
  (void)__hip_atomic_fetch_max(word, tag, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ bool merge_arrive(MergeWord* word, MergeWord tag, int records, int tid, int* flag) {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");   // (keeps the compiler from moving a store behind the wait)
  __builtin_amdgcn_s_waitcnt(0x0F70);                      // vmcnt(0): this wavefront's record stores are performed
  __syncthreads();                                         // (and so are the other wavefronts')
  if (tid == 0) {
    MergeWord before = __hip_atomic_fetch_add(word, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (merge_unmarked(before, tag)) {                     // (rare; a swap fails only because another workgroup got on)
      MergeWord seen = before + 1;
      while (merge_unmarked(seen, tag) &&
             !__hip_atomic_compare_exchange_strong(word, &seen, tag | 1ull, __ATOMIC_RELAXED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) {}
      before = merge_unmarked(seen, tag) ? tag : __hip_atomic_fetch_add(word, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    const bool last = merge_last(before, records);
    if (last) __hip_atomic_store(word, tag, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *flag = last;
  }
  __syncthreads();
  return *flag;
}
// Rows [row0, row0 + n) of a kv head from their `parts` records: 32 threads a row, four channels each, four records at a time under a running maximum.
template <int THREADS>
__device__ __forceinline__ void merge_rows(const ChunkArgs& a, int b, int h, int row0, int n, int parts, int tid) {
  const int R = a.heads_per_kv;
  for (int idx = tid; idx < 32 * n; idx += THREADS) {
    const int row = row0 + (idx >> 5), d = 4 * (idx & 31);
    const int64_t hq = ((int64_t)b * a.n_q + row / R) * a.q_heads + h * R + row % R;
    const float* rec = a.ws + hq * a.splits * kRec;
    float m = kNoMax, l = 0.0f, y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s0 = 0; s0 < parts; s0 += 4) {
      float2 ml[4], u[4], v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float* r = rec + min(s0 + k, parts - 1) * kRec;
        ml[k] = load_record2(r + kHeadDim); u[k] = load_record2(r + d); v[k] = load_record2(r + d + 2);
      }
      float top = m;
#pragma unroll
      for (int k = 0; k < 4; ++k) top = s0 + k < parts ? fmaxf(top, ml[k].x) : top;
      const float f0 = __builtin_amdgcn_exp2f(m - top);
      l *= f0;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] *= f0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float f = s0 + k < parts ? __builtin_amdgcn_exp2f(ml[k].x - top) : 0.0f;
        l = fmaf(f, ml[k].y, l);
        y[0] = fmaf(f, u[k].x, y[0]); y[1] = fmaf(f, u[k].y, y[1]); y[2] = fmaf(f, v[k].x, y[2]); y[3] = fmaf(f, v[k].y, y[3]);
      }
      m = top;
    }
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;          // (a row that sees nothing: zeros)
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] *= inv;
    store_out4(a.out, a.out_dtype, hq * kHeadDim + d, y);
  }
}

}  // namespace
}  // namespace kvq
