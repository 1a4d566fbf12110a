// Shapes of the kernel for a few query rows (kvq_few.hip) that its launches and the plan need.
#pragma once
#include "kvq_internal.h"

namespace kvq {

// Column sets of 16 rows (query token, query head) a workgroup takes at most: three where their sums and a block's registers fit.
constexpr int few_max_sets(int bits_k, int bits_v, int groups) { return bits_k + bits_v <= 8 && groups <= 2 ? 3 : 2; }

constexpr int kFewWaves = 8;
template <int B> constexpr int key_loads() { return (32 * B + 63) / 64; }            // 16-byte loads of a lane for 32 key rows
// Wavefronts per SIMD that the registers are cut for (512 of them a SIMD): the sums take 32 per column set, the next block 2 (b_K + b_V), the
// rest about 80.
constexpr int few_occupancy(int BK, int BV, int NC, int NG) {
  const bool odd = BK == 3 || BK == 6 || BV == 3 || BV == 6 || BK == 1 || BV == 1;          // (codes in two runs, lanes that share a word)
  return NC > 1 || BK + BV > 16 || (NG == 4 && BK + BV > 12) ? 2 : NG == 4 || odd || BK + BV > 8 || (NG == 1 && BK + BV > 6) ? 3 : 4;
}
// LDS of a wavefront: a block's keys, values, scales and zeros
template <int BK, int BV> constexpr int few_wave_bytes() { return 512 * BK + 512 * BV + (BK == 16 && BV == 16 ? 0 : 1024); }
// the wavefronts' sums are joined through LDS in so many parts
template <int NC> constexpr int few_join_parts() { return NC > 2 ? 2 : 1; }
template <int BK, int BV, int NC> constexpr int few_lds_bytes() {
  constexpr int walk = kFewWaves * few_wave_bytes<BK, BV>(), join = kFewWaves * 16 * NC * (kHeadDim / few_join_parts<NC>() + 4) * 4;
  return walk > join ? walk : join;
}

// One launcher per pair of widths (the units of kvq_few.hip); sets: column sets of 16 rows a workgroup takes, 1 to few_max_sets.
#define KVQ_FEW_VALUES(X, k) X(k, 1) X(k, 2) X(k, 3) X(k, 4) X(k, 6) X(k, 8) X(k, 16)
#define KVQ_FEW_PAIRS(X) KVQ_FEW_VALUES(X, 1) KVQ_FEW_VALUES(X, 2) KVQ_FEW_VALUES(X, 3) KVQ_FEW_VALUES(X, 4) KVQ_FEW_VALUES(X, 6) \
  KVQ_FEW_VALUES(X, 8) KVQ_FEW_VALUES(X, 16)
#define KVQ_FEW_DECLARE(k, v) hipError_t launch_few_k##k##v##v(const ChunkArgs& a, int sets, hipStream_t stream);
KVQ_FEW_PAIRS(KVQ_FEW_DECLARE)

#if defined(__HIPCC__)
// A lane's piece of a 32-token value block (16-byte pieces 1 KB apart; 1-bit fields: 8 bytes; 3 and 6 bits: low fields, then high ones)
template <int B> __device__ __forceinline__ void load_value_piece(uint32_t* w, const uint8_t* block, int lane) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  if constexpr (B == 3) {
    load_value_piece<2>(w, block, lane);
    load_value_piece<1>(w + 4, block + 1024, lane);
  } else if constexpr (B == 6) {
    load_value_piece<4>(w, block, lane);
    load_value_piece<2>(w + 8, block + 2048, lane);
  } else if constexpr (B == 1) {
    const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(block + 8 * lane));
    w[0] = x[0]; w[1] = x[1];
  } else {
#pragma unroll
    for (int i = 0; i < B / 2; ++i) {
      const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(block + 1024 * i + 16 * lane));
#pragma unroll
      for (int e = 0; e < 4; ++e) w[4 * i + e] = x[e];
    }
  }
}
// The same piece, stored in and read from a block in LDS.
template <int B> __device__ __forceinline__ void store_value_piece(const uint32_t* w, uint8_t* block, int lane) {
  if constexpr (B == 3) {
    store_value_piece<2>(w, block, lane);
    store_value_piece<1>(w + 4, block + 1024, lane);
  } else if constexpr (B == 6) {
    store_value_piece<4>(w, block, lane);
    store_value_piece<2>(w + 8, block + 2048, lane);
  } else if constexpr (B == 1) {
    *reinterpret_cast<uint2*>(block + 8 * lane) = make_uint2(w[0], w[1]);
  } else {
#pragma unroll
    for (int i = 0; i < B / 2; ++i) *reinterpret_cast<uint4*>(block + 1024 * i + 16 * lane) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  }
}
template <int B> __device__ __forceinline__ void read_value_piece(uint32_t* w, const uint8_t* block, int lane) {
  if constexpr (B == 3) {
    read_value_piece<2>(w, block, lane);
    read_value_piece<1>(w + 4, block + 1024, lane);
  } else if constexpr (B == 6) {
    read_value_piece<4>(w, block, lane);
    read_value_piece<2>(w + 8, block + 2048, lane);
  } else if constexpr (B == 1) {
    const uint2 x = *reinterpret_cast<const uint2*>(block + 8 * lane);
    w[0] = x.x; w[1] = x.y;
  } else {
#pragma unroll
    for (int i = 0; i < B / 2; ++i) {
      const uint4 x = *reinterpret_cast<const uint4*>(block + 1024 * i + 16 * lane);
      w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
    }
  }
}
#endif

}  // namespace kvq
