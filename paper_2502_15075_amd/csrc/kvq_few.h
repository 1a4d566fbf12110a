// Shapes of the kernel for a few query rows (kvq_few.hip) that its launches and the plan need.
#pragma once
#include "kvq_internal.h"

namespace kvq {

constexpr int kFewRows = 32;                       // rows (query token, query head) of a workgroup, in column sets of 16

template <int B> constexpr int key_loads() { return (32 * B + 63) / 64; }            // 16-byte loads of a lane for 32 key rows
template <int BK, int BV> constexpr int few_step_regs() { return 4 * key_loads<BK>() + 2 * BV + 4; }
// wavefronts of a workgroup: eight, four where the registers or the LDS of eight would not fit
template <int BK, int BV, int NC> constexpr int few_waves() { return BK + BV > 16 ? 4 : 8; }
// steps in flight per wavefront
template <int BK, int BV, int NC> constexpr int few_stages() { return NC == 1 && few_step_regs<BK, BV>() <= 40 ? 2 : 1; }
template <int BK, int BV> constexpr int few_wave_bytes() { return 1024 * key_loads<BK>() + (BK == 16 && BV == 16 ? 0 : 1024); }
template <int BK, int BV, int NC> constexpr int few_lds_bytes() {
  constexpr int NW = few_waves<BK, BV, NC>();
  constexpr int walk = NW * few_wave_bytes<BK, BV>(), join = NW / 2 * NC * 64 * 38 * 4, query = 16 * NC * 256;
  return walk > join ? (walk > query ? walk : query) : (join > query ? join : query);
}

// One launcher per pair of widths (the units of kvq_few.hip); sets: column sets of 16 rows a workgroup takes, 1 or 2.
#define KVQ_FEW_VALUES(X, k) X(k, 1) X(k, 2) X(k, 3) X(k, 4) X(k, 6) X(k, 8) X(k, 16)
#define KVQ_FEW_PAIRS(X) KVQ_FEW_VALUES(X, 1) KVQ_FEW_VALUES(X, 2) KVQ_FEW_VALUES(X, 3) KVQ_FEW_VALUES(X, 4) KVQ_FEW_VALUES(X, 6) \
  KVQ_FEW_VALUES(X, 8) KVQ_FEW_VALUES(X, 16)
#define KVQ_FEW_DECLARE(k, v) hipError_t launch_few_k##k##v##v(const ChunkArgs& a, int sets, hipStream_t stream);
KVQ_FEW_PAIRS(KVQ_FEW_DECLARE)

#if defined(__HIPCC__)
// A lane's piece of a 32-token value block (16-byte pieces 1 KB apart; 1-bit fields: 8 bytes; 3 and 6 bits: low fields, then high ones)
template <int B> __device__ __forceinline__ void load_value_piece(uint32_t* w, const uint8_t* block, int lane, uint32_t live) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  if constexpr (B == 3) {
    load_value_piece<2>(w, block, lane, live);
    load_value_piece<1>(w + 4, block + 1024, lane, live);
  } else if constexpr (B == 6) {
    load_value_piece<4>(w, block, lane, live);
    load_value_piece<2>(w + 8, block + 2048, lane, live);
  } else if constexpr (B == 1) {
    const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(block + ((8u * lane) & live)));
    w[0] = x[0]; w[1] = x[1];
  } else {
#pragma unroll
    for (int i = 0; i < B / 2; ++i) {
      const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(block + ((1024u * i + 16u * lane) & live)));
#pragma unroll
      for (int e = 0; e < 4; ++e) w[4 * i + e] = x[e];
    }
  }
}
#endif

}  // namespace kvq
