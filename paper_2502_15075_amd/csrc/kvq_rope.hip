// Append of several tokens per sequence, each sequence at its own position, with the rotation of their positions applied on the
// way (gfx950): queries and keys are rotated in binary32, queries rounded once and handed back, keys and values quantized and stored as
// kvq_quantize_append stores them.  Bound by the bytes: a row is read once from memory and written once, whatever its bits.  65536 tokens of 32 query
// and 8 kv heads, 8/8 bits: 1.2 GB in 240 to 255 us, 4.8 to 5.0 TB/s, where a copy of 1 to 4 GiB reaches 4.8 to 5.1; a query head after the other,
// loaded when its turn came, took 281.  Short calls are a chain of trips to memory: position, page, rows, the words a new code shares.
//
// A pair (x1, x2) of a row becomes (x1 c - x2 s, x2 c + x1 s).  Sixteen lanes hold a row, eight channels each; a lane reads its partners'
// eight channels once more (from the caches) instead of exchanging them between lanes, which keeps every rotary width alike.
// Contraction is off in this file: every operation is rounded once, so that codes do not depend on the compiler.
#include "kvq_stage.h"

namespace kvq {
namespace {

constexpr int kRopeSpan = 32;                      // tokens a workgroup covers: one block of value codes

// cos and sin of the eight channels of a lane at one position, signs included: y = x c + partner s
struct Turn { float c[8], s[8]; };
__device__ __forceinline__ Turn load_turn(const RopeArgs& a, int64_t p, int d0) {
  Turn t;
  const int half = a.rotary >> 1;
  if (a.interleaved) {
    const int at = min(d0, a.rotary - 8) >> 1;
    const float4 c = *reinterpret_cast<const float4*>(a.cos_t + p * half + at), s = *reinterpret_cast<const float4*>(a.sin_t + p * half + at);
    const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) { t.c[e] = cc[e >> 1]; t.s[e] = e & 1 ? ss[e >> 1] : -ss[e >> 1]; }
  } else {
    const int d = min(d0, a.rotary - 8), at = d < half ? d : d - half;
    const uint32_t flip = d < half ? 0x80000000u : 0u;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float4 c = *reinterpret_cast<const float4*>(a.cos_t + p * half + at + 4 * i), s = *reinterpret_cast<const float4*>(a.sin_t + p * half + at + 4 * i);
      const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) { t.c[4 * i + e] = cc[e]; t.s[4 * i + e] = __uint_as_float(__float_as_uint(ss[e]) ^ flip); }
    }
  }
  return t;
}
// where a lane's partners lie in its row
__device__ __forceinline__ int partner_channel(const RopeArgs& a, int d0) {
  const int half = a.rotary >> 1;
  return a.interleaved || d0 >= a.rotary ? d0 : d0 < half ? d0 + half : d0 - half;
}
template <bool BF> __device__ __forceinline__ void widen8(uint4 raw, float (&x)[8]) {
  const uint32_t rw[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = widen16((uint16_t)(rw[e >> 1] >> (16 * (e & 1))), BF);
}
// x: a lane's channels, rotated in place; `other`: its partners as they came (not read with interleaved pairs)
template <bool BF> __device__ __forceinline__ void turn8(const RopeArgs& a, const Turn& t, float (&x)[8], uint4 other, int d0) {
  if (d0 >= a.rotary) return;
  float p[8];
  if (a.interleaved) {
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = x[e ^ 1];
  } else {
    widen8<BF>(other, p);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = x[e] * t.c[e] + p[e] * t.s[e];
}
template <bool BF> __device__ __forceinline__ uint16_t narrow16(float x) { return BF ? f32_to_bf16_bits(x) : f32_to_f16_bits(x); }
template <bool BF> __device__ __forceinline__ uint4 narrow8(const float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = narrow16<BF>(x[2 * e]) | (uint32_t)narrow16<BF>(x[2 * e + 1]) << 16;
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// A key row (16 lanes): the rotation of rotate_k, the quantizer, the stores.  tv: the token's number in plane order.
template <bool BF> __device__ __forceinline__ void store_key_row(const RopeArgs& a, float (&x)[8], int64_t tv, int lane16) {
  const Geom& g = a.g;
  uint8_t* row = (uint8_t*)a.cache.k_codes + tv * (16 * g.bits_k);
  if (g.bits_k == 16) {
    store_stream16(row + 16 * lane16, narrow8<BF>(x));
    return;
  }
  if (g.rotate_k) rotate8(x, lane16, rot_sign_bits(g.signs_k, lane16));
  const int lpg = g.g_k >> 3;
  uint32_t codes[8];
  uint16_t S, Z;
  quantize8(x, g.bits_k, lpg, codes, &S, &Z);
  if ((lane16 & (lpg - 1)) == 0)
    __builtin_nontemporal_store((uint32_t)S | ((uint32_t)Z << 16), (uint32_t*)a.cache.k_meta + meta_index(tv, lane16 >> lpg_shift(lpg), g.ng_k));
  switch (g.bits_k) {
    case 1: store_key_codes<1, true>(row, lane16, codes); break;
    case 2: store_key_codes<2, true>(row, lane16, codes); break;
    case 3: store_key_codes<3, true>(row, lane16, codes); break;
    case 4: store_key_codes<4, true>(row, lane16, codes); break;
    case 6: store_key_codes<6, true>(row, lane16, codes); break;
    default: store_key_codes<8, true>(row, lane16, codes); break;
  }
}
// A value row: its codes (patterns of an unquantized plane), scale and zero stored.
template <bool BF> __device__ __forceinline__ void quantize_value_row(const RopeArgs& a, uint4 raw, int64_t tv, int bh, int lane16, uint32_t (&codes)[8]) {
  const Geom& g = a.g;
  if (g.bits_v == 16) {
    const uint32_t rw[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) codes[e] = (rw[e >> 1] >> (16 * (e & 1))) & 0xFFFFu;
    return;
  }
  float x[8];
  widen8<BF>(raw, x);
  if (g.rotate_v) rotate8(x, lane16, rot_sign_bits(g.signs_v, lane16));
  const int lpg = g.g_v >> 3;
  uint16_t S, Z;
  quantize8(x, g.bits_v, lpg, codes, &S, &Z);
  if ((lane16 & (lpg - 1)) == 0) {
    __builtin_nontemporal_store((uint32_t)S | ((uint32_t)Z << 16), (uint32_t*)a.cache.v_meta + meta_index(tv, lane16 >> lpg_shift(lpg), g.ng_v));
    note_value_scale(a.cache.v_scale_exp + bh, S);
  }
}

// One workgroup: the new tokens of one 32-token block of one (sequence, kv head), and the same tokens of its query heads, which
// share the tokens' cosines and sines in registers.
template <bool BF>
__global__ __launch_bounds__(256) void rope_append_kernel(const RopeArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t vstage[stage_total<16, kRopeSpan>()];
  static_assert(stage_total<16, kRopeSpan>() >= stage_total<6, kRopeSpan>(), "staging area");
  const Geom& g = a.g;
  const int tid = threadIdx.x, lane16 = tid & 15, d0 = 8 * lane16;
  // (a division leaves its result in vector registers, and with it every address: these are the same in all lanes)
  const int b = __builtin_amdgcn_readfirstlane(blockIdx.y / g.kv_heads), h = blockIdx.y - b * g.kv_heads;
  const int pos = a.pos[b];
  const int count = a.n_tokens ? min(max(a.n_tokens[b], 0), a.n_new) : a.n_new;
  const int first = max(pos, 0), end = (int)min((int64_t)pos + count, (int64_t)a.capacity);    // positions that are stored
  if (first >= end) return;                        // uniform (nothing to store; also keeps positions near 2^31 out of what follows)
  const int blk = first / kRopeSpan + blockIdx.x;
  const int lo = max(first - blk * kRopeSpan, 0), hi = min(end - blk * kRopeSpan, kRopeSpan);
  if (lo >= hi) return;                            // uniform
  const int64_t tv0 = virtual_token(g, a.cache.page_table, b, h, (int64_t)blk * kRopeSpan);
  const int64_t row0 = (int64_t)b * a.sb + (int64_t)h * a.sh;
  const int other = partner_channel(a, d0);
  // Many tokens: 16 lanes take a token's key, value and queries in turn.  A single one: its key goes to the first wavefront, its value to the
  // second, its query heads to 16 lanes each of the others (32 query heads, 8 kv heads: 7.2 us in turn, 4.9 so; 64 sequences 10.8 and 5.8).
  const int slot = tid >> 4;
  const bool one = hi - lo == 1, do_k = !one || slot == 0, do_v = !one || slot == 4;
  const int r_begin = !one ? 0 : slot >= 8 ? slot - 8 : a.heads_per_kv, r_end = !one ? a.heads_per_kv : min(r_begin + 1, a.heads_per_kv);
  for (int it = 0; it < (one ? 1 : 2); ++it) {
    const int row = one ? lo : slot + 16 * it;
    if (row < lo || row >= hi) continue;           // whole 16-lane rows take the same branch
    const int64_t p = (int64_t)blk * kRopeSpan + row, i = p - pos;
    const Turn t = load_turn(a, p, d0);
    const int64_t src = row0 + i * a.st;
    uint4 kraw{}, kother{}, vraw{};
    if (do_k) {
      kraw = *reinterpret_cast<const uint4*>(a.k_new + src + d0);
      kother = *reinterpret_cast<const uint4*>(a.k_new + src + other);
    }
    if (do_v) vraw = *reinterpret_cast<const uint4*>(a.v_new + src + d0);
    // query heads two at a time, the next two on their way while two are rotated (a last one of an odd number is loaded twice, stored once)
    const int64_t qs = b * a.q_sb + i * a.q_st + (int64_t)h * a.heads_per_kv * a.q_sh;
    uint4 own[2], oth[2];
    auto load_heads = [&](int r) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint16_t* const q = a.q + qs + min(r + k, r_end - 1) * a.q_sh;
        own[k] = *reinterpret_cast<const uint4*>(q + d0);
        if (!a.interleaved) oth[k] = *reinterpret_cast<const uint4*>(q + other);
      }
    };
    if (r_begin < r_end) load_heads(r_begin);      // (none: also a call without queries)
    float x[8];
    if (do_k) {
      widen8<BF>(kraw, x);
      turn8<BF>(a, t, x, kother, d0);
      store_key_row<BF>(a, x, tv0 + row, lane16);
    }
    if (do_v) {
      uint32_t codes[8];
      quantize_value_row<BF>(a, vraw, tv0 + row, blockIdx.y, lane16, codes);
      switch (g.bits_v) {
        case 1: stage_value_row<1, kRopeSpan>(vstage, row, d0, codes); break;
        case 2: stage_value_row<2, kRopeSpan>(vstage, row, d0, codes); break;
        case 3: stage_value_row<3, kRopeSpan>(vstage, row, d0, codes); break;
        case 4: stage_value_row<4, kRopeSpan>(vstage, row, d0, codes); break;
        case 6: stage_value_row<6, kRopeSpan>(vstage, row, d0, codes); break;
        case 8: stage_value_row<8, kRopeSpan>(vstage, row, d0, codes); break;
        default: stage_value_row<16, kRopeSpan>(vstage, row, d0, codes); break;
      }
    }
    uint16_t* const out = a.q_out + (((int64_t)b * a.n_new + i) * a.q_heads + (int64_t)h * a.heads_per_kv) * kHeadDim + d0;
    for (int r = r_begin; r < r_end; r += 2) {
      uint4 y[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        widen8<BF>(own[k], x);
        turn8<BF>(a, t, x, oth[k], d0);
        y[k] = narrow8<BF>(x);
      }
      if (r + 2 < r_end) load_heads(r + 2);
      *reinterpret_cast<uint4*>(out + r * kHeadDim) = y[0];
      if (r + 1 < r_end) *reinterpret_cast<uint4*>(out + (r + 1) * kHeadDim) = y[1];
    }
  }
  __syncthreads();
  uint32_t* vc = (uint32_t*)a.cache.v_codes + (tv0 >> 5) * (128 * g.bits_v);
  switch (g.bits_v) {
    case 1: store_value_span<1, kRopeSpan, true>(vc, vstage, tid, lo, hi); break;
    case 2: store_value_span<2, kRopeSpan, true>(vc, vstage, tid, lo, hi); break;
    case 3: store_value_span<3, kRopeSpan, true>(vc, vstage, tid, lo, hi); break;
    case 4: store_value_span<4, kRopeSpan, true>(vc, vstage, tid, lo, hi); break;
    case 6: store_value_span<6, kRopeSpan, true>(vc, vstage, tid, lo, hi); break;
    case 8: store_value_span<8, kRopeSpan, true>(vc, vstage, tid, lo, hi); break;
    default: store_value_span<16, kRopeSpan, true>(vc, vstage, tid, lo, hi); break;
  }
}

}  // namespace

hipError_t launch_rope_append(const RopeArgs& a, int in_dtype, hipStream_t stream) {
  // (n tokens that start anywhere touch at most (n + 30) / 32 + 1 blocks)
  const dim3 grid((a.n_new + kRopeSpan - 2) / kRopeSpan + 1, a.g.batch * a.g.kv_heads);
  if (in_dtype == KVQ_BF16) hipLaunchKernelGGL((rope_append_kernel<true>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((rope_append_kernel<false>), grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace kvq
