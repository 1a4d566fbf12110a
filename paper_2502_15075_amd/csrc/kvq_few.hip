// Attention of a few query rows per kv head over the packed cache (gfx950): single tokens behind a sliding window, the verification of
// drafted tokens, short chunks.  A workgroup takes up to 48 rows (query token, query head) of a kv head; where there are many, the tiles of
// kvq_chunk.hip take them (plan_chunk weighs both).
//
//   S[t,i] = sum_g sK[t,g] (sum_{d in g} q[i,d] cK[t,d]) + zK[t,g] (sum_{d in g} q[i,d])
//   out[i] = ( sum_t (P[t,i] sV[t,g(d)]) cV[t,d] + sum_t P[t,i] zV[t,g(d)] ) / sum_t P[t,i],   P = 2^(kappa S - m)
//
// Bound by the cache's bytes, so every byte is read once per workgroup and kept packed as long as it can be: a wavefront walks blocks of 32
// tokens of its own and holds a ring of them in registers.  Scores are tokens x rows by 16x16x32 matrix instructions, so that a lane owns one
// row (16 rows a column set) and the packed value blocks, which are in operand order already, meet its weights where they are.  Codes enter
// as binary16 whole numbers and scales multiply in binary32: nothing is rounded on the way to the scores, so they do not limit an
// output in binary32.  A weight is rounded to binary16 once, together with its value scale; for binary32 outputs (FINE) it
// travels as two binary16 parts, 2^-22 of it.
//
// A code stays a number in the low bits of a binary16 lane, i.e. a subnormal: c 2^(k - 24) with its lowest bit at bit k, so that unpacking is a
// shift and a mask; the power of two goes into the scores' factor and the final sums.  The matrix unit takes a subnormal by the exponent
// 2^-14 and loses what lies 24 bits below a sum's largest product (code_base).
//
// A wavefront's next block is on its way while it computes one: its loads land in registers, and go from there through LDS of the
// wavefront's own at the start of the next turn.  A lane needs 8 channels of every 32 of its key row (all groups alike), which would be loads
// of a few bytes; the rows' 16-byte units are permuted by the row's number so that the reads meet no bank twice.
//
// Measured: 64 sequences x 8 kv heads, 16400 visible tokens each, 4/4 bits, one set of 16 rows: 1.21 GB in 197 us, 6.1 TB/s, bound by memory.  A
// block of 32 tokens costs a compute unit's eight wavefronts 0.2 us with one set and 0.33 with three (4/2 bits: about 245 vector instructions
// with one), which binds where lengths are uneven or rows many: 16 sequences x 40 rows, 1200 to 16384 tokens, 92 us at 1.4 TB/s.
#include "kvq_attend.h"
#include "kvq_few.h"

namespace kvq {
namespace {

constexpr float kFewWeightBits = 8.0f;     // weights carry 2^8, with value scales below 64 and
constexpr float kFewSlack = 1.9f;          // a running maximum that lags by at most this they stay below binary16's bound

__device__ __forceinline__ float4v mma16(u32x4 a, u32x4 b, float4v c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8v, a), __builtin_bit_cast(half8v, b), c, 0, 0, 0);
}
__device__ __forceinline__ float over_rows_sum(float x) {       // over the four 16-lane rows of a wavefront, in every lane
  const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const float s = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(s), __float_as_uint(s), false, false);
  return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}
__device__ __forceinline__ float over_rows_max(float x) {
  const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const float s = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(s), __float_as_uint(s), false, false);
  return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}
__device__ __forceinline__ float meta_s(uint32_t m) { return (float)as_half2(m)[0]; }
__device__ __forceinline__ float meta_z(uint32_t m) { return (float)as_half2(m)[1]; }

// ---- key rows in LDS: 16 B bytes a row of B units; unit q of row r lies at place q ^ (r B / 16 mod B) of the row (B a power of two).
// All reads of a wavefront (16 rows at once) then use every bank once.
template <int B> constexpr bool key_swizzled() { return (B & (B - 1)) == 0 && B > 1; }
template <int B> __device__ __forceinline__ int key_swizzle(int row) { return key_swizzled<B>() ? (row * B / 16) & (B - 1) : 0; }

// Where the lowest bit k of a code lies in its binary16 lane.  2^(-14 - k) of a code's step is lost: for binary32 outputs (FINE) the codes go as high
// as they fit, which leaves 2^-24 of a group's range whatever the width; otherwise where they need fewest shifts.
template <int B, bool FINE> constexpr int code_base() { return FINE ? 10 - B : B == 1 || B == 2 ? 6 : B == 3 || B == 4 || B == 6 ? 4 : 0; }
template <int B, bool FINE> constexpr float code_unit() { return B == 16 ? 1.0f : 1.0f / (float)(1 << (24 - code_base<B == 16 ? 8 : B, FINE>())); }
// x >> n, n < 0: x << -n
template <int N> __device__ __forceinline__ uint32_t shifted(uint32_t x) { return N >= 0 ? x >> (N >= 0 ? N : 0) : x << (N < 0 ? -N : 0); }
// Fields of W bits at bits AT and 16 + AT of x, their lowest bits taken to BASE and 16 + BASE
template <int W, int AT, int BASE> __device__ __forceinline__ uint32_t field(uint32_t x) {
  return shifted<AT - BASE>(x) & (((1u << W) - 1u) * 0x00010001u << BASE);
}

// Operand of channels 32 kk .. 32 kk + 31 of token row `row`: this lane's eight (slots 8 j .. 8 j + 7 of the chunk).
template <int B, bool FINE> __device__ __forceinline__ u32x4 key_operand(const uint8_t* st, int row, int sw, int kk, int j, bool raw_bf) {
  constexpr int K = code_base<B == 16 ? 8 : B, FINE>();
  const uint8_t* base = st + row * (16 * B);
  if constexpr (B == 16) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(base + (((4 * kk + j) ^ sw) << 4));
    return u32x4{raw_to_half2(w[0], raw_bf), raw_to_half2(w[1], raw_bf), raw_to_half2(w[2], raw_bf), raw_to_half2(w[3], raw_bf)};
  } else if constexpr (B == 8) {
    const uint2 w = *reinterpret_cast<const uint2*>(base + (((2 * kk + (j >> 1)) ^ sw) << 4) + 8 * (j & 1));
    return u32x4{field<8, 0, K>(w.x), field<8, 8, K>(w.x), field<8, 0, K>(w.y), field<8, 8, K>(w.y)};
  } else if constexpr (B == 4 || B == 2 || B == 1) {
    const uint32_t w = B == 4 ? *reinterpret_cast<const uint32_t*>(base + ((kk ^ sw) << 4) + 4 * j)
                     : B == 2 ? *reinterpret_cast<const uint32_t*>(base + (((kk >> 1) ^ sw) << 4) + 8 * (kk & 1) + 4 * (j >> 1)) >> (8 * (j & 1))
                              : *reinterpret_cast<const uint32_t*>(base + 4 * kk) >> (4 * j);
    return u32x4{field<B, 0, K>(w), field<B, B, K>(w), field<B, 2 * B, K>(w), field<B, 3 * B, K>(w)};
  } else if constexpr (B == 3) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(base) + 3 * kk;
    const uint32_t lo = w[j >> 1] >> (8 * (j & 1)), hi = w[2] >> (16 * (j >> 1) + 4 * (j & 1));
    u32x4 out;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      out[i] = (((lo >> (2 * i)) & 0x00030003u) | (((hi >> i) & 1u) << 2) | (((hi >> (i + 8)) & 1u) << 18)) << K;
    return out;
  } else {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(base) + 6 * kk;
    const uint32_t lo = w[j], hi = w[4 + (j >> 1)] >> (16 * (j & 1));
    u32x4 out;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      out[i] = (((lo >> (4 * i)) & 0x000F000Fu) | (((hi >> (2 * i)) & 3u) << 4) | (((hi >> (2 * i + 8)) & 3u) << 20)) << K;
    return out;
  }
}

// ---- value blocks: a lane's piece, 2 b dwords; field 4 dt + v is pair v (tokens 2 v, 2 v + 1 of the lane's eight) of channel tile dt
template <int B, bool FINE> __device__ __forceinline__ u32x4 value_operand(const uint32_t* w, int dt) {
  constexpr int K = code_base<B == 16 ? 8 : B, FINE>();
  if constexpr (B == 16) return u32x4{w[4 * dt], w[4 * dt + 1], w[4 * dt + 2], w[4 * dt + 3]};
  else if constexpr (B == 8) return u32x4{field<8, 0, K>(w[2 * dt]), field<8, 8, K>(w[2 * dt]), field<8, 0, K>(w[2 * dt + 1]), field<8, 8, K>(w[2 * dt + 1])};
  else if constexpr (B == 4) return u32x4{field<4, 0, K>(w[dt]), field<4, 4, K>(w[dt]), field<4, 8, K>(w[dt]), field<4, 12, K>(w[dt])};
  else if constexpr (B == 2) {
    const uint32_t x = w[dt >> 1];
    return dt & 1 ? u32x4{field<2, 8, K>(x), field<2, 10, K>(x), field<2, 12, K>(x), field<2, 14, K>(x)}
                  : u32x4{field<2, 0, K>(x), field<2, 2, K>(x), field<2, 4, K>(x), field<2, 6, K>(x)};
  } else if constexpr (B == 1) {
    const uint32_t x = w[dt >> 2] >> (4 * (dt & 3));
    return u32x4{field<1, 0, K>(x), field<1, 1, K>(x), field<1, 2, K>(x), field<1, 3, K>(x)};
  } else if constexpr (B == 3) {
    const uint32_t x = w[dt >> 1] >> (8 * (dt & 1)), y = w[4 + (dt >> 2)] >> (4 * (dt & 3));
    return u32x4{field<2, 0, K>(x) | field<1, 0, K + 2>(y), field<2, 2, K>(x) | field<1, 1, K + 2>(y), field<2, 4, K>(x) | field<1, 2, K + 2>(y),
                 field<2, 6, K>(x) | field<1, 3, K + 2>(y)};
  } else {
    const uint32_t x = w[dt], y = w[8 + (dt >> 1)] >> (8 * (dt & 1));
    return u32x4{field<4, 0, K>(x) | field<2, 0, K + 4>(y), field<4, 4, K>(x) | field<2, 2, K + 4>(y), field<4, 8, K>(x) | field<2, 4, K + 4>(y),
                 field<4, 12, K>(x) | field<2, 6, K + 4>(y)};
  }
}

// Byte offset of a lane's i-th 16-byte load of 32 key rows (off: those of the first loads, after which the permutation repeats).
template <int BK, int N> __device__ __forceinline__ uint32_t key_load_offset(const uint32_t (&off)[N], int i, int lane) {
  if constexpr (BK == 1) return off[0];
  else if constexpr (BK == 3) return i == 0 ? off[0] : 1024u + 16u * min(lane, 31);
  else return off[i % N] + 1024u * (i / N * N);
}

template <int BK, int BV> struct Step {
  u32x4 k[key_loads<BK>()];
  uint32_t v[2 * BV];
  u32x4 meta;
};

// NG: the larger number of groups per row of the two tensors; a tensor with fewer is taken as one with NG whose scales repeat.
template <int BK, int BV, int NC, int NG, bool FINE>
__global__ __launch_bounds__((64 * kFewWaves), (few_occupancy(BK, BV, NC, NG))) void few_kernel(const ChunkArgs a) {
  constexpr int NW = kFewWaves, NK = key_loads<BK>(), kWaveBytes = few_wave_bytes<BK, BV>();
  constexpr bool RAWK = BK == 16, RAWV = BV == 16;
  constexpr bool kQueryInLds = NC > 1;
  constexpr float kUnitK = code_unit<BK, FINE>(), kUnitV = code_unit<BV, FINE>();
  __shared__ __attribute__((aligned(16))) uint8_t sm[few_lds_bytes<BK, BV, NC>()];
  __shared__ __attribute__((aligned(16))) uint8_t sm_query[16 * NC * 256];
  __shared__ __attribute__((aligned(16))) float sm_sums[16 * NC][4];
  __shared__ int sm_last;
  __shared__ int sm_pos[16 * NC];                          // positions of the rows
  __shared__ float sm_kappa[16 * NC], sm_m[NW][16 * NC], sm_l[NW][16 * NC];
  const Geom& g = a.g;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, j = lane >> 4;
  // (a division leaves its result in vector registers, and with it every address: these are the same in all lanes)
  const int b = __builtin_amdgcn_readfirstlane(blockIdx.x / g.kv_heads), h = blockIdx.x - b * g.kv_heads, split = blockIdx.y;
  const int R = a.heads_per_kv;
  const int len = a.seq_lens ? min(max(a.seq_lens[b], 0), a.seq_bound) : a.seq_bound;
  const int nq = a.q_lens ? min(max(a.q_lens[b], 0), a.n_q) : a.n_q;
  const int row0 = blockIdx.z * (16 * NC), rows = nq * R;
  if (row0 >= rows) return;
  // positions: of query token 0, of the tile's first and last row (limit: no row of it sees a token from there on)
  const int p0 = len - nq, p_first = p0 + __builtin_amdgcn_readfirstlane(row0 / R);
  const int p_last = p0 + __builtin_amdgcn_readfirstlane((min(row0 + 16 * NC, rows) - 1) / R), limit = p_last + 1;
  const bool raw_bf = g.raw_dtype == KVQ_BF16;
  __builtin_amdgcn_s_setreg(1 | (23 << 6), 1);             // binary16 results that overflow become the largest number (see kvq_chunk.hip)

  // ---- the blocks of 32 tokens that some row sees: [0, sink_blocks), [first, ...), n in all; this workgroup's, this wavefront's
  const int lo = a.window ? max(p_first - a.window + 1, 0) : 0;
  const int first = lo >> 5, sink_blocks = min((a.sinks + 31) >> 5, first);
  const int n_blocks = p_last >= 0 ? sink_blocks + (p_last >> 5) + 1 - first : 0;
  const int parts = a.splits == 1 ? 1 : max(__builtin_amdgcn_readfirstlane((n_blocks + a.per - 1) / a.per), 1);
  if (split >= parts) return;                              // uniform
  const int begin = split * a.per, end = min(begin + a.per, n_blocks);
  auto block_at = [&](int x) { return x < sink_blocks ? x : x - sink_blocks + first; };

  // ---- loads of a step
  const int nmk = RAWK ? 0 : 8 * g.ng_k, nmv = RAWV ? 0 : 8 * g.ng_v;        // 16-byte units of scales and zeros
  // (64 units are 64 / BK rows; the permutation of the units repeats every 16 rows)
  constexpr int kRepeat = BK == 8 ? 2 : BK == 16 ? 4 : 1;
  uint32_t k_off[kRepeat];
#pragma unroll
  for (int i = 0; i < kRepeat; ++i) {
    const int u = min(64 * i + lane, 32 * BK - 1), row = u / BK;
    k_off[i] = (uint32_t)(row * BK + ((u % BK) ^ key_swizzle<BK>(row))) * 16;
  }
  const int mu = min(lane, nmk + nmv - 1);
  // in LDS every tensor has NG groups: a tensor with fewer is stored once for each it stands for
  const int ngk = RAWK ? 1 : g.ng_k, ngv = RAWV ? 1 : g.ng_v, most_rep = NG / min(ngk, ngv);
  const int unit = mu - (mu < nmk ? 0 : nmk), groups = ngk + (mu < nmk ? 0 : ngv - ngk);
  const int rep = NG / groups;
  const int meta_at = (mu < nmk ? 0 : 128 * NG) + (unit / (4 * groups) * NG + (unit >> 2) % groups * rep) * 64 + (unit & 3) * 16;
  // (picked by arithmetic: a choice between words of the argument block would become a load from it, waited for in every step.  A block number
  // stays below 2^32: a block of value codes takes 512 bytes at least)
  const uint64_t pick = mu < nmk ? 0 : ~0ull;
  const uint64_t meta_base = (uint64_t)a.cache.k_meta + (((uint64_t)a.cache.v_meta - (uint64_t)a.cache.k_meta) & pick) + 16 * unit;
  const uint32_t meta_step = 128 * g.ng_k + (128 * (g.ng_v - g.ng_k) & (uint32_t)pick);
  typedef const __attribute__((address_space(4))) int32_t* TablePtr;
  const TablePtr pages = (TablePtr)(uintptr_t)(g.page_shift ? a.cache.page_table + (int64_t)b * g.pages_per_seq : nullptr);
  const int page_blocks = g.page_shift - 5;
  auto page_of = [&](int blk) -> int { return g.page_shift ? pages[blk >> page_blocks] : 0; };
  auto load = [&](Step<BK, BV>& s, int blk, int page) {
    const int64_t vb_ = g.page_shift ? (((int64_t)page * g.kv_heads + h) << page_blocks) + (blk & ((1 << page_blocks) - 1))
                                     : ((int64_t)b * g.kv_heads + h) * (g.t_cap >> 5) + blk;
    // (the choice above would leave the address in vector registers)
    const int64_t vb = ((int64_t)__builtin_amdgcn_readfirstlane((int)(vb_ >> 32)) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane((int)vb_);
    const uint8_t* kp = (const uint8_t*)a.cache.k_codes + vb * (512 * BK);
    const uint8_t* vp = (const uint8_t*)a.cache.v_codes + vb * (512 * BV);
#pragma unroll
    for (int i = 0; i < NK; ++i) s.k[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(kp + key_load_offset<BK>(k_off, i, lane)));
    load_value_piece<BV>(s.v, vp, lane);
    if constexpr (RAWK && RAWV) s.meta = u32x4{0u, 0u, 0u, 0u};
    else s.meta = __builtin_nontemporal_load((const __attribute__((address_space(1))) u32x4*)(meta_base + (uint64_t)(uint32_t)vb * meta_step));
  };

  Step<BK, BV> step;
  const int x0 = begin + wave;                             // this wavefront's blocks: x0, x0 + NW, ...
  if (x0 < end) load(step, block_at(x0), page_of(block_at(x0)));
  int page = x0 + NW < end ? page_of(block_at(x0 + NW)) : 0;
  const int scale_exp = RAWV ? 0 : a.cache.v_scale_exp[(int64_t)b * g.kv_heads + h];

  // ---- query
  stage_query<64 * NW>(a, b, h, row0, rows, 16 * NC, NG, sm_query, nullptr, sm_sums, sm_kappa);
  if (tid < 16 * NC) sm_pos[tid] = p0 + min(row0 + tid, rows - 1) / R;
  __syncthreads();
  auto query_operand = [&](int cs, int kk) { return *reinterpret_cast<const u32x4*>(sm_query + (16 * cs + c) * 256 + (((4 * kk + j) ^ c) << 4)); };
  u32x4 qb[kQueryInLds ? 1 : NC][4];
#pragma unroll
  for (int cs = 0; cs < NC; ++cs) {
    if constexpr (!kQueryInLds) {
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) qb[cs][kk] = query_operand(cs, kk);
    }
  }
  // (read where they are used: the loop has no registers for them.  Scores carry the codes' unit)
  auto query_sum = [&](int cs, int n) { return sm_sums[16 * cs + c][n] * kUnitK; };
  auto kappa = [&](int cs) { return sm_kappa[16 * cs + c] * (1.0f / kUnitK); };
  uint8_t* const st = sm + wave * kWaveBytes;
  uint8_t* const st_v = st + 512 * BK;
  uint8_t* const st_meta = st_v + 512 * BV;

  // value scales of 64 and more take their bits of room from the weights
  const float weight_bits = kFewWeightBits - (float)max(scale_exp - 20, 0);
  const int sw = key_swizzle<BK>(c);
  auto meta_k = [&](int x4, int n) { return *reinterpret_cast<const u32x4*>(st_meta + 16 * j + (x4 * NG + n) * 64); };
  auto meta_v = [&](int x4, int n) { return *reinterpret_cast<const u32x4*>(st_meta + 16 * j + 128 * NG + (x4 * NG + n) * 64); };

  float4v acc[NC][8];
  float m[NC], l[NC], zacc[NC][NG];
#pragma unroll
  for (int cs = 0; cs < NC; ++cs) {
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) acc[cs][dt] = float4v{0.f, 0.f, 0.f, 0.f};
    m[cs] = kNoMax; l[cs] = 0.0f;
#pragma unroll
    for (int n = 0; n < NG; ++n) zacc[cs][n] = 0.0f;
  }

  // A SIMD serves its oldest wavefront first: of four with 24 steps each, bound by their instructions, the first was done after 45 us, the
  // last, alone by then, after 84.  So the priority goes round, a step at each of four levels, wavefronts of a SIMD apart by their slot in it: 52 and
  // 76 us (timing only: who computes what stays fixed).
  uint32_t turn = __builtin_amdgcn_s_getreg((3 << 11) | 4);          // WAVE_ID, bits 3:0 of HW_ID
  for (int x = x0; x < end; x += NW) {
    switch (turn++ & 3) {
      case 0: __builtin_amdgcn_s_setprio(0); break;
      case 1: __builtin_amdgcn_s_setprio(1); break;
      case 2: __builtin_amdgcn_s_setprio(2); break;
      default: __builtin_amdgcn_s_setprio(3); break;
    }
    const int t0 = 32 * block_at(x);
    const bool cut = t0 + 32 > limit || t0 < lo;           // some of its tokens no row sees: what a cache holds there need be no number
    auto seen_by_some = [&](int t) { return (t < limit) & ((t >= lo) | (t < a.sinks)); };
    // ---- the block to LDS, the next one under way
#pragma unroll
    for (int i = 0; i < NK; ++i)
      if (64 * (i + 1) <= 32 * BK || lane < 32 * BK - 64 * i) *reinterpret_cast<u32x4*>(st + 1024 * i + 16 * lane) = step.k[i];
    store_value_piece<BV>(step.v, st_v, lane);
    if constexpr (!RAWK || !RAWV) {
      if (cut) {
        const int token = t0 + 16 * (meta_at % (128 * NG) / (64 * NG)) + ((meta_at >> 2) & 12);
#pragma unroll
        for (int r = 0; r < 4; ++r) step.meta[r] = seen_by_some(token + r) ? step.meta[r] : 0u;
      }
      *reinterpret_cast<u32x4*>(st_meta + meta_at) = step.meta;
      for (int r = 1; r < most_rep; ++r) *reinterpret_cast<u32x4*>(st_meta + meta_at + 64 * min(r, rep - 1)) = step.meta;
    }
    if (x + NW < end) {
      load(step, block_at(x + NW), page);
      page = x + 2 * NW < end ? page_of(block_at(x + 2 * NW)) : 0;
    }
    __builtin_amdgcn_wave_barrier();

    // ---- scores
    float sc[NC][8];
#pragma unroll
    for (int x4 = 0; x4 < 2; ++x4) {
      constexpr int NGK = RAWK ? 1 : NG;
      u32x4 ka[4];
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) ka[kk] = key_operand<BK, FINE>(st, 16 * x4 + c, sw, kk, j, raw_bf);
#pragma unroll
      for (int cs = 0; cs < NC; ++cs)
#pragma unroll
        for (int r = 0; r < 4; ++r) sc[cs][4 * x4 + r] = 0.0f;
#pragma unroll
      for (int n = 0; n < NGK; ++n) {
        u32x4 mk;
        if constexpr (!RAWK) mk = meta_k(x4, n);
#pragma unroll
        for (int cs = 0; cs < NC; ++cs) {
          float4v d = float4v{0.f, 0.f, 0.f, 0.f};
          const float qs = RAWK ? 0.0f : query_sum(cs, n);
#pragma unroll
          for (int kk = n * (4 / NGK); kk < (n + 1) * (4 / NGK); ++kk) d = mma16(ka[kk], kQueryInLds ? query_operand(cs, kk) : qb[kQueryInLds ? 0 : cs][kk], d);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            float& y = sc[cs][4 * x4 + r];
            y = RAWK ? d[r] : fmaf(meta_s(mk[r]), d[r], fmaf(meta_z(mk[r]), qs, y));
          }
        }
      }
    }
    // slot 4 x4 + r of a lane: token 16 x4 + 4 j + r of the block
    const bool whole = t0 + 31 <= p_first && (a.window == 0 || t0 > p_last - a.window);
    if (!whole) {
#pragma unroll
      for (int cs = 0; cs < NC; ++cs) {
        // (the lane's number formed anew: kept for this rare place it would cost the loop a register)
        const int me = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)), mj = me >> 4;
        const int my_p = sm_pos[16 * cs + (me & 15)], my_lo = a.window ? my_p - a.window : -1;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int t = t0 + 16 * (i >> 2) + 4 * mj + (i & 3);
          const bool seen = (t <= my_p) & ((t > my_lo) | (t < a.sinks));
          sc[cs][i] = seen ? sc[cs][i] : -INFINITY;
        }
      }
    }
    // ---- weights
#pragma unroll
    for (int cs = 0; cs < NC; ++cs) {
      const float kap = kappa(cs);
      float most = sc[cs][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) most = fmaxf(most, sc[cs][i]);
      most *= kap;
      if (__any(most > m[cs] + kFewSlack)) {
        const float m_new = fmaxf(m[cs], over_rows_max(most)), f = __builtin_amdgcn_exp2f(m[cs] - m_new);
        m[cs] = m_new;
        l[cs] *= f;
#pragma unroll
        for (int n = 0; n < NG; ++n) zacc[cs][n] *= f;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) acc[cs][dt] *= f;
      }
      const float off = weight_bits - m[cs];
#pragma unroll
      for (int i = 0; i < 8; ++i) { sc[cs][i] = __builtin_amdgcn_exp2f(fmaf(sc[cs][i], kap, off)); l[cs] += sc[cs][i]; }
    }
    // ---- weights of every part of the value rows (8 / NGV channel tiles each), and the product with its tiles
    constexpr int NGV = RAWV ? 1 : NG;
    uint32_t vw[2 * BV];
    read_value_piece<BV>(vw, st_v, lane);
#pragma unroll
    for (int n = 0; n < NGV; ++n) {
      u32x4 mv[2], hi[NC], lo2[NC];
      if constexpr (!RAWV) { mv[0] = meta_v(0, n); mv[1] = meta_v(1, n); }
#pragma unroll
      for (int cs = 0; cs < NC; ++cs) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float w0 = sc[cs][2 * i], w1 = sc[cs][2 * i + 1];
          half2v y;
          if constexpr (!RAWV) {
            const uint32_t e0 = mv[i >> 1][2 * (i & 1)], e1 = mv[i >> 1][2 * (i & 1) + 1];
            zacc[cs][n] = fmaf(w0, meta_z(e0), zacc[cs][n]);
            zacc[cs][n] = fmaf(w1, meta_z(e1), zacc[cs][n]);
            if constexpr (FINE) { w0 = as_rounded(w0 * meta_s(e0)); w1 = as_rounded(w1 * meta_s(e1)); }
            else {                                         // (product and rounding in one instruction each)
              y[0] = (_Float16)fmaf(w0, meta_s(e0), 0.0f);
              y[1] = (_Float16)fmaf(w1, meta_s(e1), 0.0f);
            }
          }
          if constexpr (RAWV || FINE) { y[0] = (_Float16)w0; y[1] = (_Float16)w1; }
          hi[cs][i] = as_u32(y);
          if constexpr (FINE) {
            half2v z;
            z[0] = (_Float16)(w0 - (float)y[0]); z[1] = (_Float16)(w1 - (float)y[1]);
            lo2[cs][i] = as_u32(z);
          }
        }
      }
#pragma unroll
      for (int dt = n * (8 / NGV); dt < (n + 1) * (8 / NGV); ++dt) {
        u32x4 va = value_operand<BV, FINE>(vw, dt);
        if constexpr (RAWV) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t y = raw_to_half2(va[i], raw_bf);
            const int at = t0 + 4 * j + 16 * (i >> 1) + 2 * (i & 1);
            if (cut) y &= (seen_by_some(at) ? 0x0000FFFFu : 0u) | (seen_by_some(at + 1) ? 0xFFFF0000u : 0u);
            va[i] = y;
          }
        }
#pragma unroll
        for (int cs = 0; cs < NC; ++cs) {
          acc[cs][dt] = mma16(va, hi[cs], acc[cs][dt]);
          if constexpr (FINE) acc[cs][dt] = mma16(va, lo2[cs], acc[cs][dt]);
        }
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
  __builtin_amdgcn_s_setprio(0);

  // (lane and thread formed anew: kept for here they would cost the loop a register)
  const int me = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)), my_tid = 64 * wave + me, mc = me & 15, mj = me >> 4;
  MergeWord* const word = a.words + (int64_t)blockIdx.z * gridDim.x + blockIdx.x;
  if (parts > 1 && my_tid == 0) merge_announce(word, a.merge_tag);
  // ---- join the wavefronts: everybody's maxima and weight sums, then sums of channels rescaled to the common maximum
#pragma unroll
  for (int cs = 0; cs < NC; ++cs) {
    l[cs] = over_rows_sum(l[cs]);
#pragma unroll
    for (int n = 0; n < NG; ++n) zacc[cs][n] = over_rows_sum(zacc[cs][n]);
    if constexpr (!RAWV) {
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) acc[cs][dt] = acc[cs][dt] * (1.0f / kUnitV) + zacc[cs][dt * NG / 8];
      if (g.rotate_v) {                                    // back to the input basis (linear, so sums of parts as well)
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
          float4v& y = acc[cs][dt];
          y = float4v{y[0] + y[1], y[0] - y[1], y[2] + y[3], y[2] - y[3]};
          y = float4v{y[0] + y[2], y[1] + y[3], y[0] - y[2], y[1] - y[3]};
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            float o = __shfl_xor(y[r], 16);
            y[r] = mj & 1 ? o - y[r] : y[r] + o;
            o = __shfl_xor(y[r], 32);
            y[r] = mj & 2 ? o - y[r] : y[r] + o;
          }
        }
#pragma unroll
        for (int half = 1; half < 8; half <<= 1)
#pragma unroll
          for (int dt = 0; dt < 8; ++dt)
            if (!(dt & half)) { const float4v u = acc[cs][dt], w = acc[cs][dt + half]; acc[cs][dt] = u + w; acc[cs][dt + half] = u - w; }
#pragma unroll
        for (int dt = 0; dt < 8; ++dt)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float y = acc[cs][dt][r] * kRotScale;
            acc[cs][dt][r] = (g.signs_v[dt >> 1] >> (16 * (dt & 1) + 4 * mj + r)) & 1u ? -y : y;
          }
      }
    }
    if (mj == 0) { sm_m[wave][16 * cs + mc] = m[cs]; sm_l[wave][16 * cs + mc] = l[cs]; }
  }
  __syncthreads();
  constexpr int kParts = few_join_parts<NC>(), kWidth = kHeadDim / kParts, kStride = kWidth + 4;
  float* const sums = reinterpret_cast<float*>(sm);
#pragma unroll
  for (int part = 0; part < kParts; ++part) {
    if (part) __syncthreads();
#pragma unroll
    for (int cs = 0; cs < NC; ++cs) {
      float top = sm_m[0][16 * cs + mc];
#pragma unroll
      for (int w = 1; w < NW; ++w) top = fmaxf(top, sm_m[w][16 * cs + mc]);
      const float f = __builtin_amdgcn_exp2f(m[cs] - top);
#pragma unroll
      for (int dt = part * (8 / kParts); dt < (part + 1) * (8 / kParts); ++dt)
        *reinterpret_cast<float4v*>(sums + (wave * (16 * NC) + 16 * cs + mc) * kStride + 16 * dt + 4 * mj - part * kWidth) = acc[cs][dt] * f;
    }
    __syncthreads();
    // 8 channels a thread, 16 (kParts = 2: 8) threads a row
    constexpr int kThreads = kWidth / 8;
    for (int r = my_tid / kThreads; r < 16 * NC; r += 64 * NW / kThreads) {
      const int d0 = 8 * (my_tid % kThreads), row = row0 + r;
      float top = sm_m[0][r], total = 0.0f;
#pragma unroll
      for (int w = 1; w < NW; ++w) top = fmaxf(top, sm_m[w][r]);
#pragma unroll
      for (int w = 0; w < NW; ++w) total += sm_l[w][r] * __builtin_amdgcn_exp2f(sm_m[w][r] - top);
      float4v y0 = float4v{0.f, 0.f, 0.f, 0.f}, y1 = y0;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float* from = sums + (w * (16 * NC) + r) * kStride + d0;
        y0 += *reinterpret_cast<const float4v*>(from);
        y1 += *reinterpret_cast<const float4v*>(from + 4);
      }
      if (row < rows) {
        const int64_t hq = ((int64_t)b * a.n_q + row / R) * a.q_heads + h * R + row % R;
        const int d = part * kWidth + d0;
        if (parts > 1) {
          float* rec = a.ws + (hq * a.splits + split) * kRec;
          store_record2(rec + d, y0[0], y0[1]); store_record2(rec + d + 2, y0[2], y0[3]);
          store_record2(rec + d + 4, y1[0], y1[1]); store_record2(rec + d + 6, y1[2], y1[3]);
          if (d == 0) store_record2(rec + kHeadDim, top, total);
        } else {
          const float inv = total > 0.0f ? 1.0f / total : 0.0f;              // (a row that sees nothing: zeros)
          const float z0[4] = {y0[0] * inv, y0[1] * inv, y0[2] * inv, y0[3] * inv}, z1[4] = {y1[0] * inv, y1[1] * inv, y1[2] * inv, y1[3] * inv};
          store_out4(a.out, a.out_dtype, hq * kHeadDim + d, z0);
          store_out4(a.out, a.out_dtype, hq * kHeadDim + d + 4, z1);
        }
      }
    }
  }
  if (parts > 1 && merge_arrive(word, a.merge_tag, parts, my_tid, &sm_last))
    merge_rows<64 * NW>(a, b, h, row0, min(16 * NC, rows - row0), parts, my_tid);
}

}  // namespace

template <int BK, int BV, int NC, int NG> hipError_t launch_few_groups(const ChunkArgs& a, hipStream_t stream) {
  const dim3 grid(a.g.batch * a.g.kv_heads, a.splits, (a.n_q * a.heads_per_kv + 16 * NC - 1) / (16 * NC)), block(64 * kFewWaves);
  if (a.out_dtype == KVQ_F32) hipLaunchKernelGGL((few_kernel<BK, BV, NC, NG, true>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((few_kernel<BK, BV, NC, NG, false>), grid, block, 0, stream, a);
  return hipGetLastError();
}
template <int BK, int BV, int NC> hipError_t launch_few_pair(const ChunkArgs& a, hipStream_t stream) {
  const int ngk = BK == 16 ? 1 : a.g.ng_k, ngv = BV == 16 ? 1 : a.g.ng_v, ng = ngk > ngv ? ngk : ngv;
  if constexpr (NC <= few_max_sets(BK, BV, 1)) if (ng == 1) return launch_few_groups<BK, BV, NC, 1>(a, stream);
  if constexpr (BK != 16 || BV != 16) {
    if constexpr (NC <= few_max_sets(BK, BV, 2)) if (ng == 2) return launch_few_groups<BK, BV, NC, 2>(a, stream);
    if constexpr (NC <= few_max_sets(BK, BV, 4)) if (ng == 4) return launch_few_groups<BK, BV, NC, 4>(a, stream);
  }
  return hipErrorInvalidValue;
}

#define KVQ_PAIR(k, v) KVQ_PAIR_(k, v)
#define KVQ_PAIR_(k, v) launch_few_k##k##v##v
hipError_t KVQ_PAIR(KVQ_INST_BK, KVQ_INST_BV)(const ChunkArgs& a, int sets, hipStream_t stream) {
  switch (sets) {
    case 1: return launch_few_pair<KVQ_INST_BK, KVQ_INST_BV, 1>(a, stream);
    case 2: return launch_few_pair<KVQ_INST_BK, KVQ_INST_BV, 2>(a, stream);
    case 3: return launch_few_pair<KVQ_INST_BK, KVQ_INST_BV, 3>(a, stream);
  }
  return hipErrorInvalidValue;
}

}  // namespace kvq
