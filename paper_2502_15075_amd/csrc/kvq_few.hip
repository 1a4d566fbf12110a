// Attention of a few query rows per kv head over the packed cache (gfx950): single tokens behind a sliding window, the verification of
// drafted tokens.  A workgroup takes up to 32 rows (query token, query head) of a kv head; where there are many, the tiles of
// kvq_chunk.hip take them.
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
// Key rows pass through a wavefront's own LDS: a lane needs 8 channels of every 32 of its token (all groups alike), which would be loads
// of a few bytes.  Their 16-byte units are permuted by the row's number so that the reads meet no bank twice.
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

// Operand of channels 32 kk .. 32 kk + 31 of token row `row`: this lane's eight (slots 8 j .. 8 j + 7 of the chunk).
template <int B> __device__ __forceinline__ u32x4 key_operand(const uint8_t* st, int row, int sw, int kk, int j, bool raw_bf) {
  constexpr uint32_t mask = B == 16 ? 0u : ((1u << (B == 3 ? 2 : B == 6 ? 4 : B)) - 1u) * 0x00010001u;
  const uint8_t* base = st + row * (16 * B);
  u32x4 out;
  if constexpr (B == 16) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(base + (((4 * kk + j) ^ sw) << 4));
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = raw_to_half2(w[i], raw_bf);
  } else if constexpr (B == 8) {
    const uint2 w = *reinterpret_cast<const uint2*>(base + (((2 * kk + (j >> 1)) ^ sw) << 4) + 8 * (j & 1));
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = as_u32(whole_to_half2(((i >> 1 ? w.y : w.x) >> (8 * (i & 1))) & mask));
  } else if constexpr (B == 4 || B == 2 || B == 1) {
    const uint32_t w = B == 4 ? *reinterpret_cast<const uint32_t*>(base + ((kk ^ sw) << 4) + 4 * j)
                     : B == 2 ? *reinterpret_cast<const uint32_t*>(base + (((kk >> 1) ^ sw) << 4) + 8 * (kk & 1) + 4 * (j >> 1)) >> (8 * (j & 1))
                              : *reinterpret_cast<const uint32_t*>(base + 4 * kk) >> (4 * j);
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = as_u32(whole_to_half2((w >> (B * i)) & mask));
  } else if constexpr (B == 3) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(base) + 3 * kk;
    const uint32_t lo = w[j >> 1] >> (8 * (j & 1)), hi = w[2] >> (16 * (j >> 1) + 4 * (j & 1));
#pragma unroll
    for (int i = 0; i < 4; ++i)
      out[i] = as_u32(whole_to_half2(((lo >> (2 * i)) & mask) | (((hi >> i) & 1u) << 2) | (((hi >> (i + 8)) & 1u) << 18)));
  } else {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(base) + 6 * kk;
    const uint32_t lo = w[j], hi = w[4 + (j >> 1)] >> (16 * (j & 1));
#pragma unroll
    for (int i = 0; i < 4; ++i)
      out[i] = as_u32(whole_to_half2(((lo >> (4 * i)) & mask) | (((hi >> (2 * i)) & 3u) << 4) | (((hi >> (2 * i + 8)) & 3u) << 20)));
  }
  return out;
}

// ---- value blocks: a lane's piece, 2 b dwords; field 4 dt + v is pair v (tokens 2 v, 2 v + 1 of the lane's eight) of channel tile dt
template <int B> __device__ __forceinline__ uint32_t value_field(const uint32_t* w, int q) {
  constexpr int P = 16 / B;
  constexpr uint32_t mask = B == 16 ? 0xFFFFFFFFu : ((1u << B) - 1u) * 0x00010001u;
  return (w[q / P] >> (B * (q % P))) & mask;
}
template <int B> __device__ __forceinline__ u32x4 value_operand(const uint32_t* w, int dt) {
  u32x4 out;
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    const int q = 4 * dt + v;
    if constexpr (B == 16) out[v] = w[q];
    else if constexpr (B == 3) out[v] = as_u32(whole_to_half2(value_field<2>(w, q) | (value_field<1>(w + 4, q) << 2)));
    else if constexpr (B == 6) out[v] = as_u32(whole_to_half2(value_field<4>(w, q) | (value_field<2>(w + 8, q) << 4)));
    else out[v] = as_u32(whole_to_half2(value_field<B>(w, q)));
  }
  return out;
}

template <int BK, int BV> struct Step {
  u32x4 k[key_loads<BK>()];
  uint32_t v[2 * BV];
  u32x4 meta;
};

// NG: the larger number of groups per row of the two tensors; a tensor with fewer is taken as one with NG whose scales repeat.
template <int BK, int BV, int NC, int NG, bool FINE>
__global__ __launch_bounds__((64 * few_waves<BK, BV, NC>()), 2) void few_kernel(const ChunkArgs a) {
  constexpr int NW = few_waves<BK, BV, NC>(), NK = key_loads<BK>(), ST = few_stages<BK, BV, NC>();
  constexpr int kWaveBytes = few_wave_bytes<BK, BV>();
  constexpr bool RAWK = BK == 16, RAWV = BV == 16;
  __shared__ __attribute__((aligned(16))) uint8_t sm[few_lds_bytes<BK, BV, NC>()];
  __shared__ __attribute__((aligned(16))) float sm_sums[16 * NC][4];
  __shared__ float sm_kappa[16 * NC];
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
  const int per = __builtin_amdgcn_readfirstlane((n_blocks + a.splits - 1) / a.splits);
  const int begin = split * per, end = min(begin + per, n_blocks);
  const int n_my = begin + wave < end ? (int)((unsigned)(end - begin - wave + NW - 1) / NW) : 0;
  auto block_of = [&](int i) { const int x = begin + wave + NW * i; return x < sink_blocks ? x : x - sink_blocks + first; };

  // ---- loads of a step
  const int nmk = RAWK ? 0 : 8 * g.ng_k, nmv = RAWV ? 0 : 8 * g.ng_v;        // 16-byte units of scales and zeros
  uint32_t k_off[NK];
#pragma unroll
  for (int i = 0; i < NK; ++i) {
    const int u = min(64 * i + lane, 32 * BK - 1), row = u / BK;
    k_off[i] = (uint32_t)(row * BK + ((u % BK) ^ key_swizzle<BK>(row))) * 16;
  }
  const int mu = min(lane, nmk + nmv - 1);
  const uint8_t* const meta_base = mu < nmk ? (const uint8_t*)a.cache.k_meta : (const uint8_t*)a.cache.v_meta;
  const int meta_step = mu < nmk ? 128 * g.ng_k : 128 * g.ng_v, meta_off = 16 * (mu < nmk ? mu : mu - nmk);
  typedef const __attribute__((address_space(4))) int32_t* TablePtr;
  const TablePtr pages = (TablePtr)(uintptr_t)(g.page_shift ? a.cache.page_table + (int64_t)b * g.pages_per_seq : nullptr);
  const int page_blocks = g.page_shift - 5;
  auto page_of = [&](int blk) -> int { return g.page_shift ? pages[blk >> page_blocks] : 0; };
  // (live = 0: a step that is not there; its loads collapse to one line)
  auto load = [&](Step<BK, BV>& s, int blk, int page, uint32_t live) {
    const int64_t vb = g.page_shift ? (((int64_t)page * g.kv_heads + h) << page_blocks) + (blk & ((1 << page_blocks) - 1))
                                    : ((int64_t)b * g.kv_heads + h) * (g.t_cap >> 5) + blk;
    const uint8_t* kp = (const uint8_t*)a.cache.k_codes + vb * (512 * BK);
    const uint8_t* vp = (const uint8_t*)a.cache.v_codes + vb * (512 * BV);
#pragma unroll
    for (int i = 0; i < NK; ++i) s.k[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(kp + (k_off[i] & live)));
    load_value_piece<BV>(s.v, vp, lane, live);
    if constexpr (RAWK && RAWV) s.meta = u32x4{0u, 0u, 0u, 0u};
    else
      s.meta = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(meta_base + vb * meta_step + (meta_off & live)));
  };

  Step<BK, BV> ring[ST];
  if (n_my > 0) {
#pragma unroll
    for (int s = 0; s < ST; ++s) {
      const int blk = block_of(s < n_my ? s : 0);
      load(ring[s], blk, page_of(blk), s < n_my ? ~0u : 0u);
    }
  }

  // ---- query
  stage_query<64 * NW>(a, b, h, row0, rows, 16 * NC, NG, sm, nullptr, sm_sums, sm_kappa);
  __syncthreads();
  u32x4 qb[NC][4];
  float qsum[NC][NG], kappa[NC];
  int my_p[NC];
#pragma unroll
  for (int cs = 0; cs < NC; ++cs) {
    const int r = 16 * cs + c;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) qb[cs][kk] = *reinterpret_cast<const u32x4*>(sm + r * 256 + (((4 * kk + j) ^ (r & 15)) << 4));
    const float4v q4 = *reinterpret_cast<const float4v*>(sm_sums[r]);
#pragma unroll
    for (int n = 0; n < NG; ++n) qsum[cs][n] = q4[n];
    kappa[cs] = sm_kappa[r];
    my_p[cs] = p0 + min(row0 + r, rows - 1) / R;
  }
  __syncthreads();                                         // (the query's place is the wavefronts' from here on)
  uint8_t* const st = sm + wave * kWaveBytes;
  uint8_t* const st_meta = st + NK * 1024;

  // value scales of 64 and more take their bits of room from the weights
  const int scale_exp = RAWV ? 0 : a.cache.v_scale_exp[(int64_t)b * g.kv_heads + h];
  const float weight_bits = kFewWeightBits - (float)max(scale_exp - 20, 0);
  const int sw = key_swizzle<BK>(c);

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

  // where the scales and zeros of part n (of NG) of a row lie: group n >> shift of the tensor's
  const int ngk = RAWK ? 1 : g.ng_k, ngv = RAWV ? 1 : g.ng_v;
  const int shift_k = NG == ngk ? 0 : NG == 2 * ngk ? 1 : 2, shift_v = NG == ngv ? 0 : NG == 2 * ngv ? 1 : 2;
  auto meta_k = [&](int x4, int n) { return *reinterpret_cast<const u32x4*>(st_meta + ((x4 * ngk + (n >> shift_k)) * 16 + 4 * j) * 4); };
  auto meta_v = [&](int x4, int n) { return *reinterpret_cast<const u32x4*>(st_meta + 16 * nmk + ((x4 * ngv + (n >> shift_v)) * 16 + 4 * j) * 4); };
  auto compute = [&](Step<BK, BV>& s, int blk) {
    const int t0 = 32 * blk;
    // keys and scales through LDS
#pragma unroll
    for (int i = 0; i < NK; ++i) *reinterpret_cast<u32x4*>(st + 1024 * i + 16 * lane) = s.k[i];
    if constexpr (!RAWK || !RAWV) *reinterpret_cast<u32x4*>(st_meta + 16 * lane) = s.meta;
    __builtin_amdgcn_wave_barrier();
    float sc[NC][8];
#pragma unroll
    for (int x4 = 0; x4 < 2; ++x4) {
      u32x4 ka[4];
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) ka[kk] = key_operand<BK>(st, 16 * x4 + c, sw, kk, j, raw_bf);
      constexpr int NGK = RAWK ? 1 : NG;
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
#pragma unroll
          for (int kk = n * (4 / NGK); kk < (n + 1) * (4 / NGK); ++kk) d = mma16(ka[kk], qb[cs][kk], d);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            float& y = sc[cs][4 * x4 + r];
            y = RAWK ? d[r] : fmaf(meta_s(mk[r]), d[r], fmaf(meta_z(mk[r]), qsum[cs][n], y));
          }
        }
      }
    }
    // slot 4 x4 + r of a lane: token 16 x4 + 4 j + r of the block
    const bool whole = t0 + 31 <= p_first && (a.window == 0 || t0 > p_last - a.window);
    if (!whole) {
#pragma unroll
      for (int cs = 0; cs < NC; ++cs) {
        const int my_lo = a.window ? my_p[cs] - a.window : -1;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int t = t0 + 16 * (i >> 2) + 4 * j + (i & 3);
          const bool seen = (t <= my_p[cs]) & ((t > my_lo) | (t < a.sinks));
          sc[cs][i] = seen ? sc[cs][i] : -INFINITY;
        }
      }
    }
    float p[NC][8];
#pragma unroll
    for (int cs = 0; cs < NC; ++cs) {
      float most = sc[cs][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) most = fmaxf(most, sc[cs][i]);
      most *= kappa[cs];
      if (__any(most > m[cs] + kFewSlack)) {
        const float m_new = fmaxf(m[cs], over_rows_max(most)), f = exp2f(m[cs] - m_new);
        m[cs] = m_new;
        l[cs] *= f;
#pragma unroll
        for (int n = 0; n < NG; ++n) zacc[cs][n] *= f;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) acc[cs][dt] *= f;
      }
      const float off = weight_bits - m[cs];
#pragma unroll
      for (int i = 0; i < 8; ++i) { p[cs][i] = __builtin_amdgcn_exp2f(fmaf(sc[cs][i], kappa[cs], off)); l[cs] += p[cs][i]; }
    }
    const bool tail = t0 + 32 > limit;
    const int valid = limit - (t0 + 4 * j);                // tokens 16 x4 + r of this lane below it exist
    // weights of every part of the value rows (8 / NGV channel tiles each), and the product with its tiles
    constexpr int NGV = RAWV ? 1 : NG;
#pragma unroll
    for (int n = 0; n < NGV; ++n) {
      u32x4 mv[2], hi[NC], lo[NC];
      if constexpr (!RAWV) {
#pragma unroll
        for (int x4 = 0; x4 < 2; ++x4) {
          mv[x4] = meta_v(x4, n);
          if (tail) {                                      // (what lies behind the sequence's end is no number)
#pragma unroll
            for (int r = 0; r < 4; ++r) mv[x4][r] = 16 * x4 + r < valid ? mv[x4][r] : 0u;
          }
        }
      }
#pragma unroll
      for (int cs = 0; cs < NC; ++cs) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float w0 = p[cs][2 * i], w1 = p[cs][2 * i + 1];
          if constexpr (!RAWV) {
            const uint32_t e0 = mv[i >> 1][2 * (i & 1)], e1 = mv[i >> 1][2 * (i & 1) + 1];
            zacc[cs][n] = fmaf(w0, meta_z(e0), zacc[cs][n]);
            zacc[cs][n] = fmaf(w1, meta_z(e1), zacc[cs][n]);
            w0 *= meta_s(e0);
            w1 *= meta_s(e1);
          }
          half2v x;
          x[0] = (_Float16)w0; x[1] = (_Float16)w1;
          hi[cs][i] = as_u32(x);
          if constexpr (FINE) {
            half2v y;
            y[0] = (_Float16)(w0 - (float)x[0]); y[1] = (_Float16)(w1 - (float)x[1]);
            lo[cs][i] = as_u32(y);
          }
        }
      }
#pragma unroll
      for (int dt = n * (8 / NGV); dt < (n + 1) * (8 / NGV); ++dt) {
        u32x4 va = value_operand<BV>(s.v, dt);
        if constexpr (RAWV) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t x = raw_to_half2(va[i], raw_bf);
            const int at = 16 * (i >> 1) + 2 * (i & 1);
            if (tail) x &= (at < valid ? 0x0000FFFFu : 0u) | (at + 1 < valid ? 0xFFFF0000u : 0u);
            va[i] = x;
          }
        }
#pragma unroll
        for (int cs = 0; cs < NC; ++cs) {
          acc[cs][dt] = mma16(va, hi[cs], acc[cs][dt]);
          if constexpr (FINE) acc[cs][dt] = mma16(va, lo[cs], acc[cs][dt]);
        }
      }
    }
    __builtin_amdgcn_wave_barrier();
  };

  for (int i0 = 0; i0 < n_my; i0 += ST) {
#pragma unroll
    for (int s = 0; s < ST; ++s) {
      const int i = i0 + s;
      if (i >= n_my) break;                                // uniform
      const int next = i + ST < n_my ? i + ST : 0;
      const int page = page_of(block_of(next));
      compute(ring[s], block_of(i));
      load(ring[s], block_of(next), page, i + ST < n_my ? ~0u : 0u);
    }
  }

  // ---- join the wavefronts, halves onto halves
  constexpr int kJoin = NC * 64 * (32 + 6) * 4;            // bytes of one wavefront's sums
  __syncthreads();
#pragma unroll
  for (int half = NW / 2; half >= 1; half >>= 1) {
    if (wave >= half && wave < 2 * half) {
      float* to = reinterpret_cast<float*>(sm + (wave - half) * kJoin);
#pragma unroll
      for (int cs = 0; cs < NC; ++cs) {
        float* q = to + cs * (64 * 38);
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) *reinterpret_cast<float4v*>(q + 256 * dt + 4 * lane) = acc[cs][dt];
        *reinterpret_cast<float4v*>(q + 2048 + 4 * lane) = float4v{zacc[cs][0], zacc[cs][NG > 1], zacc[cs][NG > 2 ? 2 : 0], zacc[cs][NG > 2 ? 3 : 0]};
        q[2304 + lane] = m[cs];
        q[2368 + lane] = l[cs];
      }
    }
    __syncthreads();
    if (wave < half) {
      const float* from = reinterpret_cast<const float*>(sm + wave * kJoin);
#pragma unroll
      for (int cs = 0; cs < NC; ++cs) {
        const float* q = from + cs * (64 * 38);
        const float m2 = q[2304 + lane], l2 = q[2368 + lane];
        const float m_new = fmaxf(m[cs], m2), f = exp2f(m[cs] - m_new), f2 = exp2f(m2 - m_new);
        m[cs] = m_new;
        l[cs] = l[cs] * f + l2 * f2;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) acc[cs][dt] = acc[cs][dt] * f + *reinterpret_cast<const float4v*>(q + 256 * dt + 4 * lane) * f2;
        const float4v z = *reinterpret_cast<const float4v*>(q + 2048 + 4 * lane);
#pragma unroll
        for (int n = 0; n < NG; ++n) zacc[cs][n] = zacc[cs][n] * f + z[n] * f2;
      }
    }
    __syncthreads();
  }
  if (wave != 0) return;

  // ---- results: acc[cs][dt][r] is channel 16 dt + 4 j + r of row 16 cs + c
#pragma unroll
  for (int cs = 0; cs < NC; ++cs) {
    l[cs] = over_rows_sum(l[cs]);
#pragma unroll
    for (int n = 0; n < NG; ++n) zacc[cs][n] = over_rows_sum(zacc[cs][n]);
    if constexpr (!RAWV) {
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) {
        acc[cs][dt] += zacc[cs][dt * NG / 8];
      }
      if (g.rotate_v) {                                    // back to the input basis (linear, so sums of parts as well)
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
          float4v& x = acc[cs][dt];
          x = float4v{x[0] + x[1], x[0] - x[1], x[2] + x[3], x[2] - x[3]};
          x = float4v{x[0] + x[2], x[1] + x[3], x[0] - x[2], x[1] - x[3]};
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            float o = __shfl_xor(x[r], 16);
            x[r] = j & 1 ? o - x[r] : x[r] + o;
            o = __shfl_xor(x[r], 32);
            x[r] = j & 2 ? o - x[r] : x[r] + o;
          }
        }
#pragma unroll
        for (int step = 1; step < 8; step <<= 1)
#pragma unroll
          for (int dt = 0; dt < 8; ++dt)
            if (!(dt & step)) { const float4v u = acc[cs][dt], w = acc[cs][dt + step]; acc[cs][dt] = u + w; acc[cs][dt + step] = u - w; }
#pragma unroll
        for (int dt = 0; dt < 8; ++dt)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float y = acc[cs][dt][r] * kRotScale;
            acc[cs][dt][r] = (g.signs_v[dt >> 1] >> (16 * (dt & 1) + 4 * j + r)) & 1u ? -y : y;
          }
      }
    }
    const int row = row0 + 16 * cs + c;
    if (row < rows) {
      const int64_t hq = ((int64_t)b * a.n_q + row / R) * a.q_heads + h * R + row % R;
      if (a.splits > 1) {
        float* rec = a.ws + (hq * a.splits + split) * kRec;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) *reinterpret_cast<float4v*>(rec + 16 * dt + 4 * j) = acc[cs][dt];
        if (j == 0) { rec[kHeadDim] = m[cs]; rec[kHeadDim + 1] = l[cs]; }
      } else {
        const float inv = l[cs] > 0.0f ? 1.0f / l[cs] : 0.0f;              // (a row that sees nothing: zeros)
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
          const float4v x = acc[cs][dt] * inv;
          const float y[4] = {x[0], x[1], x[2], x[3]};
          store_out4(a.out, a.out_dtype, hq * kHeadDim + 16 * dt + 4 * j, y);
        }
      }
    }
  }
}

}  // namespace

template <int BK, int BV, int NC, int NG> hipError_t launch_few_groups(const ChunkArgs& a, hipStream_t stream) {
  const dim3 grid(a.g.batch * a.g.kv_heads, a.splits, (a.n_q * a.heads_per_kv + 16 * NC - 1) / (16 * NC)), block(64 * few_waves<BK, BV, NC>());
  if (a.out_dtype == KVQ_F32) hipLaunchKernelGGL((few_kernel<BK, BV, NC, NG, true>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((few_kernel<BK, BV, NC, NG, false>), grid, block, 0, stream, a);
  return hipGetLastError();
}
template <int BK, int BV, int NC> hipError_t launch_few_pair(const ChunkArgs& a, hipStream_t stream) {
  const int ngk = BK == 16 ? 1 : a.g.ng_k, ngv = BV == 16 ? 1 : a.g.ng_v, ng = ngk > ngv ? ngk : ngv;
  if (ng == 1) return launch_few_groups<BK, BV, NC, 1>(a, stream);
  if constexpr (BK != 16 || BV != 16) {
    if (ng == 2) return launch_few_groups<BK, BV, NC, 2>(a, stream);
    if (ng == 4) return launch_few_groups<BK, BV, NC, 4>(a, stream);
  }
  return hipErrorInvalidValue;
}

#define KVQ_PAIR(k, v) KVQ_PAIR_(k, v)
#define KVQ_PAIR_(k, v) launch_few_k##k##v##v
hipError_t KVQ_PAIR(KVQ_INST_BK, KVQ_INST_BV)(const ChunkArgs& a, int sets, hipStream_t stream) {
  return sets == 1 ? launch_few_pair<KVQ_INST_BK, KVQ_INST_BV, 1>(a, stream) : launch_few_pair<KVQ_INST_BK, KVQ_INST_BV, 2>(a, stream);
}

}  // namespace kvq
