// Attention of several query tokens per sequence over the packed cache (gfx950): chunks of a prompt, verification of
// drafted tokens, with or without a sliding window and sinks.
//
//   S[t,i]  = sum_g sK[t,g] (sum_{d in g} q[i,d] cK[t,d]) + zK[t,g] (sum_{d in g} q[i,d])
//   out[i]  = sum_t P[t,i] V^[t,:] / sum_t P[t,i],   P = 2^(kappa S - m),  kappa = softmax_scale log2 e
//
// The rows i of a kv head are its (query token, query head) pairs, token-major, so every row of a tile sees about the same tokens and
// nothing is padded whatever the head ratio.  S is formed transposed (tokens x rows) by 32x32x16 matrix instructions: a lane then
// owns one row of the softmax (its half of a tile's tokens), and its weights are in the place where the second product, channels x rows,
// wants them.  Tokens reach the matrix rows with bits 3 and 4 of their number swapped, which makes the packed value blocks' order the
// operand's order.
//
// A tile of 64 tokens is unpacked once per workgroup into LDS: keys as binary16 codes (0 .. 255: exact, so their products with the query
// are too), values as binary16 reconstructions (rounded once, half a unit of 2^-11; the weights are rounded alike).  For outputs in
// binary32 (FINE) weights and values travel as two binary16 parts each, 2^-22 of them, and three products are summed.  Key scales are
// applied to the binary32 sums of their group, key zeros come in through one more matrix instruction against the query's group sums,
// each split into two binary16 parts.
//
// Bound by LDS, by issue and by power together.  2048 query tokens of 32 heads on 32768 tokens, 4/2 bits: 1.06 TFLOP in 1226 us (869 TFLOP/s; a
// product of 8192^3 reaches 1313).  Of its 2.9 million cycles a compute unit's LDS reads take about 1.5 (42 of 16 bytes a lane and wavefront tile, 8
// cycles each), a SIMD's vector instructions 1.4, its matrix instructions 1.1; matrix instructions of ordinary operands alone run at 20 ns
// each under sustained load, 14 with zeros.  What the steps gave: 128 rows a workgroup, two of them a compute unit, each tile loaded when
// its turn came 1640; the next tile's words on their way meanwhile 1577; 256 rows, so that unpacking is shared by eight wavefronts 1419;
// uniform addresses and a maximum that is looked for only when a sum shows that it lags 1380 on that card, 1253 on this; key scales read as
// binary16, two groups of four tokens at a time, 1226.  Nothing: unpacking before the products in half of a workgroup's wavefronts, priorities.
// Steps of four matrix instructions with the next operands read ahead and the last scores' arithmetic between them, in one wavefront's code, took
// 30 % more vector instructions and 1685 us.
#include "kvq_attend.h"
#include "kvq_few.h"

namespace kvq {
namespace {

constexpr float kWeightBits = 10.0f;     // weights carry 2^10: small ones stay clear of binary16's subnormals
constexpr float kMaxWeight = 32768.0f;   // the running maximum is raised once a lane's 16 weights sum to more: none passes binary16's range
constexpr int kTileTokens = 64;
constexpr int kRowsPerWave = 32;

__device__ __forceinline__ float16v mma32(u32x4 a, u32x4 b, float16v c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8v, a), __builtin_bit_cast(half8v, b), c, 0, 0, 0);
}

// One 32-channel chunk of a key row, B dwords, into registers ...
template <int B> __device__ __forceinline__ void load_key_chunk(uint32_t* w, const uint32_t* __restrict__ p) {
  if constexpr (B % 4 == 0) {
#pragma unroll
    for (int i = 0; i < B / 4; ++i) {
      const u32x4 x = reinterpret_cast<const u32x4*>(p)[i];
#pragma unroll
      for (int e = 0; e < 4; ++e) w[4 * i + e] = x[e];
    }
  } else if constexpr (B == 2) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    w[0] = x.x; w[1] = x.y;
  } else {
#pragma unroll
    for (int i = 0; i < B; ++i) w[i] = p[i];
  }
}
// ... and its codes as 16 binary16 pairs in slot order, four 16-byte pieces (PIECES 2: the first or the second half, B / 2 dwords).
template <int B, int PIECES = 4> __device__ __forceinline__ void unpack_key_chunk(const uint32_t* w, bool raw_bf, uint32_t one_k, u32x4 (&out)[PIECES]) {
  constexpr int LO = code_lo_bits<B>(), HI = code_hi_bits<B>();
  constexpr int P = 16 / LO;                       // pairs per dword
  constexpr uint32_t mask = B == 16 ? 0xFFFFFFFFu : ((1u << LO) - 1u) * 0x00010001u;
#pragma unroll
  for (int s = 0; s < 4 * PIECES; ++s) {
    const int dw = s / P, f = s % P;
    uint32_t x = w[dw] >> (LO * f);
    if constexpr (B == 16) {
      out[s >> 2][s & 3] = raw_to_half2(x, raw_bf);
    } else {
      if constexpr (HI != 0) {
        // channels x0 = 2 P dw + f and x0 + P: their high parts, HI bits each, at bits HI x of the high run
        constexpr uint32_t hmask = (1u << HI) - 1u;
        const int at = HI * (2 * P * dw + f), next = at + HI * P;
        x &= mask;
        x |= ((w[LO + at / 32] >> (at % 32)) & hmask) << LO;
        x |= ((w[LO + next / 32] >> (next % 32)) & hmask) << (LO + 16);
      }
      out[s >> 2][s & 3] = as_u32(whole_to_half2(x, HI != 0 ? ~0u : mask, one_k));
    }
  }
}

// The B-bit fields of four 16-channel tiles (tiles 4 half .. 4 half + 3) of a lane's piece of a value block, B dwords ...
template <int B> __device__ __forceinline__ void load_value_half(uint32_t* w, const uint32_t* __restrict__ block, int lane, int half) {
  if constexpr (B == 1) {
    w[0] = block[2 * lane + half];
  } else if constexpr (B == 2) {
    const uint2 x = *reinterpret_cast<const uint2*>(block + 4 * lane + 2 * half);
    w[0] = x.x; w[1] = x.y;
  } else {
#pragma unroll
    for (int i = 0; i < B / 4; ++i) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(block + 256 * (B / 4 * half + i) + 4 * lane);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[4 * i + e] = x[e];
    }
  }
}
// ... as pairs: pair v of tile t is the words' field 4 t + v, tokens 2 v and 2 v + 1 of the lane's eight (with what lies above the field; MASKED: cut to
// it, for what is joined with high parts).
template <int B, bool MASKED = false, int N = 16> __device__ __forceinline__ void value_fields(const uint32_t* w, uint32_t (&out)[N]) {
  constexpr int P = 16 / B;
  constexpr uint32_t mask = B == 16 ? 0xFFFFFFFFu : ((1u << B) - 1u) * 0x00010001u;
#pragma unroll
  for (int s = 0; s < N; ++s) out[s] = MASKED ? (w[s / P] >> (B * (s % P))) & mask : w[s / P] >> (B * (s % P));
}

// N consecutive words, 1, 2 or 4, aligned to as many
template <int N> __device__ __forceinline__ void load_words(uint32_t* w, const uint32_t* __restrict__ p) {
  if constexpr (N == 4) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = x[e];
  } else if constexpr (N == 2) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    w[0] = x.x; w[1] = x.y;
  } else {
    w[0] = *p;
  }
}

// What a workgroup walks: tokens [0, sink_tiles * 64) and [first * 64, ...), n tiles in all.
struct Walk { int lo, sink_tiles, first, n; };              // lo: the oldest token that a window leaves to some row
__device__ __forceinline__ Walk make_walk(int p_first, int p_last, int window, int sinks) {
  Walk w;
  w.lo = window ? max(p_first - window + 1, 0) : 0;
  w.first = w.lo / kTileTokens;
  w.sink_tiles = min((sinks + kTileTokens - 1) / kTileTokens, w.first);
  w.n = p_last < 0 ? 0 : w.sink_tiles + (p_last / kTileTokens + 1 - w.first);
  return w;
}

// The tokens of row tile `tile` of sequence b and the parts they are cut into
struct TileSpan { int rows, row0, p0, p_last, parts; Walk walk; };
__device__ __forceinline__ TileSpan tile_span(const ChunkArgs& a, int b, int tile, int tile_rows) {
  TileSpan s;
  const int R = a.heads_per_kv;
  const int len = a.seq_lens ? min(max(a.seq_lens[b], 0), a.seq_bound) : a.seq_bound;
  const int nq = a.q_lens ? min(max(a.q_lens[b], 0), a.n_q) : a.n_q;
  s.rows = nq * R;
  s.row0 = tile * tile_rows;
  s.p0 = len - nq;                                         // position of query token 0
  s.p_last = s.p0 + __builtin_amdgcn_readfirstlane((min(s.row0 + tile_rows, s.rows) - 1) / R);
  s.walk = make_walk(s.p0 + __builtin_amdgcn_readfirstlane(s.row0 / R), s.p_last, a.window, a.sinks);
  s.parts = a.splits == 1 ? 1 : max(__builtin_amdgcn_readfirstlane((s.walk.n + a.per - 1) / a.per), 1);
  return s;
}

constexpr int tile_waves(int bk) { return bk ? 8 : 4; }

// BK, BV: the widths, or 0 and 0: any, told at run time.  With widths known eight wavefronts take 256 rows, a thread's share of the next tile is
// loaded while this one is computed, and there are two tiles in LDS, one computed while the other is unpacked.
template <int BK, int BV, int NG, bool FINE>
__global__ __launch_bounds__(64 * tile_waves(BK), 2) void chunk_kernel(const ChunkArgs a) {
  constexpr bool kAhead = BK != 0;
  constexpr int kWaves = tile_waves(BK), kTileRows = kRowsPerWave * kWaves;
  constexpr int kPair = NG < 2 ? 1 : 2;
  constexpr int kTileBytes = kTileTokens * kHeadDim * 2, kBuffers = kAhead ? 2 : 1, kBufferBytes = (FINE ? 3 : 2) * kTileBytes;
  __shared__ __attribute__((aligned(16))) uint8_t sm_tile[kBuffers * kBufferBytes];            // keys, values, the values' second parts
  __shared__ __attribute__((aligned(16))) uint16_t sm_scale_[kBuffers][NG / kPair][kTileTokens * kPair];       // key scales, by matrix row, two groups side by side
  __shared__ __attribute__((aligned(16))) uint32_t sm_zero_[kBuffers][kTileTokens][4];         // key zeros, each twice
  __shared__ __attribute__((aligned(16))) uint32_t sm_qsum[kTileRows][4];                      // group sums of the query, two parts each
  __shared__ float sm_kappa[kTileRows];
  const Geom& g = a.g;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // (a division leaves its result in vector registers, and with it every address: these are the same in all lanes)
  const int b = __builtin_amdgcn_readfirstlane(blockIdx.x / g.kv_heads), h = blockIdx.x - b * g.kv_heads;
  const int R = a.heads_per_kv;
  const int split = blockIdx.z, tile = (int)gridDim.y - 1 - (int)blockIdx.y;          // later rows see more: they go first
  const TileSpan span = tile_span(a, b, tile, kTileRows);
  const int row0 = span.row0, rows = span.rows, p0 = span.p0, p_last = span.p_last, parts = span.parts;
  const Walk walk = span.walk;
  if (row0 >= rows || split >= parts) return;              // uniform
  const int t_begin = split * a.per, t_end = min(t_begin + a.per, walk.n);
  const int limit = p_last + 1;                          // no row of the tile sees a token from here on
  const bool raw_bf = g.raw_dtype == KVQ_BF16;
  // Reconstructions may lie past binary16's largest number (code * scale + zero with a scale that was rounded up): results that overflow
  // become that number, half a step off, instead of infinity (FP16_OVFL, bit 23 of the MODE register).
  __builtin_amdgcn_s_setreg(1 | (23 << 6), 1);

  stage_query<64 * kWaves>(a, b, h, row0, rows, kTileRows, NG, sm_tile, sm_qsum, nullptr, sm_kappa);
  __syncthreads();
  const int col = lane & 31, hh = lane >> 5;
  const int my_row = wave * kRowsPerWave + col;
  u32x4 qb[8], qs;
#pragma unroll
  for (int kk = 0; kk < 8; ++kk)
    qb[kk] = *reinterpret_cast<const u32x4*>(sm_tile + my_row * 256 + (((2 * kk + hh) ^ (my_row & 15)) << 4));
  qs = *reinterpret_cast<const u32x4*>(sm_qsum[my_row]);
  if (hh) qs = u32x4{0u, 0u, 0u, 0u};
  const float kappa = sm_kappa[my_row];
  const int my_p = p0 + min(row0 + my_row, rows - 1) / R;                    // position of this lane's query
  const int my_lo = a.window ? my_p - a.window : -1;                         // ... and the newest token that is too old for it
  // the wavefront's positions, for the tiles that need no mask
  const int w_first = p0 + __builtin_amdgcn_readfirstlane(min(row0 + wave * kRowsPerWave, rows - 1) / R);
  const int w_last = p0 + __builtin_amdgcn_readfirstlane(min(row0 + wave * kRowsPerWave + 31, rows - 1) / R);
  __syncthreads();

  float16v acc[4];
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[ct][i] = 0.0f;
  float m = kNoMax, l = 0.0f;
  const bool two_parts = g.bits_v != 16;                   // (patterns of an unquantized plane have no second part)
  const uint32_t one_k = one_k_pattern(), v_mask = ((1u << min(g.bits_v, 15)) - 1u) * 0x00010001u;

  // (a block of tiles: [0, sink_tiles) and [first, ...))
  auto first_token = [&](int ti) { return (ti < walk.sink_tiles ? ti : walk.first + ti - walk.sink_tiles) * kTileTokens; };
  // Thread t unpacks, of token `tok`, part `chunk` of its key row, and tiles 4 half ... of value block `vblk` as lane (j, dl) of a fragment; with
  // eight wavefronts half as much: the part's half `sub`, tiles 2 half ... .
  constexpr int kPieces = kAhead ? 2 : 4, kTiles = kAhead ? 2 : 4, kPairs = 4 * kTiles;
  const int tok = tid / (16 / kPieces), sub = kAhead ? tid & 1 : 0, chunk = (tid >> (kAhead ? 1 : 0)) & 3;
  const int vblk = tid / (128 * 4 / kTiles), half = (tid >> 6) & (8 / kTiles - 1), j = lane >> 4, dl = lane & 15;
  const int x_ = tok & 31, k_row = (tok & 32) | (x_ & 7) | ((x_ & 8) << 1) | ((x_ & 16) >> 1);        // bits 3 and 4 swapped
  const int per_group = g.g_v >> 4;                        // 16-channel tiles of a value group
  // Addresses: where the tile begins, the same for all lanes, and a 32-bit distance from there
  auto tile_base = [&](int t0) {
    const int64_t base = virtual_token(g, a.cache.page_table, b, h, t0);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((int)base), hi = __builtin_amdgcn_readfirstlane((int)(base >> 32));
    return (int64_t)(((uint64_t)hi << 32) | lo);
  };
  auto seen_by_some = [&](int t) { return (t < limit) & ((t >= walk.lo) | (t < a.sinks)); };
  auto key_distance = [&](int t0) { return (uint32_t)min(tok, limit - 1 - t0); };              // (nothing behind the last visible token is read)
  auto value_distance = [&](int t0) { return (uint32_t)min(vblk, (limit - 1 - t0) >> 5); };
  auto load_metas = [&](int64_t base, uint32_t dk, uint32_t dv, bool raw_k, bool raw_v, uint32_t& km, u32x4 (&vm)[kTiles]) {
    km = raw_k ? 0x00003C00u : ((const uint32_t*)a.cache.k_meta + base * NG)[(dk >> 4) * (16 * NG) + 16 * min(chunk, NG - 1) + (dk & 15)];                 // (unquantized: scale 1, zero 0)
    if (raw_v) return;
#pragma unroll
    for (int n = 0; n < kTiles / 2; ++n) {
      if (n == 1 && per_group != 2) break;                 // uniform: half a row is one group, or two
      const uint32_t* mp = (const uint32_t*)a.cache.v_meta + base * g.ng_v + (32 * dv * g.ng_v + 16 * (uint32_t)((kTiles * half + 2 * n) / per_group) + 4 * j);
#pragma unroll
      for (int x4 = 0; x4 < 2; ++x4) vm[2 * n + x4] = *reinterpret_cast<const u32x4*>(mp + 16 * g.ng_v * x4);
    }
  };
  auto store = [&](const u32x4 (&piece)[kPieces], uint32_t km, uint32_t (&f)[kPairs], u32x4 (&vm)[kTiles], bool raw_v, int t0, int at) {
    uint8_t* const sm_k = sm_tile + at * kBufferBytes;
    uint8_t* const sm_v = sm_k + kTileBytes + vblk * 8192 + (j * 128 + 16 * kTiles * half + dl) * 16;
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
      *reinterpret_cast<u32x4*>(sm_k + k_row * 256 + (((4 * chunk + kPieces * sub + i) ^ (k_row & 15)) << 4)) = piece[i];
    if (!seen_by_some(t0 + tok) || chunk >= NG) km = 0;
    if (chunk < NG) sm_scale_[at][chunk / kPair][k_row * kPair + chunk % kPair] = (uint16_t)km;
    sm_zero_[at][k_row][chunk] = (km >> 16) * 0x00010001u;

    const int tv = t0 + 32 * vblk + 4 * j;                 // the lane's tokens: tv + 16 x4 + r
    const bool cut = t0 + kTileTokens > limit || t0 < walk.lo;                 // uniform: some of the tile's tokens no row sees
    if (raw_v) {
#pragma unroll
      for (int s = 0; s < kPairs; ++s) {
        const int token = tv + 16 * ((s & 2) >> 1) + 2 * (s & 1);  // pair v = s % 4: tokens 2 v, 2 v + 1 of the eight (x4, r)
        uint32_t x = raw_to_half2(f[s], raw_bf);
        if (cut) x &= (seen_by_some(token) ? 0x0000FFFFu : 0u) | (seen_by_some(token + 1) ? 0xFFFF0000u : 0u);
        f[s] = x;
      }
    } else {
      if (cut) {                                           // (what a cache holds there need be no number)
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            vm[i][r] = seen_by_some(tv + 16 * (i & 1) + r) ? vm[i][r] : 0u;
      }
      half2v sc[4], ze[4];                                 // scales and zeros of the four pairs
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        u32x4 second;
        if (t == 0 || (t == 2 && per_group == 2)) {
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const uint32_t e0 = vm[t + (v >> 1)][2 * (v & 1)], e1 = vm[t + (v >> 1)][2 * (v & 1) + 1];
            sc[v] = as_half2(__builtin_amdgcn_perm(e1, e0, 0x05040100u));      // low halves
            ze[v] = as_half2(__builtin_amdgcn_perm(e1, e0, 0x07060302u));      // high halves
          }
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const half2v code = whole_to_half2(f[4 * t + v], v_mask, one_k);
          if constexpr (FINE) {
            const float x = as_rounded(fmaf((float)code[0], (float)sc[v][0], (float)ze[v][0]));
            const float y = as_rounded(fmaf((float)code[1], (float)sc[v][1], (float)ze[v][1]));
            half2v hi, lo;
            hi[0] = (_Float16)x; hi[1] = (_Float16)y;
            lo[0] = (_Float16)(x - (float)hi[0]); lo[1] = (_Float16)(y - (float)hi[1]);
            f[4 * t + v] = as_u32(hi);
            second[v] = as_u32(lo);
          } else {
            f[4 * t + v] = as_u32(__builtin_elementwise_fma(code, sc[v], ze[v]));
          }
        }
        if constexpr (FINE) *reinterpret_cast<u32x4*>(sm_v + kTileBytes + 256 * t) = second;
      }
    }
#pragma unroll
    for (int t = 0; t < kTiles; ++t) *reinterpret_cast<u32x4*>(sm_v + 256 * t) = u32x4{f[4 * t], f[4 * t + 1], f[4 * t + 2], f[4 * t + 3]};
  };
  auto compute = [&](int ti, int at) {
    const int t0 = first_token(ti);
    const uint8_t* const sm_k = sm_tile + at * kBufferBytes;
    const uint8_t* const sm_v = sm_k + kTileBytes;
    // ---- two blocks of 32 tokens
#pragma unroll
    for (int blk = 0; blk < 2; ++blk) {
      const int tb = t0 + 32 * blk;
      if (tb > w_last) break;                              // uniform in the wavefront
      const uint8_t* kt = sm_k + blk * 8192;
      float16v s;
      {
        float16v zero;
#pragma unroll
        for (int i = 0; i < 16; ++i) zero[i] = 0.0f;
        s = mma32(*reinterpret_cast<const u32x4*>(sm_zero_[at][32 * blk + col]), qs, zero);
        typedef _Float16 scales4 __attribute__((ext_vector_type(4 * kPair)));
        scales4 sc[4];                                     // of 4 tokens each, two groups
#pragma unroll
        for (int n = 0; n < NG; ++n) {
          if (n % kPair == 0) {
#pragma unroll
            for (int q = 0; q < 4; ++q) sc[q] = *reinterpret_cast<const scales4*>(&sm_scale_[at][n / kPair][(32 * blk + 8 * q + 4 * hh) * kPair]);
          }
          float16v part = zero;
#pragma unroll
          for (int kk = n * (8 / NG); kk < (n + 1) * (8 / NG); ++kk)
            part = mma32(*reinterpret_cast<const u32x4*>(kt + col * 256 + (((2 * kk + hh) ^ (col & 15)) << 4)), qb[kk], part);
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = fmaf((float)sc[i >> 2][(i & 3) * kPair + n % kPair], part[i], s[i]);
        }
      }
      // register i: token 16 (i / 4 % 2) + 8 (i / 8) + 4 hh + i % 4 of the block
      const bool whole = tb + 31 <= w_first && (a.window == 0 || tb > w_last - a.window);
      if (!whole) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int t = tb + 16 * ((i >> 2) & 1) + 8 * (i >> 3) + 4 * hh + (i & 3);
          const bool seen = (t <= my_p) & ((t > my_lo) | (t < a.sinks));
          s[i] = seen ? s[i] : -INFINITY;
        }
      }
      // Weights with the maximum as it stands; only if their sum shows that it lags is it raised, and they are formed again
      u32x4 pw[2], pl[2];
      float sum;
      auto weights = [&]() {
        const float off = kWeightBits - m;
        sum = 0.0f;
#pragma unroll
        for (int v = 0; v < 8; ++v) {
          const float x = __builtin_amdgcn_exp2f(fmaf(s[2 * v], kappa, off)), y = __builtin_amdgcn_exp2f(fmaf(s[2 * v + 1], kappa, off));
          half2v p;
          p[0] = (_Float16)x;
          p[1] = (_Float16)y;
          pw[v >> 2][v & 3] = as_u32(p);
          if constexpr (FINE) {
            sum += x + y;
            half2v q;
            q[0] = (_Float16)(x - (float)p[0]); q[1] = (_Float16)(y - (float)p[1]);
            pl[v >> 2][v & 3] = as_u32(q);
          } else {
            sum = __builtin_amdgcn_fdot2(p, half2v{(_Float16)1.0f, (_Float16)1.0f}, sum, false);
          }
        }
      };
      weights();
      if (__any(sum > kMaxWeight)) {
        float most = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) most = fmaxf(most, s[i]);
        most = fmaxf(most, other_half(most)) * kappa;
        const float m_new = fmaxf(m, most), f = exp2f(m - m_new);
        m = m_new;
        l *= f;
#pragma unroll
        for (int ct = 0; ct < 4; ++ct)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[ct][i] *= f;
        weights();
      }
      l += sum;
      const uint8_t* vt = sm_v + blk * 8192;
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) {
          const int at = ((2 * st + hh) * 128 + 32 * ct + col) * 16;
          const u32x4 va = *reinterpret_cast<const u32x4*>(vt + at);
          acc[ct] = mma32(va, pw[st], acc[ct]);
          if constexpr (FINE) {
            acc[ct] = mma32(va, pl[st], acc[ct]);
            if (two_parts) acc[ct] = mma32(*reinterpret_cast<const u32x4*>(vt + kTileBytes + at), pw[st], acc[ct]);
          }
        }
    }
  };

  if constexpr (kAhead) {
    uint32_t raw_k[BK / 2], raw_v[BV / 2], raw_km;         // what a thread loads of a tile (paged: a tile never straddles a page)
    u32x4 raw_vm[kTiles];
    auto load = [&](int ti) {
      const int t0 = first_token(ti);
      const int64_t base = tile_base(t0);
      const uint32_t dk = key_distance(t0), dv = value_distance(t0);
      load_words<BK / 2>(raw_k, (const uint32_t*)a.cache.k_codes + base * (4 * BK) + (dk * (4 * BK) + chunk * BK + sub * (BK / 2)));
      constexpr int kWords = BV / 2;                         // of the lane's 2 BV, which lie in fours: 256 words from one four to the next
      const int w = kWords * half;
      load_words<kWords>(raw_v, (const uint32_t*)a.cache.v_codes + base * (4 * BV) + (dv * (128 * BV) + 256 * (w >> 2) + 4 * lane + (w & 3)));
      load_metas(base, dk, dv, false, false, raw_km, raw_vm);
    };
    // The loaded tile, to buffer `at`
    auto unpack = [&](int ti, int at) {
      u32x4 piece[kPieces];
      uint32_t f[kPairs];
      unpack_key_chunk<BK, kPieces>(raw_k, raw_bf, one_k, piece);
      value_fields<BV, false, kPairs>(raw_v, f);
      store(piece, raw_km, f, raw_vm, false, first_token(ti), at);
    };
    if (t_begin < t_end) {
      load(t_begin);
      unpack(t_begin, 0);
      if (t_begin + 1 < t_end) load(t_begin + 1);
      __syncthreads();
    }
    auto step = [&](int ti, int at) {
      compute(ti, at);
      if (ti + 1 < t_end) unpack(ti + 1, 1 - at);
      if (ti + 2 < t_end) load(ti + 2);
      __syncthreads();
    };
    for (int ti = t_begin; ti < t_end; ti += 2) {          // (two steps a turn: `at` is a constant, addresses in LDS are)
      step(ti, 0);
      if (ti + 1 == t_end) break;
      step(ti + 1, 1);
    }
  } else {
    // A tile of widths told at run time
    auto load_and_unpack = [&](int ti) {
      const int t0 = first_token(ti), bits_k = g.bits_k, bits_v = g.bits_v;
      const int64_t base = tile_base(t0);
      const uint32_t dk = key_distance(t0), dv = value_distance(t0);
      const uint32_t* kp = (const uint32_t*)a.cache.k_codes + base * (4 * bits_k) + (dk * (4 * bits_k) + chunk * bits_k);
      const uint32_t* vp = (const uint32_t*)a.cache.v_codes + base * (4 * bits_v) + dv * (128 * bits_v);
      u32x4 piece[4], vm[4];
      uint32_t w[16], f[16], km;
      switch (bits_k) {
        case 1: load_key_chunk<1>(w, kp); unpack_key_chunk<1>(w, raw_bf, one_k, piece); break;
        case 2: load_key_chunk<2>(w, kp); unpack_key_chunk<2>(w, raw_bf, one_k, piece); break;
        case 3: load_key_chunk<3>(w, kp); unpack_key_chunk<3>(w, raw_bf, one_k, piece); break;
        case 4: load_key_chunk<4>(w, kp); unpack_key_chunk<4>(w, raw_bf, one_k, piece); break;
        case 6: load_key_chunk<6>(w, kp); unpack_key_chunk<6>(w, raw_bf, one_k, piece); break;
        case 8: load_key_chunk<8>(w, kp); unpack_key_chunk<8>(w, raw_bf, one_k, piece); break;
        default: load_key_chunk<16>(w, kp); unpack_key_chunk<16>(w, raw_bf, one_k, piece); break;
      }
      switch (bits_v) {
        case 1: load_value_half<1>(w, vp, lane, half); value_fields<1>(w, f); break;
        case 2: load_value_half<2>(w, vp, lane, half); value_fields<2>(w, f); break;
        case 4: load_value_half<4>(w, vp, lane, half); value_fields<4>(w, f); break;
        case 8: load_value_half<8>(w, vp, lane, half); value_fields<8>(w, f); break;
        case 16: load_value_half<16>(w, vp, lane, half); value_fields<16>(w, f); break;
        default: {                                           // 3 and 6 bits: a block of low parts, a block of high parts
          uint32_t hi[16];
          if (bits_v == 3) {
            load_value_half<2>(w, vp, lane, half); value_fields<2, true>(w, f);
            load_value_half<1>(w, vp + 256, lane, half); value_fields<1, true>(w, hi);
          } else {
            load_value_half<4>(w, vp, lane, half); value_fields<4, true>(w, f);
            load_value_half<2>(w, vp + 512, lane, half); value_fields<2, true>(w, hi);
          }
          const int lo = bits_v == 3 ? 2 : 4;
#pragma unroll
          for (int s = 0; s < 16; ++s) f[s] |= hi[s] << lo;
        }
      }
      load_metas(base, dk, dv, bits_k == 16, bits_v == 16, km, vm);
      store(piece, km, f, vm, bits_v == 16, t0, 0);
    };
    for (int ti = t_begin; ti < t_end; ++ti) {
      load_and_unpack(ti);
      __syncthreads();
      compute(ti, 0);
      __syncthreads();
    }
  }

  // ---- results.  acc[ct][i]: channel 32 ct + 8 (i / 4) + 4 hh + i % 4 of row `col`
  l += other_half(l);
  if (g.rotate_v) {                                        // back to the input basis: linear, so partial sums as well
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (!(i & 1)) { const float u = acc[ct][i], w = acc[ct][i + 1]; acc[ct][i] = u + w; acc[ct][i + 1] = u - w; }
#pragma unroll
    for (int step = 2; step <= 8; step <<= 1) {
      if (step == 4) {                                     // stride 4 of the channels: the other half of the wavefront
#pragma unroll
        for (int ct = 0; ct < 4; ++ct)
#pragma unroll
          for (int i = 0; i < 16; ++i) { const float o = other_half(acc[ct][i]); acc[ct][i] = hh ? o - acc[ct][i] : acc[ct][i] + o; }
      }
#pragma unroll
      for (int ct = 0; ct < 4; ++ct)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (!(i & step)) { const float u = acc[ct][i], w = acc[ct][i + step]; acc[ct][i] = u + w; acc[ct][i + step] = u - w; }
    }
#pragma unroll
    for (int step = 1; step < 4; step <<= 1)
#pragma unroll
      for (int ct = 0; ct < 4; ++ct)
        if (!(ct & step))
#pragma unroll
          for (int i = 0; i < 16; ++i) { const float u = acc[ct][i], w = acc[ct + step][i]; acc[ct][i] = u + w; acc[ct + step][i] = u - w; }
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int d = 8 * (i >> 2) + 4 * hh + (i & 3);
        const float x = acc[ct][i] * kRotScale;
        acc[ct][i] = (g.signs_v[ct] >> d) & 1u ? -x : x;
      }
  }
  const int row = row0 + my_row;
  const int64_t hq = ((int64_t)b * a.n_q + row / R) * a.q_heads + h * R + row % R;
  if (row >= rows) return;
  if (parts > 1) {                                         // (joined by the launch behind this one)
    float* rec = a.ws + (hq * a.splits + split) * kRec;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4v*>(rec + 32 * ct + 8 * q + 4 * hh) = float4v{acc[ct][4 * q], acc[ct][4 * q + 1], acc[ct][4 * q + 2], acc[ct][4 * q + 3]};
    if (hh == 0) *reinterpret_cast<float2*>(rec + kHeadDim) = make_float2(m, l);
    return;
  }
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;            // (a row that sees nothing: zeros)
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t o = hq * kHeadDim + 32 * ct + 8 * q + 4 * hh;
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = acc[ct][4 * q + e] * inv;
      store_out4(a.out, a.out_dtype, o, y);
    }
}

// Rows whose tokens were cut into parts, 16 a workgroup (one workgroup for all rows of a tile took 30 to 80 us for 2 to 16 parts of 256 rows)
constexpr int kJoinRows = 16;
__global__ __launch_bounds__(32 * kJoinRows) void join_kernel(const ChunkArgs a, int tile_rows) {
  const int b = __builtin_amdgcn_readfirstlane(blockIdx.x / a.g.kv_heads), h = blockIdx.x - b * a.g.kv_heads;
  const int row0 = kJoinRows * blockIdx.y;
  const TileSpan span = tile_span(a, b, __builtin_amdgcn_readfirstlane(row0 / tile_rows), tile_rows);
  if (row0 >= span.rows || span.parts == 1) return;
  merge_rows<32 * kJoinRows>(a, b, h, row0, min(kJoinRows, span.rows - row0), span.parts, threadIdx.x);
}

}  // namespace

// Widths 2, 4 and 8 have row tiles of 256 rows, all others share the kernel that is told them at run time, 128 rows.
static bool tile_widths(int bk, int bv) { return (bk == 2 || bk == 4 || bk == 8) && (bv == 2 || bv == 4 || bv == 8); }
static int tile_rows(const Geom& g) { return kRowsPerWave * tile_waves(tile_widths(g.bits_k, g.bits_v) ? g.bits_k : 0); }

// What a choice costs: each workgroup `fixed` ns and `unit` ns for each of its units of tokens, in rounds of as many workgroups as the device
// takes at once, `join` ns where parts are joined.  Measured at 4/2 bits (a call's time in us, predicted and measured):
//   few rows, 1 column set, 256 workgroups x 130 blocks: 33, 30; cut in three 36, 41     8 workgroups x 33 blocks: 14, 14; cut in eight 11, 11
//   few rows, 3 column sets, 48 workgroups x 256 blocks: 99, 88; cut in four 41, 39; in eight (a second round) 55, 54
//   row tiles, 8 workgroups x 128 tiles: 314, 311             16 x 16 tiles: 57, 57      64 x 4 tiles: 29, 28
struct ChunkCost { int64_t fixed, unit, step, join; };     // step: units that a workgroup takes at a time
static void cheapest_split(const ChunkCost& c, int64_t groups, int64_t at_once, int64_t share, int64_t units, int64_t* splits, int64_t* cost) {
  *cost = INT64_MAX;
  for (const int64_t s : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64}) {
    const int64_t n = groups * s;
    if (s > 1 && (s > units || n > 2 * at_once)) break;
    // (`share`: workgroups that have a compute unit's full speed between them; those beyond take turns)
    const int64_t t = (n + at_once - 1) / at_once * c.fixed + (n + share - 1) / share * c.unit * (((units + s - 1) / s + c.step - 1) / c.step * c.step) +
                      (s > 1 ? c.join : 0);
    if (t < *cost) { *cost = t; *splits = s; }
  }
}
ChunkPlan plan_chunk(const Geom& g, int heads_per_kv, int32_t n_q, int32_t seq_bound, int32_t window, int32_t sinks) {
  const int64_t rows = (int64_t)n_q * heads_per_kv, streams = (int64_t)g.batch * g.kv_heads, cus = device_compute_units();
  // the units (blocks of 32 tokens, tiles of 64) that a row tile of so many rows sees at most
  auto units_of = [&](int64_t unit, int64_t tile) {
    int64_t all = (seq_bound + unit - 1) / unit;
    if (window) {
      const int64_t tokens = (tile + heads_per_kv - 2) / heads_per_kv + 1;     // (a tile may begin inside a token's rows)
      const int64_t some = ((int64_t)window + (tokens > n_q ? n_q : tokens) - 1 + unit - 2) / unit + 1 + ((int64_t)sinks + unit - 1) / unit;
      if (some < all) all = some;
    }
    return all < 1 ? 1 : all;
  };
  // few rows: the cache stays packed, every wavefront takes blocks of its own for up to three sets of 16 rows
  const int ngk = g.bits_k == 16 ? 1 : g.ng_k, ngv = g.bits_v == 16 ? 1 : g.ng_v, ng = ngk > ngv ? ngk : ngv;
  const int64_t most = few_max_sets(g.bits_k, g.bits_v, ng), sets = (rows + 15) / 16, few_tiles = (sets + most - 1) / most;
  const int few_sets = (int)((sets + few_tiles - 1) / few_tiles);              // as few row tiles as can be, of the same size
  const int64_t blocks = units_of(32, 16 * few_sets), resident = few_occupancy(g.bits_k, g.bits_v, few_sets, ng) / 2;
  const ChunkCost few{3500 + 3500 * few_sets, (g.bits_k + g.bits_v > 8 ? 170 : 130) + 70 * few_sets, kFewWaves, 2000 * few_sets};
  int64_t few_splits = 1, few_cost;
  cheapest_split(few, streams * few_tiles, resident * cus, cus, blocks, &few_splits, &few_cost);
  if (few_tiles == 1) return ChunkPlan{few_sets, (int32_t)few_splits, (int32_t)blocks};      // (row tiles would be filled to less than a fifth)
  // more rows: tiles
  const int64_t at_once = tile_rows(g), tiles = (rows + at_once - 1) / at_once * streams, steps = units_of(kTileTokens, at_once);
  const ChunkCost tile{20000, at_once == 256 ? 2300 : 1600, 1, 10000};
  int64_t tile_splits = 1, tile_cost;
  cheapest_split(tile, tiles, 256 / at_once * cus, cus, steps, &tile_splits, &tile_cost);
  return few_cost <= tile_cost ? ChunkPlan{few_sets, (int32_t)few_splits, (int32_t)blocks} : ChunkPlan{0, (int32_t)tile_splits, (int32_t)steps};
}
size_t chunk_record_bytes(int32_t batch, int32_t n_q, int32_t q_heads, int32_t splits) {
  return splits <= 1 ? 0 : (size_t)batch * n_q * q_heads * splits * kRec * sizeof(float);
}

size_t chunk_counter_bytes(const Geom& g, int heads_per_kv, int32_t n_q) {
  const int64_t tiles = ((int64_t)n_q * heads_per_kv + 15) / 16;               // (16 rows: the smallest tile there is)
  return (size_t)((tiles * g.batch * g.kv_heads * sizeof(MergeWord) + 15) / 16 * 16);
}

namespace {
template <int BK, int BV, int NG> void launch_tiles(const ChunkArgs& a, dim3 grid, hipStream_t stream) {
  if (a.out_dtype == KVQ_F32) hipLaunchKernelGGL((chunk_kernel<BK, BV, NG, true>), grid, dim3(64 * tile_waves(BK)), 0, stream, a);
  else hipLaunchKernelGGL((chunk_kernel<BK, BV, NG, false>), grid, dim3(64 * tile_waves(BK)), 0, stream, a);
}
template <int BK, int BV> hipError_t launch_tiles_of(const ChunkArgs& a, dim3 grid, hipStream_t stream) {
  switch (a.g.ng_k) {
    case 1: launch_tiles<BK, BV, 1>(a, grid, stream); return hipSuccess;
    case 2: launch_tiles<BK, BV, 2>(a, grid, stream); return hipSuccess;
    case 4: launch_tiles<BK, BV, 4>(a, grid, stream); return hipSuccess;
  }
  return hipErrorInvalidValue;
}
hipError_t launch_few(const ChunkArgs& a, int32_t sets, hipStream_t stream) {
  switch (32 * a.g.bits_k + a.g.bits_v) {
#define KVQ_FEW_CASE(k, v) case 32 * k + v: return launch_few_k##k##v##v(a, sets, stream);
    KVQ_FEW_PAIRS(KVQ_FEW_CASE)
  }
  return hipErrorInvalidValue;
}
}  // namespace

hipError_t launch_chunk_attention(const ChunkArgs& args, const ChunkPlan& plan, hipStream_t stream) {
  ChunkArgs a = args;
  if (plan.few_sets) {
    if (a.splits > 1) a.merge_tag = next_merge_tag();
    const hipError_t e = launch_few(a, plan.few_sets, stream);
    if (e != hipSuccess) return e;
  } else {
    const int at_once = tile_rows(a.g), tiles = (a.n_q * a.heads_per_kv + at_once - 1) / at_once;
    const dim3 grid(a.g.batch * a.g.kv_heads, tiles, a.splits);
    hipError_t e;
    switch (32 * a.g.bits_k + a.g.bits_v) {                // 
      case 32 * 2 + 2: e = launch_tiles_of<2, 2>(a, grid, stream); break;
      case 32 * 2 + 4: e = launch_tiles_of<2, 4>(a, grid, stream); break;
      case 32 * 4 + 2: e = launch_tiles_of<4, 2>(a, grid, stream); break;
      case 32 * 4 + 4: e = launch_tiles_of<4, 4>(a, grid, stream); break;
      case 32 * 2 + 8: e = launch_tiles_of<2, 8>(a, grid, stream); break;
      case 32 * 4 + 8: e = launch_tiles_of<4, 8>(a, grid, stream); break;
      case 32 * 8 + 2: e = launch_tiles_of<8, 2>(a, grid, stream); break;
      case 32 * 8 + 4: e = launch_tiles_of<8, 4>(a, grid, stream); break;
      case 32 * 8 + 8: e = launch_tiles_of<8, 8>(a, grid, stream); break;
      default: e = launch_tiles_of<0, 0>(a, grid, stream); break;
    }
    if (e != hipSuccess) return e;
    if (a.splits > 1) {
      const dim3 joins(grid.x, (a.n_q * a.heads_per_kv + kJoinRows - 1) / kJoinRows);
      hipLaunchKernelGGL(join_kernel, joins, dim3(32 * kJoinRows), 0, stream, a, at_once);
    }
  }
  return hipGetLastError();
}

}  // namespace kvq
