// Attention of a chunk of new tokens over a sequence's low-bit cache and, causally, over itself (Eq. 1 over the sets of
// the decode step, and the prefill phase's attention among the prompt's own tokens).
#include "kvq_common.h"

#include <type_traits>

// (the parts of the loops are used two or three times each, and called they would keep their registers in memory)
#define KVQ_INLINE __attribute__((always_inline))

namespace kvq {

namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef __fp16 lds_half4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) lds_half4* lds_half4_ptr;
typedef float float16v __attribute__((ext_vector_type(16)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kTile = 64;            // keys per tile
constexpr int kMergeThreads = 256;
constexpr int kWaveRows = kChunkWaveRows;   // query rows of a wavefront: (token, query head) pairs, token-major
constexpr int kPitchK = 272;         // LDS rows of 128 fp16: 16 bytes more, so that 16 rows' 16-byte pieces lie in different banks
constexpr int kPitchV = 320;         // four rows' 64-byte pieces in different banks
constexpr int kPitchT = 144;         // LDS rows of 64 keys of one channel
constexpr int kBytesK = kTile * kPitchK;
constexpr int kBytesV = kTile * kPitchV > kHeadDim * kPitchT ? kTile * kPitchV : kHeadDim * kPitchT;
constexpr int kBytesBuffer = kBytesK + kBytesV;
// A row's weights are taken relative to a maximum that may lie below the true one by this much (powers of two), so that
// the outputs are rescaled only when it has grown by more.  Weights up to 2^8 keep their 11 bits in fp16.
constexpr float kSlack = 8.0f;

__device__ __forceinline__ half2v as_h2(uint32_t w) { return __builtin_bit_cast(half2v, w); }
__device__ __forceinline__ uint32_t as_u32(half2v v) { return __builtin_bit_cast(uint32_t, v); }
__device__ __forceinline__ uint32_t rotr32(uint32_t w, int n) { return __builtin_amdgcn_alignbit(w, w, n); }

// The four code pairs (x = 2v, 2v + 1 in the two halves) of a field as fp16 numbers zero + code * step, one rounding each.
// `w` is the field's word, rotated so that the pairs v = 0 .. (2-bit: all, 4-bit: 0 and 1, and 2 and 3 eight bits further)
// stand at bits 2.. of each half.  A code at bit p of the significand of 2^(10 - p) is worth itself.
template <int BITS, int V>
__device__ __forceinline__ uint32_t dequant_pair(uint32_t w, uint32_t step, uint32_t zero) {
  constexpr int p = BITS == 2 ? 2 * (V + 1) : 2 + 4 * (V & 1);
  constexpr uint32_t mask = (uint32_t)((1 << BITS) - 1) << p, one = (uint32_t)(25 - p) << 10;
  const uint32_t x = (w & (mask | (mask << 16))) | (one | (one << 16));
  constexpr _Float16 base = (_Float16)(float)(1 << (10 - p));
  const half2v code = as_h2(x) - half2v{base, base};
  return as_u32(__builtin_elementwise_fma(code, as_h2(step), as_h2(zero)));
}
template <int BITS>
__device__ __forceinline__ u32x4 dequant_field(uint32_t word, int odd, const uint32_t (&step)[4], const uint32_t (&zero)[4]) {
  u32x4 r;
  if (BITS == 2) {                                       // (`odd`: the second field of the word)
    const uint32_t w = odd ? rotr32(word, 8) : word;
    r[0] = dequant_pair<2, 0>(w, step[0], zero[0]);
    r[1] = dequant_pair<2, 1>(w, step[1], zero[1]);
    r[2] = dequant_pair<2, 2>(w, step[2], zero[2]);
    r[3] = dequant_pair<2, 3>(w, step[3], zero[3]);
  } else {
    const uint32_t high = rotr32(word, 8);
    r[0] = dequant_pair<4, 0>(word, step[0], zero[0]);
    r[1] = dequant_pair<4, 1>(word, step[1], zero[1]);
    r[2] = dequant_pair<4, 2>(high, step[2], zero[2]);
    r[3] = dequant_pair<4, 3>(high, step[3], zero[3]);
  }
  return r;
}

// The larger of two numbers, or a NaN (one instruction for three: of what comes out of a matrix instruction the ordinary
// maximum has every operand made canonical first).
__device__ __forceinline__ float largest(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// The value of lane ^ 32.
__device__ __forceinline__ float other_half(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

// What a wavefront loads for the next tile of quantized tokens: a half or (NW = 8) a quarter of a block's codes, steps and zeros.
// It has F = 8 / NW times two fields of the Keys (cb = F part .., both halves of the tokens) and as many of the Values (ct =
// 2 F part ..).
template <int BITS, int NV, int F>
struct QuantRegs {
  static constexpr int kVGroups = NV == 4 && F == 2 ? 2 : 1;
  uint32_t k[2][BITS == 2 ? 1 : F];    // [half of the tokens][2-bit: the word, 4-bit: field]
  uint32_t v[BITS == 2 ? F : 2 * F];   // 2-bit: two fields a word
  u32x4 k_step[F], k_zero[F];          // of a field's eight channels
  uint32_t v_step[4][kVGroups], v_zero[4][kVGroups];     // of token pair 4 r + v
};
template <int N>
__device__ __forceinline__ void load_words(uint32_t (&w)[N], const unsigned char* p) {
  if constexpr (N == 1) {
    w[0] = *(const uint32_t*)p;
  } else if constexpr (N == 2) {
    const u32x2 x = *(const u32x2*)p;
    w[0] = x[0], w[1] = x[1];
  } else {
    const u32x4 x = *(const u32x4*)p;
    w[0] = x[0], w[1] = x[1], w[2] = x[2], w[3] = x[3];
  }
}

// What a sequence holds, and the keys of a row tile, 64 a tile, in this order: quantized tokens; new tokens that every row of
// the tile sees; full-precision rows of the cache; the other new tokens.
struct CacheRows {
  int nq, rs, nr, n_pool, n_aux;
};
__device__ __forceinline__ CacheRows cache_rows(const ChunkArgs& a, int b, int64_t u) {
  const Dims& d = a.d;
  CacheRows c = {a.n_quant, a.res_start, a.n_res, 0, 0};
  if (a.seq) {
    const int4 own = *(const int4*)(a.seq + 4 * b);
    c.nq = min(max(own.x, 0), a.n_quant) & ~(kBlockTokens - 1);
    c.rs = own.y >= 0 && own.y < d.res_rows ? own.y : 0;
    c.nr = min(max(own.z, 0), a.n_res);
  }
  if (d.N > 0) {
    c.n_pool = min(max(a.pool_count[u], 0), d.N);
    c.n_aux = min(max(a.aux_count[u], 0), d.A);
  }
  return c;
}
struct TileKeys {
  int n_new, tq, ti, tr, tiles;
  int splits;                // workgroups that share them: as few as have a.most tiles each
};
__device__ __forceinline__ TileKeys tile_keys(const ChunkArgs& a, const CacheRows& c, int n, int first_row, int live_rows) {
  TileKeys k;
  k.n_new = a.k_new ? min(n, ((first_row + live_rows - 1) >> a.g_shift) + 1) : 0;
  k.tq = (c.nq + kTile - 1) / kTile;
  k.ti = a.k_new ? min(n, (first_row >> a.g_shift) + 1) / kTile : 0;
  k.tr = (c.n_pool + c.n_aux + c.nr + kTile - 1) / kTile;
  k.tiles = k.tq + k.tr + (k.n_new + kTile - 1) / kTile;
  k.splits = max((k.tiles + a.most - 1) / a.most, 1);
  return k;
}

// The sequence with the turn-th most work for a workgroup, of at most 64, a lane each: the longest first leave the device's
// compute units least to wait for at the end (16 sequences of different lengths, up to 700 tokens over 6000, 32 kv heads: 258 us
// as they come, 243 so; 24, up to 700 over 2000, 8 kv heads: 158, 141).  A workgroup with few rows takes about half as long per
// tile of keys as one with all of them.
__device__ __forceinline__ int ranked_sequence(const ChunkArgs& a, int turn, int rows) {
  const int lane = threadIdx.x & 63, mine = min(lane, a.d.batch - 1);
  const int n = chunk_rows(a.starts, a.total, a.max_tokens, mine).n;
  const int held = a.seq ? min(max(a.seq[4 * mine], 0), a.n_quant) : a.n_quant;
  const float work = n > 0 ? ((float)held + n) * (rows + min((int64_t)n * a.d.g, (int64_t)rows)) : 0.0f;
  int rank = 0;
  for (int j = 0; j < a.d.batch; ++j) {
    const float other = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(work), j));
    rank += other > work || (other == work && j < lane);
  }
  return __builtin_ctzll(__ballot(lane < a.d.batch && rank == turn));
}

// One wavefront has 32 query rows, whose products with 64 keys stand transposed in its registers (keys down, one query row
// per lane and half): the softmax of a row is then work inside a lane, and the weights are, as they stand, an operand of the
// second product if its keys are taken in the order in which the first one leaves them (16 s + 8 (j / 4) + 4 h + j % 4 for half
// h of the lanes, element j).  NW wavefronts share the Keys' and Values' tiles in LDS, two buffers of each.
template <int BITS, int NV, int NW>
__global__ void __launch_bounds__(64 * NW, 2) prompt_attention_kernel(ChunkArgs a) {
  constexpr int kRows = NW * kWaveRows;
  extern __shared__ __align__(16) unsigned char smem[];
  const Dims& d = a.d;
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // ---- which rows, which keys
  // Workgroups go round the eight XCDs.  An XCD takes whole units (where their number is no multiple of eight, every
  // `parts`-th row tile of them), unit after unit, so that those that share a unit's keys share an L2 cache as well, and
  // sequences of different lengths weigh on all XCDs alike.
  const uint32_t per_unit = a.part_tiles * a.splits, turn = blockIdx.x >> 3;
  const uint32_t at = turn / per_unit, in_unit = turn - at * per_unit;
  const uint32_t part_unit = 8 * at + (blockIdx.x & 7);
  const int unit_turn = part_unit / a.parts;
  const int tile_in_part = in_unit / a.splits, split = in_unit - tile_in_part * a.splits;
  const int tile_back = tile_in_part * a.parts + (part_unit - unit_turn * a.parts);
  const int seq_turn = unit_turn / d.kv_heads, h = unit_turn - seq_turn * d.kv_heads;
  const int b = a.ranked ? ranked_sequence(a, seq_turn, kRows) : seq_turn, ul = b * d.kv_heads + h;
  const ChunkRows mine = chunk_rows(a.starts, a.total, a.max_tokens, b);
  const int64_t s0 = mine.first, u = d.unit0 + ul;
  const int n = mine.n;
  const int row_tiles = (int)(((int64_t)n * d.g + kRows - 1) / kRows);
  if (tile_back >= row_tiles) return;
  const int row_tile = row_tiles - 1 - tile_back;        // the longest ones first
  const int first_row = row_tile * kRows;                // of the unit's n * g rows
  const int live_rows = (int)min((int64_t)kRows, (int64_t)n * d.g - first_row);
  const CacheRows held = cache_rows(a, b, u);
  const int nq = held.nq, rs = held.rs, n_pool = held.n_pool, n_aux = held.n_aux;
  const int n_rows = n_pool + n_aux + held.nr;           // full-precision rows of the cache
  const TileKeys keys = tile_keys(a, held, n, first_row, live_rows);
  const int n_new = keys.n_new, tq = keys.tq, ti = keys.ti, tr = keys.tr;
  const int my_splits = keys.splits;
  if (split >= my_splits) return;
  const int per = (keys.tiles + my_splits - 1) / my_splits;
  const int t_begin = min(split * per, keys.tiles), t_end = min(t_begin + per, keys.tiles);

  // ---- the wavefront's query rows, as a matrix operand: lane (row col, channels 16 s + 8 half ..)
  const int wave_row = first_row + wave * kWaveRows;
  const bool wave_live = wave * kWaveRows < live_rows;
  const int row = wave_row + col;
  const bool row_live = wave * kWaveRows + col < live_rows;
  const int token = row >> a.g_shift, head = h * d.g + (row & (d.g - 1));
  half8 q[8];
#pragma unroll
  for (int s = 0; s < 8; ++s) q[s] = half8{0, 0, 0, 0, 0, 0, 0, 0};
  if (row_live) {
    const __half* qr = a.q + (s0 + token) * a.q_stride + head * kHeadDim + 8 * half;
#pragma unroll
    for (int s = 0; s < 8; ++s) q[s] = *(const half8*)(qr + 16 * s);
  }

  float16v o[4];
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[c][r] = 0.0f;
  float m = kNegBig, l = 0.0f;                           // of the lane's row: maximum (log2), sum over the half's keys

  auto buffer = [&](int i) { return smem + (i & 1) * kBytesBuffer; };
  float scale = a.scale, one = 1.0f;
  asm volatile("" : "+v"(scale), "+v"(one));             // (in registers: read anew, every step would wait for the scale)

  // V stands as rows of channels (two transposing reads bring four keys each of a channel to a lane) or, dequantized, already by
  // channel in the order of the second product.
  auto value = [&](auto quantized, const unsigned char* buf, int s, int c) KVQ_INLINE -> half8 {
    const unsigned char* sv = buf + kBytesK;
    if constexpr (decltype(quantized)::value) return *(const half8*)(sv + (32 * c + col) * kPitchT + 32 * s + 16 * half);
    const unsigned char* at = sv + (16 * s + 4 * half + ((lane & 15) >> 2)) * kPitchV + 2 * (32 * c + (lane & 16) + 4 * (lane & 3));
    const half4 lo = __builtin_bit_cast(half4, __builtin_amdgcn_ds_read_tr16_b64_v4f16((lds_half4_ptr)at));
    const half4 hi = __builtin_bit_cast(half4, __builtin_amdgcn_ds_read_tr16_b64_v4f16((lds_half4_ptr)(at + 8 * kPitchV)));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  // The first product with the Keys in `kb` (scores to x) and the second one with the Values in `vb` (of the weights w): FIRST,
  // SECOND: which of the two.  Eight operands are on their way ahead of the matrix instructions: left to itself the compiler
  // asks for two at a time and waits for them.  Of a SIMD's two wavefronts the one that multiplies goes first, it needs few of
  // the turns (8192 tokens, 32 heads: 577 us, 617 with no order; 45 tokens over 32768 92, 101).
  float16v x[2];
  half8 w[4];
  auto multiply = [&](auto quantized, auto first, auto second, const unsigned char* kb, const unsigned char* vb) KVQ_INLINE {
    constexpr bool QUANT = decltype(quantized)::value, FIRST = decltype(first)::value, SECOND = decltype(second)::value;
    const unsigned char* sk = kb + col * kPitchK + 16 * half;
    __builtin_amdgcn_s_setprio(1);
    if (FIRST) {
#pragma unroll
      for (int r = 0; r < 16; ++r) x[0][r] = x[1][r] = 0.0f;
#pragma unroll
      for (int s = 0; s < 8; ++s)
#pragma unroll
        for (int t = 0; t < 2; ++t)
          x[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*(const half8*)(sk + 32 * t * kPitchK + 32 * s), q[s], x[t], 0, 0, 0);
    }
    if (SECOND) {
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int c = 0; c < 4; ++c) o[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(value(quantized, vb, s, c), w[s], o[c], 0, 0, 0);
    }
    constexpr int kReadsV = QUANT ? 1 : 2;
    __builtin_amdgcn_sched_group_barrier(0x100, FIRST ? 8 : 8 * kReadsV, 0);
    if constexpr (FIRST) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
    }
    if constexpr (SECOND) {
#pragma unroll
      for (int i = 0; i < (FIRST ? 16 : 8); ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, kReadsV, 0);
      }
    }
    __builtin_amdgcn_sched_group_barrier(0x008, 8, 0);
    __builtin_amdgcn_s_setprio(0);
  };
  // The softmax of a tile's scores: x to weights w, and what the outputs have taken so far to the new maximum.  `hide(x)` sets
  // the scores of keys that a row does not see to -infinity, `keep(x)` may look at the weights.  The sum is of the weights as
  // they are used, rounded.  A dot product adds two of them, but waits for the matrix unit (16 of them 80 clocks, beside another
  // wavefront's matrix instructions 600; 32 multiply-adds 160 and 194).  Where a tile takes no work to store that is what a step
  // waits for (8192 tokens: 590 us with dot products, 576 so), behind quantized tiles it is not (4 x 512 over 8192: 349, 358).
  auto softmax = [&](auto quantized, auto hide, auto keep) KVQ_INLINE {
    hide(x);
    float top = largest(x[0][0], x[1][0]);
#pragma unroll
    for (int r = 1; r < 16; ++r) top = largest(largest(top, x[0][r]), x[1][r]);
    top = largest(top, other_half(top)) * scale;
    if (__any(top > m + kSlack)) {
      const float m_new = fmaxf(m, top);
      const float down = __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      l *= down;
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[c][r] *= down;
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) x[t][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[t][r], scale, -m));
    keep(x);
    float l1 = 0.0f;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      half2v y[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2v pair = {x[s >> 1][8 * (s & 1) + 2 * j], x[s >> 1][8 * (s & 1) + 2 * j + 1]};
        y[j] = __builtin_convertvector(pair, half2v);
        if (decltype(quantized)::value) {
          l = __builtin_amdgcn_fdot2(y[j], half2v{1, 1}, l, false);
        } else {
          l = __builtin_fmaf((float)y[j][0], one, l);
          l1 = __builtin_fmaf((float)y[j][1], one, l1);
        }
      }
      w[s] = half8{y[0][0], y[0][1], y[1][0], y[1][1], y[2][0], y[2][1], y[3][0], y[3][1]};
    }
    l += l1;
  };
  const std::true_type yes;
  const std::false_type no;
  const auto nothing = [](auto&&...) KVQ_INLINE {};

  // A run of `count` tiles.  With eight wavefronts a SIMD has two of them, and these take turns: while one multiplies (the first
  // product of a tile and the second one of the tile before), the other has its softmax and stores its share of tiles to come.
  // Wavefronts 4 to 7 are half a step behind.  Step t of a wavefront: Keys t and Values t - 1 are multiplied; then Keys t + 1
  // and Values t (the ones behind: t + 2 and t + 1) are stored where Keys t - 1 and Values t - 2 (t and t - 1) were read last
  // half a step ago.  `load(j)` asks for Keys j and Values j - 1 (behind the last tile: that one again).
  // (All eight with the same tile, one step after the other: 45 tokens over 32768 96 us, 88 so; 4 x 512 over 8192 359, 348; 16
  // sequences of different lengths, 4-bit codes, 296, 257; 8192 tokens 595, 576.  Matrix and vector instructions take about as
  // long as each other, 1000 to 1300 clocks a tile, and under both the device lowers its clock.)
  const int behind = NW == 8 ? wave >> 2 : 0;
  auto work = [&](auto quantized, int count, auto load, auto put_k, auto put_v, auto hide) KVQ_INLINE {
    load(0);
    put_k(buffer(0));
    load(1);
    __syncthreads();
    if (behind) {
      put_k(buffer(1));
      put_v(buffer(0));
      load(2);
      __syncthreads();
    }
    auto store = [&](int t) KVQ_INLINE {
      put_k(buffer(t + 1 + behind));
      put_v(buffer(t + behind));
      load(t + 2 + behind);
      __syncthreads();
    };
    if (wave_live) {
      multiply(quantized, yes, no, buffer(0), nullptr);
      if (NW == 8) __syncthreads();
      softmax(quantized, hide, nothing);
      store(0);
      for (int t = 1; t < count; ++t) {
        multiply(quantized, yes, yes, buffer(t), buffer(t - 1));
        if (NW == 8) __syncthreads();
        softmax(quantized, hide, nothing);
        store(t);
      }
      multiply(quantized, no, yes, nullptr, buffer(count - 1));
    } else {
      for (int t = 0; t < count; ++t) {
        if (NW == 8) __syncthreads();
        store(t);
      }
    }
    if (NW == 8 && !behind) __syncthreads();
  };

  // ---- quantized tokens, 64 (two blocks) a tile: each wavefront turns its share of a block's Keys and Values into fp16 rows
  {
    const int last = (nq >> 5) - 1;
    const int qe = min(t_end, tq);
    const int r = lane >> 4, m16 = lane & 15, part = wave >> 1;
    constexpr int F = 8 / NW;
    QuantRegs<BITS, NV, F> R;
    // Where the blocks are: their numbers in the unit's or the page plane's run, and their mask words, of 64 blocks at a time, a
    // lane each (a look into the table for every tile would have the tile's loads wait for it).
    const int64_t run = d.page_table ? d.plane0 + h : u;
    const int in_group = (1 << d.bpg_shift) - 1;
    const int cb = F * part, ct = 2 * F * part;          // first fields
    const unsigned char* const k_run = a.k_codes + run * d.blocks_per_unit * (512 * BITS) + (BITS == 2 ? 4 * (cb >> 1) : 4 * cb);
    const unsigned char* const v_run = a.v_codes + run * d.blocks_per_unit * (512 * BITS) + (BITS == 2 ? 4 * (ct >> 1) : 1024 * (ct >> 2) + 4 * (ct & 3));
    const unsigned char* const km_run = a.k_meta + run * d.groups_per_unit * 512 + 64 * cb;
    const unsigned char* const vm_run = a.v_meta + run * d.blocks_per_unit * (128 * NV) + 4 * (ct * NV / 8);
    const uint32_t* const mask_run = a.mask + run * d.blocks_per_unit;
    int first_block = 0, blocks = 0;
    uint32_t words = 0;
    auto look_up = [&](int block) KVQ_INLINE {
      first_block = block;
      const int mine = min(block + lane, last), group = mine >> d.bpg_shift;
      int slot = group;
      if (d.page_table) slot = min(max(d.page_table[(int64_t)b * d.table_stride + group], 0), d.n_pages - 1);
      blocks = (slot << d.bpg_shift) + (mine & in_group);
      words = mask_run[blocks];
    };
    // The wavefront's block of the tile whose Keys, and of the one whose Values are asked for; the mask words of that one, and of
    // those before.
    int k_block = 0;
    uint32_t hidden[2], seen1[2] = {0, 0}, seen2[2] = {0, 0};
    auto load = [&](int j) KVQ_INLINE {
      const int tile = t_begin + j, at = min(2 * tile, last & ~1);
      const int v_block = k_block;
      if (j == 0 || at - first_block >= 64) look_up(at);
      const int i = at - first_block;
      k_block = __builtin_amdgcn_readlane(blocks, (wave & 1) && at < last ? i + 1 : i);
      hidden[0] = behind ? seen2[0] : seen1[0];
      hidden[1] = behind ? seen2[1] : seen1[1];
      seen2[0] = seen1[0];
      seen2[1] = seen1[1];
      seen1[0] = __builtin_amdgcn_readlane(words, i);
      seen1[1] = at < last ? __builtin_amdgcn_readlane(words, i + 1) : ~0u;
      const unsigned char* at_k = k_run + (((uint64_t)(uint32_t)k_block) << (BITS == 2 ? 10 : 11));
      const unsigned char* at_km = km_run + (((uint64_t)(uint32_t)k_block >> d.bpg_shift) << 9);
#pragma unroll
      for (int th = 0; th < 2; ++th) load_words(R.k[th], at_k + 16 * lane + (BITS == 2 ? 8 : 1024) * th);
#pragma unroll
      for (int e = 0; e < F; ++e) {
        R.k_step[e] = *(const u32x4*)(at_km + 64 * e + 16 * r);
        R.k_zero[e] = *(const u32x4*)(at_km + 64 * e + 16 * r + 256);
      }
      if (j == 0) return;
      const unsigned char* at_v = v_run + (((uint64_t)(uint32_t)v_block) << (BITS == 2 ? 10 : 11));
      const unsigned char* at_vm = vm_run + ((uint64_t)(uint32_t)v_block) * (128 * NV);
      load_words(R.v, at_v + 16 * lane);
      if constexpr (NV == 1) {
        const u32x4 st = *(const u32x4*)(at_vm + 16 * r), ze = *(const u32x4*)(at_vm + 16 * r + 64);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          R.v_step[v][0] = st[v];
          R.v_zero[v][0] = ze[v];
        }
      } else {
#pragma unroll
        for (int v = 0; v < 4; ++v) {                    // pair 4 r + v, the value groups of this part of the channels
          load_words(R.v_step[v], at_vm + 4 * NV * (4 * r + v));
          load_words(R.v_zero[v], at_vm + 4 * NV * (4 * r + v) + 64 * NV);
        }
      }
    };
    // A field of Keys: 8 channels from 32 cb + 8 r on of token 16 th + m16.
    const int token0 = 32 * (wave & 1);
    auto put_k = [&](unsigned char* buf) KVQ_INLINE {
#pragma unroll
      for (int th = 0; th < 2; ++th)
#pragma unroll
        for (int e = 0; e < F; ++e) {
          uint32_t st[4], ze[4];
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            st[v] = R.k_step[e][v];
            ze[v] = R.k_zero[e][v];
          }
          const int odd = BITS == 2 ? (F == 2 ? e : part & 1) : 0;
          *(u32x4*)(buf + (token0 + 16 * th + m16) * kPitchK + 64 * F * part + 64 * e + 16 * r) =
              dequant_field<BITS>(R.k[th][BITS == 2 ? 0 : e], odd, st, ze);
        }
    };
    // A field of Values: tokens 8 r .. of channel 16 (ct + s) + m16.
    auto put_v = [&](unsigned char* buf) KVQ_INLINE {
#pragma unroll
      for (int s = 0; s < 2 * F; ++s) {
        constexpr int kOf = F == 2 ? 1 : 0;
        uint32_t st[4], ze[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          st[v] = R.v_step[v][NV == 4 && kOf ? s >> 1 : 0];
          ze[v] = R.v_zero[v][NV == 4 && kOf ? s >> 1 : 0];
        }
        const u32x4 y = dequant_field<BITS>(R.v[BITS == 2 ? s >> 1 : s], BITS == 2 ? s & 1 : 0, st, ze);
        unsigned char* sv = buf + kBytesK + (32 * F * part + 16 * s + m16) * kPitchT + 2 * (token0 + 16 * (r >> 1) + 4 * (r & 1));
        *(u32x2*)sv = u32x2{y[0], y[1]};
        *(u32x2*)(sv + 16) = u32x2{y[2], y[3]};
      }
    };
    auto hide = [&](float16v (&x)[2]) KVQ_INLINE {
      if (hidden[0] | hidden[1]) {                       // uniform
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t word = hidden[i] >> (4 * half);
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (word & (1u << (8 * (r >> 2) + (r & 3)))) x[i][r] = -__builtin_inff();
        }
      }
    };
    if (t_begin < qe) work(yes, qe - t_begin, load, put_k, put_v, hide);
  }

  // ---- full-precision rows, 64 a tile
  const int piece = tid & 15, line = tid >> 4;
  constexpr int kPasses = 16 / NW, kLines = 4 * NW;      // rows of a tile: kLines at a time
  u32x4 rk[kPasses], rv[kPasses];
  auto put_k = [&](unsigned char* buf) KVQ_INLINE {
#pragma unroll
    for (int i = 0; i < kPasses; ++i) *(u32x4*)(buf + (kLines * i + line) * kPitchK + 16 * piece) = rk[i];
  };
  auto put_v = [&](unsigned char* buf) KVQ_INLINE {
#pragma unroll
    for (int i = 0; i < kPasses; ++i) *(u32x4*)(buf + kBytesK + (kLines * i + line) * kPitchV + 16 * piece) = rv[i];
  };

  // new tokens that all of the workgroup's rows see
  {
    const int nb = max(t_begin, tq), ne = min(t_end, tq + ti);
    if (nb < ne) {
      const uint32_t row_bytes = (uint32_t)a.kv_stride * 2, offset = line * row_bytes + 16 * piece;
      const int64_t first = s0 * a.kv_stride + h * kHeadDim + (int64_t)(nb - tq) * kTile * a.kv_stride;
      const int count = ne - nb;
      const unsigned char* at_k = (const unsigned char*)(a.k_new + first);
      const unsigned char* at_v = (const unsigned char*)(a.v_new + first);
      auto rows = [&](u32x4 (&x)[kPasses], const unsigned char*& at, bool more) KVQ_INLINE {
#pragma unroll
        for (int i = 0; i < kPasses; ++i) x[i] = *(const u32x4*)(at + (offset + kLines * i * row_bytes));
        at += more ? row_bytes * kTile : 0;              // (uniform)
      };
      work(no, count, [&](int j) KVQ_INLINE {
        rows(rk, at_k, j + 1 < count);
        if (j > 0) rows(rv, at_v, j < count);
      }, put_k, put_v, nothing);
    }
  }

  // the pools' members and the ring, then the new tokens that some of the rows do not see
  {
    const int fb = max(t_begin, tq + ti), rows_end = tq + ti + tr;
    const __half* pk = a.pool_k + u * d.pool_slots * kHeadDim + 8 * piece;
    const __half* pv = a.pool_v + u * d.pool_slots * kHeadDim + 8 * piece;
    const __half* ck = a.k_res + u * d.res_rows * kHeadDim + 8 * piece;
    const __half* cv = a.v_res + u * d.res_rows * kHeadDim + 8 * piece;
    const __half* nk = a.k_new + s0 * a.kv_stride + h * kHeadDim + 8 * piece;
    const __half* nv = a.v_new + s0 * a.kv_stride + h * kHeadDim + 8 * piece;
    // Where some rows see a new token and others do not, its Value must not reach the others, for 0 times an infinity is a
    // NaN: what is not finite is left out of the tile (and counted in by `late` for the rows that see it).
    auto load = [&](int tile) KVQ_INLINE -> bool {
      const bool own = tile >= rows_end;                 // uniform
      const int first = own ? (tile - rows_end + ti) * kTile : (tile - tq - ti) * kTile;
#pragma unroll
      for (int i = 0; i < kPasses; ++i) {
        const int e = first + kLines * i + line;
        rk[i] = rv[i] = u32x4{0, 0, 0, 0};
        const __half* fk;
        const __half* fv;
        if (own) {
          fk = nk + e * a.kv_stride;
          fv = nv + e * a.kv_stride;
        } else {
          int at = rs + (e - n_pool - n_aux);
          at -= at >= d.res_rows ? d.res_rows : 0;
          const bool pooled = e < n_pool + n_aux;
          if (pooled) at = e < n_pool ? e : d.pool_slots - d.A + (e - n_pool);
          fk = (pooled ? pk : ck) + at * kHeadDim;
          fv = (pooled ? pv : cv) + at * kHeadDim;
        }
        if (e < (own ? n_new : n_rows)) {
          rk[i] = *(const u32x4*)fk;
          rv[i] = *(const u32x4*)fv;
        }
      }
      return own;
    };
    auto sort_out = [&]() {
      uint32_t odd = 0;
#pragma unroll
      for (int i = 0; i < kPasses; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t w = rv[i][k], lo = (w & 0x7C00u) == 0x7C00u ? 0xFFFFu : 0u, hi = (w & 0x7C000000u) == 0x7C000000u ? 0xFFFF0000u : 0u;
          odd |= lo | hi;
          rv[i][k] = w & ~(lo | hi);
        }
      return odd;
    };
    // The Values left out of a tile, for the rows that see them.  Weights of half the keys at a time go through LDS (the buffer
    // that is not in use).
    auto late = [&](int tile, int limit, float* mine, const float16v (&x)[2]) {
      static_assert(NW * kWaveRows * 32 * 4 <= kBytesBuffer, "the weights of all wavefronts have room in a buffer");
      const int base = (tile - rows_end + ti) * kTile;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int r = 0; r < 16; ++r) mine[(8 * (r >> 2) + 4 * half + (r & 3)) * kWaveRows + col] = x[t][r];
        __builtin_amdgcn_s_waitcnt(0xc07f);              // lgkmcnt(0): the wavefront's own stores
        __builtin_amdgcn_wave_barrier();
#pragma unroll 1
        for (int k = 32 * t; k < 32 * t + 32 && base + k < n_new; ++k) {
          const float w = mine[(k & 31) * kWaveRows + col];
          const __half* vr = a.v_new + (s0 + base + k) * a.kv_stride + h * kHeadDim + 4 * half;
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
              const half4 v = *(const half4*)(vr + 32 * c + 8 * r4);
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (k < limit && w != 0.0f && !(fabsf((float)v[i]) <= 65504.0f)) o[c][4 * r4 + i] += w * (float)v[i];
            }
        }
        __builtin_amdgcn_s_waitcnt(0xc07f);
        __builtin_amdgcn_wave_barrier();
      }
    };
    if (fb < t_end) {
      if (t_begin < fb) __syncthreads();                 // (the last tile's Values)
      bool odd = load(fb) && sort_out();
      put_k(buffer(fb));
      put_v(buffer(fb));
      odd = __syncthreads_or(odd);
      for (int t = fb; t < t_end; ++t) {
        const bool more = t + 1 < t_end;
        bool next_own = false;
        if (more) next_own = load(t + 1);
        // how many of the tile's keys the lane's row sees, and the most that a row of the wavefront does
        const bool own = t >= rows_end;
        const int base = own ? (t - rows_end + ti) * kTile : (t - tq - ti) * kTile;
        const int limit = (own ? min(n_new, token + 1) : n_rows) - base;
        const int most = (own ? min(n_new, ((wave_row + kWaveRows - 1) >> a.g_shift) + 1) : n_rows) - base;
        if (wave_live && most > 0) {
          multiply(no, yes, no, buffer(t), nullptr);
          softmax(no, [&](float16v (&x)[2]) KVQ_INLINE {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int r = 0; r < 16; ++r)
                if (32 * i + 8 * (r >> 2) + (r & 3) + 4 * half >= limit) x[i][r] = -__builtin_inff();
          }, [&](float16v (&x)[2]) KVQ_INLINE {
            if (odd) late(t, limit, (float*)(buffer(t + 1) + wave * (kWaveRows * 32 * 4)), x);     // (uniform)
          });
          multiply(no, no, yes, nullptr, buffer(t));
        }
        if (more) {
          if (odd) __syncthreads();                      // (the weights' place in the other buffer)
          odd = next_own && sort_out();
          put_k(buffer(t + 1));
          put_v(buffer(t + 1));
          odd = __syncthreads_or(odd);
        }
      }
    }
  }

  // ---- the rows' results: normalized, or this split's share
  if (!row_live) return;
  l += other_half(l);
  if (my_splits == 1) {
    const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
    __half* to = a.out + ((s0 + token) * d.q_heads + head) * kHeadDim + 4 * half;
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        half4 y;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = (_Float16)(o[c][4 * r4 + i] * inv);
        *(half4*)(to + 32 * c + 8 * r4) = y;
      }
    return;
  }
  const int64_t place = ((int64_t)ul * a.unit_rows + row) * a.splits + split;
  if (half == 0) *(float2*)(a.share_ml + 2 * place) = make_float2(m, l);
  if (l == 0.0f) return;
  float* to = a.share_o + place * kHeadDim + 4 * half;
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4)
      *(float4*)(to + 32 * c + 8 * r4) = make_float4(o[c][4 * r4], o[c][4 * r4 + 1], o[c][4 * r4 + 2], o[c][4 * r4 + 3]);
}

// The shares of a row's splits put together: sum of 2^(m_i - max m) (l_i, o_i).  32 lanes a row: a lane has the maximum and the
// sum of one of 32 splits, and four channels; the splits' rows are asked for eight at a time.
__global__ void __launch_bounds__(kMergeThreads) prompt_merge_kernel(ChunkArgs a) {
  const Dims& d = a.d;
  const int sub = threadIdx.x & 31;
  const int row = blockIdx.x * (kMergeThreads / 32) + (threadIdx.x >> 5);
  const int h = blockIdx.y, b = blockIdx.z, ul = b * d.kv_heads + h;
  const ChunkRows mine = chunk_rows(a.starts, a.total, a.max_tokens, b);
  const int64_t s0 = mine.first;
  const int n = mine.n;
  if (row >= (int64_t)n * d.g) return;
  const int rows = a.waves * kWaveRows, first_row = row / rows * rows;
  const int splits = tile_keys(a, cache_rows(a, b, d.unit0 + ul), n, first_row, (int)min((int64_t)rows, (int64_t)n * d.g - first_row)).splits;
  if (splits == 1) return;                               // (written by the workgroup that had them all)
  const int64_t place = ((int64_t)ul * a.unit_rows + row) * a.splits;
  const float2* ml = (const float2*)a.share_ml + place;
  const float4* shares = (const float4*)(a.share_o + place * kHeadDim) + sub;
  float m = kNegBig, l = 0.0f, o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int first = 0; first < splits; first += 32) {
    const float2 own = first + sub < splits ? ml[first + sub] : make_float2(kNegBig, 0.0f);
    const bool some = own.y != 0.0f;                     // (a share that saw nothing has left no rows)
    float top = some ? own.x : kNegBig;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 32));
    const float m_new = fmaxf(m, top), down = __builtin_amdgcn_exp2f(m - m_new);
    m = m_new;
    const float weight = some ? __builtin_amdgcn_exp2f(own.x - m) : 0.0f;
    float sum = weight * own.y;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 32);
    l = l * down + sum;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] *= down;
    const int count = min(32, splits - first);
    for (int i0 = 0; i0 < count; i0 += 8) {
      float4 x[8];
      float w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        w[i] = __shfl(weight, i0 + i, 32);
        x[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (w[i] != 0.0f) x[i] = shares[(int64_t)(first + i0 + i) * (kHeadDim / 4)];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        o[0] += w[i] * x[i].x;
        o[1] += w[i] * x[i].y;
        o[2] += w[i] * x[i].z;
        o[3] += w[i] * x[i].w;
      }
    }
  }
  const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
  half4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = (_Float16)(o[i] * inv);
  const int token = row >> a.g_shift, head = h * d.g + (row & (d.g - 1));
  *(half4*)(a.out + ((s0 + token) * d.q_heads + head) * kHeadDim + 4 * sub) = y;
}

}  // namespace

hipError_t launch_prompt_attention(const ChunkArgs& a, hipStream_t s) {
  const int64_t units = (int64_t)a.d.units_per_layer * a.parts;
  const uint32_t grid = (uint32_t)(units * a.part_tiles * a.splits);
  auto go = [&](auto kern) {
    hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, 2 * kBytesBuffer);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3(grid), dim3(64 * a.waves), 2 * kBytesBuffer, s, a);
    return hipGetLastError();
  };
  auto of_bits = [&](auto bits) {
    constexpr int BITS = decltype(bits)::value;
    switch (a.d.vgroups) {
      case 4: return a.waves == 8 ? go(prompt_attention_kernel<BITS, 4, 8>) : go(prompt_attention_kernel<BITS, 4, 4>);
      case 2: return a.waves == 8 ? go(prompt_attention_kernel<BITS, 2, 8>) : go(prompt_attention_kernel<BITS, 2, 4>);
      default: return a.waves == 8 ? go(prompt_attention_kernel<BITS, 1, 8>) : go(prompt_attention_kernel<BITS, 1, 4>);
    }
  };
  hipError_t e = a.d.bits == 2 ? of_bits(std::integral_constant<int, 2>{}) : of_bits(std::integral_constant<int, 4>{});
  if (e != hipSuccess || a.splits == 1) return e;
  const int64_t rows = (int64_t)a.max_tokens * a.d.g;
  hipLaunchKernelGGL(prompt_merge_kernel, dim3((uint32_t)((rows + 7) / 8), a.d.kv_heads, a.d.batch), dim3(kMergeThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace kvq
