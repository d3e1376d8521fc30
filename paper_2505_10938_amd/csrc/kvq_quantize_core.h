// Quantization of one group by one workgroup, as device code shared by the kernels that quantize groups one at a time: Eq. 2
// for a value, the group's rows in LDS, mean replacement, meta, codes and mask words.
#pragma once

#include "kvq_common.h"

// The integer code decisions must not depend on how the compiler fuses multiplies and adds.
#pragma clang fp contract(off)

namespace kvq {

namespace {

// ---- Eq. 2 for one value against its group's (min, step) -------------------------------------
// step is the fp16-rounded step as float; code = number of thresholds (k + 1/2) * step reached
// by fl32(x - mn).  The products are exact in fp32, so the decision is IEEE-reproducible.
__device__ inline uint32_t quant_code(float x, float mn, float step, int levels) {
  if (step == 0.0f) return 0u;
  const float t = x - mn;
  uint32_t code = 0;
  for (int k = 0; k < levels; ++k) {
    const float thr = ((float)k + 0.5f) * step;
    code += (t >= thr) ? 1u : 0u;
  }
  return code;
}

// The same decision as quant_code, as a binary search: code k is reached when fl32(x - mn) >= (2k - 1) * h
// with h = step / 2 (exact products again: 2k - 1 has 5 bits, h 11).  Returns 2 * code as a float.  A group
// whose step is zero passes h = +infinity: no threshold is reached, the code is 0.
template <int BITS>
__device__ __forceinline__ float quant_code_twice(float x, float mn, float h) {
  const float t = x - mn;
  float acc = 0.0f;
#pragma unroll
  for (int l = BITS - 1; l >= 0; --l) {
    const float c = (float)(2 << l);
    const float w = acc + (c - 1.0f);
    acc = (t >= w * h) ? acc + c : acc;
  }
  return acc;
}
__device__ __forceinline__ float half_step_of(__half st) {
  const float s = __half2float(st);
  return s == 0.0f ? __uint_as_float(0x7F800000u) : 0.5f * s;
}
// 2 * code (as returned above) put at bit position p of a packed word (a compile-time position of the
// first field of a word; bits beyond 31 wrap around)
template <int BITS>
__device__ __forceinline__ uint32_t place_twice(float acc, int p) {
  const uint32_t b = (uint32_t)acc;
  return (b << (p - 1)) | (p + BITS > 32 ? b >> (33 - p) : 0u);
}

// fp16 step from a group's min and max: fl32(fl32(max - min) * c_b) rounded to nearest even.
__device__ inline __half step_of(float mn, float mx, int bits) {
  const float c = bits == 2 ? __uint_as_float(0x3EAAAAABu) : __uint_as_float(0x3D888889u);  // 1/3, 1/15
  const float d = mx - mn;
  float s32 = d * c;
  // Keep the fp32 product as its own rounding step: without this the compiler merges the
  // multiply and the fp16 conversion into one instruction with a single rounding.
  asm volatile("" : "+v"(s32));
  return __float2half_rn(s32);
}

constexpr int kRowB = 272;   // LDS row: 128 fp16 + 16 bytes of padding (spreads rows over the banks)

__device__ inline float half_at(const unsigned char* p) { return __half2float(*(const __half*)p); }
__device__ inline float lo_half(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)(w & 0xFFFFu))); }
__device__ inline float hi_half(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)(w >> 16))); }

constexpr int kQuantThreads = 1024;

// Minimum and maximum over groups of `n` adjacent lanes (n = 4, 8 or 16).
__device__ inline void team_minmax(float& mn, float& mx, int n) {
  mn = fminf(mn, row_partner<0>(mn));
  mx = fmaxf(mx, row_partner<0>(mx));
  mn = fminf(mn, row_partner<1>(mn));
  mx = fmaxf(mx, row_partner<1>(mx));
  if (n > 4) {
    mn = fminf(mn, row_partner<2>(mn));
    mx = fmaxf(mx, row_partner<2>(mx));
  }
  if (n > 8) {
    mn = fminf(mn, row_partner<3>(mn));
    mx = fmaxf(mx, row_partner<3>(mx));
  }
}

// LDS of the quantization: the whole group (G x 128, K and V) and its meta.
template <int G>
struct QuantLds {
  unsigned char* sk;     // [G] rows of kRowB bytes
  unsigned char* sv;     // [G] rows
  float2* skm;           // [128] K meta: {zero, step / 2 (+infinity for a zero step)}
  float2* svm;           // [vgroups][G] V meta, the same pair
  uint8_t* ssel;         // [G] selected flags
  __device__ QuantLds(unsigned char* smem, int vgroups) {
    sk = smem;
    sv = sk + G * kRowB;
    skm = (float2*)(sv + G * kRowB);
    svm = skm + kHeadDim;
    ssel = (uint8_t*)(svm + G * vgroups);
  }
};
template <int G>
size_t quant_lds_bytes(int vgroups) { return (size_t)2 * G * kRowB + kHeadDim * 8 + (size_t)G * vgroups * 8 + G; }

// The group's rows, 16 bytes per thread: K rows first, then V rows.  (Of a vector type of the compiler's: HIP's uint4 is
// a structure, which it copies as memory.  Where nothing says that the rows are not written to meanwhile, quantize_kernel
// put such copies into scratch memory with G = 64 and 128, each behind a wait for its load.  A prompt's whole call with
// structures / vectors, 16 units: G = 64, 300 tokens 15.8 / 14.6 us, 3000 37.3 / 33.8; G = 128, 700 24.6 / 20.9.)
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <int G>
struct GroupRows {
  static constexpr int kLoads = 2 * G * 16 / kQuantThreads;   // 1, 2 or 4
  u32x4 rw[kLoads];
};
template <int G>
__device__ __forceinline__ void rows_issue(GroupRows<G>& r, const __half* gk, const __half* gv, int tid) {
#pragma unroll
  for (int q = 0; q < GroupRows<G>::kLoads; ++q) {
    const int e = q * kQuantThreads + tid;
    const int kv = e / (G * 16), rem = e % (G * 16);
    r.rw[q] = *(const u32x4*)((kv ? gv : gk) + (rem >> 4) * kHeadDim + (rem & 15) * 8);
  }
}
template <int G>
__device__ __forceinline__ void rows_to_lds(const GroupRows<G>& r, const QuantLds<G>& L, int tid) {
#pragma unroll
  for (int q = 0; q < GroupRows<G>::kLoads; ++q) {
    const int e = q * kQuantThreads + tid;
    const int kv = e / (G * 16), rem = e % (G * 16);
    *(u32x4*)((kv ? L.sv : L.sk) + (rem >> 4) * kRowB + (rem & 15) * 16) = r.rw[q];
  }
}

// Quantization of the group held in LDS (rows stored, not yet synchronized): mean replacement of
// the rows flagged (`flag` = this thread's token, threads below G), meta, codes, mask words.
// Every thread of the 1024-thread workgroup calls it.  (u, group_index) say where the group is stored
// (place_of_group): the unit and the group's index, or, in a paged cache, the plane and the page.
template <int BITS, int G>
__device__ __forceinline__ void quantize_body(const Dims& d, int64_t u, int32_t group_index, const QuantLds<G>& L,
                                              uint8_t flag, uint8_t* __restrict__ k_codes,
                                              uint32_t* __restrict__ k_meta, uint8_t* __restrict__ v_codes,
                                              uint32_t* __restrict__ v_meta, uint32_t* __restrict__ mask, int tid) {
  unsigned char* sk = L.sk;
  unsigned char* sv = L.sv;
  float2* skm = L.skm;
  float2* svm = L.svm;
  uint8_t* ssel = L.ssel;
  const int gv_shift = 31 - __clz(d.Gv);             // Gv is a power of two
  if (tid < G) ssel[tid] = flag;
  const int any = __syncthreads_or(flag);

  // mean replacement: per-channel mean of the original rows of all G tokens, exact fp64 sum,
  // scaled by the power of two 1/G, rounded to fp32 then fp16.
  if (any) {
    // four adjacent lanes per (matrix, channel), each summing every fourth token (the adds are exact,
    // so the split changes nothing), then each replacing the flagged ones among its own tokens
    const int part = tid & 3, c = (tid >> 2) & 127;
    unsigned char* rows = (tid < 512) ? sk : sv;
    double sum = 0.0;
#pragma unroll 8
    for (int t = part; t < G; t += 4) sum += (double)half_at(rows + t * kRowB + 2 * c);
    sum += row_partner<0>(sum);
    sum += row_partner<1>(sum);
    const float m32 = (float)(sum / (double)G);
    const __half m16 = __float2half_rn(m32);
    for (int t = part; t < G; t += 4)
      if (ssel[t]) *(__half*)(rows + t * kRowB + 2 * c) = m16;
    __syncthreads();
  }

  // K meta: 8 adjacent lanes share a channel, each taking every 8th token.
  {
    const int c = tid >> 3, part = tid & 7;
    float mn = half_at(sk + part * kRowB + 2 * c), mx = mn;
#pragma unroll
    for (int t = part + 8; t < G; t += 8) {
      const float x = half_at(sk + t * kRowB + 2 * c);
      mn = fminf(mn, x);
      mx = fmaxf(mx, x);
    }
    team_minmax(mn, mx, 8);
    mn += 0.0f;                                        // a zero minimum is stored as +0 (-0 + +0 = +0)
    if (part == 0) {
      const __half st = step_of(mn, mx, BITS);
      skm[c] = make_float2(mn, half_step_of(st));      // (mn is an fp16 value)
      // global layout of a group's Key meta: fp16 step[128], then fp16 zero[128]
      __half* gm = (__half*)(k_meta + (u * d.groups_per_unit + group_index) * kHeadDim);
      gm[c] = st;
      gm[kHeadDim + c] = __float2half_rn(mn);
    }
  }
  // V meta: Gv / 8 adjacent lanes share a (token, channel group), 8 channels each.
  if (!d.keys_only) {
    const int lanes = d.Gv >> 3;                       // 4, 8 or 16
#pragma unroll 1
    for (int e = tid; e < G * 16; e += kQuantThreads) {
      const int t = e >> 4, c8 = e & 15;               // 8 channels from 8 * c8 on
      const uint4 w = *(const uint4*)(sv + t * kRowB + c8 * 16);
      const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
      float mn = lo_half(ww[0]), mx = mn;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float x0 = lo_half(ww[k]), x1 = hi_half(ww[k]);
        mn = fminf(mn, fminf(x0, x1));
        mx = fmaxf(mx, fmaxf(x0, x1));
      }
      team_minmax(mn, mx, lanes);
      mn += 0.0f;                                      // a zero minimum is stored as +0
      if ((c8 & (lanes - 1)) == 0) {
        const int j = (c8 * 8) >> gv_shift;
        const __half st = step_of(mn, mx, BITS);
        svm[j * G + t] = make_float2(mn, half_step_of(st));
        // global layout of a 32-token block's Value meta (NV = value groups per token):
        // fp16 step[16 token pairs][NV][2], then fp16 zero[16 token pairs][NV][2]
        const int64_t tok = (int64_t)group_index * G + t;
        const int tb = (int)(tok & 31);
        __half* gm = (__half*)(v_meta + (u * d.blocks_per_unit + (tok >> 5)) * 32 * d.vgroups);
        gm[((tb >> 1) * d.vgroups + j) * 2 + (tb & 1)] = st;
        gm[32 * d.vgroups + ((tb >> 1) * d.vgroups + j) * 2 + (tb & 1)] = __float2half_rn(mn);
      }
    }
  }
  __syncthreads();

  // codes: one field (8 codes) of one packed u32 word of K or V per thread step.  Word w of lane l
  // of block blk holds 4/BITS fields; with two fields per word, adjacent lanes hold them.
  constexpr int kWordsPerBlock = 128 * BITS;          // 512*BITS bytes / 4
  constexpr int kFieldsPerWord = 4 / BITS;            // 2 (2-bit) or 1 (4-bit)
  constexpr int nblk = G / kBlockTokens;
  constexpr int kItems = 2 * nblk * kWordsPerBlock * kFieldsPerWord;   // a multiple of 1024
  const int first_block = group_index * nblk;
  const int n_items = d.keys_only ? kItems / 2 : kItems;          // Key words first, then Value words
#pragma unroll 1
  for (int e = tid; e < n_items; e += kQuantThreads) {
    const int kv = e / (kItems / 2);
    const int wf = e % (kItems / 2);
    const int i = wf / kFieldsPerWord, ff = wf % kFieldsPerWord;
    const int blk = i / kWordsPerBlock;
    const int wi = i - blk * kWordsPerBlock;
    // invert word_byte(): byte = 4*wi
    int lane, f0;
    if (BITS == 2) {
      lane = wi >> 2;
      f0 = (wi & 3) * 2;
    } else {
      const int half = wi >> 8;                        // 256 words per 1 KiB half
      lane = (wi & 255) >> 2;
      f0 = half * 4 + (wi & 3);
    }
    const int r = lane >> 4, mn_ = lane & 15;
    const int f = f0 + ff;
    // the word as if the field were the first of its word; the second field of a 2-bit word sits 8 bits up
    uint32_t word = 0;
    float2 ms[8];
    float val[8];
    if (kv == 0) {  // Key: lane = 16 r + m, field = 4 th + cb: 8 consecutive channels of one token
      const int t = 16 * (f >> 2) + mn_;
      const int c0 = 32 * (f & 3) + 8 * r;
      const uint4 xv = *(const uint4*)(sk + (blk * kBlockTokens + t) * kRowB + 2 * c0);
      const uint32_t xs[4] = {xv.x, xv.y, xv.z, xv.w};
#pragma unroll
      for (int x = 0; x < 8; x += 2) {
        const float4 m2 = *(const float4*)(skm + c0 + x);
        ms[x] = make_float2(m2.x, m2.y);
        ms[x + 1] = make_float2(m2.z, m2.w);
      }
#pragma unroll
      for (int x = 0; x < 8; ++x) val[x] = (x & 1) ? hi_half(xs[x >> 1]) : lo_half(xs[x >> 1]);
    } else {        // Value: lane = 16 r + n, field = ct: one channel of 8 consecutive tokens
      const int c = 16 * f + mn_;
      const int t0 = blk * kBlockTokens + 8 * r;
      const float2* pm = svm + (c >> gv_shift) * G + t0;
#pragma unroll
      for (int x = 0; x < 8; x += 2) {
        const float4 m2 = *(const float4*)(pm + x);
        ms[x] = make_float2(m2.x, m2.y);
        ms[x + 1] = make_float2(m2.z, m2.w);
      }
#pragma unroll
      for (int x = 0; x < 8; ++x) val[x] = half_at(sv + (t0 + x) * kRowB + 2 * c);
    }
#pragma unroll
    for (int x = 0; x < 8; ++x)
      word |= place_twice<BITS>(quant_code_twice<BITS>(val[x], ms[x].x, ms[x].y), code_bit(BITS, 0, x));
    if (ff) word = (word << 8) | (word >> 24);
    if (kFieldsPerWord == 2) word |= row_partner_u32<0>(word);      // the word's other field (the adjacent lane)
    if (ff == 0) {
      const int64_t boff = (u * d.blocks_per_unit + first_block + blk) * (int64_t)d.block_bytes;
      ((uint32_t*)((kv ? v_codes : k_codes) + boff))[wi] = word;
    }
  }

  // mask words
  if (tid < nblk) {
    uint32_t w = 0;
    for (int t = 0; t < 32; ++t) w |= (ssel[tid * 32 + t] ? 1u : 0u) << t;
    mask[u * d.blocks_per_unit + first_block + tid] = w;
  }
}

}  // namespace

}  // namespace kvq
