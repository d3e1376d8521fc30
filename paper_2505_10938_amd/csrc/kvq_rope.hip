// The rotary position embedding for positions with several axes (text: one; images: height and width; video: time too).
// Channel pair i turns by positions[axis of i] * freq[i]; the rotation's arithmetic is rope_word's.
#include "kvq_common.h"

namespace kvq {

namespace {

constexpr int kTokens = 4;               // per workgroup, a wavefront each
constexpr int kPairs = kHeadDim / 2;
constexpr int kPairsPerLane = 8;         // 16 bytes of each half of a row: eight lanes have a row, a wavefront eight rows

// Cosine and sine of one pair's angle.  Far positions times a frequency are thousands of turns: product and reduction to one
// turn in fp64 (2 pi in two parts), then fp32 of the reduced angle, its own rounding made good to first order.
__device__ __forceinline__ float2 turn_of(int32_t position, float freq) {
  const double angle = (double)position * (double)freq;
  const double turns = rint(angle * 0.15915494309189535);
  const double left = fma(-turns, 2.4492935982947064e-16, fma(-turns, 6.283185307179586, angle));
  const float x = (float)left, rest = (float)(left - (double)x);
  float s, c;
  sincosf(x, &s, &c);
  return make_float2(c - s * rest, s + c * rest);
}

__device__ __forceinline__ float2 turn_of_token(const int32_t* positions, int32_t tokens, const PairAxes& axes, const float* freq,
                                                int64_t token, int pair) {
  return turn_of(positions[(int64_t)axes.of[pair] * tokens + token], freq[pair]);
}

// A wavefront per token: each lane works out one pair's cosine and sine, which pass through LDS to the lanes that rotate
// that pair in every head.  Bound by memory (rows read once, written once).
__global__ void __launch_bounds__(64 * kTokens) rope_axes_kernel(
    const __half* q, int64_t q_stride, int32_t q_heads, const __half* k, int64_t k_stride, int32_t k_heads, int32_t tokens,
    const int32_t* __restrict__ positions, PairAxes axes, const float* __restrict__ freq, __half* q_out, int64_t q_out_stride,
    __half* k_out, int64_t k_out_stride) {
  __shared__ float2 turns[kTokens][kPairs];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t token = (int64_t)blockIdx.x * kTokens + wave;
  if (token < tokens) turns[wave][lane] = turn_of_token(positions, tokens, axes, freq, token, lane);
  __syncthreads();
  if (token >= tokens) return;
  const int piece = lane & 7;
  float2 t[kPairsPerLane];
#pragma unroll
  for (int i = 0; i < kPairsPerLane; ++i) t[i] = turns[wave][kPairsPerLane * piece + i];
  auto rows = [&](const __half* x, int64_t stride, int heads, __half* out, int64_t out_stride) {
    const __half* from = x + token * stride + 8 * piece;
    __half* to = out + token * out_stride + 8 * piece;
#pragma unroll 2
    for (int h = lane >> 3; h < heads; h += 8) {
      const uint4 a = *(const uint4*)(from + h * kHeadDim), b = *(const uint4*)(from + h * kHeadDim + kPairs);
      const uint32_t lo[4] = {a.x, a.y, a.z, a.w}, hi[4] = {b.x, b.y, b.z, b.w};
      uint32_t y[4], z[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 c = make_float2(t[2 * i].x, t[2 * i + 1].x), s = make_float2(t[2 * i].y, t[2 * i + 1].y);
        y[i] = rope_word(lo[i], hi[i], c, s, false);
        z[i] = rope_word(hi[i], lo[i], c, s, true);
      }
      *(uint4*)(to + h * kHeadDim) = make_uint4(y[0], y[1], y[2], y[3]);
      *(uint4*)(to + h * kHeadDim + kPairs) = make_uint4(z[0], z[1], z[2], z[3]);
    }
  };
  if (q) rows(q, q_stride, q_heads, q_out, q_out_stride);
  if (k) rows(k, k_stride, k_heads, k_out, k_out_stride);
}

__global__ void __launch_bounds__(64 * kTokens) rope_rows_kernel(int32_t tokens, const int32_t* __restrict__ positions,
                                                                  PairAxes axes, const float* __restrict__ freq,
                                                                  float* __restrict__ rows) {
  const int lane = threadIdx.x & 63;
  const int64_t token = (int64_t)blockIdx.x * kTokens + (threadIdx.x >> 6);
  if (token >= tokens) return;
  const float2 t = turn_of_token(positions, tokens, axes, freq, token, lane);
  rows[token * kHeadDim + lane] = t.x;
  rows[token * kHeadDim + kPairs + lane] = t.y;
}

}  // namespace

hipError_t launch_rope_axes(const __half* q, int64_t q_stride, int32_t q_heads, const __half* k, int64_t k_stride,
                            int32_t k_heads, int32_t tokens, const int32_t* positions, const PairAxes& axes, const float* freq,
                            __half* q_out, int64_t q_out_stride, __half* k_out, int64_t k_out_stride, hipStream_t s) {
  hipLaunchKernelGGL(rope_axes_kernel, dim3((uint32_t)(((int64_t)tokens + kTokens - 1) / kTokens)), dim3(64 * kTokens), 0, s, q,
                     q_stride, q_heads, k, k_stride, k_heads, tokens, positions, axes, freq, q_out, q_out_stride, k_out,
                     k_out_stride);
  return hipGetLastError();
}

hipError_t launch_rope_rows(int32_t tokens, const int32_t* positions, const PairAxes& axes, const float* freq, float* rows,
                            hipStream_t s) {
  hipLaunchKernelGGL(rope_rows_kernel, dim3((uint32_t)(((int64_t)tokens + kTokens - 1) / kTokens)), dim3(64 * kTokens), 0, s,
                     tokens, positions, axes, freq, rows);
  return hipGetLastError();
}

}  // namespace kvq
