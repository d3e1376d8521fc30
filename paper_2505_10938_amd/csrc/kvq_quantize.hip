// Residual append and group quantization (mean replacement, Eq. 2 per group, packing), and the
// fused group step (append + outlier competition + quantization in one launch).
#include "kvq_common.h"
#include "kvq_quantize_core.h"
#include "kvq_trace_core.h"

#include <type_traits>

// The integer code decisions must not depend on how the compiler fuses multiplies and adds.
#pragma clang fp contract(off)

namespace kvq {

namespace {

// ---- residual append: one row of 128 fp16 per unit, K and V -----------------------------------
__global__ void __launch_bounds__(128) append_kernel(Dims d, const __half* __restrict__ k_new,
                                                     const __half* __restrict__ v_new, __half* __restrict__ k_res,
                                                     __half* __restrict__ v_res, int32_t row) {
  const int ul = blockIdx.x;                       // unit inside the layer
  const int64_t u = d.unit0 + ul;
  const int tid = threadIdx.x;                     // 64 threads for K, 64 for V, 4 bytes each
  const int which = tid >> 6, lane = tid & 63;
  const uint32_t* src = (const uint32_t*)((which ? v_new : k_new) + (int64_t)ul * kHeadDim);
  uint32_t* dst = (uint32_t*)((which ? v_res : k_res) + (u * d.res_rows + row) * kHeadDim);
  dst[lane] = src[lane];
}

// From this many groups in one launch on, prompt_quantize_kernel takes them (1024 threads keep a group of 128 tokens longest,
// and one workgroup of them fills half a compute unit).  Us of calls recorded in a graph, three sets of rows in turn,
// quantize_kernel / prompt_quantize_kernel; 2-bit, then 4-bit codes:
//   prompt without a pool   G = 32, 128 groups 6.7 / 5.7, 6.9 / 6.3   256 7.0 / 5.8, 7.2 / 6.5    512 9.0 / 7.2, 9.5 / 8.6    768 11.8 / 8.6, 12.4 / 10.0
//                           G = 64,  32 groups 7.8 / 5.9, 8.2 / 6.5   512 12.9 / 9.3, 14.0 / 11.0
//                           G = 128,  8 groups 10.8 / 6.5, 11.7 / 7.7 256 14.1 / 9.4, 15.3 / 11.0
//   with a pool, N = 8      G = 32, 256 groups 17.5 / 16.5, 17.7 / 17.2;  G = 64, 32 14.3 / 12.0, 14.7 / 12.8;  G = 128, 8 17.4 / 12.4, 18.3 / 13.6
//   kvq_quantize_group      G = 32, 256 units 5.0 / 4.0, 5.2 / 4.5;  G = 64, 32 5.8 / 3.9, 6.1 / 4.5;  G = 128, one 8.5 / 4.4, 9.5 / 5.4
// Its code is 29 .. 37 KB, the other's 5 .. 6.  With a decode step, products and elementwise kernels ahead of each call, so
// that neither finds its code in the instruction cache, a group of 128 tokens still gains 4 us and one of 64 tokens 1 .. 2.  With
// G = 32 the two are even at 256 groups (ten shapes, N = 0 and 8: 2-bit 0.5 us faster in the mean, -0.9 .. 1.3, 4-bit 0.3 slower,
// -1.6 .. 0.8); from 320 on it is ahead there too (4-bit 0.3 .. 1.1 us, from 640 on 2 .. 3).
constexpr int64_t prompt_groups(int G) { return G == 32 ? 256 : G == 64 ? 32 : 1; }

// One workgroup of 16 wavefronts per unit.  Every global load of the kernel is issued before the
// first wait, so a launch costs one trip to memory; the work after it is spread over all 1024
// threads because nothing else hides latency.  LDS: 2 * G * 272 bytes (<= 68 KB) + meta.
template <int BITS, int G, int LAYERS>
__global__ void __launch_bounds__(kQuantThreads) quantize_kernel(
    Dims d, int32_t group_index, int64_t unit_stride, const uint8_t* __restrict__ selected, int64_t selected_unit_stride,
    uint8_t* __restrict__ k_codes, uint32_t* __restrict__ k_meta, uint8_t* __restrict__ v_codes,
    uint32_t* __restrict__ v_meta, uint32_t* __restrict__ mask, int32_t n_groups, int32_t tail_n,
    __half* __restrict__ k_res, __half* __restrict__ v_res, LayerRows<LAYERS> rows) {
  // grid (units, groups + tail blocks, layers): workgroup (ul, gy) with gy < n_groups quantizes the G rows from row
  // gy * G of the unit's rows as group group_index + gy; its flags are
  // selected[(layer * units + ul) * selected_unit_stride + gy * G ..].  The workgroups behind them copy the tail_n
  // rows that follow the last group into ring rows 0 .. of the unit (a whole prompt: the rows that stay in full
  // precision), 16 bytes of K and of V per thread.
  extern __shared__ __align__(16) unsigned char smem[];
  const QuantLds<G> L(smem, d.vgroups);
  const int tid = threadIdx.x;
  const int ul = blockIdx.x, gy = blockIdx.y, layer = LAYERS > 1 ? blockIdx.z : 0;
  const __half* __restrict__ k_rows = rows.k[layer];
  const __half* __restrict__ v_rows = rows.v[layer];
  if (gy >= n_groups) {
    const int i = (gy - n_groups) * kQuantThreads + tid;
    if (i < tail_n * 16) {
      const int64_t src = (int64_t)ul * unit_stride + (int64_t)n_groups * G * kHeadDim;
      const int64_t dst = (d.unit0 + (int64_t)layer * d.layer_units + ul) * d.res_rows * kHeadDim;
      ((uint4*)(k_res + dst))[i] = ((const uint4*)(k_rows + src))[i];
      ((uint4*)(v_res + dst))[i] = ((const uint4*)(v_rows + src))[i];
    }
    return;
  }
  GroupRows<G> group;
  const int64_t row0 = (int64_t)ul * unit_stride + (int64_t)gy * G * kHeadDim;
  rows_issue<G>(group, k_rows + row0, v_rows + row0, tid);
  const int64_t sel0 = ((int64_t)layer * d.units_per_layer + ul) * selected_unit_stride + (int64_t)gy * G;
  uint8_t flag = 0;
  if (tid < G && selected) flag = selected[sel0 + tid];
  const GroupPlace at = place_of_group(d, ul, group_index + gy, layer);
  rows_to_lds<G>(group, L, tid);
  quantize_body<BITS, G>(d, at.row, at.slot, L, flag, k_codes, k_meta, v_codes, v_meta, mask, tid);
}

template <int BITS, int G, int LAYERS, bool ONCE>
__global__ void __launch_bounds__(4 * G) __attribute__((amdgpu_waves_per_eu(4, 8))) prompt_quantize_kernel(
    Dims d, int32_t group_index, int64_t unit_stride, const uint8_t* __restrict__ selected, int64_t selected_unit_stride,
    uint8_t* __restrict__ k_codes, uint32_t* __restrict__ k_meta, uint8_t* __restrict__ v_codes,
    uint32_t* __restrict__ v_meta, uint32_t* __restrict__ mask, int32_t n_groups, int32_t tail_n,
    __half* __restrict__ k_res, __half* __restrict__ v_res, int32_t last_first, LayerRows<LAYERS> rows) {
  // grid (units, groups + tail blocks, layers), as quantize_kernel's
  constexpr int nblk = G / kBlockTokens, kThreads = 128 * nblk;
  const int tid = threadIdx.x;
  const int ul = blockIdx.x, by = blockIdx.y, layer = LAYERS > 1 ? blockIdx.z : 0;
  const __half* __restrict__ k_rows = rows.k[layer];
  const __half* __restrict__ v_rows = rows.v[layer];
  const int gy = last_first && by < n_groups ? n_groups - 1 - by : by;
  if (gy >= n_groups) {
    const int i = (gy - n_groups) * kThreads + tid;
    if (i < tail_n * 16) {
      const int64_t src = (int64_t)ul * unit_stride + (int64_t)n_groups * G * kHeadDim;
      const int64_t dst = (d.unit0 + (int64_t)layer * d.layer_units + ul) * d.res_rows * kHeadDim;
      ((uint4*)(k_res + dst))[i] = ((const uint4*)(k_rows + src))[i];
      ((uint4*)(v_res + dst))[i] = ((const uint4*)(v_rows + src))[i];
    }
    return;
  }
  const int64_t row0 = (int64_t)ul * unit_stride + (int64_t)gy * G * kHeadDim;
  const int64_t sel0 = ((int64_t)layer * d.units_per_layer + ul) * selected_unit_stride + (int64_t)gy * G;
  quantize_rows<BITS, G, ONCE>(d, GroupOf{k_rows + row0, v_rows + row0}, selected ? selected + sel0 : nullptr,
                               place_of_group(d, ul, group_index + gy, layer), k_codes, k_meta, v_codes, v_meta, mask, tid);
}

// The n rows of every unit into ring rows 0 .. n - 1 (16 bytes per thread).  grid (units, blocks, layers).
template <int LAYERS>
__global__ void __launch_bounds__(256) tail_copy_kernel(Dims d, int64_t unit_stride, int32_t n, __half* __restrict__ k_res,
                                                        __half* __restrict__ v_res, LayerRows<LAYERS> rows) {
  const int ul = blockIdx.x, layer = LAYERS > 1 ? blockIdx.z : 0;
  const int64_t u = d.unit0 + (int64_t)layer * d.layer_units + ul;
  const uint4* sk = (const uint4*)(rows.k[layer] + (int64_t)ul * unit_stride);
  const uint4* sv = (const uint4*)(rows.v[layer] + (int64_t)ul * unit_stride);
  uint4* dk = (uint4*)(k_res + u * d.res_rows * kHeadDim);
  uint4* dv = (uint4*)(v_res + u * d.res_rows * kHeadDim);
  for (int i = blockIdx.y * 256 + threadIdx.x; i < n * 16; i += gridDim.y * 256) {
    dk[i] = sk[i];
    dv[i] = sv[i];
  }
}

// The whole group step of one unit in one launch: append the new token's row to the ring, run the
// outlier competition on the oldest G rows, quantize them.  The ring must be full after the
// append (R + G rows), its oldest G rows starting at ring row `group_row0`.
template <int BITS, int G>
__global__ void __launch_bounds__(kQuantThreads) group_step_kernel(
    Dims d, int32_t group_index, const __half* __restrict__ k_new, const __half* __restrict__ v_new, __half* k_res,
    __half* v_res, int32_t append_row, int32_t group_row0, const int32_t* __restrict__ seq, __half* pool_k,
    __half* pool_v, int32_t* pool_idx,
    double* pool_score, int32_t* pool_count, int32_t* aux_count, int32_t* frozen, uint8_t* selected,
    uint8_t* __restrict__ k_codes, uint32_t* __restrict__ k_meta, uint8_t* __restrict__ v_codes,
    uint32_t* __restrict__ v_meta, uint32_t* __restrict__ mask) {
  extern __shared__ __align__(16) unsigned char smem[];
  const QuantLds<G> L(smem, d.vgroups);
  const int tid = threadIdx.x;
  const int ul = blockIdx.x;
  const int64_t u = d.unit0 + ul;
  __half* kring = k_res + u * d.res_rows * kHeadDim;
  __half* vring = v_res + u * d.res_rows * kHeadDim;
  bool close_group = true;
  if (seq) {
    // A batch of sequences of different lengths: the unit's sequence says where its new row goes
    // and whether its ring is full with it.  A sequence that is inactive, or whose state does not
    // fit the buffers, is left alone; all of this is uniform over the workgroup.
    const int4 own = *(const int4*)(seq + 4 * (ul / d.kv_heads));
    const int nq = own.x, rs = own.y, nr = own.z;
    if (!own.w || nq < 0 || rs < 0 || rs >= d.res_rows || nr < 0 || nr >= d.res_rows) return;
    append_row = rs + nr;
    append_row -= append_row >= d.res_rows ? d.res_rows : 0;
    group_row0 = rs;
    group_index = nq / G;
    close_group = nr + 1 == d.R + G && rs % G == 0 && nq % G == 0 && nq + G <= d.max_seq;
  }
  if (tid < 128) {                                   // the new row: 64 threads for K, 64 for V, 4 bytes each
    const int which = tid >> 6, lane = tid & 63;
    const uint32_t* src = (const uint32_t*)((which ? v_new : k_new) + (int64_t)ul * kHeadDim);
    ((uint32_t*)((which ? vring : kring) + append_row * kHeadDim))[lane] = src[lane];
  }
  if (!close_group) return;
  const GroupPlace at = place_of_group(d, ul, group_index);        // where the group's codes and meta go
  if (append_row >= group_row0 && append_row < group_row0 + G) {   // R = 0: the new token closes the group
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  }
  const __half* gk = kring + group_row0 * kHeadDim;
  const __half* gv = vring + group_row0 * kHeadDim;
  GroupRows<G> rows;
  rows_issue<G>(rows, gk, gv, tid);
  uint8_t* sel = selected ? selected + (int64_t)ul * G : nullptr;
  if (d.N > 0) {
    const trace_core::UnitPool p =
        trace_core::unit_pool(d, u, pool_k, pool_v, pool_idx, pool_score, pool_count, aux_count, frozen);
    trace_core::Loaded<G> in;
    const bool ahead = d.N <= trace_core::kPoolRowsAhead;
    trace_core::load<G>(in, d, p, gk, tid, ahead);
    rows_to_lds<G>(rows, L, tid);
    trace_core::compete<G>(in, d, group_index, p, gk, gv, sel, L.ssel, tid, L.sk, L.sv, kRowB, ahead);
  } else {
    rows_to_lds<G>(rows, L, tid);
    if (tid < G) {
      L.ssel[tid] = 0;
      if (sel) sel[tid] = 0;
    }
  }
  __syncthreads();                                   // the flags are in LDS
  const uint8_t flag = tid < G ? L.ssel[tid] : (uint8_t)0;
  quantize_body<BITS, G>(d, at.row, at.slot, L, flag, k_codes, k_meta, v_codes, v_meta, mask, tid);
}

template <int BITS, int G, int LAYERS>
hipError_t launch_quantize_one(const Dims& d, int32_t group_index, int32_t n_groups, const PromptRows& rows,
                               const uint8_t* selected, int64_t selected_unit_stride,
                               const kvq_qcache& qc, int32_t tail_n, __half* k_res, __half* v_res, hipStream_t s) {
  // many groups (a prompt): the kernel that spends the fewest instructions per group; few: the one that is
  // done with a group soonest
  const int64_t groups = (int64_t)d.units_per_layer * rows.layers * n_groups;
  const bool many = groups >= prompt_groups(G) && !d.keys_only;
  const int threads = many ? 4 * G : kQuantThreads;
  const dim3 grid(d.units_per_layer, n_groups + (tail_n * 16 + threads - 1) / threads, rows.layers);
  auto go = [&](auto kern, size_t smem, auto... more) {
    hipLaunchKernelGGL(kern, grid, dim3(threads), smem, s, d, group_index, rows.unit_stride, selected,
                       selected_unit_stride, (uint8_t*)qc.k_codes, (uint32_t*)qc.k_meta, (uint8_t*)qc.v_codes,
                       (uint32_t*)qc.v_meta, (uint32_t*)qc.mask, n_groups, tail_n, k_res, v_res, more...,
                       layer_rows<LAYERS>(rows));
    return hipGetLastError();
  };
  // Two rules on the Keys' size.  (Times of the whole call, MB of 2^20 bytes; the memory-side cache holds 256.)
  // Where the competition has just read more Keys than the cache keeps besides everything else, the last groups come
  // first: their Keys are still there.  First to last / last to first, three sets of rows in turn, G = 32 2-bit, 4-bit, G = 128
  // 2-bit: 128 units x 4096 tokens (128 MB) 82.8 / 81.9 us, 96.2 / 94.9, 92.4 / 90.4; 256 x 4096 150.4 / 149.3, 173.9 / 171.2,
  // 170.4 / 167.6; 256 x 8192 286.0 / 285.0, 316.2 / 312.5, 324.0 / 321.6; 512 x 4096 319.4 / 317.7, 344.5 / 348.9, 340.5 / 340.2.
  // ONCE keeps rows that are not needed again, and the codes, from displacing the rest.  It pays where the rows have to
  // come from memory, and costs where the next call would have found the same rows in the same place in the cache (which
  // a prompt does not do).  Whole calls, three sets of rows in turn, without / with, G = 32 (64 and 128 alike):
  //   Keys   12 MB, 128 units   24, 128       36, 256       64, 32        100, 128      200, 128    400, 256    1100 MB, 512 units
  //   2-bit  26.4 / 26.1 us     31.7 / 32.2   41.2 / 38.9   60.4 / 54.7   83.4 / 77.1   153 / 134   275 / 238   745 / 688
  //   4-bit  29.0 / 28.9        35.5 / 35.6   45.5 / 44.1   67.3 / 62.4   92.7 / 88.3   166 / 150   304 / 263   794 / 732
  // With one set of rows, read again and again, it costs 2 .. 4 % from 32 to 100 MB, and gives 5 .. 13 % from 200 MB on.  Without
  // a pool, three sets that the cache holds together (32 MB): 18.5 / 20.9.  Rows that a copy has just written (the copies are
  // in the times), 128 units, without / with:
  //   Keys              32 MB         48           64              96              128             192
  //   G = 32, 2-bit     54.4 / 54.5   78.4 / 74.2  105.4 / 104.8   150.5 / 153.4   198.9 / 191.9   297.8 / 280.8
  //   G = 32, 4-bit     58.7 / 59.2   87.5 / 82.0  111.3 / 113.0   159.3 / 162.2   211.0 / 204.8   362.1 / 349.7
  //   G = 64, 2-bit     55.6 / 55.7   77.9 / 75.8  104.5 / 105.4   150.9 / 154.9   231.6 / 227.3   347.6 / 332.3
  //   G = 128, 2-bit    56.7 / 56.5   80.5 / 79.1  109.6 / 110.2   155.1 / 157.1   237.6 / 232.7   353.5 / 341.8
  //   no pool, G = 32   41.2 / 40.9   55.5 / 55.0  81.9 / 79.3     122.5 / 121.4   166.3 / 155.7   253.7 / 239.8
  // So it costs up to 4 us of about 75 there around 96 MB, where rows that are not so new gain 6, and gives on either side.
  const int64_t key_bytes = groups * G * (2 * kHeadDim);
  const int32_t last_first = key_bytes >= (1ll << 27);
  const bool once = key_bytes >= (1ll << 25);
  if (many && once) return go(prompt_quantize_kernel<BITS, G, LAYERS, true>, 0, last_first);
  if (many) return go(prompt_quantize_kernel<BITS, G, LAYERS, false>, 0, last_first);
  const size_t smem = quant_lds_bytes<G>(d.vgroups);
  if (smem > 48 * 1024) {  // more than the default limit of dynamic LDS per workgroup
    hipError_t e = hipFuncSetAttribute((const void*)quantize_kernel<BITS, G, LAYERS>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                       (int)smem);
    if (e != hipSuccess) return e;
  }
  return go(quantize_kernel<BITS, G, LAYERS>, smem);
}

}  // namespace

hipError_t launch_append(const Dims& d, const __half* k_new, const __half* v_new, __half* k_res, __half* v_res,
                         int32_t row, hipStream_t s) {
  hipLaunchKernelGGL(append_kernel, dim3(d.units_per_layer), dim3(128), 0, s, d, k_new, v_new, k_res, v_res, row);
  return hipGetLastError();
}

namespace {

template <int BITS, int G>
hipError_t launch_group_step_one(const Dims& d, int32_t group_index, const __half* k_new, const __half* v_new,
                                 __half* k_res, __half* v_res, int32_t append_row, int32_t group_row0,
                                 const int32_t* seq, const kvq_pool& pool, uint8_t* selected, const kvq_qcache& qc,
                                 hipStream_t s) {
  const size_t smem = quant_lds_bytes<G>(d.vgroups);
  if (smem > 48 * 1024) {
    hipError_t e = hipFuncSetAttribute((const void*)group_step_kernel<BITS, G>,
                                       hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((group_step_kernel<BITS, G>), dim3(d.units_per_layer), dim3(kQuantThreads), smem, s, d,
                     group_index, k_new, v_new, k_res, v_res, append_row, group_row0, seq, (__half*)pool.pool_k,
                     (__half*)pool.pool_v, pool.pool_idx, pool.pool_score, pool.pool_count, pool.aux_count,
                     pool.frozen, selected, (uint8_t*)qc.k_codes, (uint32_t*)qc.k_meta, (uint8_t*)qc.v_codes,
                     (uint32_t*)qc.v_meta, (uint32_t*)qc.mask);
  return hipGetLastError();
}

template <int BITS>
hipError_t launch_group_step_bits(const Dims& d, int32_t group_index, const __half* k_new, const __half* v_new,
                                  __half* k_res, __half* v_res, int32_t append_row, int32_t group_row0,
                                  const int32_t* seq, const kvq_pool& pool, uint8_t* selected, const kvq_qcache& qc,
                                  hipStream_t s) {
  switch (d.G) {
    case 32: return launch_group_step_one<BITS, 32>(d, group_index, k_new, v_new, k_res, v_res, append_row, group_row0, seq, pool, selected, qc, s);
    case 64: return launch_group_step_one<BITS, 64>(d, group_index, k_new, v_new, k_res, v_res, append_row, group_row0, seq, pool, selected, qc, s);
    default: return launch_group_step_one<BITS, 128>(d, group_index, k_new, v_new, k_res, v_res, append_row, group_row0, seq, pool, selected, qc, s);
  }
}

}  // namespace

// ---- per-step Value quantization ---------------------------------------------------------------
// One workgroup of 128 threads (thread = channel) per unit; the tokens of the call one after the
// other.  Per token: minimum and maximum of each group of Gv channels, step and zero, codes (Eq. 2,
// the same device functions as the group quantization), the dequantized row back into the ring, the
// steps and zeros to their places in the block's meta, and the token's 2 or 4 bits of 64 or 128
// packed words replaced (the words also hold the block's other tokens of the same 8).
template <int BITS>
__global__ void __launch_bounds__(128) value_tokens_kernel(Dims d, int32_t first_token, int32_t count,
                                                           __half* __restrict__ v_res, int32_t ring_row,
                                                           uint8_t* __restrict__ v_codes,
                                                           uint32_t* __restrict__ v_meta) {
  constexpr int kLevels = (1 << BITS) - 1;
  constexpr int kWords = 32 * BITS;                     // packed words that hold one token's codes
  __shared__ float s_mn[2], s_mx[2];
  __shared__ uint32_t s_words[kWords];
  const int ul = blockIdx.x;
  const int64_t u = d.unit0 + ul;
  const int c = threadIdx.x;                            // channel
  const int gv_shift = 31 - __clz(d.Gv);
  const int nblk_shift = d.bpg_shift;                   // blocks per Key group
  __half* ring = v_res + u * d.res_rows * kHeadDim;
  for (int i = 0; i < count; ++i) {
    const int tok = first_token + i;
    int row = ring_row + i;
    row -= row >= d.res_rows ? d.res_rows : 0;
    const float x = __half2float(ring[row * kHeadDim + c]);
    float mn = x, mx = x;
    const int team = d.Gv < 64 ? d.Gv : 64;
    for (int off = 1; off < team; off <<= 1) {
      mn = fminf(mn, __shfl_xor(mn, off));
      mx = fmaxf(mx, __shfl_xor(mx, off));
    }
    if (d.Gv == 128) {                                  // the group spans both wavefronts
      if ((c & 63) == 0) {
        s_mn[c >> 6] = mn;
        s_mx[c >> 6] = mx;
      }
      __syncthreads();
      mn = fminf(s_mn[0], s_mn[1]);
      mx = fmaxf(s_mx[0], s_mx[1]);
    }
    mn += 0.0f;                                         // a zero minimum is stored as +0
    const __half st = step_of(mn, mx, BITS);
    const float stf = __half2float(st);
    const uint32_t code = quant_code(x, mn, stf, kLevels);
    const float prod = (float)code * stf;               // exact
    ring[row * kHeadDim + c] = __float2half_rn(mn + prod);
    // where the token's block is stored
    const GroupPlace at = place_of_group(d, ul, tok / d.G);
    const int64_t blk = at.row * d.blocks_per_unit + ((int64_t)at.slot << nblk_shift) + ((tok % d.G) >> 5);
    const int tb = tok & 31;
    if ((c & (d.Gv - 1)) == 0) {
      const int j = c >> gv_shift;
      __half* gm = (__half*)(v_meta + blk * 32 * d.vgroups);
      gm[((tb >> 1) * d.vgroups + j) * 2 + (tb & 1)] = st;
      gm[32 * d.vgroups + ((tb >> 1) * d.vgroups + j) * 2 + (tb & 1)] = __float2half_rn(mn);
    }
    // codes: channel c = 16 f + n of token tb = 8 r + xx lives in lane 16 r + n, field f, code xx
    const int n = c & 15, f = c >> 4, xx = tb & 7, r = tb >> 3;
    const int slot = BITS == 2 ? n * 4 + (f >> 1) : (f >> 2) * 64 + n * 4 + (f & 3);
    __syncthreads();                                    // the previous token's words have been used
    if (c < kWords) s_words[c] = 0;
    __syncthreads();
    atomicOr(&s_words[slot], place_code(code, code_bit(BITS, f, xx)));
    __syncthreads();
    if (c < kWords) {
      const int half = BITS == 2 ? 0 : c >> 6, nn = (c & 63) >> 2, w = c & 3;
      const uint32_t clear = BITS == 2 ? (place_code(3u, code_bit(2, 0, xx)) | place_code(3u, code_bit(2, 1, xx)))
                                       : place_code(15u, code_bit(4, 0, xx));
      uint32_t* gw = (uint32_t*)(v_codes + blk * d.block_bytes + 1024 * half + 16 * (16 * r + nn) + 4 * w);
      *gw = (*gw & ~clear) | s_words[c];
    }
  }
}

hipError_t launch_value_tokens(const Dims& d, int32_t first_token, int32_t count, __half* v_res, int32_t ring_row,
                               const kvq_qcache& qc, hipStream_t s) {
  if (d.bits == 2)
    hipLaunchKernelGGL(value_tokens_kernel<2>, dim3(d.units_per_layer), dim3(128), 0, s, d, first_token, count, v_res,
                       ring_row, (uint8_t*)qc.v_codes, (uint32_t*)qc.v_meta);
  else
    hipLaunchKernelGGL(value_tokens_kernel<4>, dim3(d.units_per_layer), dim3(128), 0, s, d, first_token, count, v_res,
                       ring_row, (uint8_t*)qc.v_codes, (uint32_t*)qc.v_meta);
  return hipGetLastError();
}

// The state of every active sequence after one token has been appended to it (and its oldest group
// quantized if that filled its ring): the rule group_step_kernel applies, applied to the array.
__global__ void seq_advance_kernel(Dims d, int32_t* seq) {
  const int b = blockIdx.x * blockDim.x + threadIdx.x;
  if (b >= d.batch) return;
  int4 own = *(const int4*)(seq + 4 * b);
  if (!own.w || own.x < 0 || own.y < 0 || own.y >= d.res_rows || own.z < 0 || own.z >= d.res_rows) return;
  const bool close_group =
      own.z + 1 == d.R + d.G && own.y % d.G == 0 && own.x % d.G == 0 && own.x + d.G <= d.max_seq;
  own.z += 1;
  if (close_group) {
    own.x += d.G;
    own.z -= d.G;
    own.y += d.G;
    own.y -= own.y >= d.res_rows ? d.res_rows : 0;
  }
  *(int4*)(seq + 4 * b) = own;
}

// A launch plan for the decode attention of sequences of different lengths: `entries` workgroups per kv
// head are dealt to the sequences by the work each has (mini-chunks of quantized tokens, groups of
// full-precision rows at half a mini-chunk each), every sequence at least one; a sequence's workgroups
// share its mini-chunks equally.  The share m of one workgroup is the smallest for which the sequences'
// workgroups, ceil(work / m) each, are at most `entries` in all (found by bisection: that count does not
// grow with m).  One workgroup, one thread per sequence.  What bounds it is the bisection, one sum over the
// sequences per step: up to 64 sequences are one wavefront's, which needs neither LDS nor barriers for it
// (32 sequences of 128 .. 8192 tokens: 6.6 -> 4.6 us).
template <bool ONE_WAVE>
__global__ void __launch_bounds__(1024) seq_plan_kernel(Dims d, const int32_t* __restrict__ seq, int32_t max_nq,
                                                         int32_t max_nres, int32_t entries, int32_t* __restrict__ plan) {
  __shared__ int s_acc;
  __shared__ int s_wave[16];
  const int b = threadIdx.x;
  const bool live = b < d.batch;
  int nq = 0, rs = 0, nr = 0, w = 0, mc = 0;
  if (live) {
    const int4 own = *(const int4*)(seq + 4 * b);
    nq = min(max(own.x, 0), max_nq) & ~(kBlockTokens - 1);
    rs = (own.y >= 0 && own.y < d.res_rows) ? own.y & ~15 : 0;
    nr = min(max(own.z, 0), max_nres);
    mc = (nq + kMiniChunk - 1) / kMiniChunk;
    w = 2 * mc + ((nr + kFpGroupRows - 1) / kFpGroupRows) + ((d.pool_slots + kFpGroupRows - 1) / kFpGroupRows);
  }
  auto block_sum = [&](int v) {
    if (ONE_WAVE) return __builtin_amdgcn_readlane(wave_scan(v), 63);
    if (threadIdx.x == 0) s_acc = 0;
    __syncthreads();
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    if ((threadIdx.x & 63) == 0) atomicAdd(&s_acc, v);
    __syncthreads();
    const int r = s_acc;
    __syncthreads();
    return r;
  };
  auto block_max = [&](int v) {
    for (int off = 32; off > 0; off >>= 1) v = max(v, __shfl_xor(v, off));
    if (ONE_WAVE) return __builtin_amdgcn_readfirstlane(v);
    if (threadIdx.x == 0) s_acc = 0;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) atomicMax(&s_acc, v);
    __syncthreads();
    const int r = s_acc;
    __syncthreads();
    return r;
  };
  auto splits_for = [&](int m) { return live ? min(max((w + m - 1) / m, 1), max(mc, 1)) : 0; };
  int lo = 1, hi = max(block_max(w), 1);                // at m = hi every sequence has one workgroup: entries >= batch
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (block_sum(splits_for(mid)) <= entries) hi = mid;
    else lo = mid + 1;
  }
  const int sp = splits_for(lo);
  // exclusive prefix of the sequences' workgroup counts
  const int incl = wave_scan(sp);
  int before = 0;
  if (!ONE_WAVE) {
    if ((threadIdx.x & 63) == 63) s_wave[threadIdx.x >> 6] = incl;
    __syncthreads();
    for (int k = 0; k < (int)(threadIdx.x >> 6); ++k) before += s_wave[k];
  }
  const int first = before + incl - sp;
  if (threadIdx.x == blockDim.x - 1) plan[0] = min(first + sp, entries);
  if (live) {
    const int per = (mc + sp - 1) / sp;                  // mini-chunks per workgroup of this sequence
    for (int k = 0; k < sp && first + k < entries; ++k) {
      int4* e = (int4*)(plan + 8 + 8 * (first + k));
      e[0] = make_int4(b, k, sp, min(k * per, mc));
      e[1] = make_int4(nq, rs, nr, min((k + 1) * per, mc));
    }
  }
}

hipError_t launch_seq_plan(const Dims& d, const int32_t* seq, int32_t max_n_quant, int32_t max_n_res, int32_t entries,
                           int32_t* plan, hipStream_t s) {
  if (d.batch <= 64)
    hipLaunchKernelGGL(seq_plan_kernel<true>, dim3(1), dim3(64), 0, s, d, seq, max_n_quant, max_n_res, entries, plan);
  else
    hipLaunchKernelGGL(seq_plan_kernel<false>, dim3(1), dim3(1024), 0, s, d, seq, max_n_quant, max_n_res, entries, plan);
  return hipGetLastError();
}

hipError_t launch_seq_advance(const Dims& d, int32_t* seq, hipStream_t s) {
  hipLaunchKernelGGL(seq_advance_kernel, dim3((d.batch + 255) / 256), dim3(256), 0, s, d, seq);
  return hipGetLastError();
}

hipError_t launch_group_step(const Dims& d, int32_t group_index, const __half* k_new, const __half* v_new,
                             __half* k_res, __half* v_res, int32_t append_row, int32_t group_row0,
                             const int32_t* seq, const kvq_pool& pool, uint8_t* selected, const kvq_qcache& qc,
                             hipStream_t s) {
  return d.bits == 2 ? launch_group_step_bits<2>(d, group_index, k_new, v_new, k_res, v_res, append_row, group_row0, seq, pool, selected, qc, s)
                     : launch_group_step_bits<4>(d, group_index, k_new, v_new, k_res, v_res, append_row, group_row0, seq, pool, selected, qc, s);
}

// The entry of a sequence in the array of states, {n_quant, 0, n_res, active}.  A launch of its own, behind those that
// write what the entry speaks of: a launch on another stream that finds the sequence active finds its rows and codes
// too.  (Written by a workgroup of the quantization it is seen while others are still at work, and ahead of their loads
// it cost each of them a test.  With it a prompt of 8191 tokens, 8 kv heads, 4 layers takes 60.4 us, 59.0 without.)
__global__ void seq_entry_kernel(int4* at, int4 state) { *at = state; }
hipError_t launch_seq_entry(int32_t* at, int32_t n_quant, int32_t n_res, int32_t active, hipStream_t s) {
  hipLaunchKernelGGL(seq_entry_kernel, dim3(1), dim3(1), 0, s, (int4*)at, make_int4(n_quant, 0, n_res, active));
  return hipGetLastError();
}

hipError_t launch_quantize(const Dims& d, int32_t group_index, int32_t n_groups, const PromptRows& rows,
                           const uint8_t* selected, int64_t selected_unit_stride, const kvq_qcache& qc, hipStream_t s,
                           int32_t tail_n, __half* k_res, __half* v_res) {
  auto go = [&](auto bits, auto group) {
    constexpr int BITS = decltype(bits)::value, G = decltype(group)::value;
    const auto one = rows.layers == 1 ? launch_quantize_one<BITS, G, 1> : launch_quantize_one<BITS, G, kPromptLayers>;
    return one(d, group_index, n_groups, rows, selected, selected_unit_stride, qc, tail_n, k_res, v_res, s);
  };
  auto of_bits = [&](auto bits) {
    switch (d.G) {
      case 32: return go(bits, std::integral_constant<int, 32>{});
      case 64: return go(bits, std::integral_constant<int, 64>{});
      default: return go(bits, std::integral_constant<int, 128>{});
    }
  };
  return d.bits == 2 ? of_bits(std::integral_constant<int, 2>{}) : of_bits(std::integral_constant<int, 4>{});
}

hipError_t launch_tail_copy(const Dims& d, const PromptRows& rows, int32_t n, __half* k_res,
                            __half* v_res, hipStream_t s) {
  if (n <= 0) return hipSuccess;
  const int by = (n * 16 + 255) / 256;
  auto go = [&](auto kern, const auto& at) {
    hipLaunchKernelGGL(kern, dim3(d.units_per_layer, by > 16 ? 16 : by, rows.layers), dim3(256), 0, s, d,
                       rows.unit_stride, n, k_res, v_res, at);
    return hipGetLastError();
  };
  return rows.layers == 1 ? go(tail_copy_kernel<1>, layer_rows<1>(rows))
                          : go(tail_copy_kernel<kPromptLayers>, rows.at);
}

}  // namespace kvq
