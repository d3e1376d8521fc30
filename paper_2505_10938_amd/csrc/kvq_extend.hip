// A chunk of tokens that joins caches which may hold tokens already: the groups that it fills are traced in order and
// quantized, what is left goes to the ring.
#include "kvq_common.h"
#include "kvq_quantize_core.h"
#include "kvq_trace_core.h"

#include <type_traits>

namespace kvq {

namespace {

struct ExtendArgs {
  Dims d;
  const __half* k_new;
  const __half* v_new;
  int64_t kv_stride;
  const int32_t* starts;
  int32_t total, max_tokens;
  __half* k_res;
  __half* v_res;
  const int32_t* seq;
  int32_t n_quant, res_start, n_res;
  kvq_pool pool;
  kvq_qcache qc;
  uint8_t* selected;         // [unit][most_groups][G]
  int32_t most_groups;       // that a chunk of max_tokens tokens fills
};

// What a sequence's chunk comes to.  A state that the calls on states do not produce, an inactive sequence and one whose
// groups do not fit are left alone: no token, no group.
struct Extension {
  int64_t first;             // row of the packed arrays
  int n, nq, rs, nr, groups;
};
__device__ __forceinline__ Extension extension(const Dims& d, int4 own, ChunkRows rows) {
  Extension x = {rows.first, 0, own.x, own.y, own.z, 0};
  if (!own.w || own.x < 0 || own.x > d.max_seq || own.x % d.G != 0 || own.y < 0 || own.y >= d.res_rows || own.y % d.G != 0 ||
      own.z < 0 || own.z >= d.R + d.G)
    return x;
  const int64_t held = (int64_t)own.z + rows.n;
  const int64_t groups = held >= d.R + d.G ? (held - d.R) / d.G : 0;
  if (own.x + groups * d.G > d.max_seq) return x;
  x.n = rows.n;
  x.groups = (int)groups;
  return x;
}
__device__ __forceinline__ Extension extension_of(const ExtendArgs& a, int b) {
  const int4 own = a.seq ? *(const int4*)(a.seq + 4 * b) : make_int4(a.n_quant, a.res_start, a.n_res, 1);
  return extension(a.d, own, chunk_rows(a.starts, a.total, a.max_tokens, b));
}

// The unit's rows behind its quantized tokens, old and new: row i of them is in the ring or in the chunk.
struct JoinedRows {
  const __half* ring_k;
  const __half* ring_v;
  const __half* new_k;
  const __half* new_v;
  int64_t stride;
  int rs, nr, res_rows;
  int base;                  // row 0 of the group looked at
  __device__ __forceinline__ int64_t at(int i) const {    // elements: in the ring, or (from nr on) in the chunk
    if (i >= nr) return (i - nr) * stride;
    int r = rs + i;
    r -= r >= res_rows ? res_rows : 0;
    return (int64_t)r * kHeadDim;
  }
  __device__ __forceinline__ const __half* k(int t) const { return (base + t < nr ? ring_k : new_k) + at(base + t); }
  __device__ __forceinline__ const __half* v(int t) const { return (base + t < nr ? ring_v : new_v) + at(base + t); }
};
__device__ __forceinline__ JoinedRows joined_rows(const ExtendArgs& a, const Extension& x, int ul, int h) {
  const int64_t ring = (a.d.unit0 + ul) * a.d.res_rows * kHeadDim, first = x.first * a.kv_stride + h * kHeadDim;
  return {a.k_res + ring, a.v_res + ring, a.k_new + first, a.v_new + first, a.kv_stride, x.rs, x.nr, a.d.res_rows, 0};
}

// The competitions, a workgroup per unit, group after group.
template <int G>
__global__ void __launch_bounds__(trace_core::kWorkers) extend_trace_kernel(ExtendArgs a) {
  const Dims& d = a.d;
  const int ul = blockIdx.x, tid = threadIdx.x;
  const int b = ul / d.kv_heads, h = ul - b * d.kv_heads;
  const Extension x = extension_of(a, b);
  if (x.groups == 0) return;
  uint8_t* sel = a.selected + (int64_t)ul * a.most_groups * G;
  if (d.N == 0) {
    for (int i = tid; i < x.groups * G; i += trace_core::kWorkers) sel[i] = 0;
    return;
  }
  JoinedRows rows = joined_rows(a, x, ul, h);
  const trace_core::UnitPool p =
      trace_core::unit_pool(d, d.unit0 + ul, (__half*)a.pool.pool_k, (__half*)a.pool.pool_v, a.pool.pool_idx, a.pool.pool_score,
                            a.pool.pool_count, a.pool.aux_count, a.pool.frozen);
  for (int j = 0; j < x.groups; ++j) {
    rows.base = j * G;
    trace_core::Loaded<G> in;
    const bool ahead = d.N <= trace_core::kPoolRowsAhead;
    trace_core::load_from<G>(in, d, p, rows, tid, ahead);
    trace_core::compete_over<G>(in, d, x.nq / G + j, p, rows, sel + j * G, nullptr, tid, nullptr, nullptr, 0, ahead);
    __syncthreads();                                     // the pool's new state is in memory
  }
}

// A workgroup per (unit, group).
template <int BITS, int G>
__global__ void __launch_bounds__(kQuantThreads) extend_quantize_kernel(ExtendArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  const Dims& d = a.d;
  const QuantLds<G> L(smem, d.vgroups);
  const int ul = blockIdx.x / a.most_groups, j = blockIdx.x - ul * a.most_groups, tid = threadIdx.x;
  const int b = ul / d.kv_heads, h = ul - b * d.kv_heads;
  const Extension x = extension_of(a, b);
  if (j >= x.groups) return;
  JoinedRows rows = joined_rows(a, x, ul, h);
  rows.base = j * G;
  GroupRows<G> group;
#pragma unroll
  for (int q = 0; q < GroupRows<G>::kLoads; ++q) {
    const int e = q * kQuantThreads + tid;
    const int kv = e / (G * 16), rem = e % (G * 16);
    group.rw[q] = *(const u32x4*)((kv ? rows.v(rem >> 4) : rows.k(rem >> 4)) + (rem & 15) * 8);
  }
  const uint8_t flag = tid < G ? a.selected[((int64_t)ul * a.most_groups + j) * G + tid] : 0;
  const GroupPlace at = place_of_group(d, ul, x.nq / G + j);
  rows_to_lds<G>(group, L, tid);
  quantize_body<BITS, G>(d, at.row, at.slot, L, flag, (uint8_t*)a.qc.k_codes, (uint32_t*)a.qc.k_meta, (uint8_t*)a.qc.v_codes,
                         (uint32_t*)a.qc.v_meta, (uint32_t*)a.qc.mask, tid);
}

// The new tokens behind the last group, to the ring (a launch of its own: their places are those of tokens that the
// quantization reads).  grid (units, 16-row pieces).
__global__ void __launch_bounds__(256) extend_ring_kernel(ExtendArgs a) {
  const Dims& d = a.d;
  const int ul = blockIdx.x, tid = threadIdx.x;
  const int b = ul / d.kv_heads, h = ul - b * d.kv_heads;
  const Extension x = extension_of(a, b);
  const int from = max(x.groups * d.G, x.nr), end = x.nr + x.n;
  const int i = from + blockIdx.y * 16 + (tid >> 4), piece = tid & 15;
  if (i >= end) return;
  const JoinedRows rows = joined_rows(a, x, ul, h);
  const int64_t to = ((d.unit0 + ul) * d.res_rows + (x.rs + i) % d.res_rows) * kHeadDim + 8 * piece;
  *(uint4*)(a.k_res + to) = *(const uint4*)(rows.k(i) + 8 * piece);
  *(uint4*)(a.v_res + to) = *(const uint4*)(rows.v(i) + 8 * piece);
}

__global__ void seq_extend_kernel(Dims d, int32_t* seq, kvq_chunk chunk) {
  const int b = blockIdx.x * blockDim.x + threadIdx.x;
  if (b >= d.batch) return;
  const Extension x = extension(d, *(const int4*)(seq + 4 * b), chunk_rows(chunk.starts, chunk.total, chunk.max_tokens, b));
  if (x.n == 0) return;
  const int done = x.groups * d.G;
  *(int4*)(seq + 4 * b) = make_int4(x.nq + done, (x.rs + done) % d.res_rows, x.nr + x.n - done, 1);
}

}  // namespace

hipError_t launch_extend(const Dims& d, const __half* k_new, const __half* v_new, int64_t kv_stride, const kvq_chunk& chunk,
                         const kvq_residual& res, const int32_t* seq, int32_t n_quant, int32_t res_start, int32_t n_res,
                         const kvq_pool& pool, uint8_t* selected, const kvq_qcache& qc, hipStream_t s) {
  ExtendArgs a;
  a.d = d;
  a.k_new = k_new;
  a.v_new = v_new;
  a.kv_stride = kv_stride;
  a.starts = chunk.starts;
  a.total = chunk.total;
  a.max_tokens = chunk.max_tokens;
  a.k_res = (__half*)res.k_res;
  a.v_res = (__half*)res.v_res;
  a.seq = seq;
  a.n_quant = n_quant;
  a.res_start = res_start;
  a.n_res = n_res;
  a.pool = pool;
  a.qc = qc;
  a.selected = selected;
  a.most_groups = (chunk.max_tokens + d.G - 1) / d.G;
  auto go = [&](auto bits, auto group) -> hipError_t {
    constexpr int BITS = decltype(bits)::value, G = decltype(group)::value;
    hipLaunchKernelGGL(extend_trace_kernel<G>, dim3(d.units_per_layer), dim3(trace_core::kWorkers), 0, s, a);
    const size_t smem = quant_lds_bytes<G>(d.vgroups);
    if (smem > 48 * 1024) {
      const hipError_t e = hipFuncSetAttribute((const void*)extend_quantize_kernel<BITS, G>,
                                               hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((extend_quantize_kernel<BITS, G>), dim3((uint32_t)d.units_per_layer * a.most_groups), dim3(kQuantThreads),
                       smem, s, a);
    return hipGetLastError();
  };
  // (with uniform states the host knows whether any group fills)
  if (seq || (int64_t)n_res + chunk.max_tokens >= d.R + d.G) {
    auto of_bits = [&](auto bits) {
      switch (d.G) {
        case 32: return go(bits, std::integral_constant<int, 32>{});
        case 64: return go(bits, std::integral_constant<int, 64>{});
        default: return go(bits, std::integral_constant<int, 128>{});
      }
    };
    const hipError_t e = d.bits == 2 ? of_bits(std::integral_constant<int, 2>{}) : of_bits(std::integral_constant<int, 4>{});
    if (e != hipSuccess) return e;
  }
  const int32_t most = chunk.max_tokens < d.R + d.G ? chunk.max_tokens : d.R + d.G;
  hipLaunchKernelGGL(extend_ring_kernel, dim3(d.units_per_layer, (most + 15) / 16), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_seq_extend(const Dims& d, int32_t* seq, const kvq_chunk& chunk, hipStream_t s) {
  hipLaunchKernelGGL(seq_extend_kernel, dim3((d.batch + 255) / 256), dim3(256), 0, s, d, seq, chunk);
  return hipGetLastError();
}

}  // namespace kvq
