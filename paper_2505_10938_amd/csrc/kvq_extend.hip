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
  const int shift = 5 + d.bpg_shift, part = d.G - 1;      // (G is 32, 64 or 128)
  if (!own.w || own.x < 0 || own.x > d.max_seq || (own.x & part) || own.y < 0 || own.y >= d.res_rows || (own.y & part) ||
      own.z < 0 || own.z >= d.R + d.G)
    return x;
  const int held = own.z + rows.n;                       // (at most 2^30 new tokens)
  const int groups = held >= d.R + d.G ? (held - d.R) >> shift : 0;
  if (groups > (d.max_seq - own.x) >> shift) return x;
  x.n = rows.n;
  x.groups = groups;
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

// The competitions, a workgroup per unit.  All tokens' scores come first, kSegment at a time.  Then only groups are looked at
// that can change the pool: those with a score below its largest, or all while it is not full (with the first prefix behind
// them few are: 1 .. 2000 tokens behind 2083, N = 8, a handful of up to 31).  A group's competition ranks pool and group by
// counting, as trace_core::compete does, but on scores in LDS, and moves no rows: where each slot's row comes from is noted,
// and rows are copied once, at the end.  16 chunks of 1 .. 2000 tokens, 8 kv heads, G = 64: 184 us when every group was loaded,
// ranked and moved after the other.
constexpr int kTraceThreads = 1024;
constexpr int kSegment = 2048;
constexpr int kRowsInFlight = 8;
typedef unsigned long long u64;      // scores as their bits: they are not negative, so they are ordered alike (a NaN last)

__device__ __forceinline__ u64 largest_of_lanes(u64 v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    const u64 o = __shfl_xor(v, off);
    v = o > v ? o : v;
  }
  return v;
}

template <int G>
__global__ void __launch_bounds__(kTraceThreads) extend_trace_kernel(ExtendArgs a) {
  constexpr int kMost = 64 + G;                          // candidates: pool and group
  __shared__ u64 s_score[kSegment], s_least[kSegment / G];
  __shared__ u64 c_score[kMost], p_score[64], x_score[64];
  __shared__ int32_t c_idx[kMost], c_rank[kMost], p_idx[64], x_idx[64];
  __shared__ int32_t p_from[64], x_from[64];             // row of a slot: >= 0 the pool's as it was, < 0: -1 - joined row
  __shared__ int32_t gone[64], s_gone, s_new[kMost / 64 + 1];
  const Dims& d = a.d;
  const int tid = threadIdx.x, lane = tid & 63, team = tid >> 4, sub = tid & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ul = blockIdx.x, b = ul / d.kv_heads, h = ul - b * d.kv_heads;
  const Extension x = extension_of(a, b);
  if (x.groups == 0) return;
  uint8_t* sel = a.selected + (int64_t)ul * a.most_groups * G;
  const int64_t u = d.unit0 + ul;
  const int n_tok = x.groups * G;
  for (int i = tid; i < n_tok; i += kTraceThreads) sel[i] = 0;
  if (d.N == 0 || a.pool.frozen[u]) return;
  const int N = d.N, A = d.A;
  const int64_t slot0 = u * d.pool_slots;
  int n_old = min(max(a.pool.pool_count[u], 0), N), n_aux = min(max(a.pool.aux_count[u], 0), A);
  const int n_aux0 = n_aux;
  if (tid < N) {
    p_score[tid] = (u64)__double_as_longlong(a.pool.pool_score[slot0 + tid]);
    p_idx[tid] = a.pool.pool_idx[slot0 + tid];
    p_from[tid] = tid;
  }
  const JoinedRows rows = joined_rows(a, x, ul, h);
  bool stopped = false;
  for (int t0 = 0; t0 < n_tok && !stopped; t0 += kSegment) {
    const int n = min(kSegment, n_tok - t0);
    for (int e0 = 0; e0 < n; e0 += kRowsInFlight * kTraceThreads / 16) {
      u32x4 w[kRowsInFlight];
#pragma unroll
      for (int q = 0; q < kRowsInFlight; ++q)
        w[q] = *(const u32x4*)(rows.k(t0 + min(e0 + q * (kTraceThreads / 16) + team, n - 1)) + sub * 8);
#pragma unroll
      for (int q = 0; q < kRowsInFlight; ++q) {
        const int e = e0 + q * (kTraceThreads / 16) + team;
        if (e0 + q * (kTraceThreads / 16) >= n) break;   // uniform
        const double sc = trace_core::team_sum_f64(trace_core::abs_sum8(make_uint4(w[q][0], w[q][1], w[q][2], w[q][3])));
        if (sub == 0 && e < n) s_score[e] = (u64)__double_as_longlong(sc);
      }
    }
    __syncthreads();
    if (tid * G < n) {
      u64 least = ~0ull;
      for (int t = 0; t < G; ++t) least = min(least, s_score[tid * G + ((t + tid) & (G - 1))]);
      s_least[tid] = least;
    }
    __syncthreads();
    const int groups = n / G;
    for (int j = 0; j < groups && !stopped; ++j) {
      // the next group with something to say (every wavefront finds it for itself)
      const u64 worst = n_old < N ? ~0ull : largest_of_lanes(lane < n_old ? p_score[lane] : 0ull);
      const u64 ask = __ballot(j + lane < groups && (n_old < N || s_least[min(j + lane, groups - 1)] < worst));
      if (!ask) break;
      j += __ffsll((long long)ask) - 1;
      const int n_cand = n_old + G, first = x.nq + t0 + j * G;
      if (tid < n_cand) {
        c_score[tid] = tid < n_old ? p_score[tid] : s_score[j * G + tid - n_old];
        c_idx[tid] = tid < n_old ? p_idx[tid] : first + tid - n_old;
        c_rank[tid] = 0;
      }
      __syncthreads();
      // rank by (score, token index): lane = candidate, the wavefronts share the candidates to compare with
      for (int base = 0; base < n_cand; base += 64) {
        const int me = min(base + lane, n_cand - 1);
        const u64 sme = c_score[me];
        const int32_t ix = c_idx[me];
        int less = 0;
        for (int k = wave; k < n_cand; k += kTraceThreads / 64) less += c_score[k] < sme || (c_score[k] == sme && c_idx[k] < ix);
        if (base + lane < n_cand && less) atomicAdd(&c_rank[base + lane], less);
      }
      __syncthreads();
      const int keep = min(N, n_cand);
      const bool out = tid < n_old && c_rank[tid] >= keep;
      const bool in = tid >= n_old && tid < n_cand && c_rank[tid] < keep;
      const u64 outs = __ballot(out), ins = __ballot(in), below = (1ull << lane) - 1ull;
      int order = __popcll((out ? outs : ins) & below);  // (all members sit in wavefront 0)
      if (lane == 0 && wave < kMost / 64 + 1) s_new[wave] = __popcll(ins);
      if (tid == 0) s_gone = __popcll(outs);
      __syncthreads();
      const int n_out = s_gone;
      int n_in = 0;
      for (int k = 0; k < kMost / 64 + 1; ++k) {
        if (k < wave && in) order += s_new[k];
        n_in += s_new[k];
      }
      if (n_aux + n_out > A) {                           // (uniform) tracing stops before this group
        stopped = true;
        break;
      }
      if (out) {
        gone[order] = tid;
        x_score[n_aux - n_aux0 + order] = p_score[tid];
        x_idx[n_aux - n_aux0 + order] = p_idx[tid];
        x_from[n_aux - n_aux0 + order] = p_from[tid];
      }
      __syncthreads();
      if (in) {                                          // into the freed slots, then the free ones
        const int to = order < n_out ? gone[order] : n_old - n_out + order;
        p_score[to] = c_score[tid];
        p_idx[to] = c_idx[tid];
        p_from[to] = -1 - (t0 + j * G + tid - n_old);
        sel[t0 + j * G + tid - n_old] = 1;
      }
      n_old += n_in - n_out;
      n_aux += n_out;
      __syncthreads();
    }
    __syncthreads();                                     // (the scores' place is written again)
  }
  // the slots' new rows, a team each: every load has returned before anything is stored (a slot may be another's source)
  __half* pk = (__half*)a.pool.pool_k + slot0 * kHeadDim;
  __half* pv = (__half*)a.pool.pool_v + slot0 * kHeadDim;
  u32x4 wk[2], wv[2];
  int to[2];
#pragma unroll
  for (int q = 0; q < 2; ++q) {                          // pool slots, then those of the auxiliary pool that are new
    const int s = team;
    const bool some = q == 0 ? s < n_old && p_from[s] != s : s < n_aux - n_aux0;
    to[q] = some ? (q == 0 ? s : N + n_aux0 + s) : -1;
    wk[q] = wv[q] = u32x4{0, 0, 0, 0};
    if (some) {
      const int from = q == 0 ? p_from[s] : x_from[s];
      const __half* fk = from >= 0 ? pk + from * kHeadDim : rows.k(-1 - from);
      const __half* fv = from >= 0 ? pv + from * kHeadDim : rows.v(-1 - from);
      wk[q] = *(const u32x4*)(fk + 8 * sub);
      wv[q] = *(const u32x4*)(fv + 8 * sub);
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    if (to[q] < 0) continue;
    *(u32x4*)(pk + to[q] * kHeadDim + 8 * sub) = wk[q];
    *(u32x4*)(pv + to[q] * kHeadDim + 8 * sub) = wv[q];
    if (sub == 0) {
      a.pool.pool_idx[slot0 + to[q]] = q == 0 ? p_idx[team] : x_idx[team];
      a.pool.pool_score[slot0 + to[q]] = __longlong_as_double((long long)(q == 0 ? p_score[team] : x_score[team]));
    }
  }
  if (tid == 0) {
    a.pool.pool_count[u] = n_old;
    a.pool.aux_count[u] = n_aux;
    if (stopped) a.pool.frozen[u] = 1;
  }
}

// A workgroup per (unit, group).
template <int BITS, int G>
__global__ void __launch_bounds__(4 * G) __attribute__((amdgpu_waves_per_eu(4, 8))) extend_quantize_kernel(ExtendArgs a) {
  const Dims& d = a.d;
  const int ul = blockIdx.x / a.most_groups, j = blockIdx.x - ul * a.most_groups;
  const int b = ul / d.kv_heads, h = ul - b * d.kv_heads;
  const Extension x = extension_of(a, b);
  if (j >= x.groups) return;
  JoinedRows rows = joined_rows(a, x, ul, h);
  rows.base = j * G;
  quantize_rows<BITS, G, false>(d, rows, a.selected + ((int64_t)ul * a.most_groups + j) * G, place_of_group(d, ul, x.nq / G + j),
                                (uint8_t*)a.qc.k_codes, (uint32_t*)a.qc.k_meta, (uint8_t*)a.qc.v_codes, (uint32_t*)a.qc.v_meta,
                                (uint32_t*)a.qc.mask, threadIdx.x);
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
    hipLaunchKernelGGL(extend_trace_kernel<G>, dim3(d.units_per_layer), dim3(kTraceThreads), 0, s, a);
    hipLaunchKernelGGL((extend_quantize_kernel<BITS, G>), dim3((uint32_t)d.units_per_layer * a.most_groups), dim3(4 * G), 0, s, a);
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
