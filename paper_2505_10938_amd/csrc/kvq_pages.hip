// Sequences that take over others, and the pages of a paged cache: which are live, copies, a pool packed into another.
#include "kvq_common.h"

namespace kvq {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// ---- sequences that take over others ------------------------------------------------------------------------------------
// All pairs take effect at once, whatever chains and rings they form: a workgroup has one slice of an array for ALL pairs,
// loads it for every source before it stores it for any target, and no other workgroup touches that slice.  What says which
// rows are live (states and counts) is copied by a launch of its own behind the first.
constexpr int kForkThreads = 256;
constexpr int kForkLoads = 8;            // in flight per thread
constexpr int kForkItems = kForkThreads * kForkLoads;
constexpr int kForkJobs = 12;

enum ForkKind { kRingRows, kPoolRows, kPoolWords, kPoolPairs, kGroups, kTable };

// One array: elements of 16 or 4 bytes, `elems` of a unit (of a sequence, for the table), of which the kind says the live ones.
struct ForkJob {
  void* base;
  int64_t unit_stride;       // bytes
  int32_t kind;
  int32_t wide;              // 16-byte elements
  int32_t elems;
  int32_t per_group;         // kGroups: elements of a group
  uint32_t first_block;      // of the launch's blocks
  int32_t slices;            // blocks per plane
};
struct ForkArgs {
  Dims d;
  const int32_t* pairs;
  int32_t n_pairs;
  int32_t slice_shift;       // 1 << slice_shift elements of a unit are one block's
  const int32_t* seq;
  int32_t n_quant, res_start, n_res;
  const int32_t* pool_count;
  const int32_t* aux_count;
  int32_t n_jobs;
  ForkJob job[kForkJobs];
};

struct Live {
  int nq, rs, nr;
};
__device__ __forceinline__ Live live_of(const ForkArgs& a, int b) {
  Live s = {a.n_quant, a.res_start, a.n_res};
  if (a.seq) {
    const int4 own = *(const int4*)(a.seq + 4 * b);
    s = {own.x, own.y, own.z};
  }
  s.nq = min(max(s.nq, 0), a.d.max_seq);
  s.rs = s.rs >= 0 && s.rs < a.d.res_rows ? s.rs : 0;
  return s;
}

// UNIFORM: a wavefront's elements are of one pair (slices of 64 and more), which is then looked up by the scalar unit.  (32 layers, 8 of 32
// sequences take over others, 335 MB: 94 us with slices of any length, a division per element, and lookups by the lanes, 65 so.)
template <bool UNIFORM>
__global__ void __launch_bounds__(kForkThreads) fork_kernel(ForkArgs a) {
  const Dims& d = a.d;
  const int in_slice = (1 << a.slice_shift) - 1, group_shift = 5 + d.bpg_shift;
  int j = 0;
  while (j + 1 < a.n_jobs && blockIdx.x >= a.job[j + 1].first_block) ++j;
  const ForkJob job = a.job[j];
  const uint32_t at = blockIdx.x - job.first_block;
  const int plane = at / job.slices, e0 = (at - plane * job.slices) << a.slice_shift;
  const int layer = plane / d.kv_heads, h = plane - layer * d.kv_heads;
  auto unit_of = [&](int b) -> int64_t {
    return job.kind == kTable ? b : ((int64_t)layer * d.batch + b) * d.kv_heads + h;
  };
  u32x4 v[kForkLoads];
  int to[kForkLoads];                    // target sequence, or -1
#pragma unroll
  for (int k = 0; k < kForkLoads; ++k) {
    const int i = k * kForkThreads + threadIdx.x;
    const int p = UNIFORM ? __builtin_amdgcn_readfirstlane(i >> a.slice_shift) : i >> a.slice_shift, e = e0 + (i & in_slice);
    to[k] = -1;
    v[k] = u32x4{0, 0, 0, 0};
    if (p >= a.n_pairs || e >= job.elems) continue;
    const int src = a.pairs[2 * p], dst = a.pairs[2 * p + 1];
    if (src < 0 || src >= d.batch || dst < 0 || dst >= d.batch) continue;
    const int64_t u = unit_of(src);
    bool live;
    if (job.kind == kRingRows) {
      const Live s = live_of(a, src);
      int rel = (e >> 4) - s.rs;
      rel += rel < 0 ? d.res_rows : 0;
      live = rel < s.nr;
    } else if (job.kind == kGroups) {
      live = e < (live_of(a, src).nq >> group_shift) * job.per_group;
    } else if (job.kind == kTable) {
      live = e < live_of(a, src).nq >> group_shift;
    } else {
      const int slot = job.kind == kPoolRows ? e >> 4 : job.kind == kPoolPairs ? e >> 1 : e;
      live = slot < d.N ? slot < a.pool_count[u] : slot - d.N < a.aux_count[u];
    }
    if (!live) continue;
    const unsigned char* from = (const unsigned char*)job.base + u * job.unit_stride;
    if (job.wide) v[k] = ((const u32x4*)from)[e];
    else v[k][0] = ((const uint32_t*)from)[e];
    to[k] = dst;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // a target may be another pair's source
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kForkLoads; ++k) {
    if (to[k] < 0) continue;
    const int i = k * kForkThreads + threadIdx.x;
    const int e = e0 + (i & in_slice);
    unsigned char* p = (unsigned char*)job.base + unit_of(to[k]) * job.unit_stride;
    if (job.wide) ((u32x4*)p)[e] = v[k];
    else ((uint32_t*)p)[e] = v[k][0];
  }
}

// Counts and flags (a block per layer and kv head), and the sequences' states (the last block).
constexpr int kMostPairs = 1024;
__global__ void __launch_bounds__(kForkThreads) fork_state_kernel(Dims d, const int32_t* __restrict__ pairs, int32_t n_pairs,
                                                                  int32_t planes, int32_t* seq, int32_t* pool_count,
                                                                  int32_t* aux_count, int32_t* frozen) {
  constexpr int kPer = kMostPairs / kForkThreads;
  const int plane = blockIdx.x;
  const int layer = plane / d.kv_heads, h = plane - layer * d.kv_heads;
  int4 v[kPer];
  int to[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int p = k * kForkThreads + threadIdx.x;
    to[k] = -1;
    v[k] = make_int4(0, 0, 0, 0);
    if (p >= n_pairs) continue;
    const int src = pairs[2 * p], dst = pairs[2 * p + 1];
    if (src < 0 || src >= d.batch || dst < 0 || dst >= d.batch) continue;
    const int64_t u = ((int64_t)layer * d.batch + src) * d.kv_heads + h;
    if (plane == planes) v[k] = *(const int4*)(seq + 4 * src);
    else v[k] = make_int4(pool_count[u], aux_count[u], frozen[u], 0);
    to[k] = dst;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if (to[k] < 0) continue;
    const int64_t u = ((int64_t)layer * d.batch + to[k]) * d.kv_heads + h;
    if (plane == planes) {
      *(int4*)(seq + 4 * to[k]) = v[k];
    } else {
      pool_count[u] = v[k].x;
      aux_count[u] = v[k].y;
      frozen[u] = v[k].z;
    }
  }
}

// ---- which pages are live ---------------------------------------------------------------------------------------------
// One workgroup: a bit per page in LDS (2^20 pages: 128 KB), set through the tables of all sequences, then running counts
// per 256 pages.  What bounds it is the tables' way to one compute unit.
constexpr int kScanThreads = 1024;
constexpr int kWordsPerCount = 8;

struct PageBits {
  uint32_t* bits;            // [words], a multiple of kWordsPerCount
  int32_t* before;           // [words / kWordsPerCount]: live pages before those words
  int words;
  __device__ PageBits(unsigned char* smem, int n_pages) {
    words = (n_pages + 32 * kWordsPerCount - 1) / (32 * kWordsPerCount) * kWordsPerCount;
    bits = (uint32_t*)smem;
    before = (int32_t*)(bits + words);
  }
  __device__ bool live(int page) const { return (bits[page >> 5] >> (page & 31)) & 1u; }
  __device__ int rank(int page) const {  // live pages before this one
    const int w = page >> 5;
    int r = before[w / kWordsPerCount] + __popc(bits[w] & ((1u << (page & 31)) - 1u));
    for (int i = w / kWordsPerCount * kWordsPerCount; i < w; ++i) r += __popc(bits[i]);
    return r;
  }
};
size_t page_bits_bytes(int64_t n_pages) {
  const int64_t words = (n_pages + 32 * kWordsPerCount - 1) / (32 * kWordsPerCount) * kWordsPerCount;
  return (size_t)(words * 4 + words / kWordsPerCount * 4);
}

// Live pages of the pool, in all (every thread).
__device__ __forceinline__ int mark_pages(const PageBits& P, const Dims& d, const int32_t* seq, int32_t n_quant, int tid) {
  __shared__ int s_wave[kScanThreads / 64];
  for (int i = tid; i < P.words; i += kScanThreads) P.bits[i] = 0u;
  __syncthreads();
  const int lane = tid & 63, wave = tid >> 6;
  for (int b = wave; b < d.batch; b += kScanThreads / 64) {
    const int nq = min(max(seq ? seq[4 * b] : n_quant, 0), d.max_seq) / d.G;
    const int32_t* row = d.page_table + (int64_t)b * d.table_stride;
    for (int j = lane; j < nq; j += 64) {
      const int page = row[j];
      if (page >= 0 && page < d.n_pages) atomicOr(&P.bits[page >> 5], 1u << (page & 31));
    }
  }
  __syncthreads();
  // counts per kWordsPerCount words, each thread a run of them
  const int counts = P.words / kWordsPerCount, per = (counts + kScanThreads - 1) / kScanThreads;
  const int c0 = min(tid * per, counts), c1 = min(c0 + per, counts);
  int mine = 0;
  for (int c = c0; c < c1; ++c) {
    P.before[c] = mine;
    for (int i = 0; i < kWordsPerCount; ++i) mine += __popc(P.bits[c * kWordsPerCount + i]);
  }
  const int upto = wave_scan(mine);
  if (lane == 63) s_wave[wave] = upto;
  __syncthreads();
  int earlier = upto - mine, total = 0;
  for (int w = 0; w < kScanThreads / 64; ++w) {
    if (w < wave) earlier += s_wave[w];
    total += s_wave[w];
  }
  for (int c = c0; c < c1; ++c) P.before[c] += earlier;
  __syncthreads();
  return total;
}

__global__ void __launch_bounds__(kScanThreads) free_pages_kernel(Dims d, const int32_t* __restrict__ seq, int32_t n_quant,
                                                                  int32_t* __restrict__ free_pages,
                                                                  int32_t* __restrict__ counts) {
  extern __shared__ __align__(16) unsigned char smem[];
  const PageBits P(smem, d.n_pages);
  const int tid = threadIdx.x;
  const int live = mark_pages(P, d, seq, n_quant, tid), n_free = d.n_pages - live;
  for (int page = tid; page < d.n_pages; page += kScanThreads) {
    if (!P.live(page)) free_pages[page - P.rank(page)] = page;
    if (page >= n_free) free_pages[page] = -1;
  }
  if (tid == 0) {
    counts[0] = n_free;
    counts[1] = live;
  }
}

// The packing: sources[new page] = old page, and the new table.
__global__ void __launch_bounds__(kScanThreads) pack_pages_kernel(Dims d, const int32_t* __restrict__ seq, int32_t n_quant,
                                                                  int32_t to_pages, int32_t to_stride,
                                                                  int32_t* __restrict__ to_table, int32_t* __restrict__ counts,
                                                                  int32_t* __restrict__ sources) {
  extern __shared__ __align__(16) unsigned char smem[];
  const PageBits P(smem, d.n_pages);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int live = mark_pages(P, d, seq, n_quant, tid);
  for (int page = tid; page < d.n_pages; page += kScanThreads)
    if (P.live(page)) sources[P.rank(page)] = page;
  for (int b = wave; b < d.batch; b += kScanThreads / 64) {
    const int nq = min(max(seq ? seq[4 * b] : n_quant, 0), d.max_seq) / d.G;
    for (int j = lane; j < to_stride; j += 64) {
      int page = -1;
      if (j < nq) {
        const int old = d.page_table[(int64_t)b * d.table_stride + j];
        if (old >= 0 && old < d.n_pages) page = P.rank(old);
        if (page >= to_pages) page = -1;
      }
      to_table[(int64_t)b * to_stride + j] = page;
    }
  }
  if (tid == 0) {
    counts[0] = d.n_pages - live;
    counts[1] = live;
  }
}

// ---- copies of pages -----------------------------------------------------------------------------------------------------
// A wavefront per page and plane: codes, steps and zeros and masks of one Key group, pieces of 16 bytes, four in flight per
// lane.  Bound by memory.
struct CopyArgs {
  kvq_qcache from, to;
  int32_t code_pieces, v_meta_pieces, mask_words;      // of a page of one plane
  int32_t planes;
  const int32_t* pairs;                                // {from, to}, or null: `sources`
  const int32_t* sources;                              // page sources[i] becomes page i
  const int32_t* count;                                // device: entries of `sources` (at most n are taken)
  int32_t n;
};
__global__ void __launch_bounds__(256) copy_pages_kernel(CopyArgs a) {
  const int lane = threadIdx.x & 63;
  const int n = a.pairs ? a.n : min(*a.count, a.n);
  const int64_t items = (int64_t)n * a.planes, step = (int64_t)gridDim.x * 4;
  const int v_codes0 = a.code_pieces, k_meta0 = 2 * a.code_pieces, v_meta0 = k_meta0 + 32, all = v_meta0 + a.v_meta_pieces;
  for (int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); item < items; item += step) {
    const int64_t plane = item / n;                    // (neighbouring wavefronts: neighbouring pages)
    const int i = (int)(item - plane * n);
    const int src = a.pairs ? a.pairs[2 * i] : a.sources[i], dst = a.pairs ? a.pairs[2 * i + 1] : i;
    if (src < 0 || src >= a.from.n_pages || dst < 0 || dst >= a.to.n_pages) continue;
    const int64_t pf = plane * a.from.n_pages + src, pt = plane * a.to.n_pages + dst;
    auto piece = [&](const kvq_qcache& c, int64_t page, int e) -> u32x4* {
      if (e < v_codes0) return (u32x4*)c.k_codes + page * a.code_pieces + e;
      if (e < k_meta0) return (u32x4*)c.v_codes + page * a.code_pieces + (e - v_codes0);
      if (e < v_meta0) return (u32x4*)c.k_meta + page * 32 + (e - k_meta0);
      return (u32x4*)c.v_meta + page * a.v_meta_pieces + (e - v_meta0);
    };
    for (int e0 = 0; e0 < all; e0 += 4 * 64) {
      u32x4 v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int e = e0 + 64 * k + lane;
        if (e < all) v[k] = *piece(a.from, pf, e);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int e = e0 + 64 * k + lane;
        if (e < all) *piece(a.to, pt, e) = v[k];
      }
    }
    if (lane < a.mask_words)
      ((uint32_t*)a.to.mask)[pt * a.mask_words + lane] = ((const uint32_t*)a.from.mask)[pf * a.mask_words + lane];
  }
}

hipError_t launch_copies(const Dims& d, CopyArgs& a, int32_t planes, hipStream_t s) {
  a.planes = planes;
  a.mask_words = d.G / kBlockTokens;
  a.code_pieces = a.mask_words * d.block_bytes / 16;
  a.v_meta_pieces = a.mask_words * 128 * d.vgroups / 16;
  const int64_t blocks = ((int64_t)a.n * planes + 3) / 4;
  hipLaunchKernelGGL(copy_pages_kernel, dim3((uint32_t)(blocks < (1 << 20) ? blocks : 1 << 20)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <class Kernel>
hipError_t allow_lds(Kernel kern, size_t bytes) {
  if (bytes <= 48 * 1024) return hipSuccess;
  return hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

}  // namespace

hipError_t launch_fork(const Dims& d, int32_t layers, const int32_t* pairs, int32_t n_pairs, int32_t* seq, int32_t n_quant,
                       int32_t res_start, int32_t n_res, const kvq_residual& res, const kvq_pool& pool,
                       const kvq_qcache& qc, int32_t* page_table, hipStream_t s) {
  const int32_t planes = layers * d.kv_heads;
  ForkArgs a;
  a.d = d;
  a.pairs = pairs;
  a.n_pairs = n_pairs;
  a.slice_shift = 0;
  while ((n_pairs << (a.slice_shift + 1)) <= kForkItems) ++a.slice_shift;
  const int32_t slice = 1 << a.slice_shift;
  a.seq = seq;
  a.n_quant = n_quant;
  a.res_start = res_start;
  a.n_res = n_res;
  a.pool_count = pool.pool_count;
  a.aux_count = pool.aux_count;
  a.n_jobs = 0;
  int64_t blocks = 0;
  auto job = [&](void* base, int64_t unit_stride, ForkKind kind, bool wide, int64_t elems, int32_t per_group = 0) {
    if (elems <= 0) return;
    ForkJob& j = a.job[a.n_jobs++];
    j.base = base;
    j.unit_stride = unit_stride;
    j.kind = kind;
    j.wide = wide;
    j.elems = (int32_t)elems;
    j.per_group = per_group;
    j.first_block = (uint32_t)blocks;
    j.slices = (int32_t)((elems + slice - 1) / slice);
    blocks += (int64_t)j.slices * (kind == kTable ? 1 : planes);
  };
  const int64_t row = kHeadDim * 2;
  job(res.k_res, d.res_rows * row, kRingRows, true, d.res_rows * 16);
  job(res.v_res, d.res_rows * row, kRingRows, true, d.res_rows * 16);
  if (d.N > 0) {
    job(pool.pool_k, d.pool_slots * row, kPoolRows, true, d.pool_slots * 16);
    job(pool.pool_v, d.pool_slots * row, kPoolRows, true, d.pool_slots * 16);
    job(pool.pool_idx, d.pool_slots * 4, kPoolWords, false, d.pool_slots);
    job(pool.pool_score, d.pool_slots * 8, kPoolPairs, false, d.pool_slots * 2);
  }
  // (of the groups only those are looked at that a sequence may have)
  const int64_t groups = (seq ? d.max_seq : n_quant) / d.G, per = 1 << d.bpg_shift;
  if (page_table) {
    job(page_table, (int64_t)d.table_stride * 4, kTable, false, groups);
  } else {
    const int64_t codes = per * d.block_bytes, v_meta = per * 128 * d.vgroups, all = d.max_seq / d.G;
    job(qc.k_codes, all * codes, kGroups, true, groups * codes / 16, (int32_t)(codes / 16));
    job(qc.v_codes, all * codes, kGroups, true, groups * codes / 16, (int32_t)(codes / 16));
    job(qc.k_meta, all * 512, kGroups, true, groups * 32, 32);
    job(qc.v_meta, all * v_meta, kGroups, true, groups * v_meta / 16, (int32_t)(v_meta / 16));
    job(qc.mask, all * per * 4, kGroups, false, groups * per, (int32_t)per);
  }
  if (blocks > (1 << 24) - 1) return hipErrorInvalidConfiguration;
  const auto kern = slice >= 64 ? fork_kernel<true> : fork_kernel<false>;
  hipLaunchKernelGGL(kern, dim3((uint32_t)blocks), dim3(kForkThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(fork_state_kernel, dim3(planes + (seq ? 1 : 0)), dim3(kForkThreads), 0, s, d, pairs, n_pairs, planes, seq,
                     pool.pool_count, pool.aux_count, pool.frozen);
  return hipGetLastError();
}

hipError_t launch_free_pages(const Dims& d, const int32_t* seq, int32_t n_quant, int32_t* free_pages, int32_t* counts,
                             hipStream_t s) {
  const size_t lds = page_bits_bytes(d.n_pages);
  hipError_t e = allow_lds(free_pages_kernel, lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(free_pages_kernel, dim3(1), dim3(kScanThreads), lds, s, d, seq, n_quant, free_pages, counts);
  return hipGetLastError();
}

hipError_t launch_copy_pages(const Dims& d, int32_t planes, const kvq_qcache& from, const kvq_qcache& to, const int32_t* pairs,
                             int32_t n_pairs, hipStream_t s) {
  CopyArgs a = {};
  a.from = from;
  a.to = to;
  a.pairs = pairs;
  a.n = n_pairs;
  return launch_copies(d, a, planes, s);
}

hipError_t launch_compact_pages(const Dims& d, int32_t planes, const kvq_qcache& from, const int32_t* seq, int32_t n_quant,
                                const kvq_qcache& to, int32_t* to_table, int32_t* counts, int32_t* sources, hipStream_t s) {
  const size_t lds = page_bits_bytes(d.n_pages);
  hipError_t e = allow_lds(pack_pages_kernel, lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(pack_pages_kernel, dim3(1), dim3(kScanThreads), lds, s, d, seq, n_quant, to.n_pages, to.table_stride,
                     to_table, counts, sources);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  CopyArgs a = {};
  a.from = from;
  a.to = to;
  a.sources = sources;
  a.count = counts + 1;
  a.n = from.n_pages < to.n_pages ? from.n_pages : to.n_pages;
  return launch_copies(d, a, planes, s);
}

}  // namespace kvq
