// Pages of a cache: growing, forking, cutting and freeing sequences, and the rows that are written into their pages.
//
// The bookkeeping (table, len, refs) is a few thousand integers that one call changes a few of: what bounds it is the chain of
// dependent loads and the launch (reserving 6 us, forking, cutting 3).  The rows are bound by HBM's rate for scattered 256-byte rows,
// like compaction (half of four 24K-token prompts, 268 MB: 46 us, 5.8 TB/s), where they are many; a layer's few thousand (23 MB) by
// four dependent loads (6.7 us).
#include <limits.h>

#include "pages.cuh"

namespace {

constexpr int TABLE_THREADS = 1024;
// Bytes of K and V up to which copies on write are left to the block that keeps the books: a launch costs the host 2 us and the device
// one or two (four children of a prompt of 519 tokens: a round 13.4 -> 12.5 us on the device, 22.5 -> 20.5 from the host; a unit
// at a time by the whole block it took 19).
constexpr int64_t COPY_INSIDE = 256 * 1024;
constexpr int SCRATCH_HEAD = 4;           // words: copies on write of the latest reserve, unused x 3
// scratch: head, {old page, new page, tokens, unused} of each copy [max_seqs], offsets in the list of free pages [max_seqs], that list [n_pages]

// exclusive prefix sum of one value per thread over the block; `total`: the sum.  `part`: 33 words of shared memory.
__device__ __forceinline__ int block_scan(int v, int* part, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int s = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += u;
  }
  if (lane == 31) part[warp] = s;
  __syncthreads();
  if (warp == 0) {
    int w = part[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, w, o);
      if (lane >= o) w += u;
    }
    part[lane] = w;
  }
  __syncthreads();
  total = part[31];
  const int before = s - v + (warp ? part[warp - 1] : 0);
  __syncthreads();
  return before;
}

// The tokens held of shared last pages, in all layers: a unit is (copy, layer, kv head), its rows lie together.  Units first, first
// + step ... by `threads` threads, of which this is number `me`.
__device__ __forceinline__ void copy_units(const PagePool& g, int n_layers, const int4* cow, int n, int first, int step, int me, int threads) {
  const int64_t units = (int64_t)n * n_layers * g.n_kv_heads;
  const int64_t rows = (int64_t)g.n_pages * g.n_kv_heads << g.page_shift;
  for (int64_t u = first; u < units; u += step) {
    const int h = (int)(u % g.n_kv_heads), l = (int)(u / g.n_kv_heads % n_layers);
    const int4 c = cow[u / g.n_kv_heads / n_layers];
    const int64_t from = ((int64_t)c.x * g.n_kv_heads + h) << g.page_shift, to = ((int64_t)c.y * g.n_kv_heads + h) << g.page_shift;
    const uint4* ks = reinterpret_cast<const uint4*>(g.k + (l * rows + from) * g.k_row);
    const uint4* vs = reinterpret_cast<const uint4*>(g.v + (l * rows + from) * g.v_row);
    uint4* kd = reinterpret_cast<uint4*>(g.k + (l * rows + to) * g.k_row);
    uint4* vd = reinterpret_cast<uint4*>(g.v + (l * rows + to) * g.v_row);
    const int nk = c.z * g.k_row / 16, nv = c.z * g.v_row / 16;       // at most 128 rows of 16 vectors
    for (int i0 = me; i0 < nv; i0 += 4 * threads) {
      uint4 a[4], b[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (i0 + threads * q < nk) a[q] = __ldcg(ks + i0 + threads * q);
        if (i0 + threads * q < nv) b[q] = __ldcg(vs + i0 + threads * q);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (i0 + threads * q < nk) kd[i0 + threads * q] = a[q];
        if (i0 + threads * q < nv) vd[i0 + threads * q] = b[q];
      }
    }
  }
}
__global__ void __launch_bounds__(256) pages_copy_kernel(PagePool g, int n_layers, const int32_t* scratch) {
  pdl_wait_predecessor();
  copy_units(g, n_layers, reinterpret_cast<const int4*>(scratch + SCRATCH_HEAD), *scratch, blockIdx.x, gridDim.x, threadIdx.x, 256);
}

// One block: the free pages as a bitmap in shared memory, the slots' needs and their prefix sums, then the pages.
__global__ void __launch_bounds__(TABLE_THREADS) pages_reserve_kernel(PagePool g, const int32_t* __restrict__ want, int32_t* scratch, int copy_layers) {
  extern __shared__ uint32_t bits[];       // one bit per page: free
  __shared__ int part[33];
  __shared__ int bad;
  __shared__ unsigned long long all_s;
  pdl_wait_predecessor();
  const int tid = threadIdx.x, words = (g.n_pages + 31) / 32, page = 1 << g.page_shift;
  int4* cow = reinterpret_cast<int4*>(scratch + SCRATCH_HEAD);
  int32_t* off = scratch + SCRATCH_HEAD + 4 * g.max_seqs;
  int32_t* list = off + g.max_seqs;
  if (tid == 0) { bad = 0; scratch[0] = 0; }
  // a thread makes a byte of the bitmap from eight counts
  const int bytes = words * 4;
  uint8_t* map = reinterpret_cast<uint8_t*>(bits);
  const bool vec = (reinterpret_cast<uintptr_t>(g.refs) & 15u) == 0;
#pragma unroll 4
  for (int i = tid; i < bytes; i += TABLE_THREADS) {
    uint32_t m = 0;
    if (vec && 8 * i + 8 <= g.n_pages) {
      const int4 a = __ldcg(reinterpret_cast<const int4*>(g.refs) + 2 * i), b = __ldcg(reinterpret_cast<const int4*>(g.refs) + 2 * i + 1);
      m = (a.x == 0) | (a.y == 0) << 1 | (a.z == 0) << 2 | (a.w == 0) << 3 | (b.x == 0) << 4 | (b.y == 0) << 5 | (b.z == 0) << 6 | (b.w == 0) << 7;
    } else {
      for (int q = 0; q < 8; ++q)
        if (8 * i + q < g.n_pages && __ldcg(g.refs + 8 * i + q) == 0) m |= 1u << q;
    }
    map[i] = (uint8_t)m;
  }
  __syncthreads();
  // what every slot needs; the sign of its offset says that its last page is copied
  int need_all = 0;
  for (int s0 = 0; s0 < g.max_seqs; s0 += TABLE_THREADS) {
    const int s = s0 + tid;
    int need = 0, copies = 0;
    if (s < g.max_seqs) {
      const int n = __ldcg(g.len + s), w = __ldcg(want + s);
      if (w > n) {
        if (n < 0 || w > (int64_t)g.max_pages << g.page_shift) { bad = 1; note_error(g.err, ASL_ERR_INVALID, s); }
        else {
          need = min(pages_for(w, g.page_shift) - pages_for(n, g.page_shift), (1 << 20) + 1);      // (the pool has at most 2^20)
          if (n & (page - 1)) {
            const int last = __ldcg(g.table + (int64_t)s * g.max_pages + (n >> g.page_shift));
            if ((unsigned)last >= (unsigned)g.n_pages) { bad = 1; note_error(g.err, ASL_ERR_INVALID, s); }
            else copies = __ldcg(g.refs + last) > 1;
          }
        }
      }
    }
    int sum;
    const int before = block_scan(need + copies, part, sum);
    if (s < g.max_seqs) off[s] = copies ? ~(need_all + before) : need_all + before;
    need_all += sum;                       // (at most max_seqs * max_pages pages are needed where n_pages < 2^20 exist: clamped)
    if (need_all > (1 << 21)) need_all = 1 << 21;
  }
  // free pages before a thread's words
  const int per = (words + TABLE_THREADS - 1) / TABLE_THREADS;
  int mine = 0;
  for (int i = tid * per; i < min(words, (tid + 1) * per); ++i) mine += __popc(bits[i]);
  int free_all;
  int at = block_scan(mine, part, free_all);
  if (bad) return;
  if (need_all > free_all) {               // how many are missing: counted again, where no sum is clamped
    unsigned long long need = 0;
    for (int s = tid; s < g.max_seqs; s += TABLE_THREADS) {
      const int n = __ldcg(g.len + s), w = __ldcg(want + s);
      if (w > n) need += pages_for(w, g.page_shift) - pages_for(n, g.page_shift) + (off[s] < 0);
    }
    if (tid == 0) all_s = 0;
    __syncthreads();
    if (need) atomicAdd(&all_s, need);
    __syncthreads();
    if (tid == 0) note_error(g.err, ASL_ERR_PAGES, (int)min(all_s - free_all, (unsigned long long)INT_MAX));
    return;
  }
  if (need_all == 0) {                     // growth inside the last pages
    for (int s = tid; s < g.max_seqs; s += TABLE_THREADS) {
      const int w = __ldcg(want + s);
      if (w > __ldcg(g.len + s)) g.len[s] = w;
    }
    return;
  }
  for (int i = tid * per; i < min(words, (tid + 1) * per) && at < need_all; ++i) {
    uint32_t m = bits[i];
    while (m && at < need_all) {
      list[at++] = 32 * i + __ffs(m) - 1;
      m &= m - 1;
    }
  }
  __syncthreads();
  // a warp for 32 slots; one that needs many pages has the whole warp's lanes
  for (int s0 = (tid & ~31); s0 < g.max_seqs; s0 += TABLE_THREADS) {
    const int s = s0 + (tid & 31);
    int n = 0, w = -1, o = 0;
    if (s < g.max_seqs) { n = __ldcg(g.len + s); w = __ldcg(want + s); o = off[s]; }
    const bool grows = w > n, copies = grows && o < 0;
    if (o < 0) o = ~o;
    const int first = pages_for(n, g.page_shift), fresh = grows ? pages_for(w, g.page_shift) - first : 0;
    int32_t* row = g.table + (int64_t)s * g.max_pages;
    if (grows) {
      if (copies) {
        const int old = row[n >> g.page_shift], id = list[o];
        row[n >> g.page_shift] = id;
        g.refs[id] = 1;
        atomicSub(g.refs + old, 1);
        cow[atomicAdd(scratch, 1)] = make_int4(old, id, n & (page - 1), 0);
      }
      g.len[s] = w;
    }
    unsigned left = __ballot_sync(0xffffffffu, fresh > 0);
    if (__popc(left) > 8 && !__any_sync(0xffffffffu, fresh > 4)) {
      for (int j = 0; j < fresh; ++j) {
        const int id = list[o + copies + j];
        row[first + j] = id;
        g.refs[id] = 1;
      }
    } else {
      for (; left; left &= left - 1) {
        const int src = __ffs(left) - 1;
        const int f = __shfl_sync(0xffffffffu, fresh, src), b = __shfl_sync(0xffffffffu, first, src);
        const int from = __shfl_sync(0xffffffffu, o + copies, src);
        int32_t* to = g.table + (int64_t)(s0 + src) * g.max_pages + b;
        for (int j = tid & 31; j < f; j += 32) {
          const int id = list[from + j];
          to[j] = id;
          g.refs[id] = 1;
        }
      }
    }
  }
  if (copy_layers) {                       // few copies at most: no launch of their own
    __syncthreads();
    copy_units(g, copy_layers, cow, __ldcg(scratch), tid / 128, TABLE_THREADS / 128, tid % 128, 128);
  }
}

__global__ void __launch_bounds__(128) pages_fork_kernel(PagePool g, const int32_t* __restrict__ parent) {
  pdl_wait_predecessor();
  const int s = blockIdx.x, p = __ldcg(parent + s);
  if (p < 0) return;
  const bool fits = p < g.max_seqs && p != s && __ldcg(parent + p) < 0;
  const int n = fits ? __ldcg(g.len + p) : -1, m = pages_for(n, g.page_shift);
  if (n < 0 || m > g.max_pages || __ldcg(g.len + s) != 0) {
    if (threadIdx.x == 0) note_error(g.err, ASL_ERR_INVALID, s);
    return;
  }
  const int32_t* from = g.table + (int64_t)p * g.max_pages;
  int32_t* to = g.table + (int64_t)s * g.max_pages;
  for (int j = threadIdx.x; j < m; j += 128) {
    const int id = __ldcg(from + j);
    to[j] = id;
    if ((unsigned)id < (unsigned)g.n_pages) atomicAdd(g.refs + id, 1);
  }
  __syncthreads();                          // every thread has seen that the slot was free
  if (threadIdx.x == 0) g.len[s] = n;
}

__global__ void __launch_bounds__(128) pages_trim_kernel(PagePool g, const int32_t* __restrict__ to) {
  pdl_wait_predecessor();
  const int s = blockIdx.x, t = __ldcg(to + s), n = __ldcg(g.len + s);
  if (t < 0 || t >= n) return;
  const int32_t* row = g.table + (int64_t)s * g.max_pages;
  const int end = min(pages_for(n, g.page_shift), g.max_pages);
  for (int j = pages_for(t, g.page_shift) + threadIdx.x; j < end; j += 128) {
    const int id = __ldcg(row + j);
    if ((unsigned)id < (unsigned)g.n_pages) atomicSub(g.refs + id, 1);
  }
  __syncthreads();
  if (threadIdx.x == 0) g.len[s] = t;
}

// Where row `pos` of a slot lies, in rows of its kv head's pool; -1 where it may not be written.
__device__ __forceinline__ int place_of(const PagePool& g, int slot, int pos, int h, bool& wrong) {
  const int id = __ldcg(g.table + (int64_t)slot * g.max_pages + (pos >> g.page_shift));
  if ((unsigned)id >= (unsigned)g.n_pages || __ldcg(g.refs + id) != 1) { wrong = true; return -1; }
  return ((id * g.n_kv_heads + h) << g.page_shift) + (pos & ((1 << g.page_shift) - 1));
}

struct RowSource {
  const uint8_t* k;        // a prefill's K and V (asl_pages_store), else null: the cache's own
  const uint8_t* v;
  int64_t ks_t, ks_h, vs_t, vs_h;          // strides in bytes
  const AslReq* req;
  const asl_stat* latch;
  int cur_layer;
  const int32_t* src;      // asl_pages_compact
  const int32_t* off;
};

// Kept rows into pages.  A block takes R rows of one kv head: first a thread a row finds where it comes from and goes to (three
// dependent loads: list, table, count or table), then 16 threads move a row's 16-byte vectors, four rows' K and V in flight each
// (as compact_kv_kernel).  Found by all 16 threads of a row and 64 rows a block, half of four 24K-token prompts (268 MB
// moved) took 57 us.
template <bool CACHED, int R>
__global__ void __launch_bounds__(256) rows_to_pages_kernel(PagePool g, RowSource x, const int32_t* __restrict__ idx,
                                                            const int32_t* __restrict__ dst, int64_t sum_kept) {
  __shared__ int from_s[R], to_s[R];
  pdl_wait_predecessor();
  const int b = blockIdx.z, h = blockIdx.y, tid = threadIdx.x;
  const int slot = __ldcg(dst + b), jobs = gridDim.z;
  int kept, src = 0, n_src;
  int64_t at, tok_off = 0;
  if (CACHED) {
    src = __ldcg(x.src + b);
    const int o = __ldcg(x.off + b);
    const int end = __ldcg(x.off + b + 1);
    at = o;
    const bool listed = o >= 0 && o <= end && end <= sum_kept;
    kept = listed ? end - o : 0;
    const bool fits = (unsigned)src < (unsigned)g.max_seqs && src != slot;
    n_src = fits ? min(__ldcg(g.len + src), g.max_pages << g.page_shift) : 0;
    if (blockIdx.x == 0 && h == 0 && tid == 0 && (!listed || kept > (int64_t)gridDim.x * R)) note_error(g.err, ASL_ERR_INVALID, slot);     // or more than max_kept
  } else {
    if (x.latch && asl_finished(x.latch + b, x.cur_layer)) return;
    const AslReq rq = x.req[b];
    kept = rq.kept; at = rq.kept_off; n_src = rq.n; tok_off = rq.tok_off;
  }
  const int r0 = blockIdx.x * R;
  if (r0 >= kept) return;
  if ((unsigned)slot >= (unsigned)g.max_seqs) {
    if (tid == 0) note_error(g.err, ASL_ERR_INVALID, slot);
    return;
  }
  if (tid < R) {
    const int r = r0 + tid;
    int from = -1, to = -1;
    if (r < kept) {
      bool wrong = false;
      const int tok = __ldcg(idx + (int64_t)h * sum_kept + at + r);
      const int n_dst = min(__ldcg(g.len + slot), g.max_pages << g.page_shift);
      if (r >= n_dst || (unsigned)tok >= (unsigned)n_src) {
        wrong = true;
      } else {
        from = tok;
        if (CACHED) {
          const int id = __ldcg(g.table + (int64_t)src * g.max_pages + (tok >> g.page_shift));
          if ((unsigned)id >= (unsigned)g.n_pages) wrong = true;
          from = ((id * g.n_kv_heads + h) << g.page_shift) + (tok & ((1 << g.page_shift) - 1));
        }
        to = place_of(g, slot, r, h, wrong);
        if (wrong) to = -1;
      }
      if (wrong) note_error(g.err, ASL_ERR_INVALID, slot);
    }
    from_s[tid] = from;
    to_s[tid] = to;
  }
  // Jobs run side by side, so that a slot which another job with rows reads or writes cannot be written.  (The last threads look
  // first: where rows are few they have nothing else to do.)
  bool clash = false;
  for (int j = 255 - tid; j < jobs; j += 256)
    if ((j != b && __ldcg(dst + j) == slot) || (CACHED && __ldcg(x.src + j) == slot)) clash |= !CACHED || __ldcg(x.off + j + 1) > __ldcg(x.off + j);
  if (__syncthreads_or(clash)) {
    if (tid == 0) note_error(g.err, ASL_ERR_INVALID, slot);
    return;
  }
  const int c = tid % 16, k_vec = g.k_row / 16;
  const uint8_t* ks = CACHED ? g.k : x.k + tok_off * x.ks_t + (int64_t)h * x.ks_h;
  const uint8_t* vs = CACHED ? g.v : x.v + tok_off * x.vs_t + (int64_t)h * x.vs_h;
  const int64_t ks_t = CACHED ? g.k_row : x.ks_t, vs_t = CACHED ? g.v_row : x.vs_t;
#pragma unroll
  for (int q0 = 0; q0 < R; q0 += 64) {
    uint4 kv[4], vv[4];
    int to[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = q0 + 16 * i + tid / 16, from = from_s[r];
      to[i] = to_s[r];
      if (to[i] >= 0 && c < k_vec) kv[i] = __ldcs(reinterpret_cast<const uint4*>(ks + from * ks_t) + c);
      if (to[i] >= 0) vv[i] = __ldcs(reinterpret_cast<const uint4*>(vs + from * vs_t) + c);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (to[i] >= 0 && c < k_vec) __stcs(reinterpret_cast<uint4*>(g.k + (int64_t)to[i] * g.k_row) + c, kv[i]);
      if (to[i] >= 0) __stcs(reinterpret_cast<uint4*>(g.v + (int64_t)to[i] * g.v_row) + c, vv[i]);
    }
  }
}

// 256 rows a block where that still makes a few blocks for every SM, else 64.
template <bool CACHED>
void launch_rows(const asl_ctx* c, const PagePool& g, const RowSource& x, const int32_t* idx, const int32_t* dst, int64_t sum_kept,
                 int max_kept, int jobs, cudaStream_t st) {
  const int64_t most = max_kept < 1 || sum_kept < 1 ? 1 : max_kept < sum_kept ? max_kept : sum_kept;        // of one list
  auto columns = [&](int rows) { return dim3((unsigned)((most + rows - 1) / rows), g.n_kv_heads, jobs); };
  if (sum_kept * g.n_kv_heads >= (int64_t)c->sm_count * 4 * 256)
    launch_after(rows_to_pages_kernel<CACHED, 256>, columns(256), dim3(256), st, g, x, idx, dst, sum_kept);
  else
    launch_after(rows_to_pages_kernel<CACHED, 64>, columns(64), dim3(256), st, g, x, idx, dst, sum_kept);
}

// A step's rows at the ends of their sequences: a block column per sequence, 16 threads a (token, kv head) row.
__global__ void __launch_bounds__(128) pages_append_kernel(PagePool g, asl_batch b, const uint8_t* __restrict__ k,
                                                           const uint8_t* __restrict__ v, int64_t ks_t, int64_t ks_h,
                                                           int64_t vs_t, int64_t vs_h) {
  pdl_wait_predecessor();
  const int s = blockIdx.y, slot = __ldcg(b.slots + s);
  if ((unsigned)slot >= (unsigned)g.max_seqs) return;                  // padding
  const int t0 = __ldcg(b.cu_q + s), t1 = __ldcg(b.cu_q + s + 1), len = __ldcg(g.len + slot);
  const int c = threadIdx.x % 16;
  if (t0 < 0 || t1 > b.n_tokens) {
    if (threadIdx.x == 0) note_error(g.err, ASL_ERR_INVALID, slot);
    return;
  }
  const int64_t rows = (int64_t)max(t1 - t0, 0) * g.n_kv_heads;
  for (int64_t r = blockIdx.x * 8 + threadIdx.x / 16; r < rows; r += (int64_t)gridDim.x * 8) {
    const int t = (int)(r / g.n_kv_heads), h = (int)(r % g.n_kv_heads);
    const int pos = len - (t1 - t0) + t;
    bool wrong = pos < 0 || pos >> g.page_shift >= g.max_pages;
    const uint8_t* kr = k + (int64_t)(t0 + t) * ks_t + (int64_t)h * ks_h;
    const uint8_t* vr = v + (int64_t)(t0 + t) * vs_t + (int64_t)h * vs_h;
    uint4 kv = make_uint4(0, 0, 0, 0);
    if (c * 16 < g.k_row) kv = __ldcg(reinterpret_cast<const uint4*>(kr) + c);
    const uint4 vv = __ldcg(reinterpret_cast<const uint4*>(vr) + c);
    const int64_t to = wrong ? -1 : (int64_t)place_of(g, slot, pos, h, wrong);
    if (to >= 0) {
      if (c * 16 < g.k_row) reinterpret_cast<uint4*>(g.k + to * g.k_row)[c] = kv;
      reinterpret_cast<uint4*>(g.v + to * g.v_row)[c] = vv;
    }
    if (wrong) note_error(g.err, ASL_ERR_INVALID, slot);
  }
}

size_t scratch_bytes_of(const asl_pages* p) {
  return sizeof(int32_t) * (SCRATCH_HEAD + 5 * (size_t)p->max_seqs + (size_t)p->n_pages);
}

asl_status launched(asl_ctx* c, int n) {
  ASL_CUDA(cudaGetLastError());
  c->launches += n;
  return ASL_OK;
}

// what all calls look at
asl_status check_call(const asl_ctx* c, const asl_pages* p, int32_t layer) {
  if (!c || !asl_on_device(c)) return ASL_ERR_INVALID;
  const asl_status s = asl_check_pages(p);
  if (s != ASL_OK) return s;
  return layer < 0 || layer >= p->n_layers ? ASL_ERR_INVALID : ASL_OK;
}

struct StoreStep { const asl_pages* pages; int32_t layer; const int32_t* slots; };
asl_status store_step(asl_ctx* c, const asl_layer* l, const void* k, const void* v, const void* arg) {
  const StoreStep* s = static_cast<const StoreStep*>(arg);
  return asl_pages_store(c, s->pages, s->layer, k, v, l->idx, s->slots, l->side2);
}

}  // namespace

asl_status asl_check_pages(const asl_pages* p) {
  if (!p || !p->k || !p->v || !p->table || !p->len || !p->refs || !p->err) return ASL_ERR_INVALID;
  if (p->n_layers < 1 || p->n_kv_heads < 1 || p->n_pages < 1 || p->max_seqs < 1 || p->max_pages < 1) return ASL_ERR_INVALID;
  if (p->page_size != 16 && p->page_size != 32 && p->page_size != 64 && p->page_size != 128) return ASL_ERR_INVALID;
  if (p->k_dtype != ASL_K_BF16 && p->k_dtype != ASL_K_FP8_E4M3) return ASL_ERR_INVALID;
  if (p->k_dtype == ASL_K_FP8_E4M3 && !p->k_scale) return ASL_ERR_INVALID;
  if (!asl_aligned16(p->k) || !asl_aligned16(p->v)) return ASL_ERR_INVALID;
  if (p->head_dim < 8 || p->head_dim % 8) return ASL_ERR_INVALID;
  if (p->head_dim != 128 || p->n_pages > 1 << 20 || p->max_seqs > 65536 || p->n_kv_heads > 65535 || p->n_layers > 65535) return ASL_ERR_UNSUPPORTED;
  if ((int64_t)p->n_pages * p->n_kv_heads * p->page_size >= (int64_t)1 << 31) return ASL_ERR_UNSUPPORTED;
  if ((int64_t)p->max_pages * p->page_size >= (int64_t)1 << 31) return ASL_ERR_UNSUPPORTED;
  return ASL_OK;
}

extern "C" {

asl_status asl_pages_scratch(const asl_pages* p, size_t* bytes) {
  if (!bytes) return ASL_ERR_INVALID;
  const asl_status s = asl_check_pages(p);
  if (s == ASL_OK) *bytes = scratch_bytes_of(p);
  return s;
}

asl_status asl_pages_reserve(asl_ctx* c, const asl_pages* p, const int32_t* want, void* stream) {
  const asl_status s = check_call(c, p, 0);
  if (s != ASL_OK) return s;
  if (!want) return ASL_ERR_INVALID;
  if (!p->scratch || p->scratch_bytes < scratch_bytes_of(p) || !asl_aligned16(p->scratch)) return ASL_ERR_WORKSPACE;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const size_t smem = ((size_t)p->n_pages + 31) / 32 * 4;
  if (!c->reserve_ready) {                 // (whatever the pool: the 48 KB that need no leave hold the kernel's own arrays too)
    ASL_CUDA(cudaFuncSetAttribute(pages_reserve_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 1 << 17));
    c->reserve_ready = true;
  }
  const int64_t most = (int64_t)p->max_seqs * p->n_layers * p->n_kv_heads * p->page_size * p->head_dim * 4;      // bytes copied at most
  const bool inside = most <= COPY_INSIDE;
  launch_after_smem(pages_reserve_kernel, dim3(1), dim3(TABLE_THREADS), smem, st, page_pool(p, 0), want, p->scratch, inside ? p->n_layers : 0);
  const asl_status r = launched(c, 1);           // (without the books there is no list of copies)
  if (r != ASL_OK || inside) return r;
  launch_after(pages_copy_kernel, dim3(c->sm_count * 8), dim3(256), st, page_pool(p, 0), p->n_layers, static_cast<const int32_t*>(p->scratch));
  return launched(c, 1);
}

asl_status asl_pages_fork(asl_ctx* c, const asl_pages* p, const int32_t* parent, void* stream) {
  const asl_status s = check_call(c, p, 0);
  if (s != ASL_OK) return s;
  if (!parent) return ASL_ERR_INVALID;
  launch_after(pages_fork_kernel, dim3(p->max_seqs), dim3(128), static_cast<cudaStream_t>(stream), page_pool(p, 0), parent);
  return launched(c, 1);
}

asl_status asl_pages_trim(asl_ctx* c, const asl_pages* p, const int32_t* to, void* stream) {
  const asl_status s = check_call(c, p, 0);
  if (s != ASL_OK) return s;
  if (!to) return ASL_ERR_INVALID;
  launch_after(pages_trim_kernel, dim3(p->max_seqs), dim3(128), static_cast<cudaStream_t>(stream), page_pool(p, 0), to);
  return launched(c, 1);
}

asl_status asl_pages_store(asl_ctx* c, const asl_pages* p, int32_t layer, const void* k, const void* v, const int32_t* idx,
                           const int32_t* slots, void* stream) {
  const asl_status s = check_call(c, p, layer);
  if (s != ASL_OK) return s;
  if (!c->planned || !k || !v || !idx || !slots || !asl_aligned16(k) || !asl_aligned16(v)) return ASL_ERR_INVALID;
  const asl_params& q = c->p;
  if (p->n_kv_heads != q.n_kv_heads || p->head_dim != q.head_dim || p->k_dtype != q.k_dtype) return ASL_ERR_INVALID;
  RowSource x = {};
  x.k = static_cast<const uint8_t*>(k);
  x.v = static_cast<const uint8_t*>(v);
  x.ks_t = q.k_stride[0] * c->k_elem_bytes;
  x.ks_h = q.k_stride[1] * c->k_elem_bytes;
  x.vs_t = q.v_stride[0] * 2;
  x.vs_h = q.v_stride[1] * 2;
  x.req = c->d_req;
  x.latch = c->latch_stat;
  x.cur_layer = c->cur_layer;
  launch_rows<false>(c, page_pool(p, layer), x, idx, slots, c->sum_kept, c->max_kept, q.batch, static_cast<cudaStream_t>(stream));
  return launched(c, 1);
}

asl_status asl_pages_compact(asl_ctx* c, const asl_pages* p, int32_t layer, const int32_t* src, const int32_t* dst,
                             const int32_t* off, int32_t n_jobs, const int32_t* idx, int64_t sum_kept, int32_t max_kept,
                             void* stream) {
  const asl_status s = check_call(c, p, layer);
  if (s != ASL_OK) return s;
  if (!src || !dst || !off || (sum_kept != 0 && !idx) || n_jobs < 1 || n_jobs > 65535 || sum_kept < 0 || max_kept < 0) return ASL_ERR_INVALID;
  RowSource x = {};
  x.src = src;
  x.off = off;
  launch_rows<true>(c, page_pool(p, layer), x, idx, dst, sum_kept, max_kept, n_jobs, static_cast<cudaStream_t>(stream));
  return launched(c, 1);
}

asl_status asl_pages_append(asl_ctx* c, const asl_pages* p, int32_t layer, const asl_batch* b, const void* k_new, const void* v_new,
                            const int64_t k_stride[2], const int64_t v_stride[2], void* stream) {
  const asl_status s = check_call(c, p, layer);
  if (s != ASL_OK) return s;
  if (!b || !b->slots || !b->cu_q || !k_stride || !v_stride) return ASL_ERR_INVALID;
  if (b->n_tokens != 0 && (!k_new || !v_new)) return ASL_ERR_INVALID;             // (what is empty has no address)
  if (b->n_seqs < 1 || b->n_tokens < 0 || !asl_aligned16(k_new) || !asl_aligned16(v_new)) return ASL_ERR_INVALID;
  if (b->n_seqs > 4096) return ASL_ERR_UNSUPPORTED;
  const int kb = p->k_dtype == ASL_K_FP8_E4M3 ? 1 : 2;
  for (int i = 0; i < 2; ++i)
    if (k_stride[i] < 0 || v_stride[i] < 0 || k_stride[i] * kb % 16 || v_stride[i] * 2 % 16) return ASL_ERR_INVALID;
  if (b->n_tokens == 0) return ASL_OK;
  // one block a sequence covers a token's heads; where tokens are many (on average) more of them share a sequence
  const int64_t rows = (int64_t)(b->n_tokens + b->n_seqs - 1) / b->n_seqs * p->n_kv_heads;
  const int blocks = (int)(rows > 64 * 8 ? 64 : (rows + 7) / 8);
  launch_after(pages_append_kernel, dim3(blocks, b->n_seqs), dim3(128), static_cast<cudaStream_t>(stream), page_pool(p, layer), *b,
               static_cast<const uint8_t*>(k_new), static_cast<const uint8_t*>(v_new), k_stride[0] * kb, k_stride[1] * kb,
               v_stride[0] * 2, v_stride[1] * 2);
  return launched(c, 1);
}

asl_status asl_run_layer_pages(asl_ctx* c, const asl_layer* l, const asl_pages* p, int32_t page_layer, const int32_t* slots,
                               const void* q_obs, const void* k, const void* v, const float* lse, int32_t layer_idx,
                               int32_t n_rows, int32_t slot) {
  if (!slots) return ASL_ERR_INVALID;
  const asl_status s = check_call(c, p, page_layer);
  if (s != ASL_OK) return s;
  const StoreStep step = {p, page_layer, slots};
  return asl_run_layer_last(c, l, q_obs, k, v, lse, layer_idx, n_rows, slot, store_step, &step);
}

asl_status asl_pages_status(asl_ctx* c, const asl_pages* p, void* stream, int32_t* info) {
  if (!c || !p || !p->err) return ASL_ERR_INVALID;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  int32_t word[2] = {0, 0};
  ASL_CUDA(cudaMemcpyAsync(word, p->err, sizeof(word), cudaMemcpyDeviceToHost, st));
  ASL_CUDA(cudaStreamSynchronize(st));
  if (info) *info = word[1];
  if (word[0] == 0) return ASL_OK;
  ASL_CUDA(cudaMemsetAsync(p->err, 0, sizeof(word), st));
  return static_cast<asl_status>(word[0]);
}

}  // extern "C"
