// Attention over pages: the plan, the rows whose parts are put together, and the entry points.
#include <math.h>

#include "asl_ptx.cuh"
#include "attend.cuh"

namespace {

constexpr int PLAN_THREADS = 512;
constexpr int NARROW_CTAS = 2;             // per SM
// Least bytes of K and V that the groups' prefixes save (each its length times all its readers but one) for them to be read by
// groups: below, one more kernel and one more part per row cost more than the copies out of L2.
constexpr float SHARE_MIN_BYTES = 32e6f;
constexpr int64_t SAME_INSIDE = 16384;     // entries of the batch's rows of the table that the plan's own block compares

// Leading pages that an entry of the batch has in common with the one before it; only pages that both hold in full.
constexpr int SAME_THREADS = 256, SAME_EACH = 8;
__global__ void __launch_bounds__(SAME_THREADS) attend_same_kernel(PagePool g, asl_batch b, int32_t* same) {
  __shared__ int first[SAME_THREADS / 32];
  pdl_wait_predecessor();
  const int i = blockIdx.x, tid = threadIdx.x;
  int m = 0;
  if (i > 0) {
    const int s = __ldcg(b.slots + i), r = __ldcg(b.slots + i - 1);
    if ((unsigned)s < (unsigned)g.max_seqs && (unsigned)r < (unsigned)g.max_seqs)
      m = max(0, min(min(__ldcg(g.len + s), __ldcg(g.len + r)) >> g.page_shift, g.max_pages));
    const int32_t* x = g.table + (int64_t)s * g.max_pages;
    const int32_t* y = g.table + (int64_t)r * g.max_pages;
    for (int j0 = 0; j0 < m; j0 += SAME_THREADS * SAME_EACH) {
      int u[SAME_EACH], v[SAME_EACH], at = m;
#pragma unroll
      for (int q = 0; q < SAME_EACH; ++q) {
        const int j = j0 + q * SAME_THREADS + tid;
        u[q] = j < m ? __ldcg(x + j) : 0;
        v[q] = j < m ? __ldcg(y + j) : 0;
      }
#pragma unroll
      for (int q = SAME_EACH - 1; q >= 0; --q)
        if (u[q] != v[q]) at = j0 + q * SAME_THREADS + tid;
      at = __reduce_min_sync(0xffffffffu, at);
      if ((tid & 31) == 0) first[tid >> 5] = at;
      __syncthreads();
#pragma unroll
      for (int q = 0; q < SAME_THREADS / 32; ++q) m = min(m, first[q]);
      __syncthreads();
    }
  }
  if (tid == 0) same[i] = m;
}

// exclusive prefix sums of two values per thread over the block; x and y: the sums.  `part`: [2][warps] of shared memory.
__device__ __forceinline__ int2 scan_step(int2 v, int2* part, int2& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int2 s = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, s.x, o), y = __shfl_up_sync(0xffffffffu, s.y, o);
    if (lane >= o) { s.x += x; s.y += y; }
  }
  if (lane == 31) part[warp] = s;
  __syncthreads();
  int2 before = {0, 0};
  total = {0, 0};
#pragma unroll
  for (int k = 0; k < PLAN_THREADS / 32; ++k) {
    const int2 p = part[k];
    if (k < warp) { before.x += p.x; before.y += p.y; }
    total.x += p.x;
    total.y += p.y;
  }
  __syncthreads();
  return {before.x + s.x - v.x, before.y + s.y - v.y};
}

struct PlanArgs {
  PagePool g;
  asl_batch b;
  AttendPtrs w;
  int32_t G, n_q_heads, narrow_grid, wide_grid;
  float min_bytes;         // that groups' prefixes have to save
  int32_t share;           // 0: nothing is; what neighbours have in common comes from 1: attend_same_kernel, 2: the plan itself
};

// One block: groups of neighbours, prefix sums over sequences and groups, and where every CTA's stretch begins.  All of it in
// shared memory: what bounds it is the chain of its steps (two loads, the groups' walk entry by entry, three prefix sums).
__global__ void __launch_bounds__(PLAN_THREADS) attend_plan_kernel(PlanArgs a) {
  extern __shared__ int32_t sm[];
  __shared__ int2 part[PLAN_THREADS / 32];
  __shared__ int n_groups_s, any_full, bad;
  __shared__ unsigned long long most_s;
  pdl_wait_predecessor();
  const int tid = threadIdx.x, n = a.b.n_seqs, G = a.G, H = a.g.n_kv_heads;
  int32_t* ntok = sm;                      // per entry
  int32_t* len = sm + n;
  int32_t* slot = sm + 2 * n;
  int32_t* tok0 = sm + 3 * n;
  int32_t* grp = sm + 4 * n;
  int32_t* com = sm + 5 * n;               // shared tokens with the entry before; then narrow chunks before
  int32_t* gpfx = sm + 6 * n;              // per group: shared tokens, first entry, tokens, chunks of stripes before
  int32_t* gat = sm + 7 * n;
  int32_t* gtok = sm + 8 * n;
  int32_t* gchunk = sm + 9 * n;
  int32_t* first = sm + 10 * n;            // [n + 1] narrow tiles before
  int32_t* gcost = sm + 11 * n + 1;        // [n + 1] wide cost before
  if (tid == 0) { a.w.head->mark = 0; *a.w.open = 0; most_s = 0; any_full = 0; bad = 0; }
  for (int t = tid; t < a.b.n_tokens; t += PLAN_THREADS) a.w.tokens[t].seq.ntok = 0;
  __syncthreads();
  unsigned long long most = 0;             // tiles, were nothing shared: they are counted in 32 bits
  for (int i = tid; i < n; i += PLAN_THREADS) {
    const int s = __ldcg(a.b.slots + i), t0 = __ldcg(a.b.cu_q + i), t1 = __ldcg(a.b.cu_q + i + 1);
    const int same = a.share == 1 ? __ldcg(a.w.same + i) : 0;
    const bool slot_ok = (unsigned)s < (unsigned)a.g.max_seqs, tok_ok = t0 >= 0 && t1 >= t0 && t1 <= a.b.n_tokens;
    const int l = slot_ok ? __ldcg(a.g.len + s) : 0;
    if (!tok_ok) bad = 1;                  // (tokens that two entries own would be more rows than the workspace has room for)
    const int m = slot_ok && tok_ok ? t1 - t0 : 0;
    ntok[i] = m;
    slot[i] = m ? s : -1;
    tok0[i] = t0;
    len[i] = m ? min(max(l, 0), a.g.max_pages << a.g.page_shift) : 0;
    com[i] = same << a.g.page_shift;
    if (m) most += (unsigned long long)narrow_chunks_of(m, G) * (unsigned)(len[i] / NARROW_KEYS + 2);
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) most += __shfl_xor_sync(0xffffffffu, most, o);
  if ((tid & 31) == 0 && most) atomicAdd(&most_s, most);
  __syncthreads();
  if (bad || most_s * H >= 1ull << 30) {
    if (tid == 0) note_error(a.g.err, bad ? ASL_ERR_INVALID : ASL_ERR_UNSUPPORTED, -1);
    return;
  }
  if (a.share == 2) {                      // few pages: no launch of its own for what neighbours have in common, a warp a pair
    for (int i = 1 + (tid >> 5); i < n; i += PLAN_THREADS / 32) {
      int m = min(len[i], len[i - 1]) >> a.g.page_shift;
      const int32_t* x = a.g.table + (int64_t)slot[i] * a.g.max_pages;
      const int32_t* y = a.g.table + (int64_t)slot[i - 1] * a.g.max_pages;
      for (int j0 = 0; j0 < m; j0 += 128) {
        int u[4], v[4], at = m;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int j = j0 + q * 32 + (tid & 31);
          u[q] = j < m ? __ldcg(x + j) : 0;
          v[q] = j < m ? __ldcg(y + j) : 0;
        }
#pragma unroll
        for (int q = 3; q >= 0; --q)
          if (u[q] != v[q]) at = j0 + q * 32 + (tid & 31);
        m = min(m, __reduce_min_sync(0xffffffffu, at));
      }
      if ((tid & 31) == 0) com[i] = max(m, 0) << a.g.page_shift;
    }
    __syncthreads();
  }
  // Groups: an entry joins the group before it where that group then saves no less than without it.
  int32_t* own = gtok;                     // tokens that all of an entry's see
  for (int i = tid; i < n; i += PLAN_THREADS) {
    own[i] = max(0, len[i] - ntok[i]) >> a.g.page_shift << a.g.page_shift;
    com[i] = min(own[i], com[i]);
  }
  __syncthreads();
  if (tid == 0) {
    int ng = 0, held = 0, keys = 0;                          // of the open group: entries (0: none is open), shared tokens
    int64_t saved = 0;                                       // keys read less often, by all groups so far
    int has = ntok[0], mine = own[0], with = com[0];
    for (int i = 0; i < n; ++i) {
      const int j = min(i + 1, n - 1), has2 = ntok[j], mine2 = own[j], with2 = com[j];       // (ahead of this entry's stores)
      const int both = min(keys, with);
      const int64_t before = (int64_t)(held - 1) * keys;     // saved by the open group
      const bool joins = has && held && both > 0 && (int64_t)held * both >= before;
      if (!joins && held) {
        gpfx[ng - 1] = held > 1 ? keys : 0;
        saved += before;
      }
      if (!joins && has) gat[ng++] = i;
      held = has ? (joins ? held + 1 : 1) : 0;
      keys = joins ? both : mine;
      grp[i] = has ? ng - 1 : -1;
      has = has2; mine = mine2; with = with2;
    }
    if (held) {
      gpfx[ng - 1] = held > 1 ? keys : 0;
      saved += (int64_t)(held - 1) * keys;
    }
    if ((float)saved * H * (a.g.k_row + a.g.v_row) < a.min_bytes)
      for (int g = 0; g < ng; ++g) gpfx[g] = 0;
    n_groups_s = ng;
  }
  __syncthreads();
  const int ng = n_groups_s;
  int tiles = 0, chunks = 0;
  for (int i0 = 0; i0 < n; i0 += PLAN_THREADS) {
    const int i = i0 + tid;
    int nt = 0, nc = 0, pfx = 0;
    if (i < n && ntok[i]) {
      pfx = gpfx[grp[i]];
      nc = narrow_chunks_of(ntok[i], G);
      nt = nc * max(1, (len[i] - pfx + NARROW_KEYS - 1) / NARROW_KEYS);
    }
    int2 sum;
    const int2 at = scan_step({nt, nc}, part, sum);
    const int t0 = tiles + at.x, c0 = chunks + at.y;
    if (i < n) {
      first[i] = t0;
      com[i] = c0;
      a.w.seqs[i] = {tok0[i], ntok[i], slot[i], len[i], pfx, t0, c0, grp[i]};
    }
    tiles += sum.x;
    chunks += sum.y;
  }
  // groups: their cost, from it what a CTA has of it and the stripes, then the chunks of stripes
  int cost = 0, wchunks = 0;
  for (int i0 = 0; i0 < ng; i0 += PLAN_THREADS) {
    const int i = i0 + tid;
    int c = 0;
    if (i < ng) {
      const int at = gat[i];
      int last = i + 1 < ng ? gat[i + 1] : n;
      while (last > at + 1 && grp[last - 1] != i) --last;         // padding behind the group
      gtok[i] = tok0[last - 1] + ntok[last - 1] - tok0[at];
      const WideShape w(gtok[i], gpfx[i], G, 1);
      c = w.tiles * w.sum;
      if (gpfx[i] && gtok[i] * G > WIDE_ROWS / 2) any_full = 1;
    }
    int2 sum;
    const int c0 = cost + scan_step({c, 0}, part, sum).x;
    if (i < ng) gcost[i] = c0;
    cost += sum.x;
  }
  if (tid == 0) { first[n] = tiles; gcost[ng] = cost; }
  __syncthreads();
  const int narrow_each = max(1, (H * tiles + a.narrow_grid - 1) / a.narrow_grid);
  // (a stretch has to hold the beginning of a tile, whose cost is 2 in chunks of more than 128 rows)
  const int wide_each = max(any_full ? 2 : 1, (H * cost + a.wide_grid - 1) / a.wide_grid);
  const int stripe = (wide_each + 1) / 2;
  auto group_of = [&](int i) { return AttendGroup{tok0[gat[i]], gtok[i], slot[gat[i]], gpfx[i], gcost[i], gchunk[i], stripe, 0}; };
  if (cost) {
    for (int i0 = 0; i0 < ng; i0 += PLAN_THREADS) {
      const int i = i0 + tid;
      int nc = 0;
      if (i < ng && gpfx[i]) {
        const WideShape w(gtok[i], gpfx[i], G, stripe);
        nc = w.chunks * w.stripes;
      }
      int2 sum;
      const int n0 = wchunks + scan_step({nc, 0}, part, sum).x;
      if (i < ng) {
        gchunk[i] = n0;
        a.w.groups[i] = group_of(i);
      }
      wchunks += sum.x;
    }
  }
  __syncthreads();
  for (int i = tid; i < n; i += PLAN_THREADS) {
    if (!ntok[i]) continue;
    const int pfx = gpfx[grp[i]];
    AttendToken r = {};
    r.seq = {tok0[i], ntok[i], slot[i], len[i], pfx, first[i], com[i], grp[i]};
    if (pfx) r.group = group_of(grp[i]);
    for (int t = 0; t < ntok[i]; ++t) a.w.tokens[tok0[i] + t] = r;
  }
  for (int k = tid; k < a.narrow_grid; k += PLAN_THREADS) {
    AttendStart s = {};
    s.h = -1;
    s.items = n; s.total = tiles; s.chunks = chunks; s.more = narrow_each;
    const int64_t u = (int64_t)k * narrow_each;
    if (u < H * tiles) {
      s.h = (int)u / tiles;
      const int r = (int)u - s.h * tiles;
      int lo = 0, hi = n;                                       // last entry with first <= r that has tiles
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (first[mid] <= r) lo = mid; else hi = mid;
      }
      s.item = lo;
      const int pfx = gpfx[grp[lo]], nt = max(1, (len[lo] - pfx + NARROW_KEYS - 1) / NARROW_KEYS);
      s.chunk = (r - first[lo]) / nt;
      s.tile = r - first[lo] - s.chunk * nt;
      s.seq = {tok0[lo], ntok[lo], slot[lo], len[lo], pfx, first[lo], com[lo], grp[lo]};
    }
    a.w.narrow_start[k] = s;
  }
  for (int k = tid; k < a.wide_grid; k += PLAN_THREADS) {
    AttendStart s = {};
    s.h = -1;
    s.items = ng; s.total = cost; s.chunks = wchunks;
    const int64_t u = (int64_t)k * wide_each;
    if (u < H * cost) {
      s.h = (int)u / cost;
      const int r = (int)u - s.h * cost;
      int lo = 0, hi = ng;
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (gcost[mid] <= r) lo = mid; else hi = mid;
      }
      s.item = lo;
      s.group = group_of(lo);
      const WideShape w(s.group.ntok, s.group.pfx, G, stripe);
      const int x = r - gcost[lo];
      s.more = x / (w.stripe * w.sum);
      const int y = x - s.more * w.stripe * w.sum, nt = w.tiles_of(s.more);
      s.chunk = min(min(y / (nt * 2), w.whole), w.chunks - 1);    // full chunks first; the last one may cost less
      const int z = y - s.chunk * nt * 2, wl = w.weight(s.chunk, G);
      s.tile = s.more * w.stripe + (z + wl - 1) / wl;             // the first tile that begins in the stretch; may be the chunk's end
    }
    a.w.wide_start[k] = s;
  }
  if (tid == 0)
    *a.w.head = {ATTEND_MARK, n, a.b.n_tokens, a.n_q_heads, H, a.g.page_shift, tiles, chunks, narrow_each, cost, wchunks, wide_each,
                 a.g.max_seqs, a.g.max_pages, a.g.table};
}

// Rows whose keys were split: out = sum_i O_i 2^(m_i - m) / sum_i l_i 2^(m_i - m), m the largest m_i, and the same for lse.
// WARPS warps a row, four channels a lane, up to eight parts in flight each; parts in a fixed order, so that a row comes out the
// same on every run.  A chain of two round trips (token, parts) bounds it where rows are few.
template <int WARPS>
__global__ void __launch_bounds__(128) attend_join_kernel(AttendArgs a) {
  __shared__ float4 joined[4][32];
  pdl_wait_predecessor();
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.w.open = 0;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = WARPS == 1 ? 0 : warp;
  const int row = WARPS == 1 ? blockIdx.x * 4 + warp : blockIdx.x;
  const bool exists = row < a.n_tokens * a.n_q_heads;
  const int t = exists ? row / a.n_q_heads : 0, head = row - t * a.n_q_heads, G = a.group_heads, h = head / G, g = head - h * G;
  const AttendSeq s = load_seq(&a.w.tokens[t].seq);
  const AttendGroup gr = load_group(&a.w.tokens[t].group);
  const AttendHead hd = load_head(a.w.head);
  if (!plan_fits(a, hd) || !exists || s.ntok == 0) return;            // (the same for all warps of a row)
  const int nt = narrow_tiles_of(s), lr = (t - s.tok0) * G + g, chunk = lr / NARROW_ROWS;
  const int ta = h * hd.narrow_tiles + s.tile0 + chunk * nt;
  const int c0 = ta / hd.narrow_each, c1 = (ta + nt - 1) / hd.narrow_each;
  if (s.pfx == 0 && c0 == c1) return;                             // written where it was computed
  // Parts: narrow ones c0 .. c1, then those of the prefix: two halves each where a chunk's rows fill one; where there are
  // stripes, two CTAs each at most.
  const int64_t n_row = ((int64_t)h * hd.narrow_chunks + s.chunk0 + chunk + c0) * NARROW_ROWS + lr % NARROW_ROWS;
  const int n_parts = c1 - c0 + 1;
  const WideShape ws(gr.ntok, s.pfx, G, gr.stripe);
  int total = n_parts, halves = 1, ch = 0, wr = 0, weight = 2, x0 = 0;
  const int h_cost = h * hd.wide_cost + gr.cost0;
  if (s.pfx) {
    const int T = wide_tokens(G);
    ch = (t - gr.tok0) / T;
    wr = ((t - gr.tok0) - ch * T) * G + g;
    weight = ws.weight(ch, G);
    halves = weight == 1 ? 2 : 1;
    x0 = (h_cost + ws.before(0, ch)) / hd.wide_each;
    const int x1 = (h_cost + ws.before(0, ch) + (ws.tiles_of(0) - 1) * weight) / hd.wide_each;
    total += halves * (ws.stripes == 1 ? x1 - x0 + 1 : 2 * ws.stripes);
  }
  // where part k of the row lies (in rows; the prefixes' behind all narrow ones), -1: nowhere
  auto place = [&](int k) -> int64_t {
    if (k >= total) return -1;
    if (k < n_parts) return n_row + k * NARROW_ROWS;
    k -= n_parts;
    const int half = halves == 2 ? k & 1 : 0;
    if (halves == 2) k >>= 1;
    int stripe = 0, cta = x0 + k;
    if (ws.stripes > 1) {
      stripe = k >> 1;
      const int at = h_cost + ws.before(stripe, ch), from = at / hd.wide_each;
      cta = from + (k & 1);
      if (cta > (at + (ws.tiles_of(stripe) - 1) * weight) / hd.wide_each) return -1;
    }
    return a.w.wide_row0 + ((int64_t)h * hd.wide_chunks + gr.chunk0 + stripe * ws.chunks + ch + cta) * WIDE_ROWS + half * (WIDE_ROWS / 2) + wr;
  };
  float top = -INFINITY, sum = 0.0f;
  float4 acc = make_float4(0, 0, 0, 0);
  // up to 32 parts at a time (more than that are joined to what is there, as the parts themselves were)
  for (int k0 = 0; k0 < total; k0 += 32) {
    const int64_t at = place(k0 + lane);
    const float2 e = at >= 0 ? __ldcg(a.w.ml + at) : make_float2(-INFINITY, 0.0f);
    const int m = min(32, total - k0);
    float mx = e.x;
    float4 v[8];
    auto load = [&](int b) {
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const int k = b + sub + q * WARPS;
        const int64_t from = __shfl_sync(0xffffffffu, at, k & 31);
        v[q] = k < m && from >= 0 ? __ldcg(reinterpret_cast<const float4*>(a.w.o + from * 128) + lane) : make_float4(0, 0, 0, 0);
      }
    };
    load(0);
#pragma unroll
    for (int off = 16; off; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
    const float was = top;
    top = fmaxf(top, mx);
    const float ref = top == -INFINITY ? 0.0f : top, f = ex2(e.x - ref);
    if (k0) {
      const float back = ex2(was - ref);
      sum *= back;
      acc.x *= back; acc.y *= back; acc.z *= back; acc.w *= back;
    }
    sum += e.y * f;
    for (int b = 0; b < m; b += 8 * WARPS) {
      if (b) load(b);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const int k = b + sub + q * WARPS;
        const float fk = __shfl_sync(0xffffffffu, f, k & 31), mk = __shfl_sync(0xffffffffu, e.x, k & 31);
        if (k < m && mk != -INFINITY) {                           // a part that saw nothing may hold anything
          acc.x += v[q].x * fk; acc.y += v[q].y * fk; acc.z += v[q].z * fk; acc.w += v[q].w * fk;
        }
      }
    }
  }
  const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll
  for (int off = 16; off; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
  if (WARPS > 1) {
    joined[warp][lane] = acc;
    __syncthreads();
    if (warp) return;
#pragma unroll
    for (int k = 1; k < WARPS; ++k) {
      const float4 o = joined[k][lane];
      acc.x += o.x; acc.y += o.y; acc.z += o.z; acc.w += o.w;
    }
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  *reinterpret_cast<uint2*>(a.out + (int64_t)row * 128 + lane * 4) = make_uint2(pack2(acc.x * inv, acc.y * inv), pack2(acc.z * inv, acc.w * inv));
  if (a.lse && lane == 0) a.lse[row] = (ref + log2f(sum)) * 0.6931471805599453f;
}

AttendLayout layout_of(int sm_count, int n_kv_heads, int n_seqs, int n_tokens, int n_q_heads) {
  AttendLayout l;
  const int64_t G = n_q_heads / n_kv_heads, H = n_kv_heads;
  l.narrow_grid = NARROW_CTAS * sm_count;
  l.wide_grid = sm_count;
  // chunks at most: of a sequence's rows one is not full; no more than every token's rows on their own
  const int64_t per_token = (G + NARROW_ROWS - 1) / NARROW_ROWS;
  int64_t narrow = n_tokens * G / NARROW_ROWS + n_seqs;
  if (narrow > n_tokens * per_token) narrow = n_tokens * per_token;
  const int64_t wide = n_tokens / wide_tokens((int)G) + n_seqs / 2 + 1;
  // (chunks of stripes, where there are several: a stripe is at least half a CTA's cost long and a chunk's tile costs at least
  // 3/2 on average, so that there are 4/3 as many as CTAs at most, and one more for every chunk)
  const size_t narrow_slots = (size_t)(H * narrow + l.narrow_grid), wide_slots = (size_t)(H * wide + 3 * l.wide_grid);
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t at = off; off = asl_align256(off + bytes); return at; };
  l.head = take(128 + sizeof(uint32_t));
  l.open = l.head + 128;                   // (a line of its own: the head is read through L1)
  l.seqs = take(sizeof(AttendSeq) * n_seqs);
  l.groups = take(sizeof(AttendGroup) * n_seqs);
  l.same = take(sizeof(int32_t) * n_seqs);
  l.tokens = take(sizeof(AttendToken) * n_tokens);
  l.narrow_start = take(sizeof(AttendStart) * l.narrow_grid);
  l.wide_start = take(sizeof(AttendStart) * l.wide_grid);
  l.wide_row0 = (int64_t)(NARROW_ROWS * narrow_slots);
  l.ml = take(sizeof(float2) * (l.wide_row0 + WIDE_ROWS * wide_slots));
  l.o = take(sizeof(float) * 128 * (l.wide_row0 + WIDE_ROWS * wide_slots));
  l.total = off;
  return l;
}

AttendPtrs ptrs_of(const AttendLayout& l, void* workspace) {
  char* w = static_cast<char*>(workspace);
  AttendPtrs p;
  p.head = reinterpret_cast<AttendHead*>(w + l.head);
  p.open = reinterpret_cast<uint32_t*>(w + l.open);
  p.seqs = reinterpret_cast<AttendSeq*>(w + l.seqs);
  p.groups = reinterpret_cast<AttendGroup*>(w + l.groups);
  p.same = reinterpret_cast<int32_t*>(w + l.same);
  p.tokens = reinterpret_cast<AttendToken*>(w + l.tokens);
  p.narrow_start = reinterpret_cast<AttendStart*>(w + l.narrow_start);
  p.wide_start = reinterpret_cast<AttendStart*>(w + l.wide_start);
  p.ml = reinterpret_cast<float2*>(w + l.ml);
  p.o = reinterpret_cast<float*>(w + l.o);
  p.wide_row0 = l.wide_row0;
  return p;
}

asl_status check_attend(const asl_ctx* c, const asl_pages* p, const asl_batch* b, int n_q_heads) {
  if (!c) return ASL_ERR_INVALID;
  const asl_status s = asl_check_pages(p);
  if (s != ASL_OK) return s;
  if (!b || !b->slots || !b->cu_q || b->n_seqs < 1 || b->n_tokens < 0) return ASL_ERR_INVALID;
  if (n_q_heads < 1 || n_q_heads % p->n_kv_heads) return ASL_ERR_INVALID;
  if (b->n_seqs > ATTEND_MAX_SEQS || n_q_heads / p->n_kv_heads > 128) return ASL_ERR_UNSUPPORTED;
  if ((int64_t)b->n_tokens * n_q_heads >= (int64_t)1 << 31) return ASL_ERR_UNSUPPORTED;
  return ASL_OK;
}

// Whether neighbours could share enough, by the sizes alone, for the plan to look and the prefixes' kernel to be launched.
bool may_share(const asl_pages* p, const asl_batch* b, int share) {
  if (share == 0 || b->n_seqs < 2) return false;
  return share == 2 || (double)(b->n_seqs - 1) * p->max_pages * p->page_size * p->n_kv_heads * p->head_dim * 4 >= SHARE_MIN_BYTES;
}

}  // namespace

extern "C" {

asl_status asl_attend_workspace(const asl_ctx* c, const asl_pages* p, const asl_batch* b, int32_t n_q_heads, size_t* bytes) {
  if (!bytes) return ASL_ERR_INVALID;
  const asl_status s = check_attend(c, p, b, n_q_heads);
  if (s == ASL_OK) *bytes = layout_of(c->sm_count, p->n_kv_heads, b->n_seqs, b->n_tokens, n_q_heads).total;
  return s;
}

asl_status asl_attend_plan(asl_ctx* c, const asl_pages* p, const asl_batch* b, int32_t n_q_heads, int32_t share, void* workspace,
                           size_t workspace_bytes, void* stream) {
  const asl_status s = check_attend(c, p, b, n_q_heads);
  if (s != ASL_OK) return s;
  if (!asl_on_device(c) || share < 0 || share > 2) return ASL_ERR_INVALID;
  const AttendLayout l = layout_of(c->sm_count, p->n_kv_heads, b->n_seqs, b->n_tokens, n_q_heads);
  if (!workspace || workspace_bytes < l.total || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return ASL_ERR_WORKSPACE;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  PlanArgs a;
  a.g = page_pool(p, 0);
  a.b = *b;
  a.w = ptrs_of(l, workspace);
  a.G = n_q_heads / p->n_kv_heads;
  a.n_q_heads = n_q_heads;
  a.share = !may_share(p, b, share) ? 0 : (int64_t)b->n_seqs * p->max_pages > SAME_INSIDE ? 1 : 2;
  a.narrow_grid = l.narrow_grid;
  a.wide_grid = l.wide_grid;
  a.min_bytes = share == 2 ? 0.0f : SHARE_MIN_BYTES;
  const size_t smem = sizeof(int32_t) * (12 * (size_t)b->n_seqs + 2);
  if (!c->plan_ready) {                    // (whatever the batch: the 48 KB that need no leave hold the kernel's own arrays too)
    ASL_CUDA(cudaFuncSetAttribute(attend_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 4 * (12 * ATTEND_MAX_SEQS + 2)));
    c->plan_ready = true;
  }
  if (a.share == 1) {
    launch_after(attend_same_kernel, dim3(b->n_seqs), dim3(SAME_THREADS), st, a.g, a.b, a.w.same);
    ASL_CUDA(cudaGetLastError());          // (the plan reads what it has counted)
    c->launches += 1;
  }
  launch_after_smem(attend_plan_kernel, dim3(1), dim3(PLAN_THREADS), smem, st, a);
  ASL_CUDA(cudaGetLastError());
  c->launches += 1;
  return ASL_OK;
}

asl_status asl_attend(asl_ctx* c, const asl_pages* p, int32_t layer, const asl_batch* b, int32_t n_q_heads, int32_t share,
                      const void* q, const int64_t q_stride[2], void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  asl_status s = check_attend(c, p, b, n_q_heads);
  if (s != ASL_OK) return s;
  if (!asl_on_device(c) || share < 0 || share > 2) return ASL_ERR_INVALID;
  if (b->n_tokens != 0 && (!q || !out)) return ASL_ERR_INVALID;     // (what is empty has no address)
  if (layer < 0 || layer >= p->n_layers || !q_stride || !asl_aligned16(q) || !asl_aligned16(out)) return ASL_ERR_INVALID;
  for (int i = 0; i < 2; ++i)
    if (q_stride[i] < p->head_dim || q_stride[i] % 8) return ASL_ERR_INVALID;
  const AttendLayout l = layout_of(c->sm_count, p->n_kv_heads, b->n_seqs, b->n_tokens, n_q_heads);
  if (!workspace || workspace_bytes < l.total || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return ASL_ERR_WORKSPACE;
  if (b->n_tokens == 0) return ASL_OK;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  AttendArgs a;
  a.g = page_pool(p, layer);
  a.w = ptrs_of(l, workspace);
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.qs_t = q_stride[0];
  a.qs_h = q_stride[1];
  a.out = static_cast<__nv_bfloat16*>(out);
  a.lse = lse;
  a.k_scale = p->k_dtype == ASL_K_FP8_E4M3 ? p->k_scale + (int64_t)layer * p->n_kv_heads : nullptr;
  a.err = c->d_err;
  a.n_q_heads = n_q_heads;
  a.group_heads = n_q_heads / p->n_kv_heads;
  a.n_tokens = b->n_tokens;
  a.n_seqs = b->n_seqs;
  a.scale_log2 = (float)(1.4426950408889634 / sqrt((double)p->head_dim));
  if (!c->attend_ready) {
    if ((s = asl_attend_narrow_ready()) != ASL_OK || (s = asl_attend_wide_ready()) != ASL_OK) return s;
    c->attend_ready = true;
  }
  const bool wide = may_share(p, b, share);        // (the plan says whether they do)
  a.with_wide = wide;
  if (wide) {
    s = asl_launch_attend_wide(c, p, a, l.wide_grid, st);
    if (s != ASL_OK) return s;
  }
  s = asl_launch_attend_narrow(c, p, a, l.narrow_grid, wide, st);
  if (s != ASL_OK) return s;
  // four warps a row where they all find room at once, else one
  const int64_t rows = (int64_t)b->n_tokens * n_q_heads;
  if (rows <= 16 * c->sm_count) launch_after(attend_join_kernel<4>, dim3((unsigned)rows), dim3(128), st, a);
  else launch_after(attend_join_kernel<1>, dim3((unsigned)((rows + 3) / 4)), dim3(128), st, a);
  c->launches += 1;
  ASL_CUDA(cudaGetLastError());
  return ASL_OK;
}

}  // extern "C"
