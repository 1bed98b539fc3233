// Attention over prefixes that a group of sequences shares: the rows of all of them against keys that are read once.
//
// A chunk is up to 256 (token, query head) rows of a group's kv head.  Two accumulator pairs in tensor memory, "streams", work in
// turn so that the tensor pipe has one's products while the other's weights are computed:
//   S = Q K^T (128 rows x 128 keys), p = 2^(S c - m), written back as bf16 over S, O += P V with P from tensor memory.
// With more than 128 rows a stream has 128 of them and both meet every tile; with fewer the streams have the same rows and take
// tiles in turn, and leave two parts.  m is the reference of a row, not its maximum: it follows the maximum only when that has
// grown by more than 2^8 (p is then at most 256, and O is seldom rescaled).
// K and V tiles come by TMA, pages or pieces of pages of one kv head at a time; E4M3 keys are widened to bf16 (exactly) on their
// way by four more warps.  A prefix is a multiple of the page size, so tiles need no masks; a last tile of fewer keys makes
// fewer products.
//
// What bounds it: a tile of 256 rows is 32 products of 64 clk; the kernel takes about 3500 clk for it (2.0 us; E4M3 keys 2.4) and 17 us
// for its two ends, most of the rest a stream's round from S to its weights and back, and power: kept up, the large cases run at 1000 W
// and 1.5 to 1.7 GHz (1040 rows on 64K tokens, 8 kv heads: 294 us, 0.95 PFLOP/s; 192 rows on 128K tokens: 130 us, 4.1 TB/s), where
// schedules of fewer clocks have run at lower ones.  With up to 128 rows HBM's latency counts: 4 TB/s of 8K prompts.
#include "asl_ptx.cuh"
#include "attend.cuh"

namespace {

constexpr int K_RING = 2;
constexpr int TILE_BYTES = WIDE_KEYS * 256, TILE_HALF = WIDE_KEYS * 128;
constexpr float RESCALE = 8.0f;            // powers of two that a row's maximum may lie above its reference

template <bool FP8>
struct WideSmem {
  static constexpr int V_RING = FP8 ? 2 : 3;
  static constexpr int Q_HALF = WIDE_ROWS * 128;                    // 64 channels of 256 rows
  static constexpr int K = 2 * Q_HALF;
  static constexpr int V = K + K_RING * TILE_BYTES;
  static constexpr int CODES = V + V_RING * TILE_BYTES;             // E4M3 tiles as they come
  static constexpr int BARS = CODES + (FP8 ? 2 * TILE_HALF : 0);
  static constexpr int KF = 0, KE = KF + K_RING, VF = KE + K_RING, VE = VF + 3, SF = VE + 3, PF = SF + 2, OD = PF + 2, QF = OD + 2,
                       QE = QF + 1, CF = QE + 1, CE = CF + 2, DRAIN = CE + 2, TURN = DRAIN + 2, N_BARS = TURN + 2;
  static constexpr int MISC = BARS + 256;
  static constexpr int BYTES = MISC + 16 + 1024;
  static constexpr int THREADS = FP8 ? 512 : 384;
  // Registers a thread: a row of 128 logits stays in them.  Launched with REGS each; the warpgroups' shares are no more together.
  static constexpr int REGS = FP8 ? 128 : 168, REGS_FEW = FP8 ? 40 : 72, REGS_ROWS = 216;
  static_assert(REGS * THREADS >= REGS_FEW * (THREADS - 256) + REGS_ROWS * 256, "a warpgroup would wait for registers");
  static_assert(N_BARS * 8 <= 256 && BYTES <= 232448, "shared memory budget of one CTA");
};

// A CTA's stretch: chunk by chunk (of a stripe) the tiles tile .. end - 1.
struct Walk {
  int h, gi, stripe, chunk, tile, end;
  int weight, rows, items, total, chunks;
  int stop;                                // cost at which the stretch ends
  int n_chunks;                            // of the group
  AttendGroup g;
  __device__ __forceinline__ bool set(const AttendArgs& a, bool begins) {
    const int G = a.group_heads, T = wide_tokens(G);
    const WideShape w(g.ntok, g.pfx, G, g.stripe);
    const int t0 = stripe * w.stripe, nt = w.tiles_of(stripe), at = h * total + g.cost0 + w.before(stripe, chunk);
    weight = w.weight(chunk, G);
    rows = min(T, g.ntok - chunk * T) * G;
    if (begins) tile = t0;
    end = min(t0 + nt, t0 + (stop - at + weight - 1) / weight);
    n_chunks = w.chunks;
    return end > tile;
  }
  __device__ __forceinline__ bool begin(const AttendArgs& a) {
    const AttendHead hd = load_head(a.w.head);
    const AttendStart st = load_start(a.w.wide_start + blockIdx.x);
    if (!plan_fits(a, hd) || st.h < 0) return false;
    h = st.h; gi = st.item; chunk = st.chunk; tile = st.tile; stripe = st.more;
    g = st.group;
    items = st.items; total = st.total; chunks = st.chunks;
    stop = min(a.g.n_kv_heads * total, ((int)blockIdx.x + 1) * hd.wide_each);
    return set(a, false) || next(a);
  }
  __device__ __forceinline__ bool next(const AttendArgs& a) {
    if (++chunk == n_chunks) {
      chunk = 0;
      ++stripe;
      if (n_chunks == 1 || stripe * g.stripe * WIDE_KEYS >= g.pfx) {
        stripe = 0;
        do {
          if (++gi >= items) {
            gi = 0;
            if (++h >= a.g.n_kv_heads) return false;
          }
          g = load_group(a.w.groups + gi);
        } while (g.pfx == 0);
      }
    }
    return set(a, true);
  }
  __device__ __forceinline__ bool full() const { return weight == 2; }
  __device__ __forceinline__ int keys(int t) const { return min(WIDE_KEYS, g.pfx - t * WIDE_KEYS); }
  __device__ __forceinline__ int64_t slot() const { return (int64_t)h * chunks + g.chunk0 + stripe * n_chunks + chunk + blockIdx.x; }
};

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float row_max(const uint32_t (&x)[4][32]) {
  float m[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    m[k] = __uint_as_float(x[k][0]);
#pragma unroll
    for (int e = 1; e < 31; e += 2) m[k] = max3(m[k], __uint_as_float(x[k][e]), __uint_as_float(x[k][e + 1]));
    m[k] = max3(m[k], __uint_as_float(x[k][31]), m[k]);
  }
  return max3(max3(m[0], m[1], m[2]), m[3], m[3]);
}
template <int N>
__device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void give_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

template <bool FP8>
__global__ void __launch_bounds__(WideSmem<FP8>::THREADS, 1)
attend_wide_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                   const __grid_constant__ CUtensorMap tm_v, AttendArgs a) {
  using S = WideSmem<FP8>;
  extern __shared__ uint8_t raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  const uint32_t base = smem_u32(sm);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* s_abort = reinterpret_cast<volatile int*>(sm + S::MISC + 8);
  auto bar = [&](int i) { return base + S::BARS + 8 * i; };
  if (threadIdx.x == 0) {
    // (tiles and queries are given back by both issuing warps)
    for (int i = 0; i < K_RING; ++i) { mbar_init(bar(S::KF + i), FP8 ? 4 : 1); mbar_init(bar(S::KE + i), 2); }
    for (int i = 0; i < S::V_RING; ++i) { mbar_init(bar(S::VF + i), 1); mbar_init(bar(S::VE + i), 2); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar(S::SF + i), 1);
      mbar_init(bar(S::PF + i), 4);
      mbar_init(bar(S::OD + i), 1);
      mbar_init(bar(S::CF + i), 1);
      mbar_init(bar(S::CE + i), 4);
    }
    mbar_init(bar(S::QF), 1);
    mbar_init(bar(S::QE), 2);
    mbar_init(bar(S::DRAIN), 1);
    mbar_init(bar(S::DRAIN + 1), 1);
    mbar_init(bar(S::TURN), 1);
    mbar_init(bar(S::TURN + 1), 1);
    *s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(base + S::MISC) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<const uint32_t*>(sm + S::MISC);
  pdl_wait_predecessor();
  if (threadIdx.x == 0) {
    if (blockIdx.x == 0) others_may_read(a.w.open);      // (before it starts)
    pdl_release_successor();               // it finds room when this grid's blocks leave
  }
  const int G = a.group_heads, T = wide_tokens(G);

  if (warp >= 4 && warp < 12) {
    take_registers<S::REGS_ROWS>();
    Walk w;
    const bool any = w.begin(a);
    // =============================== weights ====================================
    const int s = (warp - 4) >> 2, row = (threadIdx.x & 127);      // stream; row of its 128 = lane of tensor memory
    const uint32_t st = tmem + s * 128 + ((uint32_t)((warp & 3) * 32) << 16), ot = st + 256;
    int it = 0;                                                     // items of the stream so far
    bool ok = true, more = true;
    while (any && ok && more) {
      const bool full = w.full();
      const int r = full ? s * 128 + row : row;                     // row of the chunk
      const bool warp_has = (r & ~31) < w.rows;                     // of this warp's rows some exist
      const float c = a.scale_log2 * (FP8 ? __ldcg(a.k_scale + w.h) : 1.0f);
      float m = -INFINITY;
      f32x2 l2 = pk(0.0f, 0.0f);
      const int t0 = full ? w.tile : w.tile + s, dt = full ? 1 : 2;
      for (int t = t0; t < w.end; t += dt, ++it) {
        const int nk = w.keys(t);
        if (!__all_sync(0xffffffffu, mbar_wait(bar(S::SF + s), it & 1, s_abort, 231, true))) { ok = false; break; }
        tc_fence_after();
        if (warp_has) {
          uint32_t x[4][32];
#pragma unroll
          for (int k = 0; k < 4; ++k) tc_ld_lane32(st + 32 * k, x[k]);
          tc_wait_loads();
#pragma unroll
          for (int k = 0; k < 4; ++k) tc_landed(x[k]);
          if (nk < WIDE_KEYS) {
#pragma unroll
            for (int k = 0; k < WIDE_KEYS; ++k)
              if (k >= nk) x[k >> 5][k & 31] = 0xff800000u;         // -inf
          }
          // the row's largest logit (a NaN, or infinity less itself, makes weights NaN below, and with them the row)
          const float mx = row_max(x) * c;
          const bool first = t == t0;
          if (first) {
            m = mx;
          } else {
            const bool grow = mx > m + RESCALE;
            if (__any_sync(0xffffffffu, grow)) {
              if (!__all_sync(0xffffffffu, mbar_wait(bar(S::OD + s), (it - 1) & 1, s_abort, 232, true))) { ok = false; break; }
              tc_fence_after();
              const float to = grow ? mx : m, f = grow ? ex2(m - (to == -INFINITY ? 0.0f : to)) : 1.0f;
              m = to;
              float lo, hi;
              upk(l2, lo, hi);
              l2 = pk(lo * f, hi * f);
              uint32_t o[16];
              for (int k = 0; k < 128; k += 16) {
                tc_ld_lane(ot + k, o);
                tc_ld_wait(o);
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                tc_st_lane(ot + k, o);
              }
              tc_st_wait();
            }
          }
          const float ref = m == -INFINITY ? 0.0f : m;
          const f32x2 c2 = pk(c, c), m2 = pk(-ref, -ref);
          f32x2 l3 = pk(0.0f, 0.0f);
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            uint32_t p[32];                                         // over columns that have been read
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              const int col = 64 * k + 2 * e;
              const f32x2 z = fma2(pku(x[col >> 5][col & 31], x[col >> 5][(col & 31) + 1]), c2, m2);
              const f32x2 y = ex2_pair_mufu(z);
              if (e & 1) l3 = add2(l3, y); else l2 = add2(l2, y);
              float lo, hi;
              upk(y, lo, hi);
              p[e] = pack2(lo, hi);                                 // rounded for the tensor core; l keeps them unrounded
            }
            tc_st_lane32(st + 32 * k, p);
          }
          l2 = add2(l2, l3);
          tc_st_wait();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(S::PF + s));
      }
      if (!ok) break;
      // the part: this stream's rows of the run
      const int64_t at = a.w.wide_row0 + w.slot() * WIDE_ROWS + s * 128 + row;
      if (t0 < w.end) {
        if (!__all_sync(0xffffffffu, mbar_wait(bar(S::OD + s), (it - 1) & 1, s_abort, 233, true))) { ok = false; break; }
        tc_fence_after();
        if (warp_has) {
          uint32_t o[2][16];
          tc_ld_lane(ot, o[0]);
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            tc_ld_wait(o[k & 1]);
            if (k < 7) tc_ld_lane(ot + 16 * (k + 1), o[(k + 1) & 1]);
            if (r < w.rows) {
              float4* to = reinterpret_cast<float4*>(a.w.o + at * 128 + 16 * k);
#pragma unroll
              for (int e = 0; e < 4; ++e)
                to[e] = make_float4(__uint_as_float(o[k & 1][4 * e]), __uint_as_float(o[k & 1][4 * e + 1]), __uint_as_float(o[k & 1][4 * e + 2]),
                                    __uint_as_float(o[k & 1][4 * e + 3]));
            }
          }
          tc_fence_before();
        }
      }
      if (r < w.rows) a.w.ml[at] = make_float2(t0 < w.end ? m : -INFINITY, hsum(l2));
      more = w.next(a);
    }
  } else {
    give_registers<S::REGS_FEW>();
    Walk w;
    const bool any = w.begin(a);
    if (any && warp == 0) {
      // =============================== copies =====================================
      const int shift = a.g.page_shift, per = WIDE_KEYS >> shift, page = 1 << shift;
      int run = 0, n = 0;                    // chunks; tiles of all chunks
      bool ok = true, more = true;
      auto queries = [&]() {
        if (run > 1 && !mbar_wait(bar(S::QE), (run - 2) & 1, s_abort, 211, true)) { --run; return false; }
        if (elect_one()) {
          mbar_expect_tx(bar(S::QF), (uint32_t)(2 * 128 * G * T));
          tma_load_3d(base, &tm_q, bar(S::QF), 0, w.h * G, w.g.tok0 + w.chunk * T);
          tma_load_3d(base + S::Q_HALF, &tm_q, bar(S::QF), 64, w.h * G, w.g.tok0 + w.chunk * T);
        }
        __syncwarp();
        return true;
      };
      while (ok && more) {
        if (++run == 1) queries();           // later ones go behind their first K: their room is free only when all S before are there
        const int32_t* row = a.g.table + (int64_t)w.g.slot * a.g.max_pages;
        const int last = w.g.pfx >> shift;   // pages of the prefix
        int first = w.tile * per;            // page numbers of 32 pages a lane each, and of the 32 after them
        int ids = first + lane < last ? page_in_pool(a.g, __ldcg(row + first + lane), w.g.slot) : 0;
        int ids2 = first + 32 + lane < last ? __ldcg(row + first + 32 + lane) : 0;
        for (int t = w.tile; t < w.end; ++t, ++n) {
          if (t * per >= first + 32) {       // (a tile has 8 pages at most, and 32 is a multiple of what it has)
            first += 32;
            ids = page_in_pool(a.g, ids2, w.g.slot);           // (looked at no earlier: it comes while the tiles before are copied)
            ids2 = first + 32 + lane < last ? __ldcg(row + first + 32 + lane) : 0;
          }
          const int ks = n % K_RING, vs = n % S::V_RING, np = w.keys(t) >> shift;
          // E4M3 tiles land in a ring of their own, from which they are widened into K's
          const uint32_t kbar = FP8 ? bar(S::CF + (n & 1)) : bar(S::KF + ks), kfree = FP8 ? bar(S::CE + (n & 1)) : bar(S::KE + ks);
          const uint32_t kd = base + (FP8 ? S::CODES + (n & 1) * TILE_HALF : S::K + ks * TILE_BYTES);
          const uint32_t kpar = ((FP8 ? n >> 1 : n / K_RING) & 1) ^ 1;
          if (!mbar_wait(kfree, kpar, s_abort, 212, true)) { ok = false; break; }
          const int r0 = (ids * a.g.n_kv_heads + w.h) << shift;
          if (elect_one()) mbar_expect_tx(kbar, (uint32_t)(np * page * a.g.k_row));
          __syncwarp();
          for (int x = 0; x < np; ++x) {
            const int r = __shfl_sync(0xffffffffu, r0, t * per + x - first);
            if (elect_one()) {
              tma_load_2d(kd + x * page * 128, &tm_k, kbar, 0, r);
              if (!FP8) tma_load_2d(kd + TILE_HALF + x * page * 128, &tm_k, kbar, 64, r);
            }
          }
          if (t == w.tile && run > 1 && !queries()) {
            ok = false;
            ++n;                             // K of this tile is in flight
            break;
          }
          if (!mbar_wait(bar(S::VE + vs), ((n / S::V_RING) & 1) ^ 1, s_abort, 213, true)) {
            ok = false;
            ++n;                             // K of this tile is in flight
            break;
          }
          if (elect_one()) mbar_expect_tx(bar(S::VF + vs), (uint32_t)(np * page * 256));
          __syncwarp();
          for (int x = 0; x < np; ++x) {
            const int r = __shfl_sync(0xffffffffu, r0, t * per + x - first);
            if (elect_one()) {
              const uint32_t vd = base + S::V + vs * TILE_BYTES + x * page * 128;
              tma_load_2d(vd, &tm_v, bar(S::VF + vs), 0, r);
              tma_load_2d(vd + TILE_HALF, &tm_v, bar(S::VF + vs), 64, r);
            }
          }
        }
        if (ok) more = w.next(a);
      }
      if (!ok || *s_abort) {                 // copies in flight land before the block ends
        for (int i = max(0, n - 3); i < n; ++i) {
          if (FP8) { if (i >= n - 2) mbar_wait(bar(S::CF + (i & 1)), (i >> 1) & 1, s_abort, 214, false); }
          else if (i >= n - K_RING) mbar_wait(bar(S::KF + i % K_RING), (i / K_RING) & 1, s_abort, 214, false);
          if (i >= n - S::V_RING) mbar_wait(bar(S::VF + i % S::V_RING), (i / S::V_RING) & 1, s_abort, 215, false);
        }
        mbar_wait(bar(S::QF), (run - 1) & 1, s_abort, 216, false);
      }
    } else if (any && warp <= 2) {
      // =============================== products ===================================
      // A warp per stream, so that one's waits are filled by the other's products (one warp for both: 3600 clk a tile of 256
      // rows, of which 800 passed in waits with the tensor pipe empty).
      // (What the products' operands follow from is shuffled, so that the compiler knows it to be the same in all lanes and
      // keeps descriptors in uniform registers: moved there one by one they cost 100 clk a product instead of 64.)
      const int s = __shfl_sync(0xffffffffu, warp - 1, 0);
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0) + s * 128;
      const uint32_t id_full = instr_desc(128, WIDE_KEYS), id_pv = instr_desc(128, 128) | B_MN_MAJOR;
      int n = 0;                           // tiles before this run
      uint32_t pv = 0, turns = 0;          // parity of the next product P V; batches given in turn
      bool ok = true, more = true;
      for (int run = 0; ok && more; ++run) {
        const bool full = __shfl_sync(0xffffffffu, (int)w.full(), 0);
        const int tile = __shfl_sync(0xffffffffu, w.tile, 0), nt = __shfl_sync(0xffffffffu, w.end, 0) - tile;
        const int pfx = __shfl_sync(0xffffffffu, w.g.pfx, 0) - tile * WIDE_KEYS;      // keys from the first tile on
        const int first = full ? 0 : s, step = full ? 1 : 2;                          // the stream's tiles
        auto keys_here = [&](int j) {
          if (ok && j < nt) ok = __all_sync(0xffffffffu, mbar_wait(bar(S::KF + (n + j) % K_RING), ((n + j) / K_RING) & 1, s_abort, 221, true));
        };
        auto values_here = [&](int j) {
          if (ok) ok = __all_sync(0xffffffffu, mbar_wait(bar(S::VF + (n + j) % S::V_RING), ((n + j) / S::V_RING) & 1, s_abort, 224, true));
        };
        // Streams of full chunks give their batches in turn: interleaved, two batches would both end when the later does, and
        // the streams would do everything else at the same time too.
        auto take_turn = [&]() {
          if (full && ok && (s == 1 || turns > 0))
            ok = __all_sync(0xffffffffu, mbar_wait(bar(S::TURN + s), (s == 1 ? turns : turns - 1) & 1, s_abort, 227, true));
        };
        auto scores = [&](int j) {         // S of tile j
          const int ks = (n + j) % K_RING, left = pfx - j * WIDE_KEYS;
          const uint64_t qd = smem_desc(base + (full ? s : 0) * 128 * 128), kd = smem_desc(base + S::K + ks * TILE_BYTES);
          const uint32_t id = left >= WIDE_KEYS ? id_full : instr_desc(128, left);
          if (elect_one()) {
#pragma unroll
            for (int x = 0; x < 8; ++x)
              tc_mma(tm, qd + ((x >> 2) * (S::Q_HALF >> 4) + (x & 3) * 2), kd + ((x >> 2) * (TILE_HALF >> 4) + (x & 3) * 2), id, x > 0);
            if (full) mbar_arrive(bar(S::TURN + (s ^ 1)));          // the other stream's turn
            tc_commit(bar(S::SF + s));
            tc_commit(bar(S::KE + ks));
            if (!full) tc_commit(bar(S::KE + ks));                  // nobody else reads it
            if (j + step >= nt) tc_commit(bar(S::QE));
          }
          __syncwarp();
        };
        ok = __all_sync(0xffffffffu, mbar_wait(bar(S::QF), run & 1, s_abort, 222, true));
        keys_here(first);
        take_turn();
        if (ok && first < nt) {
          tc_fence_after();
          scores(first);
          turns += full;
        } else if (ok && lane == 0) {
          mbar_arrive(bar(S::QE));         // a run of one tile: the other stream's
        }
        for (int j = first; ok && j < nt; j += step) {
          const int vs = (n + j) % S::V_RING, left = pfx - j * WIDE_KEYS;
          values_here(j);                  // (tiles are waited for before the weights, while the pipe still has products)
          keys_here(j + step);
          ok = ok && __all_sync(0xffffffffu, mbar_wait(bar(S::PF + s), pv, s_abort, 223, true));
          take_turn();
          if (!ok) break;
          tc_fence_after();
          const uint64_t vd = smem_desc_mn(base + S::V + vs * TILE_BYTES, TILE_HALF);
          const uint32_t old = j > first;  // there is a result to add to
          if (elect_one()) {
            if (left >= WIDE_KEYS) {
#pragma unroll
              for (int x = 0; x < 8; ++x) tc_mma_ts(tm + 256, tm + x * 8, vd + x * (2048 >> 4), id_pv, x > 0 ? 1u : old);
            } else {
              for (int x = 0; x < left >> 4; ++x) tc_mma_ts(tm + 256, tm + x * 8, vd + x * (2048 >> 4), id_pv, x > 0 ? 1u : old);
            }
            tc_commit(bar(S::OD + s));
            tc_commit(bar(S::VE + vs));
            if (!full) tc_commit(bar(S::VE + vs));
          }
          __syncwarp();
          pv ^= 1u;
          if (j + step < nt) scores(j + step);
          else if (full && lane == 0) mbar_arrive(bar(S::TURN + (s ^ 1)));
          turns += full;
        }
        n += nt;
        if (ok) more = w.next(a);
      }
      if (!ok) {                           // nothing writes tensor memory when it is freed
        if (elect_one()) {
          tc_commit(bar(S::DRAIN + s));
          mbar_wait(bar(S::DRAIN + s), 0, s_abort, 225, false);
        }
        __syncwarp();
      }
    } else if (FP8 && any && warp >= 12) {
      // =============================== widening ===================================
      const int key = threadIdx.x & 127;
      int n = 0;
      bool ok = true, more = true;
      while (ok && more) {
        for (int t = w.tile; ok && t < w.end; ++t, ++n) {
          const int cs = n & 1, ks = n % K_RING;
          ok = mbar_wait(bar(S::CF + cs), (n >> 1) & 1, s_abort, 241, true) && mbar_wait(bar(S::KE + ks), ((n / K_RING) & 1) ^ 1, s_abort, 242, true);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          const uint8_t* from = sm + S::CODES + cs * TILE_HALF + key * 128;
          uint8_t* to = sm + S::K + ks * TILE_BYTES + key * 128;
  #pragma unroll
          for (int x = 0; x < 8; ++x) {      // 16 codes: two 16-byte pieces of the key's bf16 row
            const uint4 v = *reinterpret_cast<const uint4*>(from + ((x ^ (key & 7)) << 4));
            uint8_t* half = to + (x >> 2) * TILE_HALF;
            const int pc = (x & 3) * 2;
            *reinterpret_cast<uint4*>(half + ((pc ^ (key & 7)) << 4)) =
                make_uint4(e4m3_pair(v.x), e4m3_pair(v.x >> 16), e4m3_pair(v.y), e4m3_pair(v.y >> 16));
            *reinterpret_cast<uint4*>(half + (((pc + 1) ^ (key & 7)) << 4)) =
                make_uint4(e4m3_pair(v.z), e4m3_pair(v.z >> 16), e4m3_pair(v.w), e4m3_pair(v.w >> 16));
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(bar(S::KF + ks));
            mbar_arrive(bar(S::CE + cs));
          }
        }
        if (ok) more = w.next(a);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
  if (threadIdx.x == 0 && *s_abort) atomicCAS(a.err, 0, *s_abort);
}

}  // namespace

asl_status asl_launch_attend_wide(asl_ctx* c, const asl_pages* p, const AttendArgs& a, int grid, cudaStream_t st) {
  const bool fp8 = p->k_dtype == ASL_K_FP8_E4M3;
  const cuuint64_t n_rows = (cuuint64_t)p->n_pages * p->n_kv_heads * p->page_size;
  const cuuint32_t page = (cuuint32_t)p->page_size, G = (cuuint32_t)a.group_heads, T = (cuuint32_t)wide_tokens(a.group_heads);
  CUtensorMap tm_q, tm_k, tm_v;
  const cuuint64_t dims[2] = {128, n_rows};
  const cuuint64_t ks[1] = {(cuuint64_t)a.g.k_row}, vs[1] = {(cuuint64_t)a.g.v_row};
  const cuuint32_t kbox[2] = {fp8 ? 128u : 64u, page}, vbox[2] = {64, page};
  const cuuint64_t qdims[3] = {128, (cuuint64_t)a.n_q_heads, (cuuint64_t)a.n_tokens};
  const cuuint64_t qs[2] = {(cuuint64_t)a.qs_h * 2, (cuuint64_t)a.qs_t * 2};
  const cuuint32_t qbox[3] = {64, G, T};
  if (!asl_make_map(&tm_q, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, a.q, 3, qdims, qs, qbox)) return ASL_ERR_CUDA;
  if (!asl_make_map(&tm_k, fp8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, a.g.k, 2, dims, ks, kbox)) return ASL_ERR_CUDA;
  if (!asl_make_map(&tm_v, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, a.g.v, 2, dims, vs, vbox)) return ASL_ERR_CUDA;
  auto kernel = fp8 ? attend_wide_kernel<true> : attend_wide_kernel<false>;
  const int smem = fp8 ? WideSmem<true>::BYTES : WideSmem<false>::BYTES;
  launch_after_smem(kernel, dim3(grid), dim3(fp8 ? WideSmem<true>::THREADS : WideSmem<false>::THREADS), smem, st, tm_q, tm_k, tm_v, a);
  c->launches += 1;
  ASL_CUDA(cudaGetLastError());
  return ASL_OK;
}

asl_status asl_attend_wide_ready() {
  ASL_CUDA(cudaFuncSetAttribute(attend_wide_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, WideSmem<false>::BYTES));
  ASL_CUDA(cudaFuncSetAttribute(attend_wide_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, WideSmem<true>::BYTES));
  return ASL_OK;
}
