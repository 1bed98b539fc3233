// Attention of few rows: the keys that one sequence reads by itself, 16 (token, query head) rows of a kv head at a time.
//
// Per row r and key j: x = q_r . k_j * log2(e)/sqrt(d), running maximum m, p = 2^(x - m), l = sum p, O = sum p v.  Four warps
// take 16 keys each of a 64-key tile (m16n8k16 products, rows padded to 16) and keep m, l and O of their own; a part's end joins
// them.  16 rows do 16 operations per byte of K and V, so HBM bounds it (its rate asks for 0.1 PFLOP/s): 24 sequences of 4100 to 4600
// tokens, 8 kv heads: 278 MB in 49 us, 5.6 TB/s.  Two blocks an SM with three tiles of 32 KB on their way each.  Short tails are
// bound by what a part costs besides its tiles; the copying warp therefore brings a part's queries and description as well (five
// draft tokens on six prompts 139 -> 135 us), and runs up to a part ahead.  Many tokens of one sequence read its keys once for every
// 16 rows, from L2: 512 of them on 8K, 32 query and 8 kv heads, 332 us where the products would take 41.
#include "asl_ptx.cuh"
#include "attend.cuh"

namespace {

constexpr int WARPS = 4;                   // that compute; one more copies
constexpr int STAGES = 3;
constexpr int Q_PITCH = 272;               // bytes from one query row to the next, so that eight of them lie in different banks
constexpr int O_STRIDE = 68;               // floats from one row to the next where parts of four warps are joined

template <bool FP8>
struct NarrowSmem {
  static constexpr int K_BYTES = NARROW_KEYS * (FP8 ? 128 : 256), V_BYTES = NARROW_KEYS * 256;
  static constexpr int STAGE = K_BYTES + V_BYTES;
  static constexpr int JOIN = STAGES * STAGE;                       // float[4][8][O_STRIDE]
  static constexpr int ML = JOIN + WARPS * 8 * O_STRIDE * 4;        // float2[4][16]
  static constexpr int Q = ML + WARPS * 16 * 8;                      // the next chunk's rows
  static constexpr int PART = Q + NARROW_ROWS * Q_PITCH;            // what they are
  static constexpr int BARS = PART + 64;
  static constexpr int QF = 2 * STAGES, QE = QF + 1;
  static constexpr int MISC = BARS + (QE + 1) * 8;
  static constexpr int BYTES = MISC + 32 + 1024;                    // and the alignment of its base
};

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// A CTA's stretch: its chunks one after another.
struct Walk {
  int h, i, chunk, tile, left;
  AttendSeq s;
  int nt, nch, items, total, chunks, each;
  __device__ __forceinline__ void sizes(const AttendArgs& a) {
    nt = narrow_tiles_of(s);
    nch = narrow_chunks_of(s.ntok, a.group_heads);
  }
  __device__ __forceinline__ bool begin(const AttendArgs& a) {
    const AttendHead hd = load_head(a.w.head);
    const AttendStart st = load_start(a.w.narrow_start + blockIdx.x);
    if (!plan_fits(a, hd) || st.h < 0) return false;
    h = st.h; i = st.item; chunk = st.chunk; tile = st.tile;
    s = st.seq;
    items = st.items; total = st.total; chunks = st.chunks; each = st.more;
    left = min(each, a.g.n_kv_heads * total - (int)blockIdx.x * each);
    sizes(a);
    return true;
  }
  __device__ __forceinline__ int here() const { return min(nt - tile, left); }     // tiles of this part
  // the sequence after this one, asked for early (the one before the last head's end is loaded for nothing)
  __device__ __forceinline__ AttendSeq ahead(const AttendArgs& a) const { return load_seq(a.w.seqs + (i + 1 < items ? i + 1 : 0)); }
  // the next chunk; false at the end
  __device__ __forceinline__ bool next(const AttendArgs& a, const AttendSeq& coming) {
    left -= here();
    if (left <= 0) return false;
    tile = 0;
    if (++chunk < nch) return true;
    chunk = 0;
    bool first = true;
    do {
      if (++i >= items) {
        i = 0;
        if (++h >= a.g.n_kv_heads) return false;
      }
      s = first ? coming : load_seq(a.w.seqs + i);
      first = false;
      sizes(a);
    } while (nch == 0);
    return true;
  }
  // A chunk whose keys nobody else has part of: its rows are written at once.
  __device__ __forceinline__ bool sole() const {
    const int at = h * total + s.tile0 + chunk * nt;
    return s.pfx == 0 && at / each == (at + nt - 1) / each;
  }
  __device__ __forceinline__ int64_t slot() const { return (int64_t)h * chunks + s.chunk0 + chunk + blockIdx.x; }
};

// A part, as the copying warp describes it to the others.
struct Part {
  int32_t tok0, ntok, len, pfx, h, chunk, tile, tiles;   // tiles 0: there is none any more
  int32_t sole, pad;
  int64_t slot;
};
static_assert(sizeof(Part) <= 64, "room for a part's description");

template <bool FP8>
__global__ void __launch_bounds__(WARPS * 32 + 32, 2)
attend_narrow_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, AttendArgs a, int beside) {
  using S = NarrowSmem<FP8>;
  extern __shared__ uint8_t raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  const uint32_t base = smem_u32(sm);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* s_abort = reinterpret_cast<volatile int*>(sm + S::MISC);
  auto full = [&](int st) { return base + S::BARS + 8 * st; };
  auto empty = [&](int st) { return base + S::BARS + 8 * (STAGES + st); };
  const uint32_t q_full = base + S::BARS + 8 * S::QF, q_empty = base + S::BARS + 8 * S::QE;
  Part* part = reinterpret_cast<Part*>(sm + S::PART);
  // Behind the prefixes' kernel (`beside`) the copying warp, from which the others have all that they know, asks whether that kernel
  // has seen the end of all before it; neither writes what the other reads.
  const bool may_read = !beside || warp != WARPS || narrow_may_read(a.w.open);
  if (threadIdx.x == 0) {
    for (int i = 0; i < STAGES; ++i) { mbar_init(full(i), 1); mbar_init(empty(i), WARPS); }
    mbar_init(q_full, 1);
    mbar_init(q_empty, WARPS);
    *s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  if (!beside || !may_read) pdl_wait_predecessor();
  const int n_kv = a.g.n_kv_heads, G = a.group_heads;
  if (warp == WARPS) {
    Walk w;
    const bool any = w.begin(a);
    // ---- copies: tiles of whole pages' pieces; pages behind the sequence's end are not read ----
    const int piece = min(1 << a.g.page_shift, NARROW_KEYS), per = NARROW_KEYS / piece;
    int n = 0, parts = 0;
    bool more = any;
    // rows and description of a part (null: there is none any more) to the others, who have taken over the one before
    auto tell = [&](const Part& what, int rows) {
      if (parts > 0 && !mbar_wait(q_empty, (parts - 1) & 1, s_abort, 204, true)) return false;
      ++parts;
      if (lane == 0) {
        *part = what;
        mbar_expect_tx(q_full, (uint32_t)(rows * 256));
      }
      __syncwarp();
      if (lane < rows) {
        const int lr = what.chunk * NARROW_ROWS + lane;
        const __nv_bfloat16* q = a.q + (int64_t)(what.tok0 + lr / G) * a.qs_t + (int64_t)(what.h * G + lr % G) * a.qs_h;
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], 256, [%2];" ::"r"(base + S::Q + lane * Q_PITCH),
                     "l"(q), "r"(q_full)
                     : "memory");
      }
      __syncwarp();
      return true;
    };
    while (more) {
      const int nt = w.here();
      const AttendSeq coming = w.ahead(a);
      const Part what = {w.s.tok0, w.s.ntok, w.s.len, w.s.pfx, w.h, w.chunk, w.tile, nt, w.sole(), 0, w.slot()};
      if (!tell(what, min(NARROW_ROWS, w.s.ntok * G - w.chunk * NARROW_ROWS))) break;
      const int32_t* row = a.g.table + (int64_t)w.s.slot * a.g.max_pages;
      const int end = min(pages_for(w.s.len, a.g.page_shift), a.g.max_pages);
      int ids = 0, first = -64;
      for (int t = 0; t < nt; ++t, ++n) {
        const int st = n % STAGES, key0 = w.s.pfx + (w.tile + t) * NARROW_KEYS;
        const int p0 = key0 >> a.g.page_shift;
        if (p0 + (NARROW_KEYS - 1 >> a.g.page_shift) >= first + 32) {        // page numbers of the next tiles, a lane each
          first = p0;
          ids = first + lane < end ? page_in_pool(a.g, __ldcg(row + first + lane), w.s.slot) : 0;
        }
        if (n >= STAGES && !mbar_wait(empty(st), (n / STAGES - 1) & 1, s_abort, 201, true)) { more = false; break; }
        const int count = min(per, max(0, ((end << a.g.page_shift) - key0 + piece - 1) / piece));       // pieces of pages that it has
        if (elect_one()) mbar_expect_tx(full(st), (uint32_t)(count * piece * (a.g.k_row + a.g.v_row)));
        __syncwarp();
        for (int x = 0; x < per; ++x) {
          const int key = key0 + x * piece, pg = key >> a.g.page_shift;
          const int id = __shfl_sync(0xffffffffu, ids, (pg - first) & 31);
          if (pg < end && elect_one()) {
            const int r = ((id * n_kv + w.h) << a.g.page_shift) + (key & ((1 << a.g.page_shift) - 1));
            // both 64-channel halves of a piece by one copy, one behind the other
            const uint32_t kd = base + st * S::STAGE, vd = kd + S::K_BYTES + x * piece * 256;
            if (FP8) tma_load_2d(kd + x * piece * 128, &tm_k, full(st), 0, r);
            else tma_load_3d(kd + x * piece * 256, &tm_k, full(st), 0, r, 0);
            tma_load_3d(vd, &tm_v, full(st), 0, r, 0);
          }
        }
      }
      if (more) more = w.next(a, coming);
    }
    const Part none = {};
    if (!*s_abort) tell(none, 0);
    if (*s_abort) {                                    // copies in flight land before the block ends
      for (int i = max(0, n - STAGES); i < n; ++i) mbar_wait(full(i % STAGES), (i / STAGES) & 1, s_abort, 202, false);
      if (parts) mbar_wait(q_full, (parts - 1) & 1, s_abort, 205, false);
    }
  } else {
    // ---- arithmetic ----
    const int gid = lane >> 2, tig = lane & 3;
    // where the rows that a lane loads lie in a stage: piece after piece, a piece's first halves before its second ones
    const int krow = warp * 16 + (lane >> 4) * 8 + (lane & 7), vrow = warp * 16 + ((lane >> 3) & 1) * 8 + (lane & 7);
    const int piece = min(1 << a.g.page_shift, NARROW_KEYS), half_bytes = piece * 128;
    const int k_at = (krow / piece * piece + krow) * 128, v_at = (vrow / piece * piece + vrow) * 128;
    int* there = reinterpret_cast<int*>(sm + S::MISC + 16);
    int n = 0;
    for (int parts = 0;; ++parts) {
      // (a part is begun by all four warps or by none: they meet at barriers until its end)
      const bool here = mbar_wait(q_full, parts & 1, s_abort, 206, true);
      if (lane == 0) there[warp] = here;
      bar_sync(1, WARPS * 32);                         // and join and ml, of the part before, are free
      if (!(there[0] && there[1] && there[2] && there[3])) break;
      const Part w = *part;
      if (w.tiles == 0) break;
      const int nt = w.tiles;
      const float c = a.scale_log2 * (FP8 ? __ldcg(a.k_scale + w.h) : 1.0f);
      const int rows = w.ntok * G, lr0 = w.chunk * NARROW_ROWS;
      // the chunk's rows gid and gid + 8: token, keys it sees (rows that do not exist: none)
      int lim[2], tok[2];
      uint32_t qf[8][4];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int lr = lr0 + gid + 8 * i;
        tok[i] = lr / G;
        lim[i] = lr < rows ? max(0, w.len - w.ntok + tok[i] + 1) : 0;
      }
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) {
        if (FP8) {         // a lane's codes are four channels in a row: so are its queries'
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint2 v = *reinterpret_cast<const uint2*>(sm + S::Q + (gid + 8 * i) * Q_PITCH + ks * 32 + tig * 8);
            qf[ks][i] = v.x;
            qf[ks][2 + i] = v.y;
          }
        } else {
          ldsm4(base + S::Q + ((lane & 7) + ((lane >> 3) & 1) * 8) * Q_PITCH + ks * 32 + (lane >> 4) * 16, qf[ks]);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(q_empty);
      const int lr1 = min(lr0 + NARROW_ROWS, rows) - 1;                      // last row of the chunk
      const int tok_a = lr0 / G, tok_b = lr1 / G;
      const int lim_a = max(0, w.len - w.ntok + tok_a + 1), lim_b = max(0, w.len - w.ntok + tok_b + 1);
      float o[16][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < 16; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] = 0.0f;

      for (int t = 0; t < nt; ++t, ++n) {
        const int st = n % STAGES;
        const int key0 = w.pfx + (w.tile + t) * NARROW_KEYS + warp * 16;
        mbar_wait(full(st), (n / STAGES) & 1, s_abort, 203, true);
        if (key0 < lim_b) {
          const uint32_t ks_ = base + st * S::STAGE, vs_ = ks_ + S::K_BYTES;
          float x[2][4] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
          if (FP8) {
            // matrices: keys 0-7 and 8-15 of 16 channels, two steps of channels
            const int row = warp * 16 + ((lane >> 3) & 1) * 8 + (lane & 7);
#pragma unroll
            for (int ks = 0; ks < 8; ks += 2) {
              uint32_t b[4];
              ldsm4(ks_ + row * 128 + (((ks + (lane >> 4)) ^ (row & 7)) << 4), b);
              mma16(x[0], qf[ks], e4m3_pair(b[0]), e4m3_pair(b[0] >> 16));
              mma16(x[1], qf[ks], e4m3_pair(b[1]), e4m3_pair(b[1] >> 16));
              mma16(x[0], qf[ks + 1], e4m3_pair(b[2]), e4m3_pair(b[2] >> 16));
              mma16(x[1], qf[ks + 1], e4m3_pair(b[3]), e4m3_pair(b[3] >> 16));
            }
          } else {
            const int row = krow;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) {
              uint32_t b[4];
              const int ch = 2 * ks + ((lane >> 3) & 1);                      // 16-byte piece of the row
              ldsm4(ks_ + k_at + (ch >> 3) * half_bytes + (((ch & 7) ^ (row & 7)) << 4), b);
              mma16(x[0], qf[ks], b[0], b[1]);
              mma16(x[1], qf[ks], b[2], b[3]);
            }
          }
          const bool careful = key0 + 16 > lim_a;      // a row of the chunk does not see all of them
          float ref[2], corr[2], p[2][4];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int nb = 0; nb < 2; ++nb)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                float& v = x[nb][2 * i + e];
                v *= c;
                if (careful && key0 + nb * 8 + tig * 2 + e >= lim[i]) v = -INFINITY;
              }
            float mx = fmaxf(fmaxf(x[0][2 * i], x[0][2 * i + 1]), fmaxf(x[1][2 * i], x[1][2 * i + 1]));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
            mx = fmaxf(m[i], fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2)));
            ref[i] = mx == -INFINITY ? 0.0f : mx;                               // nothing seen so far: every p is 0
            corr[i] = ex2(m[i] - ref[i]);
            m[i] = mx;
          }
          if (__any_sync(0xffffffffu, corr[0] != 1.0f || corr[1] != 1.0f)) {
            l[0] *= corr[0];
            l[1] *= corr[1];
#pragma unroll
            for (int j = 0; j < 16; ++j) { o[j][0] *= corr[0]; o[j][1] *= corr[0]; o[j][2] *= corr[1]; o[j][3] *= corr[1]; }
          }
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int nb = 0; nb < 2; ++nb)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                p[nb][2 * i + e] = ex2(x[nb][2 * i + e] - ref[i]);
                l[i] += p[nb][2 * i + e];
              }
          // P rounded to bf16 for the tensor core (by half a step, up to 2^-8 of a weight); l keeps the weights unrounded
          uint32_t pf[4] = {pack2(p[0][0], p[0][1]), pack2(p[0][2], p[0][3]), pack2(p[1][0], p[1][1]), pack2(p[1][2], p[1][3])};
          if (!careful) {
#pragma unroll
            for (int jb = 0; jb < 8; ++jb) {
              uint32_t b[4];
              const int ch = 2 * jb + (lane >> 4);
              ldsm4_t(vs_ + v_at + (ch >> 3) * half_bytes + (((ch & 7) ^ (vrow & 7)) << 4), b);
              mma16(o[2 * jb], pf, b[0], b[1]);
              mma16(o[2 * jb + 1], pf, b[2], b[3]);
            }
          } else {
            // Keys that a row does not see count for nothing, whatever their V holds (0 x NaN would not): token by token with
            // the unseen keys' V cleared, and only that token's rows are taken.
            for (int tt = tok_a; tt <= tok_b; ++tt) {
              const int see = w.len - w.ntok + tt + 1 - key0;               // of the warp's 16 keys
              uint32_t keep[2];
#pragma unroll
              for (int e = 0; e < 2; ++e)
                keep[e] = (tig * 2 + 8 * e < see ? 0x0000ffffu : 0u) | (tig * 2 + 1 + 8 * e < see ? 0xffff0000u : 0u);
#pragma unroll
              for (int jb = 0; jb < 8; ++jb) {
                uint32_t b[4];
                const int ch = 2 * jb + (lane >> 4);
                ldsm4_t(vs_ + v_at + (ch >> 3) * half_bytes + (((ch & 7) ^ (vrow & 7)) << 4), b);
                float d0[4] = {0, 0, 0, 0}, d1[4] = {0, 0, 0, 0};
                mma16(d0, pf, b[0] & keep[0], b[1] & keep[1]);
                mma16(d1, pf, b[2] & keep[0], b[3] & keep[1]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  o[2 * jb][e] += tok[e >> 1] == tt ? d0[e] : 0.0f;
                  o[2 * jb + 1][e] += tok[e >> 1] == tt ? d1[e] : 0.0f;
                }
              }
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(empty(st));
      }

      // ---- the part's end: four warps' rows joined ----
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
        l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
      }
      float2* ml = reinterpret_cast<float2*>(sm + S::ML);
      float* join = reinterpret_cast<float*>(sm + S::JOIN);
      if (tig == 0) {
        ml[warp * 16 + gid] = make_float2(m[0], l[0]);
        ml[warp * 16 + gid + 8] = make_float2(m[1], l[1]);
      }
      const bool sole = w.sole;
      const int64_t slot = w.slot;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (lr0 + 8 * i >= rows) break;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          bar_sync(1, WARPS * 32);
#pragma unroll
          for (int j = 0; j < 8; ++j)
            *reinterpret_cast<float2*>(join + (warp * 8 + gid) * O_STRIDE + j * 8 + tig * 2) =
                make_float2(o[half * 8 + j][2 * i], o[half * 8 + j][2 * i + 1]);
          bar_sync(1, WARPS * 32);
          const int r8 = threadIdx.x >> 4, ch = (threadIdx.x & 15) * 4, r = 8 * i + r8, lr = lr0 + r;
          if (lr < rows) {
            float2 e[WARPS];
            float top = -INFINITY, sum = 0.0f;
#pragma unroll
            for (int k = 0; k < WARPS; ++k) {
              e[k] = ml[k * 16 + r];
              top = fmaxf(top, e[k].x);
            }
            const float at = top == -INFINITY ? 0.0f : top;
            float4 acc = make_float4(0, 0, 0, 0);
#pragma unroll
            for (int k = 0; k < WARPS; ++k) {
              const float f = ex2(e[k].x - at);
              const float4 v = *reinterpret_cast<const float4*>(join + (k * 8 + r8) * O_STRIDE + ch);
              sum += e[k].y * f;
              acc.x += v.x * f; acc.y += v.y * f; acc.z += v.z * f; acc.w += v.w * f;
            }
            const int hc = half * 64 + ch;
            if (sole) {
              const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
              const int64_t row = (int64_t)(w.tok0 + lr / G) * a.n_q_heads + w.h * G + lr % G;
              const uint2 v = make_uint2(pack2(acc.x * inv, acc.y * inv), pack2(acc.z * inv, acc.w * inv));
              *reinterpret_cast<uint2*>(a.out + row * 128 + hc) = v;
              if (a.lse && half == 0 && ch == 0) a.lse[row] = (at + log2f(sum)) * 0.6931471805599453f;
            } else {
              *reinterpret_cast<float4*>(a.w.o + (slot * NARROW_ROWS + r) * 128 + hc) = acc;
              if (half == 0 && ch == 0) a.w.ml[slot * NARROW_ROWS + r] = make_float2(top, sum);
            }
          }
        }
      }
    }
  }
  __syncthreads();
  if (threadIdx.x == 0 && *s_abort) atomicCAS(a.err, 0, *s_abort);
  if (beside) pdl_wait_predecessor();                  // the end of this kernel is the end of all before it
}

}  // namespace

asl_status asl_launch_attend_narrow(asl_ctx* c, const asl_pages* p, const AttendArgs& a, int grid, bool beside, cudaStream_t st) {
  const bool fp8 = p->k_dtype == ASL_K_FP8_E4M3;
  const cuuint64_t n_rows = (cuuint64_t)p->n_pages * p->n_kv_heads * p->page_size;
  const cuuint32_t piece = p->page_size < NARROW_KEYS ? p->page_size : NARROW_KEYS;
  CUtensorMap tm_k, tm_v;
  // E4M3 rows are 128 bytes; bf16 rows two halves of that, the outermost dimension
  const cuuint64_t dims8[2] = {128, n_rows}, stride8[1] = {128};
  const cuuint64_t dims[3] = {64, n_rows, 2}, strides[2] = {256, 128};
  const cuuint32_t box8[2] = {128, piece}, box[3] = {64, piece, 2};
  const bool k_map = fp8 ? asl_make_map(&tm_k, CU_TENSOR_MAP_DATA_TYPE_UINT8, a.g.k, 2, dims8, stride8, box8)
                         : asl_make_map(&tm_k, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, a.g.k, 3, dims, strides, box);
  if (!k_map || !asl_make_map(&tm_v, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, a.g.v, 3, dims, strides, box)) return ASL_ERR_CUDA;
  auto kernel = fp8 ? attend_narrow_kernel<true> : attend_narrow_kernel<false>;
  const int smem = fp8 ? NarrowSmem<true>::BYTES : NarrowSmem<false>::BYTES;
  launch_after_smem(kernel, dim3(grid), dim3(WARPS * 32 + 32), smem, st, tm_k, tm_v, a, beside);
  c->launches += 1;
  ASL_CUDA(cudaGetLastError());
  return ASL_OK;
}

asl_status asl_attend_narrow_ready() {
  ASL_CUDA(cudaFuncSetAttribute(attend_narrow_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, NarrowSmem<false>::BYTES));
  ASL_CUDA(cudaFuncSetAttribute(attend_narrow_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, NarrowSmem<true>::BYTES));
  return ASL_OK;
}
