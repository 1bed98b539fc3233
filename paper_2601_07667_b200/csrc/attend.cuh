// Attention over pages: the plan on the device, and where the parts of rows whose keys are split lie in the workspace.
//
// Work is two rows of tiles, one behind another, that are cut into equal stretches, one per CTA:
//   narrow  the keys a sequence reads by itself, [pfx, len): chunks of 16 (token, query head) rows of one kv head, tiles of
//           64 keys; per kv head sum over sequences of chunks x tiles.
//   wide    the prefixes that groups of neighbours share, [0, pfx): chunks of up to 256 rows of the group, tiles of 128 keys
//           that count 2 where a chunk has more than 128 rows (both halves multiply) and 1 else (the halves take keys in turn).
//           Where a group has several chunks its keys are cut into stripes of about a CTA's stretch, and a stripe's chunks come
//           one behind another: CTAs that read the same keys do so at the same time, once from HBM and then from L2.
// A CTA's stretch of a chunk (of a stripe) is a part; parts of a chunk have the running maximum, the sum and the unnormalised result of
// their keys, and lie at (number of the chunk + number of the CTA): either grows by one from part to part.
#pragma once
#include "pages.cuh"

constexpr int NARROW_ROWS = 16, NARROW_KEYS = 64;
constexpr int WIDE_ROWS = 256, WIDE_KEYS = 128;
constexpr int ATTEND_MAX_SEQS = 4096;

struct __align__(16) AttendHead {        // one per plan, on the device
  int32_t mark, n_seqs, n_tokens, n_q_heads;          // what the layout follows from: see plan_fits
  int32_t n_kv_heads, page_shift, narrow_tiles, narrow_chunks;       // tiles and chunks per kv head
  int32_t narrow_each, wide_cost, wide_chunks, wide_each;      // tiles and cost per CTA; cost and chunks per kv head
  int32_t max_seqs, max_pages;             // of the cache whose slots the plan names, and its table
  const int32_t* table;
};
static_assert(sizeof(AttendHead) == 64, "load_head reads four vectors");
constexpr int ATTEND_MARK = 0x41534c50;
struct __align__(16) AttendSeq {
  int32_t tok0, ntok, slot, len;       // ntok 0: padding
  int32_t pfx, tile0, chunk0, group;   // shared tokens read by the group; narrow tiles and chunks before
};
struct __align__(16) AttendGroup {
  int32_t tok0, ntok, slot, pfx;
  int32_t cost0, chunk0, stripe, pad0; // wide cost and chunks (of stripes) before; tiles of a stripe
};
// What the joining of a token's rows needs to know, in one round trip (seq.ntok 0: nobody's token).
struct __align__(16) AttendToken { AttendSeq seq; AttendGroup group; };
// Where a CTA's stretch begins (h < 0: it has none), with all that it needs to know there: one round trip to memory.
struct __align__(16) AttendStart {
  int32_t h, item, chunk, tile;
  union { AttendSeq seq; AttendGroup group; };
  int32_t items, total, chunks, more;  // sequences or groups; tiles or cost, and chunks, per kv head; tiles per CTA, or the stripe
};

struct AttendLayout {      // byte offsets in the workspace
  size_t head, open, seqs, groups, same, tokens, narrow_start, wide_start, ml, o, total;
  int64_t wide_row0;
  int32_t narrow_grid, wide_grid;
};

struct AttendPtrs {
  AttendHead* head;
  uint32_t* open;          // 1 while the prefixes' kernel of a call has seen the end of all before it, else 0 (see narrow_may_read)
  AttendSeq* seqs;
  AttendGroup* groups;
  int32_t* same;           // [n_seqs] leading pages that an entry has in common with the one before
  AttendToken* tokens;     // [n_tokens]
  AttendStart* narrow_start;
  AttendStart* wide_start;
  float2* ml;              // of every part's rows: 16 of a narrow slot, then, from wide_row0 on, 256 of a wide one:
  float* o;                // (maximum in powers of two, sum); [128] unnormalised result
  int64_t wide_row0;
};

struct AttendArgs {
  PagePool g;
  AttendPtrs w;
  const __nv_bfloat16* q;
  int64_t qs_t, qs_h;      // element strides
  __nv_bfloat16* out;
  float* lse;              // or null
  const float* k_scale;    // [H_k] of the layer, or null; the kernel before may write it, so that it is read by coherent loads
  int32_t* err;            // the context's word of bounded waits
  int32_t n_q_heads, group_heads, n_tokens, n_seqs;
  int32_t with_wide;       // the prefixes' kernel is launched
  float scale_log2;
};

// Tokens of a chunk of a group's rows (at least two, since a token has at most 128).
ASL_HD inline int wide_tokens(int G) { return WIDE_ROWS / G; }

// A group's tiles, chunks and cost.  All chunks but the last have as many tokens as fit (and more than 128 rows).
struct WideShape {
  int tiles, whole, rest, chunks, stripe, stripes;
  int sum;                                 // cost of one tile of every chunk
  ASL_HD inline WideShape(int ntok, int pfx, int G, int stripe_) {
    const int T = wide_tokens(G);
    tiles = (pfx + WIDE_KEYS - 1) / WIDE_KEYS;
    whole = ntok / T;
    rest = ntok - whole * T;
    chunks = whole + (rest > 0);
    sum = 2 * whole + (rest ? weight_of(rest, G) : 0);
    stripe = chunks > 1 && stripe_ < tiles ? stripe_ : tiles;        // (so that stripe x sum is no more than the group's cost)
    stripes = tiles ? (tiles + stripe - 1) / stripe : 0;
  }
  static ASL_HD inline int weight_of(int tokens, int G) { return tokens * G > WIDE_ROWS / 2 ? 2 : 1; }
  ASL_HD inline int weight(int chunk, int G) const { return chunk < whole ? 2 : weight_of(rest, G); }
  ASL_HD inline int tiles_of(int s) const { return tiles - s * stripe < stripe ? tiles - s * stripe : stripe; }
  // cost before a chunk of a stripe
  ASL_HD inline int before(int s, int chunk) const { return s * stripe * sum + tiles_of(s) * 2 * chunk; }
};

#ifdef __CUDACC__
// The kernel of the sequences' own keys runs beside the prefixes' one, which has waited for all before it and writes nothing that
// it reads.  griddepcontrol makes earlier grids' writes visible only behind a wait of its own, which would be for the end of the
// prefixes' kernel too (five prefixes' cases: 115 -> 121, 159 -> 169, 355 -> 373, 137 -> 149, 67 -> 73 us).  So the one that has
// waited says so by a release, behind which all that it may see is seen by who acquires it; who does not find it said waits.  The
// kernel that joins the parts takes it back.
__device__ __forceinline__ void others_may_read(uint32_t* open) { asm volatile("st.release.gpu.global.u32 [%0], 1;" ::"l"(open) : "memory"); }
__device__ __forceinline__ bool narrow_may_read(const uint32_t* open) {        // by a whole warp
  uint32_t v;
  asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(open) : "memory");
  asm volatile("fence.proxy.async;" ::: "memory");                             // (its copies read by the async proxy)
  return __all_sync(0xffffffffu, v == 1u);
}
// Every warp reads the head, behind its kernel's wait (or acquire) for the one that wrote it: by loads that L1 keeps, since thousands
// of requests for one line wait for one another in L2 (the joined rows of 32 sequences with 32 heads: 13 us, of which 8.7 were these loads).
__device__ __forceinline__ AttendHead load_head(const AttendHead* h) {
  AttendHead r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    int4& q = reinterpret_cast<int4*>(&r)[i];
    asm volatile("ld.global.ca.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "l"(reinterpret_cast<const int4*>(h) + i) : "memory");
  }
  return r;
}
// A workspace that holds no plan, or one for other sizes or another cache (whose slots this one's table may not have), is refused
// before anything is read through it, and so is one with shared prefixes where their kernel is not launched.
__device__ __forceinline__ bool plan_fits(const AttendArgs& a, const AttendHead& h) {
  const bool fits = h.mark == ATTEND_MARK && h.n_seqs == a.n_seqs && h.n_tokens == a.n_tokens && h.n_q_heads == a.n_q_heads &&
                    h.n_kv_heads == a.g.n_kv_heads && h.page_shift == a.g.page_shift && h.max_seqs == a.g.max_seqs &&
                    h.max_pages == a.g.max_pages && h.table == a.g.table && (h.wide_cost == 0 || a.with_wide);
  if (!fits && threadIdx.x == 0) note_error(a.g.err, ASL_ERR_WORKSPACE, -1);
  return fits;
}
__device__ __forceinline__ AttendStart load_start(const AttendStart* s) {
  AttendStart r;
#pragma unroll
  for (int i = 0; i < 4; ++i) reinterpret_cast<int4*>(&r)[i] = __ldcg(reinterpret_cast<const int4*>(s) + i);
  return r;
}
__device__ __forceinline__ AttendSeq load_seq(const AttendSeq* s) {
  AttendSeq r;
  reinterpret_cast<int4*>(&r)[0] = __ldcg(reinterpret_cast<const int4*>(s));
  reinterpret_cast<int4*>(&r)[1] = __ldcg(reinterpret_cast<const int4*>(s) + 1);
  return r;
}
__device__ __forceinline__ AttendGroup load_group(const AttendGroup* s) {
  AttendGroup r;
  reinterpret_cast<int4*>(&r)[0] = __ldcg(reinterpret_cast<const int4*>(s));
  reinterpret_cast<int4*>(&r)[1] = __ldcg(reinterpret_cast<const int4*>(s) + 1);
  return r;
}
// A page number out of a table: one that the pool does not have is noted, and page 0 read in its place.
__device__ __forceinline__ int page_in_pool(const PagePool& g, int id, int slot) {
  if ((unsigned)id < (unsigned)g.n_pages) return id;
  note_error(g.err, ASL_ERR_INVALID, slot);
  return 0;
}
__device__ __forceinline__ int narrow_tiles_of(const AttendSeq& s) { return max(1, (s.len - s.pfx + NARROW_KEYS - 1) / NARROW_KEYS); }
__device__ __forceinline__ int narrow_chunks_of(int ntok, int G) { return (ntok * G + NARROW_ROWS - 1) / NARROW_ROWS; }
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// Two E4M3 codes (the lower 16 bits) as bf16, exactly: bits moved into place, then times 2^(127-7), which also makes the
// subnormal codes' values; a NaN code (0x7f, 0xff) comes out as 480, the value its bits would have, and is not in a cache.
__device__ __forceinline__ uint32_t e4m3_pair(uint32_t two) {
  const uint32_t w = __byte_perm(two, 0, 0x1404);                         // codes in the upper bytes of the halves
  const uint32_t b = (w & 0x80008000u) | ((w & 0x7f007f00u) >> 4);
  uint32_t r;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(b), "r"(0x7b807b80u), "r"(0x80008000u));   // x 2^120 (+ -0)
  return r;
}

#endif

// `beside`: right behind the prefixes' kernel, whose end it does not wait for
asl_status asl_launch_attend_narrow(asl_ctx* c, const asl_pages* p, const AttendArgs& a, int grid, bool beside, cudaStream_t st);
asl_status asl_launch_attend_wide(asl_ctx* c, const asl_pages* p, const AttendArgs& a, int grid, cudaStream_t st);
// The kernels' shared memory on the current device, once per context.
asl_status asl_attend_narrow_ready();
asl_status asl_attend_wide_ready();
