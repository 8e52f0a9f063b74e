// Decode attention of a batch whose sequences share a prefix (spkv_decode_attention_shared).
//
// Three launches:
//   prefix  the compact-cache pages that all sequences have in common, once for the batch: the B * G query
//           rows of a KV head are the M side of tcgen05 tiles, a block takes 128 or 256 of them over one
//           share of the head's common pages and leaves (m, l, O) per row;
//   tail    what is left of every unit, its own pages and its ring: one small block per unit (several for a long
//           one), mma.sync tiles of the unit's G query heads as in the decode kernel; leaves (m, l, O) too;
//   merge   joins a row's parts by their log-sum-exp weights.
// The tail does not depend on the prefix launch.  Its blocks are small (4 warps, two page buffers), so that with up to 8
// query heads per KV head (96 registers a thread) one fits on an SM beside a prefix block; with 9 - 16 (168 registers)
// it does not and the tail runs as the prefix blocks leave.  They are launched as programmatic dependents: the prefix
// kernel has waited for everything earlier on the stream before it lets them start.
// The tail launch is not complete before the prefix launch is, so that the merge, which waits for the tail,
// may read both.
//
// Prefix kernel.  Per page and 128-row slot: S = Q K^T (8 MMAs M128 N64 K16 into tensor memory), softmax
// in registers (thread = row = TMEM lane), P in fp16 back over the scores, O += P V with the page's values
// rescaled to fp16 by converter warps, or two bf16 terms for a unit of wide-ranging values
// (value_scale).  No masks: common pages are full and every query sees all of them.
// One fp16 term: a weight is rounded by at most 2^-11 of itself, so an output by at most 2^-11 sum w|v| before its own
// rounding to bf16 (2^-8), and by far less where roundings average out.  Two bf16 terms (2^-16, what the tail's
// mma.sync tiles take) would double P.V's MMAs and P's stores in the chain that bounds the kernel;
// SPKV_FLAG_PREFILL_PV_BF16 asks for them.
//   * More than 128 rows in the tile (kAlt = false): slot h holds rows [128 h, 128 h + 128), both walk
//     every page.
//   * At most 128 rows (kAlt): both slots hold the same rows and take alternate pages, which halves the
//     softmax time per page.  One of the two is joined into the other through shared memory at the end.
// Shared memory: Q (64 KB; kAlt 32 KB) + rings of 3 (4) key and 3 (4) value blocks, which leaves 66 KB to a tail
// block.  Tensor memory: score buffer b of slot h at
// [64 (2h + b), +64), O of slot h at [256 + 128 h, +128).
// Warps: 0 / 2 MMA issue of slot 0 / 1, 1 page loader, 3 tensor memory, 4-7 / 8-11 softmax of slot 0 / 1, 12-15 value
// conversion.  All waits are bounded.
//
// What bounds it (B200; device time of a call in a graph, three caches in turn): up to 128 rows, memory while the pages
// stream (8 sequences of 64/8 heads on 65536 common tokens, 59 MB: 19.6 us, of which 10 at 5.8 TB/s, 3 until
// the first scores, 6 for the end of the tail and the merge); beyond, the chain scores -> softmax -> P -> MMA
// (2050 cycles per page and 256 rows; the tensor pipe is busy half of that) and then the tail's mma.sync tiles, which
// get little of the tensor pipe beside the prefix (64 sequences of 32/8 heads on 131072: 36.9 us).
#include <algorithm>
#include <atomic>
#include <math.h>

#include "spkv_share.cuh"
#include "spkv_tc5.cuh"

namespace spkv {

namespace shp {
// Sixteen warps, four on each of the SM's register files: at 104 registers a thread a tail block of four warps of
// 96 finds room beside them (with 13 warps of 128 one file was full, and the tail ran after the prefix).  At 104 the two
// prefix kernels spill 36 and 68 bytes a thread.
// (Two converter warps instead of four, or the MMA warps on other schedulers: within 2 %.)
constexpr int kThreads = 512, kRegs = 104;
constexpr int kMmaWarp0 = 0, kLoaderWarp = 1, kMmaWarp1 = 2, kTmemWarp = 3;
constexpr int kConvThreads = 128;   // warps 12-15
constexpr int kTmemCols = 512;
constexpr float kPBias = 7.f;   // P is stored as 2^7 p
enum { B_K_FULL = 0, B_K_EMPTY = 4, B_V_FULL = 8, B_V_EMPTY = 12, B_V_READY = 16, B_S_FULL = 20 /* [2h+b] */, B_P_FULL = 24,
       B_O_DONE = 28, B_COUNT = 32 };
// Key and value blocks travel in rings of their own: a key block is free again as soon as the scores are made, two
// pages before the values of its page are needed, so nearly every buffer has a copy in flight (a page
// takes about 2 us to arrive under load; in one ring of four whole pages three were in use, one in flight).
__host__ __device__ constexpr int ring(bool alt) { return alt ? 4 : 3; }   // key blocks; as many value blocks
constexpr int kBlockBytes = kPageBytes / 2;
// keys are loaded this many pages ahead of values: as far as a slot's scores run ahead of its P.V
__host__ __device__ constexpr int key_lead(bool alt) { return alt ? 4 : 2; }
__host__ __device__ constexpr int off_k(bool alt) { return alt ? 32768 : 65536; }
__host__ __device__ constexpr int off_v(bool alt) { return off_k(alt) + ring(alt) * kBlockBytes; }
__host__ __device__ constexpr int off_bar(bool alt) { return off_v(alt) + ring(alt) * kBlockBytes; }
__host__ __device__ constexpr int smem_bytes(bool alt) { return off_bar(alt) + 512; }
constexpr int kRowStride = 132;   // floats per row of the results in shared memory
}  // namespace shp

struct SharedArgs {
  CacheView c;
  int layer, B, n_items, n_tiles, rows_per_block, sig;
  unsigned long long g_inv;     // ceil(2^32 / G): row / G as a product and a shift (rows < 2^15, G <= 16)
  const int32_t *seq_ids;
  const __nv_bfloat16 *q;       // [B][Hq][128]
  const int32_t *rec;           // the layer's record of the plan
  float scale_log2;
  int force_wide;
  float *part_o, *part_ml;      // prefix: [block][rows_per_block][128], [block][rows_per_block][2]: m (log2 domain), l
  int max_blocks;
  float *tail_o, *tail_ml;      // tail: [share][item][G][128], [share][item][G][2]
  int max_tail;                 // shares the workspace holds
  int tail_blocks;              // blocks of the tail launch that take items; those behind join prefix parts
  float *pre_o, *pre_ml;        // a query row's prefix parts joined: [B * Hq][128], [B * Hq][2]
  int row_base, row_heads;      // page-table rows of the layer: row_base + seq * row_heads + rank of the KV head
  unsigned long long local_mask;
  int32_t *item_skip;           // [n_items] common pages the tail left out (0: it read the unit in full)
  __nv_bfloat16 *out;
  float *lse;
};

// Weight of a part (m, l) against the common maximum M >= m.  A part without a visible key has m = -inf and
// l = 0; m = -inf with another l means that its scores were NaN (a maximum passes over NaN), which stays NaN.
__device__ inline float part_weight(float m, float l, float M) {
  return m == -INFINITY ? (l == 0.f ? 0.f : NAN) : fast_exp2(m - M);
}
__device__ inline int4 ldcg4(const int32_t *p) { return __ldcg(reinterpret_cast<const int4 *>(p)); }

// key (half = 0) or value block of page j of a share into its ring (one thread)
template <bool kAlt>
__device__ inline void load_block(const SharedArgs &a, unsigned char *smem, uint64_t *bar, int half, int j, int gp, uint64_t pol) {
  using namespace shp;
  const int s = j % ring(kAlt);
  unsigned char *dst = smem + (half ? off_v(kAlt) : off_k(kAlt)) + s * kBlockBytes;
  const __nv_bfloat16 *src = a.c.pages + (int64_t)gp * kPageElems + half * kBlockElems;
  uint64_t *full = &bar[(half ? B_V_FULL : B_K_FULL) + s];
  mbar_arrive_expect_tx(full, kBlockBytes);
  // a page that several row tiles read stays in L2 for the others
  if (a.n_tiles == 1) bulk_load_hint(dst, src, kBlockBytes, full, pol);
  else bulk_load(dst, src, kBlockBytes, full);
}

template <bool kAlt>
__global__ void __maxnreg__(shp::kRegs) shared_prefix_kernel(SharedArgs a) {
  using namespace tc5;
  using namespace shp;
  constexpr int kRing = ring(kAlt), kKeyLead = key_lead(kAlt);
  constexpr int kAhead = 2;                  // how many of a slot's pages its scores run ahead of P.V
  extern __shared__ __align__(1024) unsigned char smem[];
  const CacheView &c = a.c;
  uint64_t *bar = reinterpret_cast<uint64_t *>(smem + off_bar(kAlt));
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bar + B_COUNT);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  volatile int *s_desc = reinterpret_cast<volatile int *>(tmem_slot + 1);   // [8] descriptor, [8] share is valid, [9] vmax
  // ---- block-local set-up, then this block's share.  The loader warp goes ahead: descriptor (one trip to
  // memory), page-table entries (the second), first pages; the others load Q meanwhile.
  if (warp == kLoaderWarp && lane == 0) {
    for (int i = 0; i < kRing; ++i) {
      mbar_init(&bar[B_K_FULL + i], 1);
      mbar_init(&bar[B_V_FULL + i], 1);
      mbar_init(&bar[B_V_READY + i], kConvThreads);
    }
    // per slot and parity of the slot's page count: one phase per two of its pages
    for (int i = 0; i < 4; ++i) {
      mbar_init(&bar[B_S_FULL + i], 1);
      mbar_init(&bar[B_P_FULL + i], 128);
      mbar_init(&bar[B_O_DONE + i], 1);
    }
  }
  pdl_wait();
  pdl_trigger();   // (only now: what follows may then rely on everything before this launch)
  if (warp == kLoaderWarp) {
    // (pages were written through generic stores)
    asm volatile("fence.proxy.async;" ::: "memory");
    const int32_t *dp = share_desc(c, a.rec, blockIdx.x);
    if (lane < 8) s_desc[lane] = __ldcg(dp + lane);
    __syncwarp();
    // one commit per MMA warp that uses a page
    if (lane == 0) {
      const int left = a.B * c.G - s_desc[1] * kShareRows;
      for (int i = 0; i < kRing; ++i) {
        mbar_init(&bar[B_K_EMPTY + i], (!kAlt && left > 128) ? 2 : 1);
        mbar_init(&bar[B_V_EMPTY + i], (!kAlt && left > 128) ? 2 : 1);
      }
      mbar_fence_init();
    }
  }
  __syncthreads();
  const int kvh = s_desc[0], tile = s_desc[1], j_begin = s_desc[2], n_pages = s_desc[3];
  const int common = s_desc[4], trow = s_desc[5], u = s_desc[6];
  const int row_base = tile * kShareRows, n_rows = min(kShareRows, a.B * c.G - row_base);
  // (no work, another batch's plan, or not a plan at all)
  if (n_pages <= 0 || s_desc[7] != a.sig || kvh < 0 || kvh >= c.Hkv || n_rows <= 0 || j_begin < 0 ||
      j_begin + n_pages > min(common, c.max_pages) || u < 0 || u >= c.n_units || trow < 0 || trow >= c.n_units)
    return;
  const bool two = kAlt ? n_pages > 1 : n_rows > 128;     // is slot 1 in use
  uint64_t pol = 0;
  int first_entry = 0;
  if (warp == kLoaderWarp) {
    pol = l2_evict_first_policy();
    const int len = ldcg_keep(&c.len[u]);
    const uint32_t vm = __ldcg(&c.vmax[u]);
    if (lane < n_pages) first_entry = ldcg_keep(&unit_table(c, trow)[j_begin + lane]);
    // (stale plan: the unit is shorter by now; the tail sees the same and nobody reads this share's result)
    const bool valid = len / kP >= common;
    if (valid && lane < n_pages) first_entry = checked_page(c, first_entry, (int)ring_page(c, u, 0));   // (the others hold none)
    // the keys that the first scores need; the rest follows when Q is in place (every block's rings at once are 20 MB
    // of requests, behind which the tail's first look at its units would wait 3 us)
    for (int j = 0; j < kKeyLead && valid; ++j) {
      const int gk = __shfl_sync(0xffffffffu, first_entry, j);
      if (lane == 0 && j < n_pages) load_block<kAlt>(a, smem, bar, 0, j, gk, pol);
    }
    if (lane == 0) { s_desc[8] = valid; s_desc[9] = (int)vm; }
  } else {
    // Q rows -> two slabs of 128 rows x 128 B per slot, 128-byte swizzle; rows past the last are zero
    // (asynchronous copies, all in flight at once: as loads, one after the other, they took 3 us, 7 for two slots)
    const int qt = warp == 0 ? lane : tid - 32;   // the threads but for the loader warp
    for (int x = qt; x < (kAlt ? 1 : 2) * 128 * 16; x += kThreads - 32) {
      const int tr = x >> 4, h = x >> 11, r = tr & 127, ch = x & 15;   // row of the tile; slot, row in it, chunk
      const int R = row_base + min(tr, n_rows - 1), b = (int)(((unsigned long long)R * a.g_inv) >> 32), g = R - b * c.G;
      const __nv_bfloat16 *src = a.q + ((size_t)b * c.Hq + kvh * c.G + g) * kD + ch * 8;
      const uint32_t dst = smem_u32(smem + h * 32768 + (ch >> 3) * 16384 + r * 128 + (((ch & 7) ^ (r & 7)) << 4));
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(tr < n_rows ? 16 : 0) : "memory");
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    fence_async_smem();
    if (warp == kTmemWarp) {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                   "n"(kTmemCols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tbase = *tmem_slot;
  const bool valid = s_desc[8] != 0;
  float v_scale, v_unscale;
  const bool wide = value_scale((uint32_t)s_desc[9], a.force_wide, v_scale, v_unscale);
  bool failed = false;
  // pages of slot h: local page i is page h + 2 i of the share (kAlt), or page i
  auto slot_pages = [&](int h) { return kAlt ? (n_pages + 1 - h) / 2 : (h == 0 || two ? n_pages : 0); };
  auto page_of = [&](int h, int i) { return kAlt ? 2 * i + h : i; };

  if (!valid) {
    // nothing to do but to give the tensor memory back
  } else if (warp == kLoaderWarp) {
    // ---------------------------------------------------------------- page loader
    // step j: the keys of page j, the values of page j - kKeyLead
    int entry = first_entry, older = 0;   // global page indices of this lane in the current and the previous 32 pages
    int j = kKeyLead;
    auto wait_empty = [&](int which, int jj) {
      return jj < kRing || mbar_wait_bounded(&bar[which + jj % kRing], ((jj / kRing) - 1) & 1);
    };
    for (; j < n_pages + kKeyLead; ++j) {
      if ((j & 31) == 0) {
        older = entry;
        if (j + lane < n_pages)
          entry = checked_page(c, ldcg_keep(&unit_table(c, trow)[j_begin + j + lane]), (int)ring_page(c, u, 0));
      }
      const int jv = j - kKeyLead;
      const int gk = __shfl_sync(0xffffffffu, entry, j & 31);
      const int gv = __shfl_sync(0xffffffffu, (jv >> 5) == (j >> 5) ? entry : older, jv & 31);
      if (lane == 0) {
        if (jv >= 0 && jv < n_pages) {
          failed = !wait_empty(B_V_EMPTY, jv);
          if (!failed) load_block<kAlt>(a, smem, bar, 1, jv, gv, pol);
        }
        if (!failed && j < n_pages) {
          failed = !wait_empty(B_K_EMPTY, j);
          if (!failed) load_block<kAlt>(a, smem, bar, 0, j, gk, pol);
        }
      }
      failed = __shfl_sync(0xffffffffu, (int)failed, 0) != 0;
      if (failed) break;
    }
    if (failed && lane == 0) {   // do not leave while copies may still be landing
      for (int k = max(0, j - kRing); k < min(j, n_pages); ++k) mbar_wait_bounded(&bar[B_K_FULL + (k % kRing)], (k / kRing) & 1);
      for (int k = max(0, j - kKeyLead - kRing); k < min(j - kKeyLead + 1, n_pages); ++k)
        mbar_wait_bounded(&bar[B_V_FULL + (k % kRing)], (k / kRing) & 1);
    }
  } else if (warp == kMmaWarp0 || warp == kMmaWarp1) {
    // ---------------------------------------------------------------- MMA issue (whole warp, one elected lane issues)
    const int h = warp == kMmaWarp1, n_mine = slot_pages(h);
    constexpr uint32_t idesc_qk = instr_desc(128, 64, false), idesc_pv = instr_desc(128, 128, true, true),
                       idesc_pv_bf16 = instr_desc(128, 128, true, false);
    constexpr uint32_t kUnits = kBlockBytes >> 4;   // a block in descriptor address units
    const uint64_t dQ = smem_desc(smem_u32(smem + (kAlt ? 0 : h * 32768)), 16, 1024);
    const uint64_t dK = smem_desc(smem_u32(smem + off_k(kAlt)), 16, 1024), dV = smem_desc(smem_u32(smem + off_v(kAlt)), 8192, 1024);
    auto issue_qk = [&](int i) {   // S = Q . K^T of the slot's page i into score buffer i & 1, committed at once
      const int j = page_of(h, i), s = j % kRing, b = i & 1;
      if (!mbar_wait_bounded(&bar[B_K_FULL + s], (j / kRing) & 1)) { failed = true; return; }
      fence_after();
      umma_qk_page<16384 / 16, 8192 / 16>(tbase + (2 * h + b) * 64, dQ, dK + (uint64_t)s * kUnits, idesc_qk);
      umma_commit(&bar[B_S_FULL + 2 * h + b]);
      umma_commit(&bar[B_K_EMPTY + s]);    // this slot has no use for the keys any more
    };
    for (int i = 0; i < min(kAhead, n_mine) && !failed; ++i) issue_qk(i);
    for (int i = 0; i < n_mine && !failed; ++i) {
      const int j = page_of(h, i), s = j % kRing, b = i & 1;
      if (!mbar_wait_bounded(&bar[B_V_READY + s], (j / kRing) & 1)) { failed = true; break; }
      if (!mbar_wait_bounded(&bar[B_P_FULL + 2 * h + b], (i >> 1) & 1)) { failed = true; break; }
      fence_after();
      const uint32_t t_p = tbase + (2 * h + b) * 64, t_o = tbase + 256 + h * 128;
      if (wide) umma_pv_page(t_o, t_p, dV + (uint64_t)s * kUnits, idesc_pv_bf16, i > 0 ? 1u : 0u);
      else umma_pv_page_f16(t_o, t_p, dV + (uint64_t)s * kUnits, idesc_pv, i > 0 ? 1u : 0u);
      umma_commit(&bar[B_V_EMPTY + s]);    // ... nor for the values
      if (i + kAhead < n_mine) issue_qk(i + kAhead);   // (behind P.V(i): the pipe runs a thread's instructions in order)
      else umma_commit(&bar[B_O_DONE + 2 * h + b]);
    }
  } else if (warp >= 12) {
    // ---------------------------------------------------------------- value converter: bf16 -> scaled fp16, in place
    for (int j = 0; j < n_pages; ++j) {
      const int s = j % kRing;
      if (!mbar_wait_bounded(&bar[B_V_FULL + s], (j / kRing) & 1)) { failed = true; break; }
      uint4 *vb = reinterpret_cast<uint4 *>(smem + off_v(kAlt) + s * kBlockBytes) + (tid - 384);
#pragma unroll
      for (int x = 0; x < (wide ? 0 : 1024 / kConvThreads); ++x) {
        uint4 r = vb[x * kConvThreads];
        r.x = bf16x2_to_f16x2(r.x, v_scale); r.y = bf16x2_to_f16x2(r.y, v_scale);
        r.z = bf16x2_to_f16x2(r.z, v_scale); r.w = bf16x2_to_f16x2(r.w, v_scale);
        vb[x * kConvThreads] = r;
      }
      fence_async_smem();
      mbar_arrive(&bar[B_V_READY + s]);
    }
  } else if (warp >= 4) {
    // ---------------------------------------------------------------- softmax of slot 0 (warps 4-7) and slot 1 (8-11)
    const int h = (warp >> 2) - 1, row = tid & 127, n_mine = slot_pages(h);
    const uint32_t t_lane = tbase + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t t_o = t_lane + 256 + h * 128;
    // a warp without a single live row only keeps the barriers going
    const bool live = (kAlt ? 0 : h * 128) + (row & ~31) < n_rows;
    float m_ref = -INFINITY, l = 0.f;
    for (int i = 0; i < n_mine; ++i) {
      const int b = i & 1;
      if (!mbar_wait_bounded(&bar[B_S_FULL + 2 * h + b], (i >> 1) & 1)) { failed = true; break; }
      fence_after();
      if (!live) { fence_before(); mbar_arrive(&bar[B_P_FULL + 2 * h + b]); continue; }
      const uint32_t t_s = t_lane + (2 * h + b) * 64;
      float v[64];
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        float t16[16];
        tmem_ld16(t_s + q4 * 16, t16);
#pragma unroll
        for (int x = 0; x < 16; ++x) v[q4 * 16 + x] = t16[x];
      }
      tmem_ld_wait();
      float mx0 = -INFINITY, mx1 = -INFINITY, mx2 = -INFINITY, mx3 = -INFINITY;
#pragma unroll
      for (int x = 0; x < 64; x += 8) {
        mx0 = max3(mx0, v[x], v[x + 1]);
        mx1 = max3(mx1, v[x + 2], v[x + 3]);
        mx2 = max3(mx2, v[x + 4], v[x + 5]);
        mx3 = max3(mx3, v[x + 6], v[x + 7]);
      }
      const float mx = fmaxf(fmaxf(mx0, mx1), fmaxf(mx2, mx3)) * a.scale_log2;
      // the reference maximum moves only when the row maximum outgrows it by 2^8
      const bool grow = mx > m_ref + 8.f;
      const float m_new = grow ? mx : m_ref;
      if (i > 0 && __any_sync(0xffffffffu, grow)) {
        // O is stable between the completion of P.V(i-1) and the hand-over of P(i).  The scores of the slot's next page
        // were issued behind P.V(i-1); its last page has a barrier of its own.
        if (!(i + 1 < n_mine ? mbar_wait_bounded(&bar[B_S_FULL + 2 * h + (b ^ 1)], ((i + 1) >> 1) & 1)
                             : mbar_wait_bounded(&bar[B_O_DONE + 2 * h + (b ^ 1)], 0))) {
          failed = true;
          break;
        }
        fence_after();
        const float f = grow ? fast_exp2(m_ref - m_new) : 1.f;   // m_ref = -inf -> 0
#pragma unroll
        for (int q8 = 0; q8 < 8; ++q8) {
          float t16[16];
          tmem_ld16(t_o + q8 * 16, t16);
          tmem_ld_wait();
#pragma unroll
          for (int x = 0; x < 16; ++x) t16[x] *= f;
          tmem_st16(t_o + q8 * 16, t16);
        }
        l *= f;
      }
      m_ref = m_new;
      const float ms = m_ref == -INFINITY ? 0.f : m_ref;
      const float bias = wide ? 0.f : kPBias;
      const uint64_t sc2 = pack2(a.scale_log2, a.scale_log2), nms2 = pack2(bias - ms, bias - ms);
      uint64_t l2a = pack2(0.f, 0.f), l2b = l2a;
      if (wide) {   // hi in the first 32 columns of the score buffer, lo in the other 32
#pragma unroll
        for (int q2 = 0; q2 < 2; ++q2) {
          uint32_t hi[16], lo[16];
#pragma unroll
          for (int x = 0; x < 16; ++x) {
            float e0, e1, r0, r1;
            unpack2(fma2(pack2(v[q2 * 32 + 2 * x], v[q2 * 32 + 2 * x + 1]), sc2, nms2), e0, e1);
            const float p0 = fast_exp2(e0), p1 = fast_exp2(e1);
            const uint64_t p2 = pack2(p0, p1);
            if (x & 1) l2b = add2(l2b, p2); else l2a = add2(l2a, p2);
            hi[x] = pack_bf16(p0, p1);
            unpack2(sub2(p2, pack2(__uint_as_float(hi[x] << 16), __uint_as_float(hi[x] & 0xffff0000u))), r0, r1);
            lo[x] = pack_bf16(r0, r1);
          }
          tmem_st16u(t_s + q2 * 16, hi);
          tmem_st16u(t_s + 32 + q2 * 16, lo);
        }
      } else {
#pragma unroll
        for (int q2 = 0; q2 < 2; ++q2) {
          uint32_t ph[16];
#pragma unroll
          for (int x = 0; x < 16; ++x) {
            float e0, e1;
            unpack2(fma2(pack2(v[q2 * 32 + 2 * x], v[q2 * 32 + 2 * x + 1]), sc2, nms2), e0, e1);
            const float p0 = fast_exp2(e0), p1 = fast_exp2(e1);
            const uint64_t p2 = pack2(p0, p1);
            if (x & 1) l2b = add2(l2b, p2); else l2a = add2(l2a, p2);
            ph[x] = pack_f16(p0, p1);
          }
          tmem_st16u(t_s + q2 * 16, ph);
        }
      }
      float la, lb;
      unpack2(add2(l2a, l2b), la, lb);
      l += la + lb;
      tmem_st_wait();
      fence_before();
      mbar_arrive(&bar[B_P_FULL + 2 * h + b]);
    }
    // ---- the row's part: O and l without the bias of P and the value scale
    const float o_scale = wide ? 1.f : v_unscale * 0.0078125f, l_scale = wide ? 1.f : 0.0078125f;
    const bool have = n_mine > 0;
    if (have && !failed && !mbar_wait_bounded(&bar[B_O_DONE + 2 * h + ((n_mine - 1) & 1)], 0)) failed = true;
    fence_after();
    // Both slots are through with Q, keys and values before their shared memory is written to.
    asm volatile("bar.sync 1, 256;" ::: "memory");
    float *stage = reinterpret_cast<float *>(smem);          // [row][132]: a row's O, and (m, l) of slot 1
    float *mine = stage + (size_t)((kAlt ? 0 : h * 128) + row) * kRowStride;
    float M = m_ref, f0 = o_scale, f1 = 0.f;
    if (kAlt) {   // slot 1 hands its rows over
      if (h == 1) {
        if (have && live && !failed) {
#pragma unroll
          for (int q8 = 0; q8 < 8; ++q8) {
            float t16[16];
            tmem_ld16(t_o + q8 * 16, t16);
            tmem_ld_wait();
#pragma unroll
            for (int x = 0; x < 4; ++x)
              *reinterpret_cast<float4 *>(mine + q8 * 16 + 4 * x) =
                  make_float4(t16[4 * x], t16[4 * x + 1], t16[4 * x + 2], t16[4 * x + 3]);
          }
        }
        mine[128] = have ? m_ref : -INFINITY;
        mine[129] = l;
      }
      asm volatile("bar.sync 1, 256;" ::: "memory");
    }
    if (have && !failed && live && (!kAlt || h == 0)) {
      l *= l_scale;
      if (kAlt) {
        const float m1 = mine[128], l1 = mine[129];
        M = fmaxf(m_ref, m1);
        const float w0 = part_weight(m_ref, l, M), w1 = part_weight(m1, l1, M);
        l = l * w0 + l1 * l_scale * w1;
        f0 = o_scale * w0;
        f1 = o_scale * w1;
      }
#pragma unroll
      for (int q8 = 0; q8 < 8; ++q8) {
        float t16[16];
        tmem_ld16(t_o + q8 * 16, t16);
        tmem_ld_wait();
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          float4 o = make_float4(t16[4 * x] * f0, t16[4 * x + 1] * f0, t16[4 * x + 2] * f0, t16[4 * x + 3] * f0);
          float4 *at = reinterpret_cast<float4 *>(mine + q8 * 16 + 4 * x);
          if (kAlt && f1 != 0.f) {
            const float4 p = *at;
            o.x = fmaf(p.x, f1, o.x); o.y = fmaf(p.y, f1, o.y); o.z = fmaf(p.z, f1, o.z); o.w = fmaf(p.w, f1, o.w);
          }
          *at = o;
        }
      }
      // out row by row, 512 bytes at a time (a thread per row would write 32 rows' sixteenths at once: 19 MB of
      // parts took 5 us to drain, and no tail block could start before)
      __syncwarp();
      const int r0 = (kAlt ? 0 : h * 128) + (row & ~31);
      const size_t at = (size_t)blockIdx.x * a.rows_per_block + r0;
#pragma unroll 4
      for (int r = 0; r < min(32, n_rows - r0); ++r)
        *reinterpret_cast<float4 *>(a.part_o + (at + r) * kD + lane * 4) =
            *reinterpret_cast<const float4 *>(stage + (size_t)(r0 + r) * kRowStride + lane * 4);
      if (r0 + lane < n_rows) *reinterpret_cast<float2 *>(a.part_ml + (at + lane) * 2) = make_float2(M, l);
    }
  }
  if (failed) set_status(c, SPKV_E_TIMEOUT);
  fence_before();
  __syncthreads();
  if (warp == kTmemWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tbase), "n"(shp::kTmemCols) : "memory");
}

// ---- joining parts -----------------------------------------------------------------------------------
// Adds parts first, first + stride, ... < n of a query row to (M, L, O), kBatch of them in one round of loads; one warp,
// lane l owns dims 4l .. 4l + 3.  at(p, o, ml): where part p's row and its (m, l) lie; use(p): does it count.
template <int kBatch, class At, class Use>
__device__ inline void join_parts(int first, int stride, int n, At at, Use use, float &M, float &L, float4 &O) {
  const int lane = threadIdx.x & 31;
  for (int p0 = first; p0 < n; p0 += kBatch * stride) {
    const int mine = p0 + lane * stride;
    const float *po, *pml;
    float2 ml = make_float2(-INFINITY, 0.f);
    if (lane < kBatch && mine < n) {
      at(mine, po, pml);
      ml = __ldcg(reinterpret_cast<const float2 *>(pml));
    }
    float4 v[kBatch];
#pragma unroll
    for (int x = 0; x < kBatch; ++x) {
      at(min(p0 + x * stride, n - 1), po, pml);
      v[x] = __ldcg(reinterpret_cast<const float4 *>(po) + lane);
    }
    if (!use(mine)) ml = make_float2(-INFINITY, 0.f);
    float top = ml.x;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float Mn = fmaxf(M, top), old = part_weight(M, L, Mn);
    M = Mn;
    const float f = part_weight(ml.x, ml.y, M);
    float fl = f == 0.f ? 0.f : f * ml.y;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) fl += __shfl_xor_sync(0xffffffffu, fl, o);
    L = L * old + fl;
    O.x *= old; O.y *= old; O.z *= old; O.w *= old;
#pragma unroll
    for (int x = 0; x < kBatch; ++x) {
      const float fx = __shfl_sync(0xffffffffu, f, x);
      if (fx != 0.f) {   // (a part of weight 0 may never have been written)
        O.x = fmaf(v[x].x, fx, O.x); O.y = fmaf(v[x].y, fx, O.y); O.z = fmaf(v[x].z, fx, O.z); O.w = fmaf(v[x].w, fx, O.w);
      }
    }
  }
}

// Where prefix part p of a query row lies: row R = b * G + g of its KV head.
__device__ inline size_t prefix_part_row(const SharedArgs &a, int first, int R, int p) {
  const int last_block = a.max_blocks - 1;   // (a plan that was overwritten reads no further than the workspace)
  return (size_t)max(0, min(first + p * a.n_tiles + R / kShareRows, last_block)) * a.rows_per_block + R % kShareRows;
}

// With more than 128 query rows a KV head, the last blocks of the tail launch make one part of a row's prefix parts, a
// warp per row.  They wait for the prefix launch and run beside the last tail blocks, so that the merge finds
// little left to read (64 sequences of 32 heads on 8 KV heads: 18 parts a row, 19 MB; 40.1 -> 37.7 us a call.
// With fewer rows the tail ends with the prefix and nothing would hide it: 19 -> 23 us).
__device__ inline void join_prefix_parts(const SharedArgs &a, int block, int n_blocks) {
  const CacheView &c = a.c;
  const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  for (int r = block * warps + (threadIdx.x >> 5); r < a.B * c.Hq; r += n_blocks * warps) {
    const int b = r / c.Hq, j = r - b * c.Hq, kvh = j / c.G, R = b * c.G + j - kvh * c.G;
    const int4 parts = ldcg4(share_head(a.rec, kvh) + 4);
    const int first = __ldcg(share_head(a.rec, kvh) + 1), n = parts.z == a.sig ? max(parts.x, 0) : 0;
    float M = -INFINITY, L = 0.f;
    float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
    join_parts<8>(0, 1, n, [&](int p, const float *&o, const float *&ml) {
      const size_t at = prefix_part_row(a, first, R, p);
      o = a.part_o + at * kD;
      ml = a.part_ml + at * 2;
    }, [](int) { return true; }, M, L, O);
    *reinterpret_cast<float4 *>(a.pre_o + (size_t)r * kD + lane * 4) = O;
    if (lane == 0) *reinterpret_cast<float2 *>(a.pre_ml + (size_t)r * 2) = make_float2(M, L);
  }
}

// ---- tail ------------------------------------------------------------------------------------------
namespace sht {
constexpr int kThreads = 128, kWarps = 4;
// two pages, over which the four warps join their G rows of 132 floats at the end (33 KB at G = 16)
constexpr int off_bar = 2 * kPageBytes, kSmemBytes = off_bar + 128;
}  // namespace sht

// Item = share * n_items + unit.  A unit's pages are what its compact cache holds behind the common pages,
// then its ring; they are cut into up to `shares` (plan) pieces of at least kTailMinPages.  The four warps take 16
// pairs each of every page and join at the end through the page buffers.  64 sequences of 32/8
// heads with a page of their own and a ring of two: 50 MB, 7.8 us at the copy rate, which the prefix launch hides but for
// some 3 us.
template <int NH>
__global__ void __launch_bounds__(sht::kThreads, NH == 1 ? 5 : 3) shared_tail_kernel(SharedArgs a) {
  using namespace sht;
  extern __shared__ __align__(1024) unsigned char smem[];
  const CacheView &c = a.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, G = c.G;
  uint64_t *full = reinterpret_cast<uint64_t *>(smem + off_bar);   // [2 buffer + half]: keys, values
  volatile int *s_it = reinterpret_cast<volatile int *>(full + 4);   // share exists, skip, compact pages, length behind
                                                                     // the common pages, ring pairs, first page, pages, `ahead` holds
  if (tid == 0) {
    for (int i = 0; i < 4; ++i) mbar_init(&full[i], 1);
    mbar_fence_init();
  }
  pdl_trigger();
  if ((int)blockIdx.x >= a.tail_blocks) {
    pdl_wait();
    join_prefix_parts(a, (int)blockIdx.x - a.tail_blocks, (int)gridDim.x - a.tail_blocks);
    return;
  }
  // everything before the prefix launch is complete and was written through generic stores
  asm volatile("fence.proxy.async;" ::: "memory");
  const uint64_t pol = l2_evict_first_policy();
  int loads = 0;        // pages of the items before: page i of this one is in buffer (loads + i) & 1, phase (loads + i) >> 1 & 1
  bool failed = false;
  for (int item = blockIdx.x;; item += a.tail_blocks) {
    const int unit = item % a.n_items, share = item / a.n_items;
    const int b = unit / c.Hkv, kvh = unit - b * c.Hkv;
    __syncthreads();    // the previous item's stages and s_it have been read
    if (share >= a.max_tail) break;
    int u = 0, trow = -1, ahead = 0;   // ahead: page-table entry common + lane, fetched before it is known to be needed
    if (warp == 0) {
      // trip 1: the plan and the sequence
      const int4 head = ldcg4(share_head(a.rec, kvh)), parts = ldcg4(share_head(a.rec, kvh) + 4);
      const int seq = a.seq_ids[b], n_shares = parts.y;
      const bool fits = parts.z == a.sig;
      if (share >= (fits ? n_shares : 1)) {
        if (lane == 0) s_it[0] = 0;
      } else {
        int common = fits ? min(head.x, c.max_pages) : 0;
        const int row0 = head.z, u0 = head.w;
        if (common < 0 || row0 < 0 || row0 >= c.n_units || u0 < 0 || u0 >= c.n_units) common = 0;
        const bool ok = seq >= 0 && seq < c.S;
        if (!ok && lane == 0 && share == 0) set_status(c, SPKV_E_BOUNDS);
        u = unit_index(c, a.layer, ok ? seq : 0, kvh);
        // the unit's page-table row as spkv_cache_create laid the rows out: no trip for it
        const bool local = kvh < 64 && ((a.local_mask >> kvh) & 1);
        const int below = kvh < 64 ? __popcll(a.local_mask & ((1ULL << kvh) - 1ULL)) : 0;
        trow = local ? -1 : a.row_base + (ok ? seq : 0) * a.row_heads + kvh - below;
        // trip 2: the unit; do it and the batch's first sequence still hold the common pages (the last one names
        // them all); the unit's own first pages
        int len = ldcg_keep(&c.len[u]), n_ring = min(ldcg_keep(&c.t[u]), c.w);
        if (trow >= 0 && common + lane < c.max_pages) ahead = ldcg_keep(&unit_table(c, trow)[common + lane]);
        int skip = 0;
        if (common > 0 && trow >= 0) {
          const int len0 = ldcg_keep(&c.len[u0]), last0 = ldcg_keep(&unit_table(c, row0)[common - 1]),
                    last = ldcg_keep(&unit_table(c, trow)[common - 1]);
          if (len / kP >= common && len0 / kP >= common && last == last0) skip = common;
        }
        if (!ok) { len = 0; n_ring = 0; skip = 0; }
        len -= skip * kP;
        const int nk = (len + kP - 1) / kP, np = nk + (n_ring + kP - 1) / kP;
        const int ku = max(1, min(np / kTailMinPages, fits ? n_shares : 1));
        const int p0 = share < ku ? (int)((long long)np * share / ku) : 0;
        const int p1 = share < ku ? (int)((long long)np * (share + 1) / ku) : 0;
        if (lane == 0) {
          s_it[0] = 1; s_it[1] = skip; s_it[2] = nk; s_it[3] = len; s_it[4] = n_ring; s_it[5] = p0; s_it[6] = p1 - p0;
          s_it[7] = skip == common && p0 == 0;
          if (share == 0) a.item_skip[unit] = skip;
        }
        __syncwarp();
      }
    }
    __syncthreads();
    if (!s_it[0]) break;   // (items are laid out share by share: the ones behind do not exist either)
    const int skip = s_it[1], nk = s_it[2], len = s_it[3], n_ring = s_it[4], p0 = s_it[5], n = s_it[6];
    const size_t row0 = ((size_t)share * a.n_items + unit) * G;
    if (n == 0) {          // nothing to attend to in this share
      for (int g = tid; g < G; g += kThreads) *reinterpret_cast<float2 *>(a.tail_ml + (row0 + g) * 2) = make_float2(-INFINITY, 0.f);
      continue;
    }
    int entry = 0;
    auto fetch_entries = [&](int i) {   // warp 0: global page indices of the share's pages i .. i + 31, one per lane
      const int p = p0 + i + lane;
      if (i + lane < n)
        entry = p < nk ? checked_page(c, i == 0 && s_it[7] ? ahead : ldcg_keep(&unit_table(c, trow)[skip + p]),
                                      (int)ring_page(c, u, 0))
                       : (int)ring_page(c, u, p - nk);
    };
    auto load = [&](int i, int half) {  // warp 0: keys (half = 0; first) or values of page i
      if (half == 0 && (i & 31) == 0) fetch_entries(i);
      const int gp = __shfl_sync(0xffffffffu, entry, i & 31);
      if (lane == 0) {
        const int bf = (loads + i) & 1;
        uint64_t *bar = &full[2 * bf + half];
        mbar_arrive_expect_tx(bar, kPageBytes / 2);
        bulk_load_hint(smem + bf * kPageBytes + half * (kPageBytes / 2), c.pages + (int64_t)gp * kPageElems + half * kBlockElems,
                       kPageBytes / 2, bar, pol);
      }
    };
    if (warp == 0) {
      load(0, 0);
      load(0, 1);
      if (n > 1) {
        load(1, 0);
        load(1, 1);
      }
    }
    uint32_t qb[NH][8][2];
    float m[NH][2], l[NH][2], o[NH][8][4];
    const __nv_bfloat16 *q = a.q + ((size_t)b * c.Hq + (size_t)kvh * G) * kD;
    load_q_frags_t<NH>(qb, [&](int h) -> const __nv_bfloat16 * { return h < G ? q + h * kD : nullptr; }, lane);
#pragma unroll
    for (int hn = 0; hn < NH; ++hn) {
      m[hn][0] = m[hn][1] = -INFINITY;
      l[hn][0] = l[hn][1] = 0.f;
#pragma unroll
      for (int mt = 0; mt < 8; ++mt) o[hn][mt][0] = o[hn][mt][1] = o[hn][mt][2] = o[hn][mt][3] = 0.f;
    }
    for (int i = 0; i < n; ++i) {
      const int p = p0 + i;
      const int valid = p < nk ? min(kP, len - p * kP) : min(kP, n_ring - (p - nk) * kP);
      const int bf = (loads + i) & 1;
      const uint32_t ph = ((loads + i) >> 1) & 1;
      const int tok0 = warp * 16;
      const uint32_t sK = smem_u32(smem + bf * kPageBytes), sV = sK + kBlockElems * 2;
      float s[NH][4];
      if (!mbar_wait_bounded(&full[2 * bf], ph)) failed = true;
      if (!failed && tok0 < valid) qk_tile_t<NH>(s, qb, sK, tok0, lane);
      failed = __syncthreads_or(failed);   // all four warps are done with the keys
      if (!failed) {
        if (warp == 0 && i + 2 < n) load(i + 2, 0);
        if (!mbar_wait_bounded(&full[2 * bf + 1], ph)) failed = true;
        if (!failed && tok0 < valid) softmax_pv_tile_t<NH>(s, valid, a.scale_log2, m, l, o, sV, tok0, lane);
        failed = __syncthreads_or(failed);   // ... and with the values
      }
      if (failed) {
        // do not leave while copies may still be landing (keys up to page i + 2, values up to i + 1)
        if (tid == 0)
          for (int k = i; k < min(i + 3, n); ++k)
            for (int half = 0; half < 2; ++half)
              mbar_wait_bounded(&full[2 * ((loads + k) & 1) + half], ((loads + k) >> 1) & 1);
        break;
      }
      if (warp == 0 && i + 2 < n) load(i + 2, 1);
    }
    if (failed) break;
    loads += n;
    // join the four warps: rows [warp][G][132] over the pages (every copy of the item has landed)
    float *red = reinterpret_cast<float *>(smem);
    segment_hand_over<NH>(red, warp, G, G, m, l, o, lane);
    __syncthreads();
    for (int g = warp; g < G; g += kWarps) {
      float M = -INFINITY, L = 0.f;
      float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) M = fmaxf(M, red[((size_t)w * G + g) * 132 + 128]);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float *src = red + ((size_t)w * G + g) * 132;
        const float f = part_weight(src[128], src[129], M);
        const float4 v = *reinterpret_cast<const float4 *>(src + lane * 4);
        L += src[129] * f;
        O.x = fmaf(v.x, f, O.x); O.y = fmaf(v.y, f, O.y); O.z = fmaf(v.z, f, O.z); O.w = fmaf(v.w, f, O.w);
      }
      *reinterpret_cast<float4 *>(a.tail_o + (row0 + g) * kD + lane * 4) = O;
      if (lane == 0) *reinterpret_cast<float2 *>(a.tail_ml + (row0 + g) * 2) = make_float2(M, L);
    }
    tc5::fence_async_smem();   // these reads and writes come before the next item's copies into the stages
  }
  if (failed) set_status(c, SPKV_E_TIMEOUT);
  // The merge reads the prefix launch's parts too: this launch is not complete before that one is (its joining blocks
  // wait for it, or else its first block, at its end: all of them would keep others out while the prefix runs).
  if (blockIdx.x == 0) pdl_wait();
}

// ---- merge -----------------------------------------------------------------------------------------
// One block per query row: its prefix parts (kJoined: one, made by the tail launch) and the parts of the tail, kWarps warps
// taking every kWarps-th.  The plan's line is read before the launch waits for the tail (it was complete
// before the prefix launch let anything start); everything behind the wait is loaded at once: one trip to L2.
template <int kWarps, int kBatch, bool kJoined>
__global__ void __launch_bounds__(32 * kWarps) shared_merge_kernel(SharedArgs a) {
  const CacheView &c = a.c;
  __shared__ float s_ml[kWarps][2];
  __shared__ float4 s_o[kWarps][32];
  pdl_trigger();
  const int r = blockIdx.x, b = r / c.Hq, j = r - b * c.Hq, kvh = j / c.G, g = j - kvh * c.G;
  const int unit = b * c.Hkv + kvh, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // (through L1: the rows of a head that meet on an SM share the line)
  const int4 parts = *reinterpret_cast<const int4 *>(share_head(a.rec, kvh) + 4);
  const int first = share_head(a.rec, kvh)[1];
  const bool fits = parts.z == a.sig;
  const int n_pre = kJoined ? 1 : fits ? max(parts.x, 0) : 0, n = n_pre + (fits ? max(1, min(parts.y, a.max_tail)) : 1);
  pdl_wait();
  const int skip = __ldcg(a.item_skip + unit);
  float M = -INFINITY, L = 0.f;
  float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
  join_parts<kBatch>(warp, kWarps, n, [&](int p, const float *&o, const float *&ml) {
    const bool pre = p < n_pre;
    const size_t at = !pre ? ((size_t)(p - n_pre) * a.n_items + unit) * c.G + g
                           : kJoined ? (size_t)r : prefix_part_row(a, first, b * c.G + g, p);
    o = (!pre ? a.tail_o : kJoined ? a.pre_o : a.part_o) + at * kD;
    ml = (!pre ? a.tail_ml : kJoined ? a.pre_ml : a.part_ml) + at * 2;
  }, [&](int p) { return p >= n_pre || skip > 0; /* otherwise the tail read this unit in full */ }, M, L, O);
  if (kWarps > 1) {
    s_o[warp][lane] = O;
    if (lane == 0) { s_ml[warp][0] = M; s_ml[warp][1] = L; }
    __syncthreads();
    if (warp) return;
    float Mx = M;
#pragma unroll
    for (int x = 1; x < kWarps; ++x) Mx = fmaxf(Mx, s_ml[x][0]);
    const float w0 = part_weight(M, L, Mx);
    L *= w0; O.x *= w0; O.y *= w0; O.z *= w0; O.w *= w0;
#pragma unroll
    for (int x = 1; x < kWarps; ++x) {
      const float f = part_weight(s_ml[x][0], s_ml[x][1], Mx);
      const float4 v = s_o[x][lane];
      L = fmaf(s_ml[x][1], f, L);
      O.x = fmaf(v.x, f, O.x); O.y = fmaf(v.y, f, O.y); O.z = fmaf(v.z, f, O.z); O.w = fmaf(v.w, f, O.w);
    }
    M = Mx;
  }
  const bool none = M == -INFINITY && L == 0.f;   // a sequence that has received nothing: zeros, -inf
  const float inv = none ? 0.f : 1.f / L;
  uint2 pk;
  pk.x = pack_bf16(O.x * inv, O.y * inv);
  pk.y = pack_bf16(O.z * inv, O.w * inv);
  *reinterpret_cast<uint2 *>(a.out + (size_t)r * kD + lane * 4) = pk;
  if (a.lse && lane == 0) a.lse[r] = none ? -INFINITY : (M + log2f(L)) * kLn2;
}

struct SharedWs { size_t off_ml, off_o, off_tml, off_to, off_pml, off_po, total; int max_blocks, rows, max_tail; };
static SharedWs shared_ws_layout(const spkv_config_t *cfg, int B) {
  SharedWs w;
  auto a256 = [](size_t x) { return (x + 255) / 256 * 256; };
  const int G = cfg->n_q_heads / cfg->n_kv_heads, items = std::max(1, B * cfg->n_kv_heads);
  w.max_blocks = std::max(kMaxGrid, cfg->n_kv_heads * share_row_tiles(B, G));
  w.rows = std::min(kShareRows, B * G);
  w.max_tail = std::max(1, kMaxTailItems / items);
  size_t o = a256((size_t)items * 4);   // the units' skips first
  w.off_ml = o; o += a256((size_t)w.max_blocks * w.rows * 8);
  w.off_o = o; o += a256((size_t)w.max_blocks * w.rows * kD * 4);
  w.off_tml = o; o += a256((size_t)w.max_tail * items * G * 8);
  w.off_to = o; o += a256((size_t)w.max_tail * items * G * kD * 4);
  w.off_pml = o; o += a256((size_t)items * G * 8);
  w.off_po = o; o += a256((size_t)items * G * kD * 4);
  w.total = o;
  return w;
}

}  // namespace spkv

using namespace spkv;

namespace {
// Attributes of the two kernels, set once per device (a bit each).
std::atomic<unsigned long long> g_ready[2][2];

// The kernel may use `smem` bytes and gets the whole of an SM's shared memory to share out: with the default
// split, which fits one prefix block, a tail block finds none left beside it.
int whole_shared_memory(const void *kernel, int smem, std::atomic<unsigned long long> *ready) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return SPKV_E_CUDA;
  const unsigned long long bit = dev < 64 ? 1ULL << dev : 0;
  if (bit & ready->load(std::memory_order_acquire)) return SPKV_OK;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess ||
      cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared) != cudaSuccess)
    return SPKV_E_CUDA;
  ready->fetch_or(bit, std::memory_order_release);
  return SPKV_OK;
}
}  // namespace

extern "C" size_t spkv_decode_shared_workspace_bytes(const spkv_config_t *cfg, int32_t B) {
  if (!cfg || B < 0 || cfg->n_kv_heads < 1 || cfg->n_q_heads < cfg->n_kv_heads) return 0;
  return shared_ws_layout(cfg, B).total;
}

extern "C" int spkv_decode_attention_shared(spkv_cache_t *cache, int32_t layer, const int32_t *d_seq_ids, int32_t B,
                                            const void *d_q, void *d_out, float *d_lse_opt, float sm_scale,
                                            const void *d_plan, size_t plan_bytes, void *d_workspace,
                                            size_t workspace_bytes, spkv_stream_t stream) {
  bool empty;
  const int rc_args = decode_check_args(cache, layer, d_seq_ids, B, d_q, d_out, nullptr, &empty);
  if (rc_args) return rc_args;
  if (!(sm_scale > 0.f) || !isfinite(sm_scale)) return SPKV_E_INVALID;
  if (empty) return SPKV_OK;
  if (!d_plan || ((uintptr_t)d_plan & 15)) return SPKV_E_INVALID;
  const SharedWs w = shared_ws_layout(&cache->cfg, B);
  if (plan_bytes < spkv_share_plan_bytes(&cache->cfg)) return SPKV_E_WORKSPACE;
  if (!d_workspace || ((uintptr_t)d_workspace & 255) || workspace_bytes < w.total) return SPKV_E_WORKSPACE;
  const CacheView &v = cache->view;
  char *ws = static_cast<char *>(d_workspace);
  cudaStream_t s = as_stream(stream);
  SharedArgs a = {};
  a.c = v; a.layer = layer; a.B = B; a.n_items = B * v.Hkv;
  a.n_tiles = share_row_tiles(B, v.G);
  a.rows_per_block = w.rows;
  a.sig = share_signature(cache, B);
  a.g_inv = ((1ULL << 32) + v.G - 1) / v.G;
  a.seq_ids = d_seq_ids;
  a.q = static_cast<const __nv_bfloat16 *>(d_q);
  a.rec = share_record(v, static_cast<const int32_t *>(d_plan), layer);
  a.scale_log2 = sm_scale * kLog2e;
  a.force_wide = (cache->cfg.flags & SPKV_FLAG_PREFILL_PV_BF16) ? 1 : 0;
  a.item_skip = reinterpret_cast<int32_t *>(ws);
  a.part_ml = reinterpret_cast<float *>(ws + w.off_ml);
  a.part_o = reinterpret_cast<float *>(ws + w.off_o);
  a.tail_ml = reinterpret_cast<float *>(ws + w.off_tml);
  a.tail_o = reinterpret_cast<float *>(ws + w.off_to);
  a.pre_ml = reinterpret_cast<float *>(ws + w.off_pml);
  a.pre_o = reinterpret_cast<float *>(ws + w.off_po);
  a.max_blocks = w.max_blocks;
  a.max_tail = w.max_tail;
  for (int l = 0; l < layer; ++l) a.row_base += (v.Hkv - __builtin_popcountll(cache->local_mask[l])) * v.S;
  a.row_heads = v.Hkv - __builtin_popcountll(cache->local_mask[layer]);
  a.local_mask = cache->local_mask[layer];
  a.out = static_cast<__nv_bfloat16 *>(d_out);
  a.lse = d_lse_opt;
  // blocks: one share each (the plan never cuts into more)
  const int sms = std::min(kMaxGrid, cache->sm_count), grid = std::max(sms, v.Hkv * a.n_tiles);
  const bool alt = w.rows <= 128;
  auto prefix = alt ? shared_prefix_kernel<true> : shared_prefix_kernel<false>;
  const int smem = shp::smem_bytes(alt);
  auto tail = v.G > 8 ? shared_tail_kernel<2> : shared_tail_kernel<1>;
  const int tail_smem = sht::kSmemBytes;
  if (const int rc = whole_shared_memory(reinterpret_cast<const void *>(prefix), smem, &g_ready[0][alt])) return rc;
  if (const int rc = whole_shared_memory(reinterpret_cast<const void *>(tail), tail_smem, &g_ready[1][v.G > 8])) return rc;
  // Overlap mode: kernels before the last one may still be running, which griddepcontrol.wait does not
  // cover; a plain launch waits for all of them.
  const bool plain = (cache->cfg.flags & SPKV_FLAG_OVERLAP) != 0;
  cache->last_kind = kLastOther;
  if (launch_link(!plain, prefix, dim3(grid), dim3(shp::kThreads), (size_t)smem, s, a) != cudaSuccess) return SPKV_E_CUDA;
  // one block per unit, and enough of them that the pieces of long units find a block each; behind them, with many query
  // rows, the blocks that join the prefix parts: a warp per row up to two blocks per SM
  a.tail_blocks = std::max(a.n_items, 2 * sms);
  const int joiners = alt ? 0 : std::min((B * v.Hq + sht::kWarps - 1) / sht::kWarps, 2 * sms);
  if (launch_overlapped(tail, dim3(a.tail_blocks + joiners), dim3(sht::kThreads), (size_t)tail_smem, s, a) != cudaSuccess)
    return SPKV_E_CUDA;
  // With the prefix parts joined few parts are left; otherwise up to 40 go in one round of loads.
  auto merge = joiners ? shared_merge_kernel<1, 4, true> : shared_merge_kernel<8, 5, false>;
  return check_stream_error(launch_overlapped(merge, dim3(B * v.Hq), dim3(joiners ? 32 : 256), 0, s, a));
}
