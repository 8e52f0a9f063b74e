// Decode attention of a batch whose sequences share a prefix (spkv_decode_attention_shared).
//
// Three launches:
//   prefix  (here)  the compact-cache pages that all sequences have in common, once for the batch: the
//           B * G query rows of a KV head are the M side of tcgen05 tiles, a block takes 128 or 256 of
//           them over one share of the head's common pages and leaves (m, l, O) per row;
//   suffix  (spkv_decode.cu)  the decode kernel over what is left of every unit: its own pages and ring;
//   merge   (here)  joins a row's parts by their log-sum-exp weights.
// The suffix launch does not depend on the prefix launch and starts on every SM as the prefix block there
// leaves (programmatic dependent launch; the prefix kernel has waited for everything earlier on the
// stream before it lets dependents start); it waits for the prefix launch at its own end, so that
// the merge, which waits for the suffix, may read both.
//
// Prefix kernel.  Per page and 128-row slot: S = Q K^T (8 MMAs M128 N64 K16 into tensor memory), softmax
// in registers (thread = row = TMEM lane), P in fp16 back over the scores, O += P V with the page's values
// rescaled to fp16 by two converter warps, or two bf16 terms for a unit of wide-ranging values
// (value_scale).  No masks: common pages are full and every query sees all of them.
//   * More than 128 rows in the tile (kAlt = false): slot h holds rows [128 h, 128 h + 128), both walk
//     every page.  Scores of page j + 2 are issued behind P.V(j), so a slot's next scores are ready.
//   * At most 128 rows (kAlt): both slots hold the same rows and take alternate pages, which halves the
//     softmax time per page; scores of a slot's next page are issued behind P.V of its last one.  One of the two
//     is joined into the other through shared memory at the end.
// Shared memory: Q (64 KB; kAlt 32 KB) + 5 (6) page stages.  Tensor memory: score buffer b of slot h at
// [64 (2h + b), +64), O of slot h at [256 + 128 h, +128).
// Warps: 0 MMA issue slot 0, 1 page loader + TMEM, 2-3 value conversion, 4-7 / 8-11 softmax of slot 0 / 1,
// 12 MMA issue slot 1.  All waits are bounded.
#include <algorithm>
#include <math.h>

#include "spkv_decode_common.cuh"
#include "spkv_share.cuh"
#include "spkv_tc5.cuh"

namespace spkv {

namespace shp {
constexpr int kThreads = 416;
constexpr int kMmaWarp0 = 0, kMmaWarp1 = 12, kLoaderWarp = 1;
constexpr int kTmemCols = 512, kConvThreads = 64;
constexpr float kPBias = 7.f;   // P is stored as 2^7 p
enum { B_KV_FULL = 0, B_KV_EMPTY = 8, B_V_READY = 16, B_S_FULL = 24 /* [2h+b] */, B_P_FULL = 28, B_O_DONE = 32, B_COUNT = 36 };
__host__ __device__ constexpr int stages(bool alt) { return alt ? 6 : 5; }
__host__ __device__ constexpr int off_kv(bool alt) { return alt ? 32768 : 65536; }
__host__ __device__ constexpr int off_bar(bool alt) { return off_kv(alt) + stages(alt) * kPageBytes; }
__host__ __device__ constexpr int smem_bytes(bool alt) { return off_bar(alt) + 512; }
constexpr int kJoinStride = 132;   // floats per row of the hand-over between the slots (kAlt)
}  // namespace shp

struct SharedArgs {
  CacheView c;
  int layer, B, n_tiles, rows_per_block;
  const int32_t *seq_ids;
  const __nv_bfloat16 *q;       // [B][Hq][128]
  const int32_t *plan;
  float scale_log2;
  int force_wide;
  float *part_o, *part_ml;      // [block][rows_per_block][128], [block][rows_per_block][2]: m (log2 domain), l
  int max_blocks;
  // merge
  const float *suf_o, *suf_lse;       // [B * Hq][128], [B * Hq]
  const int32_t *item_skip;           // [B * Hkv] common pages the suffix left out (0: it read the unit in full)
  __nv_bfloat16 *out;
  float *lse;
};

// A plan that was made for this batch size and configuration
__device__ inline bool plan_fits(const CacheView &c, const int32_t *plan, int B) {
  return __ldcg(plan) == B && __ldcg(plan + 1) == c.L && __ldcg(plan + 2) == c.Hkv;
}

template <bool kAlt>
__global__ void __launch_bounds__(shp::kThreads, 1) shared_prefix_kernel(SharedArgs a) {
  using namespace tc5;
  using namespace shp;
  constexpr int kStages = stages(kAlt), kSKV = off_kv(kAlt);
  constexpr int kAhead = kAlt ? 1 : 2;       // how many of a slot's pages its scores run ahead of P.V
  extern __shared__ __align__(1024) unsigned char smem[];
  const CacheView &c = a.c;
  uint64_t *bar = reinterpret_cast<uint64_t *>(smem + off_bar(kAlt));
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bar + B_COUNT);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();
  pdl_trigger();   // (only now: what follows may then rely on everything before this launch)
  // ---- this block's share
  const int32_t *rec = share_record(a.plan, c.Hkv, a.layer);
  if (!plan_fits(c, a.plan, a.B)) return;
  const int per_share = max(1, __ldcg(rec)), n_blocks = min(__ldcg(rec + 1), a.max_blocks);
  if ((int)blockIdx.x >= n_blocks) return;
  int kvh = 0;
  {
    int lo = 0, hi = c.Hkv;   // last head whose first block is <= this one
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (__ldcg(rec + kShareHdr + c.Hkv + mid) <= (int)blockIdx.x) lo = mid; else hi = mid;
    }
    kvh = lo;
    while (kvh > 0 && __ldcg(rec + kShareHdr + kvh) == 0) --kvh;   // (heads without common pages start where the next one does)
  }
  const int common = min(__ldcg(rec + kShareHdr + kvh), c.max_pages);
  const int rem = (int)blockIdx.x - __ldcg(rec + kShareHdr + c.Hkv + kvh);
  const int tile = rem % a.n_tiles, share = rem / a.n_tiles;
  const int seq0 = a.seq_ids[0];
  if (common <= 0 || rem < 0 || seq0 < 0 || seq0 >= c.S) return;
  const int u = unit_index(c, a.layer, seq0, kvh), trow = unit_table_row(c, u);
  // (stale plan: the unit is shorter by now; nobody reads this share's result)
  if (trow < 0 || ldcg_keep(&c.len[u]) / kP < common) return;
  const int j_begin = share * per_share, n_pages = min(per_share, common - j_begin);
  if (n_pages <= 0) return;
  const int rows_all = a.B * c.G, row_base = tile * kShareRows;
  const int n_rows = min(kShareRows, rows_all - row_base);
  const bool two = kAlt ? n_pages > 1 : n_rows > 128;     // is slot 1 in use
  float v_scale, v_unscale;
  const bool wide = value_scale(__ldcg(&c.vmax[u]), a.force_wide, v_scale, v_unscale);

  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&bar[B_KV_FULL + i], 1);
      mbar_init(&bar[B_KV_EMPTY + i], (!kAlt && two) ? 2 : 1);   // one commit per MMA warp that uses the page
      mbar_init(&bar[B_V_READY + i], kConvThreads);
    }
    // per slot and parity of the slot's page count: one phase per two of its pages
    for (int i = 0; i < 4; ++i) {
      mbar_init(&bar[B_S_FULL + i], 1);
      mbar_init(&bar[B_P_FULL + i], 128);
      mbar_init(&bar[B_O_DONE + i], 1);
    }
    mbar_fence_init();
  }
  // Q rows -> two slabs of 128 rows x 128 B per slot, 128-byte swizzle; rows past the last are zero
  for (int x = tid; x < (kAlt ? 1 : 2) * 128 * 16; x += kThreads) {
    const int h = x >> 11, r = (x >> 4) & 127, ch = x & 15;
    const int R = row_base + h * 128 + r;
    uint4 val = make_uint4(0, 0, 0, 0);
    if (h * 128 + r < n_rows) {
      const int b = R / c.G, g = R - b * c.G;
      val = *reinterpret_cast<const uint4 *>(a.q + ((size_t)b * c.Hq + kvh * c.G + g) * kD + ch * 8);
    }
    *reinterpret_cast<uint4 *>(smem + h * 32768 + (ch >> 3) * 16384 + r * 128 + (((ch & 7) ^ (r & 7)) << 4)) = val;
  }
  fence_async_smem();
  if (warp == kLoaderWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                 "n"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tbase = *tmem_slot;
  bool failed = false;
  // pages of slot h: local page i is page h + 2 i of the share (kAlt), or page i
  auto slot_pages = [&](int h) { return kAlt ? (n_pages + 1 - h) / 2 : (h == 0 || two ? n_pages : 0); };
  auto page_of = [&](int h, int i) { return kAlt ? 2 * i + h : i; };

  if (warp == kLoaderWarp) {
    // ---------------------------------------------------------------- page loader
    const uint64_t pol = l2_evict_first_policy();
    int j = 0;
    for (int base = 0; base < n_pages && !failed; base += 32) {
      int page = 0;
      if (base + lane < n_pages)
        page = checked_page(c, ldcg_keep(&unit_table(c, trow)[j_begin + base + lane]), (int)ring_page(c, u, 0));
      const int cnt = min(32, n_pages - base);
      for (int x = 0; x < cnt; ++x, ++j) {
        const int gp = __shfl_sync(0xffffffffu, page, x);
        if (lane == 0) {
          const int s = j % kStages;
          if (j >= kStages && !mbar_wait_bounded(&bar[B_KV_EMPTY + s], ((j / kStages) - 1) & 1)) failed = true;
          if (!failed) {
            mbar_arrive_expect_tx(&bar[B_KV_FULL + s], kPageBytes);
            const __nv_bfloat16 *src = c.pages + (int64_t)gp * kPageElems;
            // a page that several row tiles read stays in L2 for the others
            if (a.n_tiles == 1) bulk_load_hint(smem + kSKV + s * kPageBytes, src, kPageBytes, &bar[B_KV_FULL + s], pol);
            else bulk_load(smem + kSKV + s * kPageBytes, src, kPageBytes, &bar[B_KV_FULL + s]);
          }
        }
        failed = __shfl_sync(0xffffffffu, (int)failed, 0) != 0;
        if (failed) break;
      }
    }
    if (failed && lane == 0)   // do not leave while copies may still be landing
      for (int k = max(0, j - kStages); k < j; ++k)
        mbar_wait_bounded(&bar[B_KV_FULL + (k % kStages)], (k / kStages) & 1);
  } else if (warp == kMmaWarp0 || warp == kMmaWarp1) {
    // ---------------------------------------------------------------- MMA issue (whole warp, one elected lane issues)
    const int h = warp == kMmaWarp0 ? 0 : 1, n_mine = slot_pages(h);
    constexpr uint32_t idesc_qk = instr_desc(128, 64, false), idesc_pv = instr_desc(128, 128, true, true),
                       idesc_pv_bf16 = instr_desc(128, 128, true, false);
    constexpr uint32_t kStageUnits = kPageBytes >> 4;
    const uint32_t kv0 = smem_u32(smem + kSKV);
    const uint64_t dQ = smem_desc(smem_u32(smem + (kAlt ? 0 : h * 32768)), 16, 1024);
    const uint64_t dK = smem_desc(kv0, 16, 1024), dV = smem_desc(kv0 + kBlockElems * 2, 8192, 1024);
    auto issue_qk = [&](int i) {   // S = Q . K^T of the slot's page i into score buffer i & 1, committed at once
      const int j = page_of(h, i), s = j % kStages, b = i & 1;
      if (!mbar_wait_bounded(&bar[B_KV_FULL + s], (j / kStages) & 1)) { failed = true; return; }
      fence_after();
      umma_qk_page<16384 / 16, 8192 / 16>(tbase + (2 * h + b) * 64, dQ, dK + (uint64_t)s * kStageUnits, idesc_qk);
      umma_commit(&bar[B_S_FULL + 2 * h + b]);
    };
    for (int i = 0; i < min(kAhead, n_mine) && !failed; ++i) issue_qk(i);
    for (int i = 0; i < n_mine && !failed; ++i) {
      const int j = page_of(h, i), s = j % kStages, b = i & 1;
      if (!mbar_wait_bounded(&bar[B_V_READY + s], (j / kStages) & 1)) { failed = true; break; }
      if (!mbar_wait_bounded(&bar[B_P_FULL + 2 * h + b], (i >> 1) & 1)) { failed = true; break; }
      fence_after();
      const uint32_t t_p = tbase + (2 * h + b) * 64, t_o = tbase + 256 + h * 128;
      if (wide) umma_pv_page(t_o, t_p, dV + (uint64_t)s * kStageUnits, idesc_pv_bf16, i > 0 ? 1u : 0u);
      else umma_pv_page_f16(t_o, t_p, dV + (uint64_t)s * kStageUnits, idesc_pv, i > 0 ? 1u : 0u);
      umma_commit(&bar[B_KV_EMPTY + s]);   // this slot has no use for the page any more
      if (i + kAhead < n_mine) issue_qk(i + kAhead);   // (behind P.V(i): the pipe runs a thread's instructions in order)
      else umma_commit(&bar[B_O_DONE + 2 * h + b]);
    }
  } else if (warp == 2 || warp == 3) {
    // ---------------------------------------------------------------- value converter: bf16 -> scaled fp16, in place
    const int ct = tid - 64;
    for (int j = 0; j < n_pages; ++j) {
      const int s = j % kStages;
      if (!mbar_wait_bounded(&bar[B_KV_FULL + s], (j / kStages) & 1)) { failed = true; break; }
      uint4 *vb = reinterpret_cast<uint4 *>(smem + kSKV + s * kPageBytes + kBlockElems * 2) + ct;
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
  } else {
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
        // O is stable between the completion of P.V(i-1) and the hand-over of P(i).  kAlt: the scores of
        // this page were issued behind P.V(i-1).  Otherwise those of the next page were; the last page
        // has a barrier of its own.
        if (!kAlt && !(i + 1 < n_mine ? mbar_wait_bounded(&bar[B_S_FULL + 2 * h + (b ^ 1)], ((i + 1) >> 1) & 1)
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
    float *join = reinterpret_cast<float *>(smem + kSKV);   // kAlt: slot 1's rows, over the page stages
    if (kAlt) {
      // slot 1 hands its rows over; every page has been consumed by both slots before that
      asm volatile("bar.sync 1, 256;" ::: "memory");
      if (h == 1) {
        if (have && live && !failed) {
#pragma unroll
          for (int q8 = 0; q8 < 8; ++q8) {
            float t16[16];
            tmem_ld16(t_o + q8 * 16, t16);
            tmem_ld_wait();
#pragma unroll
            for (int x = 0; x < 4; ++x)
              *reinterpret_cast<float4 *>(join + row * kJoinStride + q8 * 16 + 4 * x) =
                  make_float4(t16[4 * x], t16[4 * x + 1], t16[4 * x + 2], t16[4 * x + 3]);
          }
        }
        join[row * kJoinStride + 128] = have ? m_ref : -INFINITY;
        join[row * kJoinStride + 129] = l;
      }
      asm volatile("bar.sync 1, 256;" ::: "memory");
    }
    const int r_out = (kAlt ? 0 : h * 128) + row;
    if (have && !failed && live && (!kAlt || h == 0)) {
      float f0 = o_scale, f1 = 0.f, M = m_ref;
      l *= l_scale;
      if (kAlt) {
        const float m1 = join[row * kJoinStride + 128], l1 = join[row * kJoinStride + 129];
        M = fmaxf(m_ref, m1);
        const float w0 = m_ref == -INFINITY ? 0.f : fast_exp2(m_ref - M), w1 = m1 == -INFINITY ? 0.f : fast_exp2(m1 - M);
        l = l * w0 + l1 * l_scale * w1;
        f0 = o_scale * w0;
        f1 = o_scale * w1;
      }
      const size_t at = (size_t)blockIdx.x * a.rows_per_block + r_out;
      const bool write = r_out < n_rows;
#pragma unroll
      for (int q8 = 0; q8 < 8; ++q8) {
        float t16[16];
        tmem_ld16(t_o + q8 * 16, t16);
        tmem_ld_wait();
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          float4 o = make_float4(t16[4 * x] * f0, t16[4 * x + 1] * f0, t16[4 * x + 2] * f0, t16[4 * x + 3] * f0);
          if (kAlt && f1 != 0.f) {
            const float4 p = *reinterpret_cast<const float4 *>(join + row * kJoinStride + q8 * 16 + 4 * x);
            o.x = fmaf(p.x, f1, o.x); o.y = fmaf(p.y, f1, o.y); o.z = fmaf(p.z, f1, o.z); o.w = fmaf(p.w, f1, o.w);
          }
          if (write) *reinterpret_cast<float4 *>(a.part_o + at * kD + q8 * 16 + 4 * x) = o;
        }
      }
      if (write) *reinterpret_cast<float2 *>(a.part_ml + at * 2) = make_float2(M, l);
    }
  }
  if (failed) set_status(c, SPKV_E_TIMEOUT);
  fence_before();
  __syncthreads();
  if (warp == kLoaderWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tbase), "n"(shp::kTmemCols) : "memory");
}

// One warp per query row: its shares of the common pages and its suffix.  Lane l owns dims 4l .. 4l + 3.
__global__ void __launch_bounds__(256) shared_merge_kernel(SharedArgs a) {
  const CacheView &c = a.c;
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, r = blockIdx.x * 8 + (threadIdx.x >> 5);
  if (r >= a.B * c.Hq) return;
  const int b = r / c.Hq, j = r % c.Hq, kvh = j / c.G, g = j % c.G;
  const float lse = __ldcg(a.suf_lse + r);
  const float4 so = __ldcg(reinterpret_cast<const float4 *>(a.suf_o + (size_t)r * kD) + lane);
  const int skip = __ldcg(a.item_skip + b * c.Hkv + kvh);
  float M = lse * kLog2e, L = 1.f;
  float4 O = so;
  if (skip > 0) {
    const int32_t *rec = share_record(a.plan, c.Hkv, a.layer);
    const int per = max(1, __ldcg(rec)), n = (skip + per - 1) / per;
    const int R = b * c.G + g, tile = R / kShareRows, row = R % kShareRows;
    const int first = __ldcg(rec + kShareHdr + c.Hkv + kvh) + tile;
    const int last = a.max_blocks - 1;   // (a plan that was overwritten reads no further than the workspace)
    auto at = [&](int s) { return (size_t)max(0, min(first + s * a.n_tiles, last)) * a.rows_per_block + row; };
    float pm = -INFINITY;
    for (int s = lane; s < n; s += 32) pm = fmaxf(pm, __ldcg(a.part_ml + at(s) * 2));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) pm = fmaxf(pm, __shfl_xor_sync(0xffffffffu, pm, o));
    const float top = fmaxf(M, pm);
    const float w = M == -INFINITY ? 0.f : exp2f(M - top);
    M = top;
    L = w;
    O = make_float4(so.x * w, so.y * w, so.z * w, so.w * w);
    for (int s0 = 0; s0 < n; s0 += 32) {
      float2 ml = make_float2(-INFINITY, 0.f);
      if (s0 + lane < n) ml = __ldcg(reinterpret_cast<const float2 *>(a.part_ml) + at(s0 + lane));
      const float f = ml.x == -INFINITY ? 0.f : exp2f(ml.x - top), fl = f * ml.y;
      const int cnt = min(32, n - s0);
#pragma unroll 8
      for (int x = 0; x < cnt; ++x) {
        const float4 p = __ldcg(reinterpret_cast<const float4 *>(a.part_o + at(s0 + x) * kD) + lane);
        const float fx = __shfl_sync(0xffffffffu, f, x);
        L += __shfl_sync(0xffffffffu, fl, x);
        if (fx != 0.f) {
          O.x = fmaf(p.x, fx, O.x); O.y = fmaf(p.y, fx, O.y); O.z = fmaf(p.z, fx, O.z); O.w = fmaf(p.w, fx, O.w);
        }
      }
    }
  }
  const float inv = L > 0.f ? 1.f / L : 0.f;   // (the suffix' rows come normalised: l = 1)
  uint2 pk;
  pk.x = pack_bf16(O.x * inv, O.y * inv);
  pk.y = pack_bf16(O.z * inv, O.w * inv);
  *reinterpret_cast<uint2 *>(a.out + (size_t)r * kD + lane * 4) = pk;
  if (a.lse && lane == 0) a.lse[r] = skip > 0 ? (M + log2f(L)) * kLn2 : lse;
}

struct SharedWs { size_t off_lse, off_skip, off_ml, off_o, off_dec, total; int max_blocks, rows; };
static SharedWs shared_ws_layout(const spkv_config_t *cfg, int B) {
  SharedWs w;
  auto a256 = [](size_t x) { return (x + 255) / 256 * 256; };
  const int G = cfg->n_q_heads / cfg->n_kv_heads, tiles = share_row_tiles(B, G);
  w.max_blocks = std::max(kMaxGrid, cfg->n_kv_heads * tiles);
  w.rows = std::min(kShareRows, B * G);
  size_t o = a256((size_t)B * cfg->n_q_heads * kD * 4);   // suffix rows first
  w.off_lse = o; o += a256((size_t)B * cfg->n_q_heads * 4);
  w.off_skip = o; o += a256((size_t)B * cfg->n_kv_heads * 4);
  w.off_ml = o; o += a256((size_t)w.max_blocks * w.rows * 8);
  w.off_o = o; o += a256((size_t)w.max_blocks * w.rows * kD * 4);
  w.off_dec = o; o += spkv_decode_workspace_bytes(cfg, B);
  w.total = o;
  return w;
}

}  // namespace spkv

using namespace spkv;

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
  a.c = v; a.layer = layer; a.B = B;
  a.n_tiles = share_row_tiles(B, v.G);
  a.rows_per_block = w.rows;
  a.seq_ids = d_seq_ids;
  a.q = static_cast<const __nv_bfloat16 *>(d_q);
  a.plan = static_cast<const int32_t *>(d_plan);
  a.scale_log2 = sm_scale * kLog2e;
  a.force_wide = (cache->cfg.flags & SPKV_FLAG_PREFILL_PV_BF16) ? 1 : 0;
  a.part_o = reinterpret_cast<float *>(ws + w.off_o);
  a.part_ml = reinterpret_cast<float *>(ws + w.off_ml);
  a.max_blocks = w.max_blocks;
  a.suf_o = reinterpret_cast<float *>(ws);
  a.suf_lse = reinterpret_cast<float *>(ws + w.off_lse);
  a.item_skip = reinterpret_cast<int32_t *>(ws + w.off_skip);
  a.out = static_cast<__nv_bfloat16 *>(d_out);
  a.lse = d_lse_opt;
  // blocks: one share each (the plan never cuts into more)
  const int grid = std::max(std::min(kMaxGrid, cache->sm_count), v.Hkv * a.n_tiles);
  const bool alt = w.rows <= 128;
  auto prefix = alt ? shared_prefix_kernel<true> : shared_prefix_kernel<false>;
  const int smem = shp::smem_bytes(alt);
  if (cudaFuncSetAttribute(prefix, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return SPKV_E_CUDA;
  // Overlap mode: kernels before the last one may still be running, which griddepcontrol.wait does not
  // cover; a plain launch waits for all of them.
  const bool plain = (cache->cfg.flags & SPKV_FLAG_OVERLAP) != 0;
  cache->last_kind = kLastOther;
  if (launch_link(!plain, prefix, dim3(grid), dim3(shp::kThreads), (size_t)smem, s, a) != cudaSuccess) return SPKV_E_CUDA;
  const SharedDecode sd = {a.plan, reinterpret_cast<int32_t *>(ws + w.off_skip)};
  int rc = decode_suffix(cache, layer, d_seq_ids, B, d_q, d_out, reinterpret_cast<float *>(ws),
                         reinterpret_cast<float *>(ws + w.off_lse), sm_scale, ws + w.off_dec,
                         workspace_bytes - w.off_dec, sd, stream);
  cache->last_kind = kLastOther;
  if (rc) return rc;
  return check_stream_error(
      launch_overlapped(shared_merge_kernel, dim3((B * v.Hq + 7) / 8), dim3(256), 0, s, a));
}
