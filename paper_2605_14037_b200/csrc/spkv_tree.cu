// Attention of a tree of drafted tokens over the cache (spkv_decode_attention_tree).
//
// A unit's (sequence, KV head) queries are the rows (node, head of the group) -> node * G + g, cut into tiles of 128 that
// are the M side of tcgen05 MMAs.  Its keys are pages of 64: those of the compact cache, those of the ring, and one
// page of the drafts themselves.  The pages of all units of the launch stand in one line per row tile, cut into
// equal ranges, one per block, two blocks an SM.  (Where all tiles have the same lines, the blocks of a range are
// neighbours, so that the second finds its pages in L2; where trees of different sizes leave a tile few rows, it
// gets few blocks: 13 sequences with up to 135 rows 47 -> 44.5 us.)  Where a unit lies inside a range its rows are written at
// once; otherwise the pieces leave (m, l, O) per row and tree_merge_kernel joins them by their log-sum-exp weights.
//
// Per page: S = Q K^T (8 MMAs M128 N64 K16 into tensor memory), softmax in registers (row = lane of tensor memory, two
// threads a row), P as two bf16 terms back over the scores, O += P V.  Two score buffers: the scores of the next page are
// made while this one's softmax runs.
//   * Two bf16 terms (2^-16 of a weight) take the values as they lie in the cache: one fp16 term would halve P V's MMAs but
//     wants the values converted to fp16 under a scale that fits all of them.
//   * Masks: every query sees a compact page's pairs.  Of a ring page a row sees the slots in its node's window and those
//     whose pair is kept (a bit each, by ballot over the stored logits), of the drafts' page its path.  64 bits a row
//     and page, applied to the scores.
//   * A pair that is masked has P = 0, which an infinite or NaN value would turn into NaN (as would a weight's second
//     term, which is often 0): whatever the rest of the row holds, the result is not finite then.  So the epilogue looks at
//     the results, and rows of a segment with such a one are computed again key by key (tree_rows_again).  Finite caches
//     pay one multiply-add for two results.
//   * The reference maximum is a scaled score rounded, the exponents are taken from the unrounded products: at scores of 2^31
//     the difference alone empties a row's weights or overflows them.  Rows whose reference is 2^24 or more in size (off by 1)
//     are computed again likewise, from scaled scores that are rounded alike.
//
// Warps: 0-7 softmax, 8 MMA issue and tensor memory, 9 page loader, 10 query rows, drafts and paths.
// Shared memory (113 KB, two blocks an SM): Q 32 KB, ring of five 16 KB key or value blocks in the order in which the
// MMAs want them.  Tensor memory (256 columns): score buffers at [0, 64) and [64, 128), O at [128, 256).  All waits on copies
// and MMAs are bounded; the two threads of a row, which meet at a barrier without a limit, go through the same meetings
// whether or not a wait has run out.
//
// What bounds it (B200): the first scores come after 5 - 8 us (lengths two trips to memory, page table one, page one); then
// memory, with up to 128 rows a unit (16 sequences on 16384 and on 32768 tokens: 5.0 ns a page between the two, 6.5 TB/s; 32768: 77
// us a call on the device, of which the joining kernel 6).  Called for seconds on end this draws 990 W and the clock goes down to
// 1.5 GHz: 91 us.  With several tiles nothing is full: 4 sequences on 32768 tokens, 512 rows a unit, issue in 50 % of the active
// cycles, the tensor pipe is busy 42 % of the time, DRAM 15 %; what is waited for is a page's chain (scores, softmax, P V), of two
// blocks an SM (8 x 65536, 512 rows a unit: 226 us).
#include <math.h>

#include <algorithm>
#include <atomic>

#include "spkv_tc5.cuh"
#include "spkv_tree.cuh"

namespace spkv {

namespace tree {
constexpr int kThreads = 352, kBlocksPerSm = 2;
constexpr int kMmaWarp = 8, kLoaderWarp = 9, kRowWarp = 10;   // 0-7: softmax
constexpr int kTmemCols = 256;
constexpr int kBlockBytes = kPageBytes / 2, kSlots = 5;
enum { B_FULL = 0, B_EMPTY = 5, B_S_FULL = 10 /* [page & 1] */, B_P_FULL = 12, B_O_DONE = 14, B_Q_FULL = 16, B_Q_EMPTY,
       B_TREE_FULL, B_TREE_EMPTY, B_COUNT };
constexpr int kUnitsHere = 8;       // units of a block that shared memory holds; the others stand in the workspace
constexpr int off_ring = 32768, off_bar = off_ring + kSlots * kBlockBytes, off_info = off_bar + B_COUNT * 8,
              off_path = off_info + 32, off_depth = off_path + 64 * 8, off_grow = off_depth + 64,
              off_bad = off_grow + 2 * 8 * 4, off_units = off_bad + 32, kSmemBytes = off_units + kUnitsHere * 16;
static_assert(kSmemBytes <= off_bar + 1024 && off_units % 16 == 0 && off_path % 8 == 0, "two blocks an SM");
constexpr int kPerThread = (1024 + kThreads - 1) / kThreads;   // items a thread looks at while the line is cut
// What a segment costs beside its pages, in pages: its queries, its first scores, its results.
// (13 ragged 53.6 us with 3, 51.2 with 5, 47.1 with 7, 46.6 with 10; 64 x 4096 63.0, 63.4, 62.8, 64.4.)
constexpr int kSegmentCost = 7;

// Where page i of a segment of n stands in the order in which a segment's blocks are loaded and used:
// K0 K1 V0 K2 V1 ... K(n-1) V(n-2) V(n-1)
__device__ inline int key_at(int i) { return i == 0 ? 0 : 2 * i - 1; }
__device__ inline int value_at(int i, int n) { return i == n - 1 ? 2 * n - 1 : 2 * i + 2; }
}  // namespace tree

// mbar_wait_bounded for warps that wait long and often beside others that compute: the hardware may hold a try back for
// up to 20 us before it is made again (0 - 2 % against the default limit).
__device__ inline bool tree_wait(uint64_t *bar, uint32_t parity) {
  auto attempt = [&]() {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity), "r"(20000u) : "memory");
    return ok != 0;
  };
  if (attempt()) return true;
  const long long t0 = clock64();
  while (!attempt())
    if (clock64() - t0 > kWaitClocks) return false;
  return true;
}

// A unit as the plan sees it: {its place in the line, sequence | nodes << 25, pairs received, kept pairs}.  In the line a
// unit takes kSegmentCost places and then one per page.
struct TreeUnit {
  int pre, seq, n, t, len, nk, nr, np;   // nk, nr: compact and ring pages; np: all of them, 0 if the tile has no rows
  __device__ inline TreeUnit(const TreeArgs &a, int4 m, int tile) {
    pre = m.x; seq = m.y & 0x1ffffff; n = (unsigned)m.y >> 25; t = m.z; len = m.w;
    nk = (len + kP - 1) / kP;
    nr = (min(t, a.c.w) + kP - 1) / kP;
    np = n * a.c.G > tile * kTreeRows ? nk + nr + 1 : 0;
  }
};

// the unit's page table, null for a head that keeps nothing
__device__ inline const int32_t *tree_table(const TreeArgs &a, const TreeUnit &x, int item) {
  const int kvh = item % a.c.Hkv;
  if (kvh < 64 && ((a.local_mask >> kvh) & 1)) return nullptr;
  const int below = kvh < 64 ? __popcll(a.local_mask & ((1ULL << kvh) - 1ULL)) : 0;
  return unit_table(a.c, a.row_base + x.seq * a.row_heads + kvh - below);
}
__device__ inline int tree_node_of(const TreeArgs &a, int R) { return (int)(((unsigned long long)R * a.g_inv) >> 32); }
// row of the results that query row R of an item belongs to
__device__ inline size_t tree_out_row(const TreeArgs &a, int item, int R) {
  const int b = item / a.c.Hkv, kvh = item - b * a.c.Hkv, node = tree_node_of(a, R);
  return ((size_t)b * a.T + node) * a.c.Hq + kvh * a.c.G + R - node * a.c.G;
}
// Of the 32 slots of half h of ring page p: the stored logit of this lane's.  (No ring page: anything.)
__device__ inline float tree_logit(const TreeArgs &a, const TreeUnit &x, int item, int p, int h) {
  const int at = (p - x.nk) * kP + h * 32 + (threadIdx.x & 31);
  if (p < x.nk || at >= min(x.t, a.c.w)) return 0.f;
  return __ldcg(&a.c.ring_logit[(size_t)unit_index(a.c, a.layer, x.seq, item % a.c.Hkv) * a.c.w + at]);
}
// The keys of half h of page p that query row R sees; z = tree_logit(.., p, h).  Whole warps.
__device__ inline uint32_t tree_sees(const TreeArgs &a, const TreeUnit &x, int item, int p, int h, float z,
                                     const volatile uint64_t *s_path, const volatile uint8_t *s_depth, int R) {
  const CacheView &c = a.c;
  if (p < x.nk) return (uint32_t)(bits_below(x.len - p * kP) >> (32 * h));
  const int node = min(tree_node_of(a, R), kMaxDraft - 1);
  if (p >= x.nk + x.nr) return (uint32_t)(s_path[node] >> (32 * h));
  const int kvh = item % c.Hkv, rp = p - x.nk, at = rp * kP + h * 32 + (threadIdx.x & 31);
  const bool keeps = !(kvh < 64 && ((a.local_mask >> kvh) & 1));
  const float thr = head_threshold(c, a.layer, kvh, a.tau_logit);
  const unsigned kept = __ballot_sync(0xffffffffu, keeps && (z >= thr || ring_position(x.t, c.w, at) < c.n_sink));
  return (uint32_t)(bits_below(min(x.t, c.w) - rp * kP) >> (32 * h)) &
         (~(uint32_t)(ring_out_of_window(x.t, s_depth[node], c.w, rp) >> (32 * h)) | kept);
}
// The weight f > 0 of x, which may have vanished: a finite x vanishes with it, an infinite one is infinite all the same.  (A NaN
// weight makes the row's sum, and with it the row, NaN.)
__device__ inline float weight_for(float x, float f) { return fabsf(x) == INFINITY ? 1.f : f; }
// One warp's share (every second row of a quarter of the tile) of a segment whose results are not all finite, or whose scores
// are too large for the tile's arithmetic, once more, key by key: a pair that a row does not see is not touched, and an infinite value that it sees counts with its weight, however
// small.  (P V multiplies what is masked by 0, and a weight's second term is often 0 too.)  Rare.
__device__ __noinline__ void tree_rows_again(const TreeArgs &a, int seq_nodes, int t, int len, int tile, int item, int p0, int n, int quarter,
                                             int half, int part, const volatile uint64_t *s_path, const volatile uint8_t *s_depth) {
  const TreeUnit x(a, make_int4(0, seq_nodes, t, len), tile);
  const CacheView &c = a.c;
  const int lane = threadIdx.x & 31, b = item / c.Hkv, kvh = item - b * c.Hkv, u = unit_index(c, a.layer, x.seq, kvh);
  for (int row = quarter * 32 + half; row < quarter * 32 + 32; row += 2) {   // lane: dims 4 lane .. 4 lane + 3
    const int R = tile * kTreeRows + row;
    if (R >= x.n * c.G) return;
    const int node = tree_node_of(a, R);
    const __nv_bfloat16 *qr = a.q + ((int64_t)b * a.T + node) * a.q_tok + (int64_t)(kvh * c.G + R - node * c.G) * a.q_head + lane * 4;
    float q[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
    for (int z = 0; z < 4; ++z) q[z] = __bfloat162float(qr[z]);
    for (int p = p0; p < p0 + n; ++p) {
      uint64_t mask = (uint64_t)tree_sees(a, x, item, p, 1, tree_logit(a, x, item, p, 1), s_path, s_depth, R) << 32 |
                      tree_sees(a, x, item, p, 0, tree_logit(a, x, item, p, 0), s_path, s_depth, R);
      const bool draft = p >= x.nk + x.nr;
      const int64_t page = draft ? 0 : p < x.nk ? checked_page(c, ldcg_keep(&tree_table(a, x, item)[p]), (int)ring_page(c, u, 0))
                                                : (int)ring_page(c, u, p - x.nk);
      for (; mask; mask &= mask - 1) {
        const int y = __ffsll((long long)mask) - 1;
        const __nv_bfloat16 *kr, *vr;
        if (draft) {
          const int64_t tok = (int64_t)b * a.T + y;
          kr = a.k + tok * a.k_tok + (int64_t)kvh * a.k_head + lane * 4;
          vr = a.v + tok * a.v_tok + (int64_t)kvh * a.v_head + lane * 4;
        } else {
          kr = c.pages + page * kPageElems + swz_off(y, lane >> 1) + (lane & 1) * 4;
          vr = kr + kBlockElems;
        }
        float s = 0.f;
        for (int z = 0; z < 4; ++z) s = fmaf(q[z], __bfloat162float(kr[z]), s);
        s = warp_sum(s) * a.scale_log2;
        const float top = s > m ? s : m;
        const float f = m == -INFINITY ? 1.f : fast_exp2(m - top), w = fast_exp2(s - (top == -INFINITY ? 0.f : top));
        l = l * f + w;
        for (int z = 0; z < 4; ++z) {   // (a score of -infinity: a weight that is 0)
          const float val = __bfloat162float(vr[z]);
          o[z] = fmaf(val, s == -INFINITY ? w : weight_for(val, w), o[z] * weight_for(o[z], f));
        }
        m = top;
      }
    }
    if (part < 0) {
      const size_t at = tree_out_row(a, item, R);
      const float inv = 1.f / l;
      *reinterpret_cast<uint2 *>(a.out + at * kD + lane * 4) = make_uint2(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv));
      if (a.lse && lane == 0) a.lse[at] = (m + log2f(l)) * kLn2;
    } else {
      reinterpret_cast<float4 *>(a.part_o)[((size_t)part * (kD / 4) + lane) * a.rows_pad + row] = make_float4(o[0], o[1], o[2], o[3]);
      float *ml = a.part_ml + (size_t)part * 3 * a.rows_pad + row;
      if (lane == 0) { ml[0] = m; ml[a.rows_pad] = l; ml[2 * a.rows_pad] = 0.f; }
    }
  }
}

__global__ void __launch_bounds__(tree::kThreads, tree::kBlocksPerSm) tree_attention_kernel(const __grid_constant__ TreeArgs a) {
  using namespace tc5;
  using namespace tree;
  extern __shared__ __align__(1024) unsigned char smem[];
  const CacheView &c = a.c;
  uint64_t *bar = reinterpret_cast<uint64_t *>(smem + off_bar);
  // tensor memory, first and last unit, drafts' blocks let in, range (two), tile, step between the tile's blocks
  volatile int *s_info = reinterpret_cast<volatile int *>(smem + off_info);
  volatile uint64_t *s_path = reinterpret_cast<volatile uint64_t *>(smem + off_path);   // [node] nodes it sees
  volatile uint8_t *s_depth = smem + off_depth;
  volatile unsigned *s_grow = reinterpret_cast<volatile unsigned *>(smem + off_grow);   // [page & 1][warp] rows whose maximum moves
  volatile uint8_t *s_bad = smem + off_bad;   // [page & 1, 2, 3][warp] a wait ran out; 3: a result is not finite
  int4 *s_units = reinterpret_cast<int4 *>(smem + off_units);
  volatile int *s_plan = reinterpret_cast<volatile int *>(smem + off_path);     // (before the paths are)
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < B_COUNT; ++i) mbar_init(&bar[i], i == B_P_FULL || i == B_P_FULL + 1 ? 256 : i == B_TREE_EMPTY ? 8 : 1);
    mbar_fence_init();
  }
  pdl_wait();
  pdl_trigger();   // (only now: what follows may then rely on everything before this launch)
  // ---- the line of pages, its cut, and this block's units.  Thread x holds items kPerThread x and on.
  {
    int4 meta[kPerThread];
    int cost[kPerThread], sum = 0;
    int seq[kPerThread], n[kPerThread];
    bool bad = false;
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
      const int i = tid * kPerThread + k, b = i < a.n_items ? i / c.Hkv : 0;
      seq[k] = i < a.n_items ? a.seq_ids[b] : -1;
      n[k] = i < a.n_items ? tree_nodes(a, b, &bad) : 0;
    }
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
      const int i = tid * kPerThread + k;
      const bool ok = seq[k] >= 0 && seq[k] < c.S;
      meta[k] = make_int4(0, ok ? seq[k] | n[k] << 25 : 0, 0, 0);
      if (i < a.n_items) {
        bad = bad || !ok;
        const int u = unit_index(c, a.layer, ok ? seq[k] : 0, i % c.Hkv);
        meta[k].z = ldcg_keep(&c.t[u]);
        meta[k].w = ldcg_keep(&c.len[u]);
      }
    }
    if (bad && blockIdx.x == 0) set_status(c, SPKV_E_BOUNDS);
    auto cost_of = [&](int k, int of_tile) {
      const int np = TreeUnit(a, meta[k], of_tile).np;
      return np ? np + kSegmentCost : 0;
    };
    // This block's tile and its place among the tile's blocks.  Tiles of (nearly) the same length take turns block by block, so
    // that the blocks that read the same pages do so at the same time; otherwise each tile gets blocks by its length.
    int tile = 0, range = blockIdx.x, n_blocks = gridDim.x, step = 1;
    if (a.n_tiles > 1) {
      for (int x = 0; x < a.n_tiles; ++x) {
        int length = 0;
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) length += cost_of(k, x);
        length = __reduce_add_sync(0xffffffffu, length);
        if (lane == 0) s_plan[x * 16 + warp] = length;
      }
      __syncthreads();
      long long all = 0, before = 0;
      int longest = 0, shortest = 0x7fffffff;
      for (int pass = 0; pass < 2; ++pass) {
        for (int x = 0; x < a.n_tiles; ++x) {
          int length = 0;
          for (int w = 0; w < kThreads / 32; ++w) length += s_plan[x * 16 + w];
          if (pass == 0) {
            all += length;
            longest = max(longest, length);
            shortest = min(shortest, length);
          } else {
            // blocks [from, to) of those that every tile does not get anyway are this one's
            const int spare = gridDim.x - a.n_tiles;
            const int from = (int)(spare * before / all) + x, to = (int)(spare * (before + length) / all) + x + 1;
            if ((int)blockIdx.x >= from && (int)blockIdx.x < to) { tile = x; range = blockIdx.x - from; n_blocks = to - from; }
            before += length;
          }
        }
        if (pass == 0 && (all == 0 || shortest >= longest - longest / 8)) {
          step = a.n_tiles;
          n_blocks = gridDim.x / a.n_tiles;
          range = blockIdx.x / a.n_tiles;
          tile = blockIdx.x - range * a.n_tiles;
          break;
        }
      }
      __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
      cost[k] = cost_of(k, tile);
      meta[k].x = sum;
      sum += cost[k];
      if (blockIdx.x == 0)
        for (int x = 0; x < a.n_tiles; ++x)   // nothing to join
          if (tid * kPerThread + k < a.n_items && cost_of(k, x) == 0) a.ends[(size_t)x * a.n_items + tid * kPerThread + k] = make_int4(-1, -1, 1, 0);
    }
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += x;
    }
    if (lane == 31) s_plan[warp] = incl;
    if (tid == 0) s_info[1] = s_info[2] = 0;
    __syncthreads();
    int total = 0, before = incl - sum;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
      const int x = s_plan[w];
      total += x;
      if (w < warp) before += x;
    }
    const int nb = min(n_blocks, (total + a.min_cost - 1) / a.min_cost);
    if (range >= nb) return;
    // equal lengths, but for a cut that falls next to the border of two units: it moves onto it
    const int snap = total / nb / 16;
    auto cut = [&](int x) { return total < 1 << 22 ? (int)((unsigned)x * (unsigned)total / (unsigned)nb) : (int)((long long)x * total / nb); };
    const int c0 = cut(range), c1 = cut(range + 1);
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
      meta[k].x += before;
      const int from = meta[k].x, to = from + cost[k];
      if (from <= c0 && c0 < to) {
        s_info[1] = tid * kPerThread + k;
        s_info[4] = c0 - from <= snap ? from : to - c0 <= snap ? to : c0;
      }
      if (from < c1 && c1 <= to) {
        s_info[2] = tid * kPerThread + k;
        // (a cut on a border stays there: the block behind it sees it as the start of the next unit)
        s_info[5] = c1 == to ? to : c1 - from <= snap ? from : to - c1 <= snap ? to : c1;
      }
    }
    __syncthreads();
    if (s_info[4] >= s_info[5]) return;
    // (a range may hold no page, only a part of what a segment costs)
    const int u0 = s_info[1], u1 = s_info[2];
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
      const int i = tid * kPerThread + k - u0;
      if (i < 0 || i > u1 - u0) continue;
      if (i < kUnitsHere) s_units[i] = meta[k];
      else a.units[(size_t)blockIdx.x * a.n_items + i] = meta[k];
    }
    if (tid == 0) {
      s_info[3] = 0;
      s_info[6] = tile;
      s_info[7] = step;
    }
    if (tid < 32) s_bad[tid] = 0;
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(smem + off_info)),
                 "n"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tbase = (uint32_t)s_info[0];
  bool failed = false;   // (the block's units and range are read where they are needed: no register to spare)
  auto unit_at = [&](int i) { return TreeUnit(a, i < kUnitsHere ? s_units[i] : a.units[(size_t)blockIdx.x * a.n_items + i], s_info[6]); };
  auto part_of = [&](const TreeUnit &x, int &s, int &e) {   // of the unit's pages, those of this block's range: [s, e) in the line
    s = max(x.pre + kSegmentCost, s_info[4]);
    e = min(x.pre + kSegmentCost + x.np, s_info[5]);
    return s < e;
  };
  auto first_unit = [&](int &i) {   // the unit of the block's first segment
    int s, e;
    for (;; ++i) {
      const TreeUnit x = unit_at(i);
      if (i == s_info[2] - s_info[1] || part_of(x, s, e)) return x;
    }
  };
  // f(segment, unit's place among all, unit, first page in the unit, pages) for every segment of this block; f returns false to stop
  auto segments = [&](auto f) {
    int seg = 0;
    for (int i = 0; i <= s_info[2] - s_info[1]; ++i) {
      const TreeUnit x = unit_at(i);
      int s, e;
      if (!part_of(x, s, e)) continue;
      if (!f(seg, s_info[1] + i, x, s - x.pre - kSegmentCost, e - s)) return;
      ++seg;
    }
  };
  auto copy = [&](uint32_t dst, const __nv_bfloat16 *src, bool live) {   // 16 bytes (not live: zeros)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
  };
  // Query rows r, r + step, ... of an item with n nodes -> two slabs of 128 rows x 128 B, 128-byte swizzle; lanes 0-15 and
  // 16-31 of a warp take a row each.  (Rows behind the last keep what they hold: a row of a tile does not touch another.)
  auto copy_queries = [&](int item, int n, int r, int step) {
    const int b = item / c.Hkv, kvh = item - b * c.Hkv, ch = lane & 15, tile = s_info[6], n_rows = min(kTreeRows, n * c.G - tile * kTreeRows);
    const uint32_t sQ = smem_u32(smem) + (ch >> 3) * 16384;
    const __nv_bfloat16 *src = a.q + (int64_t)b * a.T * a.q_tok + (int64_t)kvh * c.G * a.q_head + ch * 8;
#pragma unroll 4
    for (; r < n_rows; r += step) {
      const int R = tile * kTreeRows + r, i = tree_node_of(a, R);
      copy(sQ + r * 128 + (((ch & 7) ^ (r & 7)) << 4), src + i * a.q_tok + (R - i * c.G) * a.q_head, true);
    }
  };
  auto wait_slot = [&](int at) {   // the at-th block may be written to its slot
    return at < kSlots || tree_wait(&bar[B_EMPTY + at % kSlots], ((at / kSlots) - 1) & 1);
  };

  if (warp == kLoaderWarp) {
    // ---------------------------------------------------------------- page loader
    asm volatile("fence.proxy.async;" ::: "memory");   // (pages were written through generic stores)
    const uint64_t pol = l2_evict_first_policy();
    int base = 0, go = 0;     // blocks of the segments before; drafts' blocks let in
    segments([&](int, int item, const TreeUnit &x, int p0, int n) {
      const int kvh = item % c.Hkv, u = unit_index(c, a.layer, x.seq, kvh);
      const int32_t *table = tree_table(a, x, item);
      auto entry_of = [&](int i) {   // global page index of page i of the segment, -1: the drafts' page or none
        const int p = p0 + i;
        if (i >= n || p >= x.nk + x.nr) return -1;
        return p < x.nk ? checked_page(c, ldcg_keep(&table[p]), (int)ring_page(c, u, 0)) : (int)ring_page(c, u, p - x.nk);
      };
      int entry = entry_of(lane), older = entry;   // of this lane in the current and the previous 32 pages
      auto load = [&](int at, int gp, int half) {  // lane 0
        if (!wait_slot(at)) { failed = true; return; }
        if (gp < 0) {   // the drafts' page is the row warp's (which cannot wait for the slot: it would have to follow every use)
          __threadfence_block();
          s_info[3] = ++go;
          return;
        }
        uint64_t *full = &bar[B_FULL + at % kSlots];
        unsigned char *dst = smem + off_ring + at % kSlots * kBlockBytes;
        const __nv_bfloat16 *src = c.pages + (int64_t)gp * kPageElems + half * kBlockElems;
        mbar_arrive_expect_tx(full, kBlockBytes);
        // a page that several row tiles read stays in L2 for the others
        if (a.n_tiles == 1) bulk_load_hint(dst, src, kBlockBytes, full, pol);
        else bulk_load(dst, src, kBlockBytes, full);
      };
      int i = 0;
      for (; i <= n && !failed; ++i) {   // keys of page i, values of page i - 1
        if (i && (i & 31) == 0) {
          older = entry;
          entry = entry_of(i + lane);
        }
        const int gk = __shfl_sync(0xffffffffu, entry, i & 31);
        const int gv = __shfl_sync(0xffffffffu, (i & 31) == 0 ? older : entry, (i - 1) & 31);
        if (lane == 0) {
          if (i < n) load(base + key_at(i), gk, 0);
          if (i > 0 && !failed) load(base + value_at(i - 1, n), gv, 1);
        }
        failed = __shfl_sync(0xffffffffu, (int)failed, 0) != 0;
      }
      base += 2 * n;
      if (failed && lane == 0)   // do not leave while copies may still be landing
        for (int at = max(0, base - 2 * n + 2 * i - 2 - kSlots); at < base - 2 * n + 2 * i; ++at)
          tree_wait(&bar[B_FULL + at % kSlots], (at / kSlots) & 1);
      return !failed;
    });
  } else if (warp == kMmaWarp) {
    // ---------------------------------------------------------------- MMA issue (whole warp, one elected lane issues)
    constexpr uint32_t idesc_qk = instr_desc(128, 64, false), idesc_pv = instr_desc(128, 128, true);
    constexpr uint32_t kUnits = kBlockBytes >> 4;   // a block in descriptor address units
    const uint64_t dQ = smem_desc(smem_u32(smem), 16, 1024);
    const uint64_t dK = smem_desc(smem_u32(smem + off_ring), 16, 1024), dV = smem_desc(smem_u32(smem + off_ring), 8192, 1024);
    int base = 0, j0 = 0;   // blocks and pages of the segments before
    segments([&](int seg, int, const TreeUnit &, int, int n) {
      auto issue_qk = [&](int i) {   // S = Q . K^T of page i into its score buffer
        const int at = base + key_at(i), s = at % kSlots, b = (j0 + i) & 1;
        if (!tree_wait(&bar[B_FULL + s], (at / kSlots) & 1)) { failed = true; return; }
        fence_after();
        umma_qk_page<16384 / 16, 8192 / 16>(tbase + b * 64, dQ, dK + (uint64_t)s * kUnits, idesc_qk);
        umma_commit(&bar[B_S_FULL + b]);
        umma_commit(&bar[B_EMPTY + s]);
        if (i == n - 1) umma_commit(&bar[B_Q_EMPTY]);
      };
      if (seg == 0) asm volatile("bar.sync 9, 288;" ::: "memory");   // the softmax warps have fetched the queries
      else if (!tree_wait(&bar[B_Q_FULL], (seg - 1) & 1)) failed = true;
      for (int i = 0; i < min(2, n) && !failed; ++i) issue_qk(i);
      for (int i = 0; i < n && !failed; ++i) {
        const int j = j0 + i, at = base + value_at(i, n), s = at % kSlots, b = j & 1;
        if (!tree_wait(&bar[B_FULL + s], (at / kSlots) & 1) || !tree_wait(&bar[B_P_FULL + b], (j >> 1) & 1)) {
          failed = true;
          break;
        }
        fence_after();
        umma_pv_page_halves(tbase + 128, tbase + b * 64, dV + (uint64_t)s * kUnits, idesc_pv, i > 0 ? 1u : 0u);
        umma_commit(&bar[B_EMPTY + s]);
        if (i + 2 < n) issue_qk(i + 2);   // (behind P V: the pipe runs a thread's instructions in order)
        else umma_commit(&bar[B_O_DONE + b]);
      }
      base += 2 * n;
      j0 += n;
      return !failed;
    });
  } else if (warp == kRowWarp) {
    // ---------------------------------------------------------------- query rows, drafts and paths
    int base = 0, go = 0, masked = 0;   // blocks of the segments so far; drafts' blocks waited for; segments with ring or drafts
    segments([&](int seg, int item, const TreeUnit &x, int p0, int n) {
      const int b = item / c.Hkv, kvh = item - b * c.Hkv, ch = lane & 15;
      auto landed = [&]() {
        asm volatile("cp.async.wait_all;" ::: "memory");
        fence_async_smem();
        __syncwarp();
      };
      if (seg > 0 && !tree_wait(&bar[B_Q_EMPTY], (seg - 1) & 1)) failed = true;
      if (failed) return false;
      const int64_t tok0 = (int64_t)b * a.T;
      if (seg > 0) {   // (the softmax warps have fetched the first segment's)
        copy_queries(item, x.n, lane >> 4, 2);
        landed();
        if (lane == 0) mbar_arrive(&bar[B_Q_FULL]);
      }
      base += 2 * n;
      if (p0 + n <= x.nk) return true;   // compact pages only
      ++masked;
      // paths: lane holds nodes lane and lane + 32; a round doubles the stretch of ancestors known
      int up[2];
      uint64_t anc[2];
      bool bad = false;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int i = lane + 32 * h;
        up[h] = i < x.n ? (a.parent ? __ldg(&a.parent[tok0 + i]) : i - 1) : -1;
        if (up[h] < -1 || up[h] >= i) { bad = bad || i < x.n; up[h] = -1; }
        anc[h] = 1ull << i;
      }
      if (bad) set_status(c, SPKV_E_BOUNDS);
      while (__any_sync(0xffffffffu, up[0] >= 0 || up[1] >= 0)) {
        uint64_t more[2];
        int far[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int from = max(up[h], 0);
          const uint64_t m0 = __shfl_sync(0xffffffffu, anc[0], from & 31), m1 = __shfl_sync(0xffffffffu, anc[1], from & 31);
          const int f0 = __shfl_sync(0xffffffffu, up[0], from & 31), f1 = __shfl_sync(0xffffffffu, up[1], from & 31);
          more[h] = up[h] < 0 ? 0 : from < 32 ? m0 : m1;
          far[h] = up[h] < 0 ? -1 : from < 32 ? f0 : f1;
        }
        anc[0] |= more[0]; anc[1] |= more[1];
        up[0] = far[0]; up[1] = far[1];
      }
      const int depth[2] = {__popcll(anc[0]) - 1, __popcll(anc[1]) - 1};
      // ancestors that have left a node's window, but for those that are kept
      if (__any_sync(0xffffffffu, max(depth[0], depth[1]) >= c.w)) {
        const bool keeps = tree_table(a, x, item) != nullptr;
        const float thr = head_threshold(c, a.layer, kvh, a.tau_logit);
        unsigned kept[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int i = lane + 32 * h;
          kept[h] = __ballot_sync(0xffffffffu, keeps && i < x.n && (__ldg(&a.logits[(tok0 + i) * c.Hkv + kvh]) >= thr ||
                                                                    x.t + depth[h] < c.n_sink));
        }
        const uint64_t keep = (uint64_t)kept[1] << 32 | kept[0];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint64_t rest = anc[h];
          for (int left = depth[h] + 1 - c.w; left > 0; --left) {   // (an ancestor's index is lower: the lowest are the oldest)
            const uint64_t oldest = rest & (0 - rest);
            rest ^= oldest;
            if (!(keep & oldest)) anc[h] ^= oldest;
          }
        }
      }
      if (masked > 1 && !tree_wait(&bar[B_TREE_EMPTY], masked & 1)) failed = true;
      if (failed) return false;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        s_path[lane + 32 * h] = anc[h];
        s_depth[lane + 32 * h] = (uint8_t)depth[h];
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&bar[B_TREE_FULL]);
      // the drafts' page, if it is in the segment: its last
      if (p0 + n == x.np) {
        for (int half = 0; half < 2; ++half) {
          const int at = base - 2 * n + (half ? value_at(n - 1, n) : key_at(n - 1));
          ++go;
          for (const long long since = clock64(); s_info[3] < go && !failed;) failed = clock64() - since > kWaitClocks;
          if (__any_sync(0xffffffffu, failed)) { failed = true; return false; }
          __threadfence_block();
          const uint32_t dst = smem_u32(smem + off_ring + at % kSlots * kBlockBytes);
          const __nv_bfloat16 *src = (half ? a.v + (int64_t)kvh * a.v_head : a.k + (int64_t)kvh * a.k_head) + ch * 8;
          const int64_t tok = half ? a.v_tok : a.k_tok;
          for (int r = lane >> 4; r < kP; r += 2) copy(dst + blk_off(r, ch), src + (tok0 + min(r, x.n - 1)) * tok, r < x.n);
          landed();
          if (lane == 0) mbar_arrive(&bar[B_FULL + at % kSlots]);
        }
      }
      return true;
    });
  } else {
    // ---------------------------------------------------------------- softmax
    // A row belongs to two threads, one in warps 0-3 (half 0) and one in warps 4-7: each has 32 of a page's 64 scores and 64
    // of the row's 128 output dims.  They meet once a page: whether the row's reference maximum has to move, which
    // it rarely does.
    const int half = warp >> 2, quarter = warp & 3, row = quarter * 32 + lane, R = s_info[6] * kTreeRows + row;
    const uint32_t t_lane = tbase + ((uint32_t)(quarter * 32) << 16), t_o = t_lane + 128 + half * 64;
    {   // the first segment's queries
      int i = 0;
      const TreeUnit x = first_unit(i);
      copy_queries(s_info[1] + i, x.n, warp * 2 + (lane >> 4), 16);
      asm volatile("cp.async.wait_all;" ::: "memory");
      fence_async_smem();
      asm volatile("bar.arrive 9, 288;" ::: "memory");
    }
    auto meet = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(1 + quarter) : "memory"); };
    // a number from the row's other thread, by way of tensor memory (`mine`, `its`: a free column of either)
    auto swap = [&](uint32_t mine, uint32_t its, float x) {
      tmem_st1(mine, x);
      tmem_st_wait();
      fence_before();
      meet();
      fence_after();
      x = tmem_ld1(its);
      tmem_ld_wait();
      fence_before();
      meet();      // (both have read before the columns are used again)
      fence_after();
      return x;
    };
    // pages of the segments before; segments with ring or drafts; parity of the commits so far of the two O_DONE barriers
    int j0 = 0, masked = 0, od = 0;
    segments([&](int seg, int item, const TreeUnit &x, int p0, int n) {
      // (What is needed for masks only is read again where it is needed: the loop over pages has no register to spare, and a
      // spilled one comes back from L2.)
      const int nk = x.nk;
      const bool row_live = R < x.n * c.G;
      const bool live = R - lane < x.n * c.G;   // warps without a live row only keep the barriers going
      float lg = tree_logit(a, x, item, p0, half);   // stored logit of this lane's slot of the page that comes next, if of the ring
      float m_ref = -INFINITY, l = 0.f;
      bool left_together = false;
      for (int i = 0; i < n; ++i) {
        const int j = j0 + i, bf = j & 1, p = p0 + i;
        uint32_t mask = 0xffffffffu;   // the keys that this row sees
        if (p >= nk - 1) {
          if (p >= nk && (i == 0 || p == nk) && !tree_wait(&bar[B_TREE_FULL], masked & 1)) failed = true;
          mask = tree_sees(a, x, item, p, half, lg, s_path, s_depth, R);
          lg = tree_logit(a, x, item, p + 1, half);
        }
        if (!failed && !tree_wait(&bar[B_S_FULL + bf], (j >> 1) & 1)) failed = true;
        fence_after();
        if (!live) {
          if (failed) break;
          fence_before();
          mbar_arrive(&bar[B_P_FULL + bf]);
          continue;
        }
        const uint32_t t_s = t_lane + bf * 64;
        float v[32];
        auto fetch_scores = [&]() {
#pragma unroll
          for (int q2 = 0; q2 < 2; ++q2) {
            float t16[16];
            tmem_ld16(t_s + half * 32 + q2 * 16, t16);
#pragma unroll
            for (int y = 0; y < 16; ++y) v[q2 * 16 + y] = t16[y];
          }
          tmem_ld_wait();
        };
        auto apply_mask = [&]() {
          if (p >= nk - 1) {
#pragma unroll
            for (int y = 0; y < 32; ++y) v[y] = (mask >> y) & 1 ? v[y] : -INFINITY;
          }
        };
        fetch_scores();
        apply_mask();
        float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
        for (int y = 0; y < 32; y += 4) {
          mx0 = max3(mx0, v[y], v[y + 1]);
          mx1 = max3(mx1, v[y + 2], v[y + 3]);
        }
        const float mx = fmaxf(mx0, mx1) * a.scale_log2;
        // the reference maximum moves only when the row maximum outgrows it by 2^8
        unsigned grown = __ballot_sync(0xffffffffu, failed || (mx > m_ref + 8.f && row_live));
        if (lane == 0) s_grow[bf * 8 + warp] = grown;
        if (failed && lane == 0) s_bad[bf * 8 + warp] = 1;
        fence_before();
        meet();
        fence_after();
        grown |= s_grow[bf * 8 + (warp ^ 4)];
        if (grown) {
          // (a wait that ran out stays noted: the row's threads leave together, `meet` has no limit)
          failed = left_together = failed || s_bad[bf * 8 + (warp ^ 4)];
          if (failed) break;
          const float first = v[0];   // (its column is used for the exchange)
          const float both = fmaxf(mx, swap(t_s + half * 32, t_s + (half ^ 1) * 32, mx));
          const bool grow = both > m_ref + 8.f && row_live;
          const float m_new = grow ? both : m_ref;
          if (i > 0) {
            // O is stable between the completion of P V of the page before and the hand-over of P.  The scores of the next
            // page were issued behind that P V; before the last page it has a barrier of its own.
            if (!(i + 1 < n ? tree_wait(&bar[B_S_FULL + (bf ^ 1)], ((j + 1) >> 1) & 1)
                            : tree_wait(&bar[B_O_DONE + (bf ^ 1)], (od >> (bf ^ 1)) & 1)))
              failed = true;   // (noticed by both at their next meeting)
            fence_after();
            const float f = grow ? fast_exp2(m_ref - m_new) : 1.f;   // m_ref = -inf -> 0
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
              float t16[16];
              tmem_ld16(t_o + q4 * 16, t16);
              tmem_ld_wait();
#pragma unroll
              for (int y = 0; y < 16; ++y) t16[y] *= f;
              tmem_st16(t_o + q4 * 16, t16);
            }
            l *= f;
          }
          m_ref = m_new;
          fetch_scores();             // again: kept across all this they would not fit the registers
          v[0] = first;
          apply_mask();
        }
        const float ms = m_ref == -INFINITY ? 0.f : m_ref;
        const float2 sc2 = make_float2(a.scale_log2, a.scale_log2), nms2 = make_float2(-ms, -ms);
        float2 l2a = make_float2(0.f, 0.f), l2b = l2a;
        // two terms, two keys a column, over the half's own scores (the other half may still have to fetch its own, again
        // if the reference moved): 16 columns the first, 16 the second
#pragma unroll
        for (int q2 = 0; q2 < 2; ++q2) {
          uint32_t hi[8], lo[8];
#pragma unroll
          for (int y = 0; y < 8; ++y) {
            const float2 e = __ffma2_rn(make_float2(v[q2 * 16 + 2 * y], v[q2 * 16 + 2 * y + 1]), sc2, nms2);
            const float2 w = make_float2(fast_exp2(e.x), fast_exp2(e.y));
            if (y & 1) l2b = __fadd2_rn(l2b, w); else l2a = __fadd2_rn(l2a, w);
            hi[y] = pack_bf16(w.x, w.y);
            const float2 r = __fadd2_rn(w, make_float2(-__uint_as_float(hi[y] << 16), -__uint_as_float(hi[y] & 0xffff0000u)));
            lo[y] = pack_bf16(r.x, r.y);
          }
          tmem_st8u(t_s + half * 32 + q2 * 8, hi);
          tmem_st8u(t_s + half * 32 + 16 + q2 * 8, lo);
        }
        l2a = __fadd2_rn(l2a, l2b);
        l += l2a.x + l2a.y;
        tmem_st_wait();
        fence_before();
        mbar_arrive(&bar[B_P_FULL + bf]);
      }
      // ---- the rows' results, or their parts
      if (failed && left_together) return false;
      const int last = (j0 + n - 1) & 1;
      if (!failed && !tree_wait(&bar[B_O_DONE + last], (od >> last) & 1)) failed = true;
      fence_after();
      od ^= n > 1 ? 3 : 1 << last;
      j0 += n;
      const bool whole = n == x.np, starts = p0 == 0, ends = p0 + n == x.np;
      if (warp == 0 && lane == 0 && (starts || ends)) {
        int *e = reinterpret_cast<int *>(&a.ends[(size_t)s_info[6] * a.n_items + item]);
        if (starts) { e[0] = blockIdx.x; e[2] = s_info[7]; }
        if (ends) e[1] = blockIdx.x;
      }
      if (live) {
        const int part = whole ? -1 : (int)blockIdx.x * 2 + (starts ? 1 : 0);
        uint64_t finite = 0;   // 0 times everything: 0, or NaN
        float t16[16];
        tmem_ld16(t_o, t16);
        tmem_ld_wait();
        if (whole) {
          // (the sums are exchanged through the first column of O, once that is in registers)
          const float sum = l + swap(t_o, t_lane + 128 + (half ^ 1) * 64, l), inv = 1.f / sum;
          const size_t at = tree_out_row(a, item, row_live ? R : 0);
          uint4 *o = reinterpret_cast<uint4 *>(a.out + at * kD + half * 64);
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            if (q4) {
              tmem_ld16(t_o + q4 * 16, t16);
              tmem_ld_wait();
            }
            uint32_t w[8];
#pragma unroll
            for (int y = 0; y < 8; ++y) {
              finite = fma2(pack2(t16[2 * y], t16[2 * y + 1]), 0, finite);
              w[y] = pack_bf16(t16[2 * y] * inv, t16[2 * y + 1] * inv);
            }
            if (row_live) {
              o[2 * q4] = make_uint4(w[0], w[1], w[2], w[3]);
              o[2 * q4 + 1] = make_uint4(w[4], w[5], w[6], w[7]);
            }
          }
          if (row_live && half == 0 && a.lse) a.lse[at] = (m_ref + log2f(sum)) * kLn2;
        } else {
          float4 *o = reinterpret_cast<float4 *>(a.part_o) + ((size_t)part * (kD / 4) + half * 16) * a.rows_pad + row;
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            if (q4) {
              tmem_ld16(t_o + q4 * 16, t16);
              tmem_ld_wait();
            }
#pragma unroll
            for (int y = 0; y < 8; ++y) finite = fma2(pack2(t16[2 * y], t16[2 * y + 1]), 0, finite);
#pragma unroll
            for (int y = 0; y < 4; ++y, o += a.rows_pad) *o = make_float4(t16[4 * y], t16[4 * y + 1], t16[4 * y + 2], t16[4 * y + 3]);
          }
          float *ml = a.part_ml + (size_t)part * 3 * a.rows_pad + row;   // m, and the two halves' l
          if (half == 0) ml[0] = m_ref;
          ml[(1 + half) * a.rows_pad] = l;
        }
        float f0, f1;
        unpack2(finite, f0, f1);
        const bool odd = __any_sync(0xffffffffu, row_live && (f0 + f1 + 0.f * l != 0.f || (fabsf(m_ref) >= 0x1p24f && m_ref != -INFINITY)));
        if (lane == 0) s_bad[3 * 8 + warp] = odd | failed << 1;
        meet();
        const int both = odd | failed << 1 | s_bad[3 * 8 + (warp ^ 4)];
        failed = both >> 1;
        if (both == 1)
          tree_rows_again(a, x.seq | x.n << 25, x.t, x.len, s_info[6], item, p0, n, quarter, half, part, s_path, s_depth);
      }
      if (failed) return false;
      if (p0 + n > nk) {   // the segment's paths are done with
        ++masked;
        __syncwarp();
        if (lane == 0) mbar_arrive(&bar[B_TREE_EMPTY]);
      }
      return true;
    });
  }
  if (failed) set_status(c, SPKV_E_TIMEOUT);
  fence_before();
  __syncthreads();
  if (warp == kMmaWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tbase), "n"(tree::kTmemCols) : "memory");
}

// ---- joining parts -----------------------------------------------------------------------------------
// A block joins 32 rows x kDims dims of a unit that several ranges hold pieces of: its warps take every kWarps-th piece
// (lane = row, all its dims of kAhead pieces asked for at once), then add up through shared memory.
template <int kWarps, int kDims, int kAhead>
__global__ void __launch_bounds__(32 * kWarps) tree_merge_kernel(const __grid_constant__ TreeArgs a) {
  __shared__ float s_o[kWarps][kDims][33], s_m[kWarps][32], s_l[kWarps][32];
  const CacheView &c = a.c;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int item = blockIdx.x / a.n_tiles, tile = blockIdx.x - item * a.n_tiles;
  const int row = blockIdx.y * 32 + lane, dim0 = blockIdx.z * kDims;
  const int b = item / c.Hkv, kvh = item - b * c.Hkv;
  bool bad = false;
  const int n_rows = tree_nodes(a, b, &bad) * c.G - tile * kTreeRows;
  pdl_trigger();
  pdl_wait();
  const int4 ends = __ldcg(&a.ends[(size_t)tile * a.n_items + item]);
  if (ends.x == ends.y || (int)blockIdx.y * 32 >= n_rows) return;   // whole: written already
  // (after a wait that ran out the entry may be what the workspace held before)
  if (ends.x < 0 || ends.y >= tree::kBlocksPerSm * kMaxGrid || ends.z < 1 || ends.z > a.n_tiles) return;
  float M = -INFINITY, L = 0.f, O[kDims];
#pragma unroll
  for (int x = 0; x < kDims; ++x) O[x] = 0.f;
  // A part's weight against the common maximum.  A part without a visible pair (`none`) has l = 0; m = -inf with another l
  // means NaN scores.
  auto none = [](float m, float l) { return m == -INFINITY && l == 0.f; };
  auto weight = [&](float m, float l, float to) { return none(m, l) ? 0.f : m == -INFINITY ? NAN : fast_exp2(m - to); };
  for (int r0 = ends.x + warp * ends.z; r0 <= ends.y; r0 += kWarps * kAhead * ends.z) {
    float v[kAhead][kDims], m[kAhead], l[kAhead], to = M;
#pragma unroll
    for (int y = 0; y < kAhead; ++y) {
      const int r = min(r0 + y * kWarps * ends.z, ends.y);
      const size_t part = (size_t)r * 2 + (r == ends.x ? 1 : 0);
      const float *ml = a.part_ml + part * 3 * a.rows_pad + row;
      const float4 *o = reinterpret_cast<const float4 *>(a.part_o) + (part * (kD / 4) + dim0 / 4) * a.rows_pad + row;
      m[y] = __ldcg(ml);
      l[y] = __ldcg(ml + a.rows_pad) + __ldcg(ml + 2 * a.rows_pad);
#pragma unroll
      for (int x = 0; x < kDims; x += 4) {
        const float4 q = __ldcg(o + x / 4 * a.rows_pad);
        v[y][x] = q.x; v[y][x + 1] = q.y; v[y][x + 2] = q.z; v[y][x + 3] = q.w;
      }
      if (r0 + y * kWarps * ends.z > ends.y) { m[y] = -INFINITY; l[y] = 0.f; }
    }
#pragma unroll
    for (int y = 0; y < kAhead; ++y) to = fmaxf(to, m[y]);
    const float old = weight(M, L, to);
    M = to;
    L *= old;
#pragma unroll
    for (int x = 0; x < kDims; ++x) O[x] *= weight_for(O[x], old);
#pragma unroll
    for (int y = 0; y < kAhead; ++y) {
      if (none(m[y], l[y])) continue;
      const float f = weight(m[y], l[y], M);
      L = fmaf(l[y], f, L);
#pragma unroll
      for (int x = 0; x < kDims; ++x) O[x] = fmaf(v[y][x], weight_for(v[y][x], f), O[x]);
    }
  }
#pragma unroll
  for (int x = 0; x < kDims; ++x) s_o[warp][x][lane] = O[x];
  s_m[warp][lane] = M;
  s_l[warp][lane] = L;
  __syncthreads();
  for (int z = threadIdx.x; z < 32 * kDims / 8; z += 32 * kWarps) {   // eight dims of a row
    const int r = z / (kDims / 8), q = z % (kDims / 8), at_row = blockIdx.y * 32 + r;
    if (at_row >= n_rows) return;
    float Mr = -INFINITY, Lr = 0.f, o[8] = {};
#pragma unroll
    for (int w = 0; w < kWarps; ++w) Mr = fmaxf(Mr, s_m[w][r]);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      if (none(s_m[w][r], s_l[w][r])) continue;
      const float f = weight(s_m[w][r], s_l[w][r], Mr);
      Lr = fmaf(s_l[w][r], f, Lr);
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const float v = s_o[w][q * 8 + x][r];
        o[x] = fmaf(v, weight_for(v, f), o[x]);
      }
    }
    const int R = tile * kTreeRows + at_row, node = (int)(((unsigned long long)R * a.g_inv) >> 32);
    const size_t at = ((size_t)b * a.T + node) * c.Hq + kvh * c.G + R - node * c.G;
    const float inv = 1.f / Lr;
    *reinterpret_cast<uint4 *>(a.out + at * kD + dim0 + q * 8) =
        make_uint4(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv), pack_bf16(o[4] * inv, o[5] * inv),
                   pack_bf16(o[6] * inv, o[7] * inv));
    if (a.lse && dim0 == 0 && q == 0) a.lse[at] = (Mr + log2f(Lr)) * kLn2;
  }
}

template <int kWarps, int kDims, int kAhead>
static cudaError_t launch_tree_merge(const TreeArgs &a, cudaStream_t s) {
  static std::atomic<unsigned long long> ready;
  auto kernel = tree_merge_kernel<kWarps, kDims, kAhead>;
  // (with another split of an SM's memory than the attention kernel's, the SM would have to change it between the two)
  if (whole_shared_memory(reinterpret_cast<const void *>(kernel), 0, &ready)) return cudaErrorUnknown;
  return launch_overlapped(kernel, dim3(a.n_items * a.n_tiles, a.rows_pad / 32, kD / kDims), dim3(32 * kWarps), 0, s, a);
}

struct TreeWs { size_t off_units, off_ml, off_o, total; int n_tiles, rows_pad; };
static TreeWs tree_ws_layout(const spkv_config_t *cfg, int B, int T, int blocks) {
  TreeWs w;
  auto a256 = [](size_t x) { return (x + 255) / 256 * 256; };
  const int G = cfg->n_q_heads / cfg->n_kv_heads;
  const size_t items = (size_t)B * cfg->n_kv_heads;
  w.n_tiles = std::max(1, (T * G + kTreeRows - 1) / kTreeRows);
  w.rows_pad = std::min(kTreeRows, (T * G + 31) / 32 * 32);
  w.off_units = a256(items * w.n_tiles * sizeof(int4));
  w.off_ml = w.off_units + a256((size_t)blocks * items * sizeof(int4));
  w.off_o = w.off_ml + a256((size_t)blocks * 6 * w.rows_pad * 4);
  w.total = w.off_o + a256((size_t)blocks * 2 * kD * w.rows_pad * 4);
  return w;
}
constexpr int kMaxTreeBlocks = tree::kBlocksPerSm * kMaxGrid;

}  // namespace spkv

using namespace spkv;

static std::atomic<unsigned long long> g_tree_ready;   // devices on which the kernel's attributes are set, a bit each

extern "C" size_t spkv_decode_tree_workspace_bytes(const spkv_config_t *cfg, int32_t B, int32_t T) {
  if (!cfg || B < 0 || T < 0 || T > kMaxDraft || cfg->n_kv_heads < 1 || cfg->n_q_heads < cfg->n_kv_heads) return 0;
  if (B == 0 || T == 0) return 0;
  return tree_ws_layout(cfg, B, T, kMaxTreeBlocks).total;
}

extern "C" int spkv_decode_attention_tree(spkv_cache_t *cache, int32_t layer, const int32_t *d_seq_ids, int32_t B, int32_t T,
                                          const int32_t *d_n_nodes, const int32_t *d_parent, const spkv_rows_t *q,
                                          const spkv_rows_t *k, const spkv_rows_t *v, const float *d_logits, void *d_out,
                                          float *d_lse_opt, float sm_scale, void *d_workspace, size_t workspace_bytes,
                                          spkv_stream_t stream) {
  if (!cache || layer < 0 || layer >= cache->cfg.n_layers || B < 0 || B > cache->cfg.max_seqs || T < 0 || T > kMaxDraft)
    return SPKV_E_INVALID;
  if (!(sm_scale > 0.f) || !isfinite(sm_scale)) return SPKV_E_INVALID;
  if (B == 0 || T == 0) return SPKV_OK;
  const CacheView &view = cache->view;
  if (!d_seq_ids || !bf16_rows_ok(q) || !bf16_rows_ok(k) || !bf16_rows_ok(v) || !d_out || ((uintptr_t)d_out & 15)) return SPKV_E_INVALID;
  if (!d_logits && T > view.w) return SPKV_E_INVALID;
  if (B * view.Hkv > 1024) return SPKV_E_UNSUPPORTED;
  if (!d_workspace || ((uintptr_t)d_workspace & 255) || workspace_bytes < spkv_decode_tree_workspace_bytes(&cache->cfg, B, T))
    return SPKV_E_WORKSPACE;
  const TreeWs w = tree_ws_layout(&cache->cfg, B, T, kMaxTreeBlocks);
  char *ws = static_cast<char *>(d_workspace);
  TreeArgs a = {};
  a.c = view; a.layer = layer; a.B = B; a.T = T; a.n_items = B * view.Hkv;
  a.seq_ids = d_seq_ids; a.n_nodes = d_n_nodes; a.parent = d_parent;
  a.q = static_cast<const __nv_bfloat16 *>(q->ptr); a.q_tok = q->token_stride; a.q_head = q->head_stride;
  a.k = static_cast<const __nv_bfloat16 *>(k->ptr); a.k_tok = k->token_stride; a.k_head = k->head_stride;
  a.v = static_cast<const __nv_bfloat16 *>(v->ptr); a.v_tok = v->token_stride; a.v_head = v->head_stride;
  a.logits = d_logits;
  a.out = static_cast<__nv_bfloat16 *>(d_out);
  a.lse = d_lse_opt;
  a.scale_log2 = sm_scale * kLog2e;
  a.tau_logit = cache->tau_logit;
  a.g_inv = ((1ULL << 32) + view.G - 1) / view.G;
  for (int l = 0; l < layer; ++l) a.row_base += (view.Hkv - __builtin_popcountll(cache->local_mask[l])) * view.S;
  a.row_heads = view.Hkv - __builtin_popcountll(cache->local_mask[layer]);
  a.local_mask = cache->local_mask[layer];
  a.ends = reinterpret_cast<int4 *>(ws);
  a.units = reinterpret_cast<int4 *>(ws + w.off_units);
  a.part_ml = reinterpret_cast<float *>(ws + w.off_ml);
  a.part_o = reinterpret_cast<float *>(ws + w.off_o);
  a.rows_pad = w.rows_pad;
  a.n_tiles = w.n_tiles;
  const int blocks = tree::kBlocksPerSm * std::min(kMaxGrid, cache->sm_count);
  // Shortest range, in pages: shorter ones go to more blocks and leave more pieces to join.  With 1 / 5 / 8 (us): 1 x 131072 tokens,
  // 16 nodes 29.8 / 26.0 / 27.9, 16 x 1000 with 8 nodes 25.5 / 22.2 / 24.9; but 1 x 8000 with 16 nodes 19.3 / 22.7 / 24.3, 4 x 2000
  // 20.0 / 23.1 / 24.8, 8 x 8000 with 32 36.4 / 38.5 / 34.3; 1 x 300, and from 24 x 16384 on: alike.
  a.min_cost = 5 + tree::kSegmentCost;
  if (const int rc = whole_shared_memory(reinterpret_cast<const void *>(tree_attention_kernel), tree::kSmemBytes, &g_tree_ready)) return rc;
  // Overlap mode: kernels before the last one may still be running, which griddepcontrol.wait does not
  // cover; a plain launch waits for all of them.
  const bool plain = (cache->cfg.flags & SPKV_FLAG_OVERLAP) != 0;
  cache->last_kind = kLastOther;
  cudaStream_t s = as_stream(stream);
  if (launch_link(!plain, tree_attention_kernel, dim3(blocks), dim3(tree::kThreads), (size_t)tree::kSmemBytes, s, a) !=
      cudaSuccess)
    return SPKV_E_CUDA;
  // Pieces of a unit's tile: about blocks / tiles + 1.  Few: two warps a block, 32 dims; many: eight warps and 16 dims, so that more of
  // them are on their way (16 x 32768 78 / 86 us, 24 x 16384 63 / 74, 16 x 1000 22.1 / 23.0; 1 x 131072 40.4 / 26.0, 1 x 32768
  // 25.4 / 24.1).  Between, at 4.6 blocks a tile, the first would still be the faster one (8 x 8000 33.5 / 38.5).
  return check_stream_error(blocks < 4 * a.n_items * a.n_tiles ? launch_tree_merge<2, 32, 1>(a, s) : launch_tree_merge<8, 16, 2>(a, s));
}
