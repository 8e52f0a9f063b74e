// What the drafted-tree attention's kernels share: arguments, paths of a tree, and which pairs of the window a node sees.
#pragma once
#include "spkv_decode_common.cuh"

namespace spkv {

constexpr int kMaxDraft = SPKV_MAX_DRAFT;
constexpr int kTreeRows = 128;     // query rows (node, head of the group) of a tile: the lanes of tensor memory
static_assert(kMaxDraft == kP, "a sequence's drafts are one page, a path is one bit per row of it");

struct TreeArgs {
  CacheView c;
  int layer, B, T, n_items;
  const int32_t *seq_ids, *n_nodes, *parent;   // n_nodes, parent: may be null
  const __nv_bfloat16 *q, *k, *v;
  int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head;   // strides in elements
  const float *logits;          // [B][T][Hkv] or null (T <= window)
  __nv_bfloat16 *out;           // [B][T][Hq][128]
  float *lse;                   // [B][T][Hq] or null
  float scale_log2, tau_logit;
  // ---- the tensor-core form
  int n_tiles, min_cost;                       // row tiles of kTreeRows; shortest range that the line of pages is cut into
  unsigned long long g_inv;                    // ceil(2^32 / G): row / G as a product and a shift
  int row_base, row_heads;                     // page-table rows of the layer: row_base + seq * row_heads + rank of the KV head
  unsigned long long local_mask;
  int4 *units;                                 // [blocks][n_items]: a block's units behind the first few
  int4 *ends;                                  // [n_tiles][n_items]: blocks of a unit's first and last page, step between its blocks
  float *part_o, *part_ml;                     // [blocks][2][32][rows_pad][4 dims], [blocks][2][3][rows_pad]: m, two shares of l
  int rows_pad;
};

// bf16 rows that are read sixteen bytes at a time
inline bool bf16_rows_ok(const spkv_rows_t *r) {
  return r && r->ptr && !((uintptr_t)r->ptr & 15) && !((r->token_stride | r->head_stride) & 7);
}

// nodes of sequence b; *bad is set for a count outside [0, T]
__device__ inline int tree_nodes(const TreeArgs &a, int b, bool *bad) {
  if (!a.n_nodes) return a.T;
  const int n = __ldg(&a.n_nodes[b]), m = max(0, min(n, a.T));
  if (m != n) *bad = true;
  return m;
}

// Ring slots that a node of depth d does not see by its window are those of positions <= t + d - w: a run of slots,
// around the end of the ring, from the oldest pair's on.  Bits of ring page p.
__device__ inline uint64_t bits_below(int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1ull; }
__device__ inline uint64_t ring_out_of_window(int t, int d, int w, int p) {
  const int first = t >= w ? t % w : 0, n = t >= w ? min(d + 1, w) : max(0, t + d - w + 1);
  const int e = first + n - p * 64, s = first - p * 64;
  uint64_t m = bits_below(min(e, w - p * 64)) & ~bits_below(s);
  if (first + n > w) m |= bits_below(first + n - w - p * 64);
  return m;
}
// position of the pair in ring slot x of a unit that has received t pairs
__device__ inline int ring_position(int t, int w, int x) {
  if (t <= w) return x;
  const int at = t % w;
  return x >= at ? t - w + x - at : t - at + x;
}

}  // namespace spkv
