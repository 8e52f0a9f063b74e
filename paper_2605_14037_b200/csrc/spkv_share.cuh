// What a batch with a common prefix decodes by: the plan's layout and the cut of the common pages.
//
// Plan (int32): header {B, layers, KV heads, row tiles, 0 ...}, then one record per layer:
//   {pages per share, blocks, 0, 0, common pages [Hkv], first block [Hkv]}.
// The queries of KV head h are the rows (b, g) -> b * G + g of its group in every sequence, cut into tiles
// of kShareRows.  A block takes one share of one head's common pages for one row tile; block first[h] +
// share * row_tiles + tile.  The tiles of a share are neighbours, so that they find its pages in L2.
#pragma once
#include "spkv_internal.cuh"

namespace spkv {

constexpr int kSharePlanHdr = 8, kShareHdr = 4;
constexpr int kShareRows = 256;       // query rows per block: two slots of 128
constexpr int kMinSharedPages = 1;    // fewer common pages than this are read per sequence
constexpr int kMinSharePages = 4;     // a share is not cut shorter

__host__ __device__ inline int share_row_tiles(int B, int G) { return (B * G + kShareRows - 1) / kShareRows; }
template <class I>
__host__ __device__ inline I *share_record(I *plan, int Hkv, int layer) {
  return plan + kSharePlanHdr + (size_t)layer * (kShareHdr + 2 * Hkv);
}

// What the decode kernel needs to leave a batch's common pages out.
struct SharedDecode {
  const int32_t *plan;
  int32_t *item_skip;   // [B * Hkv] out: the pages each unit left out
};
int decode_check_args(const spkv_cache_t *cache, int32_t layer, const int32_t *d_seq_ids, int32_t B, const void *d_q,
                      const void *d_out, const float *d_out_f32, bool *empty);
int decode_suffix(spkv_cache *cache, int32_t layer, const int32_t *d_seq_ids, int32_t B, const void *d_q, void *d_out,
                  float *d_out_f32, float *d_lse, float sm_scale, void *d_workspace, size_t workspace_bytes,
                  const SharedDecode &sd, spkv_stream_t stream);

}  // namespace spkv
