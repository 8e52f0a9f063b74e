// What a batch with a common prefix decodes by: the plan's layout and the cut of the common pages.
//
// Plan (int32): kSharePlanHdr words that nobody reads (records start at a multiple of 32 bytes), then one record per layer:
//   {pages per share, blocks, 0, 0}
//   per KV head  {common pages, first block, page-table row and unit of the batch's first sequence},
//                {prefix shares, tail shares, signature, 0}
//   per block    {KV head, row tile, first page, pages (0: no work)}, {common pages, row, unit, signature}
// The queries of KV head h are the rows (b, g) -> b * G + g of its group in every sequence, cut into tiles
// of kShareRows.  A block takes one share of one head's common pages for one row tile; block first[h] +
// share * row_tiles + tile.  The tiles of a share are neighbours, so that they find its pages in L2.
// A block's descriptor holds all it needs to know, so that it costs one trip to memory and its first
// page-table entries the second (148 blocks that each walk the plan by themselves queue up at the
// same few L2 lines: measured, 8 us of an 18 us launch).
#pragma once
#include "spkv_decode_common.cuh"

namespace spkv {

constexpr int kSharePlanHdr = 8, kShareHdr = 4, kShareHead = 8, kShareDesc = 8;
constexpr int kShareRows = 256;       // query rows per block: two slots of 128
constexpr int kMinSharedPages = 1;    // fewer common pages than this are read per sequence
constexpr int kMinSharePages = 2;     // a share is not cut shorter (2 sequences on 4096 tokens: 10.4 us on the device, 10.9 with 4)
constexpr int kTailPages = 8;         // a unit's own pages are cut into pieces of about this many, more while SMs are left
constexpr int kTailMinPages = 2;      // ... not into shorter ones than this
constexpr int kMaxTailItems = 1024;   // ... and not into more pieces than this, all units together

__host__ __device__ inline int share_row_tiles(int B, int G) { return (B * G + kShareRows - 1) / kShareRows; }
// blocks a layer's record has room for, whatever the batch (B * Hkv <= 1024, B <= max_seqs)
__host__ __device__ inline int share_max_blocks(int max_seqs, int Hkv, int G) {
  const int B = max_seqs < 1024 / Hkv ? max_seqs : (1024 / Hkv > 1 ? 1024 / Hkv : 1);
  const int n = Hkv * share_row_tiles(B, G);
  return n > kMaxGrid ? n : kMaxGrid;
}
__host__ __device__ inline size_t share_record_ints(int max_seqs, int Hkv, int G) {
  return kShareHdr + (size_t)kShareHead * Hkv + (size_t)kShareDesc * share_max_blocks(max_seqs, Hkv, G);
}
template <class I>
__host__ __device__ inline I *share_record(const CacheView &c, I *plan, int layer) {
  return plan + kSharePlanHdr + (size_t)layer * share_record_ints(c.S, c.Hkv, c.G);
}
template <class I> __host__ __device__ inline I *share_head(I *rec, int h) { return rec + kShareHdr + kShareHead * h; }
template <class I> __host__ __device__ inline I *share_desc(const CacheView &c, I *rec, int block) {
  return rec + kShareHdr + kShareHead * c.Hkv + kShareDesc * (size_t)block;
}
// What a plan must agree on with a call: the batch size, the cache's layout, which fixes where units and page tables
// lie, and the number of SMs the shares were cut for (never 0: a zero-filled buffer is no plan).
inline int share_signature(const spkv_cache *cache, int B) {
  return (int)(((uint32_t)B * 2654435761u ^ cache->share_salt ^ (uint32_t)cache->sm_count * 0x9e3779b1u << 1) | 1u);
}

}  // namespace spkv
