// Sequences that share pages: the fork itself, and the plan a batch of forked sequences decodes by.
#include <algorithm>
#include <new>

#include "spkv_share.cuh"

namespace spkv {

constexpr int kForkBatch = 64;   // destinations per launch (their ids travel by value)
struct ForkDst { int32_t id[kForkBatch]; };

// One block per (layer, KV head) and destination.  Copies the ring (ring_pages x 32 KB), its logits and the
// partly filled last page; takes shares of the full pages.  The source's bytes come from L2 for all
// destinations but the first: bound by the 64 - 96 KB each block writes.
__global__ void __launch_bounds__(256) seq_fork_kernel(CacheView c, int src, ForkDst dst) {
  const int layer = blockIdx.x / c.Hkv, kvh = blockIdx.x % c.Hkv;
  const int us = unit_index(c, layer, src, kvh), ud = unit_index(c, layer, dst.id[blockIdx.y], kvh);
  const int tid = threadIdx.x;
  // The whole block decides, behind a barrier: thread 0 writes these two words at the end, and a warp that came to them
  // later would take the finished unit for one that was not empty and leave its part uncopied.
  if (__syncthreads_or(c.t[ud] != 0 || c.len[ud] != 0)) {
    if (tid == 0) set_status(c, SPKV_E_FORK);
    return;
  }
  const int len = c.len[us], t = c.t[us];
  const int n_full = len / kP, tail = len % kP;
  const int32_t *ts = unit_table(c, len ? c.table_row[us] : 0);
  int32_t *td = unit_table(c, len ? c.table_row[ud] : 0);
  __shared__ int s_page;
  if (tail) {
    if (tid == 0) {
      int page = -1;
      const int top = atomicSub(&c.status[1], 1);
      if (top <= 0) {
        atomicAdd(&c.status[1], 1);
        set_status(c, SPKV_E_POOL_EXHAUSTED);
      } else {
        page = checked_page(c, __ldcg(&c.free_stack[top - 1]), -1);
      }
      s_page = page;
    }
    __syncthreads();
    const int page = s_page;
    if (page < 0) return;   // the unit stays empty
    const int from = checked_page(c, ts[n_full], (int)ring_page(c, us, 0));
    const uint4 *ps = reinterpret_cast<const uint4 *>(c.pages + (int64_t)from * kPageElems);
    uint4 *pd = reinterpret_cast<uint4 *>(c.pages + (int64_t)page * kPageElems);
#pragma unroll 8
    for (int i = tid; i < kPageBytes / 16; i += 256) pd[i] = ps[i];   // (rows past `tail` are zeros, as in any page)
    if (pool_page_ok(c, from) && tid < tail)
      c.pos_pool[((int64_t)page - c.n_ring_pages_total) * kP + tid] =
          c.pos_pool[((int64_t)from - c.n_ring_pages_total) * kP + tid];
    if (tid == 0) td[n_full] = page;
  }
  for (int j = tid; j < n_full; j += 256) {
    const int page = ts[j];
    td[j] = page;
    if (checked_page(c, page, -1) >= 0) atomicAdd(&c.extra_owners[page - c.n_ring_pages_total], 1);
  }
  const uint4 *rs = reinterpret_cast<const uint4 *>(c.pages + ring_page(c, us, 0) * kPageElems);
  uint4 *rd = reinterpret_cast<uint4 *>(c.pages + ring_page(c, ud, 0) * kPageElems);
  const int n16 = c.ring_pages * (kPageBytes / 16);
#pragma unroll 8
  for (int i = tid; i < n16; i += 256) rd[i] = rs[i];
  for (int i = tid; i < c.w; i += 256) c.ring_logit[(size_t)ud * c.w + i] = c.ring_logit[(size_t)us * c.w + i];
  if (tid == 0) {
    c.len[ud] = len;
    c.t[ud] = t;
    c.vmax[ud] = c.vmax[us];
  }
}

// Common leading pages of a batch, one block per (layer, KV head).  A full page sits at the same index in
// every table that holds it, and whoever holds it holds the pages before it too (a fork copies a
// table's leading entries), so "entry c - 1 agrees" means "the first c pages agree" and is a binary search.
__global__ void __launch_bounds__(128) share_common_kernel(CacheView c, const int32_t *seq_ids, int B, int32_t *plan) {
  const int layer = blockIdx.x / c.Hkv, kvh = blockIdx.x % c.Hkv;
  __shared__ int s_min;
  if (threadIdx.x == 0) s_min = 0x7fffffff;
  __syncthreads();
  const int seq0 = seq_ids[0];
  const bool ok0 = seq0 >= 0 && seq0 < c.S;
  const int u0 = unit_index(c, layer, ok0 ? seq0 : 0, kvh), row0 = c.table_row[u0];
  const int n0 = ok0 && row0 >= 0 ? c.len[u0] / kP : 0;
  for (int b = threadIdx.x; b < B; b += 128) {
    const int seq = seq_ids[b];
    int lo = 0;
    if (seq < 0 || seq >= c.S) {
      set_status(c, SPKV_E_BOUNDS);
    } else {
      const int u = unit_index(c, layer, seq, kvh), row = c.table_row[u];
      int hi = row >= 0 ? min(n0, c.len[u] / kP) : 0;   // the answer lies in [lo, hi]
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (unit_table(c, row)[mid - 1] == unit_table(c, row0)[mid - 1]) lo = mid; else hi = mid - 1;
      }
    }
    atomicMin(&s_min, lo);
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    int32_t *head = share_head(share_record(c, plan, layer), kvh);
    head[0] = (B < 2 || s_min < kMinSharedPages) ? 0 : s_min;
    head[2] = row0;
    head[3] = u0;
  }
}

// Cuts a layer's common pages into shares: the fewest pages per share, p, for which all shares of all KV
// heads and row tiles are no more than one block per SM (blocks take one share each, so the longest
// share is the launch).  Likewise the number of shares a unit's own pages are cut into, by the longest
// unit.  One block per layer.
__global__ void __launch_bounds__(256) share_cut_kernel(CacheView c, const int32_t *seq_ids, int B, int n_tiles,
                                                        int max_blocks, int sig, int32_t *plan) {
  int32_t *rec = share_record(c, plan, blockIdx.x);
  const int lane = threadIdx.x & 31;
  __shared__ int s_longest;
  if (threadIdx.x == 0) s_longest = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < B * c.Hkv; i += 256) {
    const int seq = seq_ids[i / c.Hkv];
    if (seq < 0 || seq >= c.S) continue;
    const int u = unit_index(c, blockIdx.x, seq, i % c.Hkv);
    atomicMax(&s_longest, (c.len[u] + kP - 1) / kP - share_head(rec, i % c.Hkv)[0] + (min(c.t[u], c.w) + kP - 1) / kP);
  }
  auto blocks = [&](int p) {   // (every warp computes the same)
    int n = 0;
    for (int h = lane; h < c.Hkv; h += 32) n += (share_head(rec, h)[0] + p - 1) / p;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
    return n * n_tiles;
  };
  int heads = 0, longest = 1;
  for (int h = lane; h < c.Hkv; h += 32) {
    heads += share_head(rec, h)[0] > 0;
    longest = max(longest, share_head(rec, h)[0]);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    heads += __shfl_xor_sync(0xffffffffu, heads, o);
    longest = max(longest, __shfl_xor_sync(0xffffffffu, longest, o));
  }
  // (more walks than SMs: every walk whole)
  const int limit = max(max_blocks, heads * n_tiles);
  int lo = kMinSharePages, hi = max(longest, kMinSharePages);
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (blocks(mid) <= limit) hi = mid; else lo = mid + 1;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    const int units = B * c.Hkv;
    const int n_tail = max(1, min(max((s_longest + kTailPages - 1) / kTailPages, max_blocks / units), kMaxTailItems / units));
    int at = 0;
    for (int h = 0; h < c.Hkv; ++h) {
      int32_t *hd = share_head(rec, h);
      const int n_pre = (hd[0] + lo - 1) / lo;
      hd[1] = at;
      hd[4] = n_pre;
      hd[5] = n_tail;
      hd[6] = sig;
      hd[7] = 0;
      at += n_pre * n_tiles;
    }
    rec[0] = lo;
    rec[1] = at;
    rec[2] = rec[3] = 0;
  }
  __syncthreads();
  const int n_room = share_max_blocks(c.S, c.Hkv, c.G);
  for (int x = threadIdx.x; x < n_room; x += 256) {
    int4 d0 = make_int4(0, 0, 0, 0), d1 = d0;
    if (x < rec[1]) {
      int h = c.Hkv - 1;   // the last head that starts at or before this block and has pages
      while (h > 0 && (share_head(rec, h)[1] > x || share_head(rec, h)[0] == 0)) --h;
      const int32_t *hd = share_head(rec, h);
      const int r = x - hd[1], j = r / n_tiles * lo;
      d0 = make_int4(h, r % n_tiles, j, min(lo, hd[0] - j));
      d1 = make_int4(hd[0], hd[2], hd[3], sig);
    }
    int4 *d = reinterpret_cast<int4 *>(share_desc(c, rec, x));
    d[0] = d0;
    d[1] = d1;
  }
}

}  // namespace spkv

using namespace spkv;

extern "C" int spkv_seq_fork(spkv_cache_t *cache, int32_t src, const int32_t *h_dst, int32_t n, spkv_stream_t stream) {
  if (!cache || src < 0 || src >= cache->cfg.max_seqs || n < 0 || n > cache->cfg.max_seqs || (n && !h_dst))
    return SPKV_E_INVALID;
  if (!cache->view.extra_owners) return SPKV_E_UNSUPPORTED;
  if (n == 0) return SPKV_OK;
  bool *seen = new (std::nothrow) bool[cache->cfg.max_seqs]();
  if (!seen) return SPKV_E_INVALID;
  bool ok = true;
  for (int i = 0; i < n && ok; ++i) {
    const int d = h_dst[i];
    ok = d >= 0 && d < cache->cfg.max_seqs && d != src && !seen[d];
    if (ok) seen[d] = true;
  }
  delete[] seen;
  if (!ok) return SPKV_E_INVALID;
  cache->last_kind = kLastOther;
  for (int i = 0; i < n; i += kForkBatch) {
    ForkDst dst = {};
    const int m = std::min(kForkBatch, n - i);
    for (int x = 0; x < m; ++x) dst.id[x] = h_dst[i + x];
    seq_fork_kernel<<<dim3(cache->view.L * cache->view.Hkv, m), 256, 0, as_stream(stream)>>>(cache->view, src, dst);
    if (cudaGetLastError() != cudaSuccess) return SPKV_E_CUDA;
  }
  return SPKV_OK;
}

extern "C" size_t spkv_share_plan_bytes(const spkv_config_t *cfg) {
  if (!cfg || cfg->n_layers < 1 || cfg->max_seqs < 1 || cfg->n_kv_heads < 1 || cfg->n_q_heads < cfg->n_kv_heads) return 0;
  return (kSharePlanHdr + (size_t)cfg->n_layers * share_record_ints(cfg->max_seqs, cfg->n_kv_heads,
                                                                    cfg->n_q_heads / cfg->n_kv_heads)) * 4;
}

extern "C" int spkv_share_plan(spkv_cache_t *cache, const int32_t *d_seq_ids, int32_t B, void *d_plan, size_t plan_bytes,
                               spkv_stream_t stream) {
  if (!cache || B < 1 || B > cache->cfg.max_seqs || !d_seq_ids || !d_plan || ((uintptr_t)d_plan & 15)) return SPKV_E_INVALID;
  const CacheView &v = cache->view;
  if (B * v.Hkv > 1024) return SPKV_E_UNSUPPORTED;
  if (plan_bytes < spkv_share_plan_bytes(&cache->cfg)) return SPKV_E_WORKSPACE;
  cache->last_kind = kLastOther;
  int32_t *plan = static_cast<int32_t *>(d_plan);
  share_common_kernel<<<v.L * v.Hkv, 128, 0, as_stream(stream)>>>(v, d_seq_ids, B, plan);
  share_cut_kernel<<<v.L, 256, 0, as_stream(stream)>>>(v, d_seq_ids, B, share_row_tiles(B, v.G),
                                                       std::min(kMaxGrid, cache->sm_count), share_signature(cache, B), plan);
  return check_stream_error(cudaGetLastError());
}
