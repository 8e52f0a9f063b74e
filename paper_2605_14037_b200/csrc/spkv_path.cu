// Accepted drafts: which nodes of a tree the target confirms (spkv_tree_accept), and their way into the cache
// (spkv_append_path: n_path[b] appends of a sequence's units in one go, every layer in one launch).
#include <math.h>

#include "spkv_tree.cuh"

namespace spkv {

struct PathArgs {
  CacheView c;
  int layer0, n_layers, B, T;
  const int32_t *seq_ids, *path, *n_path;   // path, n_path: may be null
  const __nv_bfloat16 *k, *v;
  int64_t k_tok, k_head, k_layer, v_tok, v_head, v_layer;   // strides in elements
  const float *logits;                      // [n_layers][B][T][Hkv]
  float tau_logit;
};

// ---- append ------------------------------------------------------------------------------------------
// One warp owns a unit, as in spkv_append_evict; lanes 0-15 move a key row, lanes 16-31 the value row.  With n new pairs
// the n_leave = max(0, t + n - w) - max(0, t - w) <= 64 pairs from position max(0, t - w) on leave the window: the
// oldest of the ring, and the first drafts themselves where n > w.  Lane x decides for leaving pairs x and x + 32; the
// kept ones go to the compact cache in order, at most one fresh page among them (64 pairs end in at most one page that
// was not begun).  Only then are the ring's slots written over, by the last min(n, w) drafts.
// What bounds it: latency.  A pair is 512 B read and 512 written, a kept one that leaves as much again.  32 layers of 24 sequences
// and 8 KV heads, keys and values apart and from memory, 1 / 4 / 16 pairs each, half of the leaving ones kept: 9.1 / 14.7 / 42 us on
// the device; at 16 that is 152 MB, 3.6 TB/s (23 us at the copy rate; none kept 24 us, 4.2 TB/s; all kept 53 us, 3.8 TB/s), with
// 49 % of the issue slots taken and a third of a warp's time spent on loads that are on their way.
constexpr int kPathWarps = 4;
constexpr int kPathAhead = 4;   // rows a lane asks for before it writes the first of them

__global__ void __launch_bounds__(kPathWarps * 32) append_path_kernel(PathArgs a) {
  pdl_wait();
  pdl_trigger();
  const CacheView &c = a.c;
  const int lane = threadIdx.x & 31, items = a.B * c.Hkv;
  const long long g = (long long)blockIdx.x * kPathWarps + (threadIdx.x >> 5);
  const int at_layer = (int)(g / items), item = (int)(g % items), b = item / c.Hkv, kvh = item % c.Hkv;
  if (at_layer >= a.n_layers) return;
  const int layer = a.layer0 + at_layer;
  const int seq = a.seq_ids[b];
  int n = a.n_path ? a.n_path[b] : a.T, node0 = lane, node1 = lane + 32;   // path entries lane and lane + 32
  if (a.path) {
    node0 = lane < a.T ? a.path[(size_t)b * a.T + lane] : 0;
    node1 = lane + 32 < a.T ? a.path[(size_t)b * a.T + lane + 32] : 0;
  }
  if (seq < 0 || seq >= c.S) {
    if (lane == 0) set_status(c, SPKV_E_BOUNDS);
    return;
  }
  const int u = unit_index(c, layer, seq, kvh);
  const int t = ldcg_keep(&c.t[u]), len = ldcg_keep(&c.len[u]), trow = unit_table_row(c, u);
  const float thr = head_threshold(c, layer, kvh, a.tau_logit);
  bool bad = n < 0 || n > a.T;
  n = max(0, min(n, a.T));
  const unsigned off0 = __ballot_sync(0xffffffffu, lane < n && (node0 < 0 || node0 >= a.T)),
                 off1 = __ballot_sync(0xffffffffu, lane + 32 < n && (node1 < 0 || node1 >= a.T));
  if (off0 || off1) {
    bad = true;
    n = off0 ? __ffs(off0) - 1 : 31 + __ffs(off1);
  }
  if (bad && lane == 0) set_status(c, SPKV_E_BOUNDS);
  if (n == 0) return;
  auto node = [&](int i) {   // of path entry i (the same for all lanes)
    const int x = __shfl_sync(0xffffffffu, i < 32 ? node0 : node1, i & 31);
    return x;
  };
  const int chunk = lane & 15, blk = (lane >> 4) * kBlockElems;
  const __nv_bfloat16 *src = lane < 16 ? a.k + (int64_t)at_layer * a.k_layer + (int64_t)kvh * a.k_head
                                       : a.v + (int64_t)at_layer * a.v_layer + (int64_t)kvh * a.v_head;
  src += (int64_t)b * a.T * (lane < 16 ? a.k_tok : a.v_tok) + chunk * 8;
  const int64_t tok = lane < 16 ? a.k_tok : a.v_tok;
  const float *lg = a.logits + ((size_t)at_layer * a.B + b) * a.T * c.Hkv + kvh;
  auto ring_cell = [&](int slot) {
    return reinterpret_cast<uint4 *>(c.pages + ring_page(c, u, slot / kP) * kPageElems + blk + swz_off(slot % kP, chunk));
  };
  float *ring_logit = c.ring_logit + (size_t)u * c.w;

  // ---- the pairs that leave the window
  const int p0 = max(0, t - c.w), n_leave = trow >= 0 ? max(0, t + n - c.w) - p0 : 0;
  if (n_leave > 0) {
    const int nodes_x[2] = {node0, node1};
    unsigned keep[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int x = lane + 32 * half, e = p0 + x - t;   // e >= 0: path entry e, already out of the window
      // (entry e of the path lies in another lane; all lanes take part in the exchange)
      const int from0 = __shfl_sync(0xffffffffu, nodes_x[0], e & 31), from1 = __shfl_sync(0xffffffffu, nodes_x[1], e & 31);
      float z = 0.f;
      if (x < n_leave) z = e < 0 ? __ldcg(&ring_logit[(p0 + x) % c.w]) : lg[(size_t)(e < 32 ? from0 : from1) * c.Hkv];
      keep[half] = __ballot_sync(0xffffffffu, x < n_leave && (z >= thr || p0 + x < c.n_sink));
    }
    int n_keep = __popc(keep[0]) + __popc(keep[1]);
    // room: what is left of the page begun, then one page more
    const int pj = len / kP, prow = len % kP, room = prow ? kP - prow : 0;
    int page = -1, fresh = -1, fresh_j = prow ? pj + 1 : pj;
    if (n_keep && prow) {
      page = checked_page(c, ldcg_keep(&unit_table(c, trow)[pj]), -1);
      if (page < 0) n_keep = 0;   // debug bounds: recorded, nothing is stored
    }
    if (n_keep > room) {
      int err = 0;
      if (fresh_j >= c.max_pages) {
        err = SPKV_E_CONTEXT_OVERFLOW;
      } else {
        fresh = alloc_page(c, lane);
        if (fresh < 0) err = fresh == -1 ? SPKV_E_POOL_EXHAUSTED : SPKV_E_BOUNDS_PAGE;
        else if (lane == 0) unit_table(c, trow)[fresh_j] = fresh;
      }
      if (err) {
        if (lane == 0) set_status(c, err);
        n_keep = room;
      }
      __syncwarp();   // (the fresh page's value block has been cleared)
    }
    uint32_t vm = 0;
    uint64_t left = (uint64_t)keep[1] << 32 | keep[0];
    for (int done = 0; done < n_keep; done += kPathAhead) {
      uint4 cell[kPathAhead];
      int pos[kPathAhead];
#pragma unroll
      for (int y = 0; y < kPathAhead; ++y) {
        if (done + y >= n_keep) break;
        const int x = __ffsll((long long)left) - 1;
        left &= left - 1;
        pos[y] = p0 + x;
        const int e = pos[y] - t;
        cell[y] = e < 0 ? __ldcg(ring_cell(pos[y] % c.w)) : *reinterpret_cast<const uint4 *>(src + (int64_t)node(e) * tok);
      }
#pragma unroll
      for (int y = 0; y < kPathAhead; ++y) {
        if (done + y >= n_keep) break;
        const int r = prow + done + y;   // row from the start of the page begun (or of the fresh one)
        const int row = r % kP, to = prow && r < kP ? page : fresh;
        *reinterpret_cast<uint4 *>(c.pages + (int64_t)to * kPageElems + blk + swz_off(row, chunk)) = cell[y];
        if (lane >= 16) vm = max(vm, chunk_abs_max_bf16(cell[y]));
        if (lane == 0) c.pos_pool[((int64_t)to - c.n_ring_pages_total) * kP + row] = pos[y];
      }
    }
    vm = __reduce_max_sync(0xffffffffu, vm);
    if (lane == 0 && n_keep) {
      c.len[u] = len + n_keep;
      note_vmax(c, u, vm);
    }
    __syncwarp();   // the ring has been read
  }
  // ---- the new pairs
  for (int i0 = max(0, n - c.w); i0 < n; i0 += kPathAhead) {
    uint4 cell[kPathAhead];
#pragma unroll
    for (int y = 0; y < kPathAhead; ++y)
      if (i0 + y < n) cell[y] = *reinterpret_cast<const uint4 *>(src + (int64_t)node(i0 + y) * tok);
#pragma unroll
    for (int y = 0; y < kPathAhead; ++y)
      if (i0 + y < n) *ring_cell((t + i0 + y) % c.w) = cell[y];
  }
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int i = lane + 32 * half;
    // (a head declared local-only keeps no logits)
    if (i < n && i >= n - c.w) ring_logit[(t + i) % c.w] = trow >= 0 ? lg[(size_t)(half ? node1 : node0) * c.Hkv] : 0.f;
  }
  if (lane == 0) c.t[u] = t + n;
}

// ---- accept ------------------------------------------------------------------------------------------
// One warp per sequence; lane x holds nodes x and x + 32.  Every step of the walk is two ballots: which nodes
// are children of the current one with the wanted token.  500 trees of 64: 2.9 us on the device, a launch and two
// trips to memory.
constexpr int kAcceptWarps = 4;

__global__ void __launch_bounds__(kAcceptWarps * 32)
tree_accept_kernel(int B, int T, const int32_t *n_nodes, const int32_t *parent, const int32_t *tokens, const int32_t *target,
                   int32_t *path, int32_t *n_path, int32_t *next) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, b = blockIdx.x * kAcceptWarps + (threadIdx.x >> 5);
  if (b >= B) return;
  const int n = n_nodes ? max(0, min(n_nodes[b], T)) : T;
  const size_t row = (size_t)b * T;
  int up[2], token[2], want[2], line[2] = {-1, -1};
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int x = lane + 32 * h;
    up[h] = -1; token[h] = 0; want[h] = -1;
    if (x < n) {
      up[h] = parent ? parent[row + x] : x - 1;
      if (up[h] >= x) up[h] = -1;   // (no parent of its own: out of range)
      token[h] = tokens[row + x];
      want[h] = target[row + x];
    }
  }
  int cur = 0, len = 0, then = -1;
  if (n > 0) {
    for (;;) {   // (cur grows: at most n steps)
      if (lane == (len & 31)) line[len >> 5] = cur;
      ++len;
      const int w0 = __shfl_sync(0xffffffffu, want[0], cur & 31), w1 = __shfl_sync(0xffffffffu, want[1], cur & 31);
      then = cur < 32 ? w0 : w1;
      const unsigned m0 = __ballot_sync(0xffffffffu, up[0] == cur && token[0] == then),
                     m1 = __ballot_sync(0xffffffffu, up[1] == cur && token[1] == then);
      if (!(m0 | m1)) break;
      cur = m0 ? __ffs(m0) - 1 : 31 + __ffs(m1);
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h)
    if (lane + 32 * h < T) path[row + lane + 32 * h] = line[h];
  if (lane == 0) {
    n_path[b] = len;
    next[b] = then;
  }
}

}  // namespace spkv

using namespace spkv;

extern "C" int spkv_append_path(spkv_cache_t *cache, int32_t layer0, int32_t n_layers, const int32_t *d_seq_ids, int32_t B,
                                int32_t T, const int32_t *d_path, const int32_t *d_n_path, const spkv_rows_t *k,
                                int64_t k_layer_stride, const spkv_rows_t *v, int64_t v_layer_stride, const float *d_logits,
                                spkv_stream_t stream) {
  if (!cache || layer0 < 0 || n_layers < 0 || layer0 > cache->cfg.n_layers - n_layers || B < 0 || B > cache->cfg.max_seqs ||
      T < 0 || T > kMaxDraft)
    return SPKV_E_INVALID;
  if (B == 0 || T == 0 || n_layers == 0) return SPKV_OK;
  if (!d_seq_ids || !bf16_rows_ok(k) || !bf16_rows_ok(v) || ((k_layer_stride | v_layer_stride) & 7) || !d_logits) return SPKV_E_INVALID;
  PathArgs a = {};
  a.c = cache->view; a.layer0 = layer0; a.n_layers = n_layers; a.B = B; a.T = T;
  a.seq_ids = d_seq_ids; a.path = d_path; a.n_path = d_n_path;
  a.k = static_cast<const __nv_bfloat16 *>(k->ptr); a.k_tok = k->token_stride; a.k_head = k->head_stride; a.k_layer = k_layer_stride;
  a.v = static_cast<const __nv_bfloat16 *>(v->ptr); a.v_tok = v->token_stride; a.v_head = v->head_stride; a.v_layer = v_layer_stride;
  a.logits = d_logits;
  a.tau_logit = cache->tau_logit;
  // (overlap mode: kernels before the last one may still be running, which griddepcontrol.wait does not cover)
  const bool plain = (cache->cfg.flags & SPKV_FLAG_OVERLAP) != 0;
  cache->last_kind = kLastOther;
  const long long warps = (long long)n_layers * B * cache->view.Hkv;
  return check_stream_error(launch_link(!plain, append_path_kernel, dim3((unsigned)((warps + kPathWarps - 1) / kPathWarps)),
                                        dim3(kPathWarps * 32), 0, as_stream(stream), a));
}

extern "C" int spkv_tree_accept(int32_t B, int32_t T, const int32_t *d_n_nodes, const int32_t *d_parent,
                                const int32_t *d_tokens, const int32_t *d_target, int32_t *d_path, int32_t *d_n_path,
                                int32_t *d_next, spkv_stream_t stream) {
  if (B < 0 || T < 0 || T > kMaxDraft) return SPKV_E_INVALID;
  if (B == 0) return SPKV_OK;
  if (!d_n_path || !d_next || (T && (!d_tokens || !d_target || !d_path))) return SPKV_E_INVALID;
  note_cacheless_call();
  tree_accept_kernel<<<(B + kAcceptWarps - 1) / kAcceptWarps, kAcceptWarps * 32, 0, as_stream(stream)>>>(
      B, T, d_n_nodes, d_parent, d_tokens, d_target, d_path, d_n_path, d_next);
  return check_stream_error(cudaGetLastError());
}
