// Attention of a tree of drafted tokens over the cache (spkv_decode_attention_tree).
#include <math.h>

#include "spkv_tree.cuh"

namespace spkv {

// One warp per query row (node, query head): lane l owns dims 4l .. 4l + 3, keys one after the other.
__global__ void __launch_bounds__(128) tree_rows_kernel(TreeArgs a) {
  const CacheView &c = a.c;
  const int lane = threadIdx.x & 31, r = blockIdx.x * 4 + (threadIdx.x >> 5), b = blockIdx.y;
  const int i = r / c.Hq, j = r - i * c.Hq, kvh = j / c.G;
  bool bad = false;
  const int n = tree_nodes(a, b, &bad);
  const int seq = a.seq_ids[b];
  if (seq < 0 || seq >= c.S) bad = true;
  if (bad && r == 0 && lane == 0) set_status(c, SPKV_E_BOUNDS);
  if (i >= n || seq < 0 || seq >= c.S) return;
  const int u = unit_index(c, a.layer, seq, kvh), t = __ldcg(&c.t[u]), len = __ldcg(&c.len[u]), trow = unit_table_row(c, u);
  const float thr = head_threshold(c, a.layer, kvh, a.tau_logit);
  uint64_t path = 0;
  for (int x = i; x >= 0;) {
    path |= 1ull << x;
    int p = a.parent ? a.parent[(size_t)b * a.T + x] : x - 1;
    if (p < -1 || p >= x) {
      if (lane == 0) set_status(c, SPKV_E_BOUNDS);
      p = -1;
    }
    x = p;
  }
  const int d = __popcll(path) - 1;
  const __nv_bfloat16 *qr = a.q + ((int64_t)b * a.T + i) * a.q_tok + (int64_t)j * a.q_head + lane * 4;
  float q[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
  for (int x = 0; x < 4; ++x) q[x] = __bfloat162float(qr[x]);
  auto take = [&](const __nv_bfloat16 *kr, const __nv_bfloat16 *vr) {   // this lane's four elements of a row
    float s = 0.f;
    for (int x = 0; x < 4; ++x) s = fmaf(q[x], __bfloat162float(kr[x]), s);
    s = warp_sum(s) * a.scale_log2;
    const float mn = s > m ? s : m, f = m == -INFINITY ? 0.f : fast_exp2(m - mn), p = fast_exp2(s - (mn == -INFINITY ? 0.f : mn));
    l = l * f + p;
    for (int x = 0; x < 4; ++x) o[x] = o[x] * f + p * __bfloat162float(vr[x]);
    m = mn;
  };
  auto take_row = [&](int64_t page, int row) {
    const __nv_bfloat16 *kr = c.pages + page * kPageElems + swz_off(row, lane >> 1) + (lane & 1) * 4;
    take(kr, kr + kBlockElems);
  };
  for (int x = 0; x < len; ++x)
    take_row(checked_page(c, unit_table(c, trow)[x / kP], (int)ring_page(c, u, 0)), x % kP);
  const int n_ring = min(t, c.w);
  for (int x = 0; x < n_ring; ++x) {
    const bool out = (ring_out_of_window(t, d, c.w, x / kP) >> (x % kP)) & 1;
    if (out && !(trow >= 0 && (__ldcg(&c.ring_logit[(size_t)u * c.w + x]) >= thr || ring_position(t, c.w, x) < c.n_sink))) continue;
    take_row(ring_page(c, u, x / kP), x % kP);
  }
  int dx = 0;
  for (int x = 0; x < n; ++x) {
    if (!((path >> x) & 1)) continue;
    const size_t tok = (size_t)b * a.T + x;
    if (d - dx < c.w || (trow >= 0 && (a.logits[tok * c.Hkv + kvh] >= thr || t + dx < c.n_sink)))
      take(a.k + (int64_t)tok * a.k_tok + (int64_t)kvh * a.k_head + lane * 4, a.v + (int64_t)tok * a.v_tok + (int64_t)kvh * a.v_head + lane * 4);
    ++dx;
  }
  const size_t row = ((size_t)b * a.T + i) * c.Hq + j;
  for (int x = 0; x < 4; ++x) a.out[row * kD + lane * 4 + x] = __float2bfloat16(o[x] / l);
  if (a.lse && lane == 0) a.lse[row] = (m + log2f(l)) * kLn2;
}

}  // namespace spkv

using namespace spkv;

extern "C" size_t spkv_decode_tree_workspace_bytes(const spkv_config_t *cfg, int32_t B, int32_t T) {
  if (!cfg || B < 0 || T < 0 || T > kMaxDraft || cfg->n_kv_heads < 1 || cfg->n_q_heads < cfg->n_kv_heads) return 0;
  return 256;
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
  cache->last_kind = kLastOther;
  tree_rows_kernel<<<dim3((T * view.Hq + 3) / 4, B), 128, 0, as_stream(stream)>>>(a);
  return check_stream_error(cudaGetLastError());
}
