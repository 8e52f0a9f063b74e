// Per-head RMS norm of queries and keys and their position rotation, in one pass over the rows of a
// projection, and the backward pass of it.
//
//   u = x / sqrt(mean(x^2) + eps),  y = w u                                  (norm, optional per side)
//   (y_lo, y_hi) -> scale (y_lo cos t - y_hi sin t, y_hi cos t + y_lo sin t)  (first rot_dim dims)
//   t = pos[axis of the pair][token] * inv_freq[pair]
//
// and, for g = the rotation's transpose applied to the upstream gradient,
//   dx = r (w g - u mean(w g u)),  r = 1 / sqrt(mean(x^2) + eps),   dw = sum over rows of g u.
//
// A row of head_dim elements belongs to TPR neighbouring lanes; a lane holds two 16-byte chunks of it,
// chosen so that both halves of every rotated pair are in the same lane: with pairs (i, i + rot/2)
// chunks j and j + rot/2, with pairs (2i, 2i + 1) two chunks side by side.  The row is read
// once, its sum of squares goes through log2(TPR) shuffles, everything else stays in registers, all in
// fp32, and is rounded once on the way out.
//
// Angles.  A frequency is held as a fraction of a turn per position in 64-bit fixed point, so that
// position * frequency modulo one turn is one exact integer product; what is left -- 32 bits of a turn -- goes
// through sincospif.  Far positions lose nothing (in fp32 a position of 10^6 is 0.06 rad off).  A block
// computes the sines and cosines of its tokens once, into shared memory, for all its heads: no table
// in memory, no position limit.
//
// What bounds it: bytes.  Each row is read and written once; about 35 issue slots per 512 B moved.
#include <math.h>

#include <algorithm>

#include <cuda_fp16.h>

#include "spkv_internal.cuh"

namespace spkv {

constexpr int kRowThreads = 256;
constexpr int kMaxTile = 8;         // tokens per block and pass
constexpr int kMaxBwdBlocks = 2048; // partial sums of the weight gradients the workspace holds

struct RowArgs {
  spkv_rope_t rope;
  int n_tok, Hq, Hkv, Hv, D, tile;
  int norm;                    // bit 0: queries, bit 1: keys
  int w_dtype;
  float eps, inv_d;
  const void *wq, *wk;         // null = ones
  const int32_t *pos;          // [n_axes][n_tok]
  spkv_rows_t x[3], g[3], y[3];   // q, k, v: inputs, (backward) upstream gradients, results
  float *part;                 // backward: [gridDim.x][2][D] partial sums of g u, or null
};

template <class T> struct Elem;
template <> struct Elem<__nv_bfloat16> {
  static constexpr int kChunk = 8;
  static __device__ inline void unpack(const uint4 &v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  }
  static __device__ inline uint32_t pack2(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
  }
  static __device__ inline uint4 pack(const float (&f)[8]) {
    return make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
  }
};
template <> struct Elem<__half> {
  static constexpr int kChunk = 8;
  static __device__ inline void unpack(const uint4 &v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 p = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
      f[2 * i] = p.x; f[2 * i + 1] = p.y;
    }
  }
  static __device__ inline uint32_t pack2(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
  }
  static __device__ inline uint4 pack(const float (&f)[8]) {
    return make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
  }
};
template <> struct Elem<float> {
  static constexpr int kChunk = 4;
  static __device__ inline void unpack(const uint4 &v, float (&f)[4]) {
    f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
  }
  static __device__ inline uint4 pack(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};

__device__ inline float load_weight(const void *w, int dtype, int i) {
  if (!w) return 1.f;
  if (dtype == SPKV_BF16) return __bfloat162float(static_cast<const __nv_bfloat16 *>(w)[i]);
  if (dtype == SPKV_F16) return __half2float(static_cast<const __half *>(w)[i]);
  return static_cast<const float *>(w)[i];
}

// Where lane j of a row finds its two chunks (element offsets), and whether its pairs are rotated.
struct LaneChunks { int c0, c1; bool live, rot; };
template <int CE>
__device__ inline LaneChunks lane_chunks(const RowArgs &a, int j) {
  LaneChunks l;
  const int n_rot = a.rope.rot_dim / (2 * CE);   // lanes whose pairs are rotated
  l.live = j < a.D / (2 * CE);
  l.rot = j < n_rot;
  if (l.rot && !a.rope.interleaved) { l.c0 = j * CE; l.c1 = a.rope.rot_dim / 2 + j * CE; }
  else { l.c0 = 2 * j * CE; l.c1 = l.c0 + CE; }
  return l;
}

// Element e of a lane's chunk 0 / 1 is half of the lane's pair pair_of(e): (i, i + rot/2): lo of pair e and
// hi of pair e; adjacent pairs: chunk 0 holds pairs 0 .. CE/2-1, chunk 1 the others.
// Rotates the CE pairs of a lane in place; cs holds (cos, sin) of its pairs, sgn = -1 for the transpose.
template <int CE>
__device__ inline void rotate(float (&f0)[CE], float (&f1)[CE], const float2 (&cs)[CE], bool interleaved, float sgn) {
  if (!interleaved) {
#pragma unroll
    for (int e = 0; e < CE; ++e) {
      const float c = cs[e].x, s = sgn * cs[e].y, lo = f0[e], hi = f1[e];
      f0[e] = lo * c - hi * s;
      f1[e] = hi * c + lo * s;
    }
  } else {
#pragma unroll
    for (int e = 0; e < CE / 2; ++e) {
      const float c = cs[e].x, s = sgn * cs[e].y, lo = f0[2 * e], hi = f0[2 * e + 1];
      f0[2 * e] = lo * c - hi * s;
      f0[2 * e + 1] = hi * c + lo * s;
      const float c2 = cs[CE / 2 + e].x, s2 = sgn * cs[CE / 2 + e].y, lo2 = f1[2 * e], hi2 = f1[2 * e + 1];
      f1[2 * e] = lo2 * c2 - hi2 * s2;
      f1[2 * e + 1] = hi2 * c2 + lo2 * s2;
    }
  }
}

// Shared memory of a block: (cos, sin) of [tile][pairs] and the two weights as floats, both ordered so that
// the lanes of a row read neighbouring 16-byte vectors: vector i of lane j at (i * TPR + j).
template <int CE, int TPR>
__device__ inline int cs_slot(int pair) {   // pair -> float2 index inside a token's table
  const int j = pair / CE, e = pair % CE;
  return ((e >> 1) * TPR + j) * 2 + (e & 1);
}
template <int CE, int TPR>
__device__ inline void load_cs(const float2 *tab, int j, float2 (&cs)[CE]) {
#pragma unroll
  for (int i = 0; i < CE / 2; ++i) {
    const float4 v = *reinterpret_cast<const float4 *>(tab + (i * TPR + j) * 2);
    cs[2 * i] = make_float2(v.x, v.y);
    cs[2 * i + 1] = make_float2(v.z, v.w);
  }
}
template <int CE, int TPR>
__device__ inline void fill_cs(const RowArgs &a, float2 *s_cs, int tok0, int n_here) {
  const int P = a.rope.rot_dim / 2;
  for (int x = threadIdx.x; x < n_here * P; x += kRowThreads) {
    const int t = x / P, p = x % P;
    const int pos = a.pos[(size_t)a.rope.axis[p] * a.n_tok + tok0 + t];
    // turns modulo one, 64-bit fixed point; the upper 32 bits as half turns in [-1, 1)
    const uint64_t turns = (uint64_t)(int64_t)pos * a.rope.turn[p];
    float s, c;
    sincospif((float)(int32_t)(turns >> 32) * 4.656612873077393e-10f, &s, &c);
    s_cs[t * (CE * TPR) + cs_slot<CE, TPR>(p)] = make_float2(c * a.rope.scale, s * a.rope.scale);
  }
}
template <int CE, int TPR>
__device__ inline void fill_weights(const RowArgs &a, float *s_w) {   // [2][2 chunks * CE * TPR]
  for (int x = threadIdx.x; x < 2 * TPR * 2 * CE; x += kRowThreads) {
    const int side = x / (2 * CE * TPR), r = x % (2 * CE * TPR), j = r / (2 * CE), e = r % (2 * CE);
    const LaneChunks l = lane_chunks<CE>(a, j);
    const int d = e < CE ? l.c0 + e : l.c1 + e - CE;
    const float w = l.live ? load_weight(side ? a.wk : a.wq, a.w_dtype, d) : 0.f;
    s_w[side * 2 * CE * TPR + ((e >> 2) * TPR + j) * 4 + (e & 3)] = w;
  }
}
template <int CE, int TPR>
__device__ inline void load_w(const float *s_w, int j, float (&w0)[CE], float (&w1)[CE]) {
#pragma unroll
  for (int i = 0; i < CE / 4; ++i) {
    const float4 v = *reinterpret_cast<const float4 *>(s_w + (i * TPR + j) * 4);
    w0[4 * i] = v.x; w0[4 * i + 1] = v.y; w0[4 * i + 2] = v.z; w0[4 * i + 3] = v.w;
    const float4 u = *reinterpret_cast<const float4 *>(s_w + ((i + CE / 4) * TPR + j) * 4);
    w1[4 * i] = u.x; w1[4 * i + 1] = u.y; w1[4 * i + 2] = u.z; w1[4 * i + 3] = u.w;
  }
}

template <int TPR>
__device__ inline float row_sum(float v) {
#pragma unroll
  for (int o = TPR / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// row r of a tile -> side (0 q, 1 k, 2 v), token of the tile, head
struct RowAt { int side, tok, head; };
__device__ inline RowAt row_at(const RowArgs &a, int r, int n_here) {
  RowAt w;
  int H = a.Hq;
  w.side = 0;
  if (r >= n_here * a.Hq) {
    r -= n_here * a.Hq; H = a.Hkv; w.side = 1;
    if (r >= n_here * a.Hkv) { r -= n_here * a.Hkv; H = a.Hv; w.side = 2; }
  }
  w.tok = r / H;
  w.head = r - w.tok * H;
  return w;
}
template <class T>
__device__ inline T *row_ptr(const spkv_rows_t &v, int tok, int head) {
  return static_cast<T *>(v.ptr) + (int64_t)tok * v.token_stride + (int64_t)head * v.head_stride;
}
__device__ inline const spkv_rows_t &side_of(const spkv_rows_t (&v)[3], int side) {
  return side == 0 ? v[0] : side == 1 ? v[1] : v[2];
}

template <class T, int TPR>
__global__ void __launch_bounds__(kRowThreads) norm_rope_kernel(const __grid_constant__ RowArgs a) {
  constexpr int CE = Elem<T>::kChunk, kRowsPerPass = kRowThreads / TPR;
  extern __shared__ __align__(16) unsigned char smem[];
  float2 *s_cs = reinterpret_cast<float2 *>(smem);
  float *s_w = reinterpret_cast<float *>(s_cs + a.tile * CE * TPR);
  pdl_trigger();
  const int tok0 = blockIdx.x * a.tile, n_here = min(a.tile, a.n_tok - tok0);
  fill_cs<CE, TPR>(a, s_cs, tok0, n_here);
  if (a.norm) fill_weights<CE, TPR>(a, s_w);
  __syncthreads();
  const int j = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  const LaneChunks l = lane_chunks<CE>(a, j);
  const int n_rows = n_here * (a.Hq + a.Hkv + a.Hv);
  for (int base = 0; base < n_rows; base += kRowsPerPass) {
    // (every lane takes part in the shuffles; lanes past the last row or the row's end hold zeros)
    const int r = base + sub;
    const bool on = r < n_rows && l.live;
    const RowAt w = row_at(a, min(r, n_rows - 1), n_here);
    const T *src = row_ptr<const T>(side_of(a.x, w.side), tok0 + w.tok, w.head);
    uint4 r0 = make_uint4(0, 0, 0, 0), r1 = r0;
    if (on) {
      r0 = __ldcs(reinterpret_cast<const uint4 *>(src + l.c0));
      r1 = __ldcs(reinterpret_cast<const uint4 *>(src + l.c1));
    }
    float f0[CE], f1[CE];
    Elem<T>::unpack(r0, f0);
    Elem<T>::unpack(r1, f1);
    float rr = 1.f;
    if (a.norm) {   // (uniform; a warp's rows may lie on several sides, all lanes shuffle)
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < CE; ++e) { ss = fmaf(f0[e], f0[e], ss); ss = fmaf(f1[e], f1[e], ss); }
      rr = rsqrtf(row_sum<TPR>(ss) * a.inv_d + a.eps);
    }
    if (w.side < 2) {
      if ((a.norm >> w.side) & 1) {
        float w0[CE], w1[CE];
        load_w<CE, TPR>(s_w + w.side * 2 * CE * TPR, j, w0, w1);
#pragma unroll
        for (int e = 0; e < CE; ++e) { f0[e] *= rr * w0[e]; f1[e] *= rr * w1[e]; }
      }
      if (l.rot) {
        float2 cs[CE];
        load_cs<CE, TPR>(s_cs + w.tok * CE * TPR, j, cs);
        rotate<CE>(f0, f1, cs, a.rope.interleaved != 0, 1.f);
      }
      r0 = Elem<T>::pack(f0);
      r1 = Elem<T>::pack(f1);
    }
    if (on) {
      T *dst = row_ptr<T>(side_of(a.y, w.side), tok0 + w.tok, w.head);
      *reinterpret_cast<uint4 *>(dst + l.c0) = r0;
      *reinterpret_cast<uint4 *>(dst + l.c1) = r1;
    }
  }
}

// Backward.  Blocks walk the token tiles with a stride of the grid, so that the partial sums of the weight
// gradients are a fixed split of the rows whatever the timing: the result is the same every time.  A
// lane keeps the sums of its 2 CE columns for both sides in registers over all its rows; at the end the
// lanes that share columns are added up, first through shuffles, then through shared memory in warp order.
template <class T, int TPR>
__global__ void __launch_bounds__(kRowThreads) norm_rope_backward_kernel(const __grid_constant__ RowArgs a) {
  constexpr int CE = Elem<T>::kChunk, kRowsPerPass = kRowThreads / TPR, kWarps = kRowThreads / 32;
  extern __shared__ __align__(16) unsigned char smem[];
  float2 *s_cs = reinterpret_cast<float2 *>(smem);
  float *s_w = reinterpret_cast<float *>(s_cs + a.tile * CE * TPR);
  float *s_dw = s_w + 2 * 2 * CE * TPR;   // [warp][2 CE * TPR], one side at a time
  pdl_trigger();
  if (a.norm) fill_weights<CE, TPR>(a, s_w);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int j = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  const LaneChunks l = lane_chunks<CE>(a, j);
  float dw[2][2 * CE];
#pragma unroll
  for (int e = 0; e < 2 * CE; ++e) dw[0][e] = dw[1][e] = 0.f;
  const int n_tiles = (a.n_tok + a.tile - 1) / a.tile;
  for (int tile = blockIdx.x; tile < n_tiles; tile += gridDim.x) {
    const int tok0 = tile * a.tile, n_here = min(a.tile, a.n_tok - tok0);
    __syncthreads();   // the previous tile's table has been read
    fill_cs<CE, TPR>(a, s_cs, tok0, n_here);
    __syncthreads();
    // one side after the other, so that the rows of a pass all add to the same sums
#pragma unroll
    for (int side = 0; side < 3; ++side) {
      const int H = side == 0 ? a.Hq : side == 1 ? a.Hkv : a.Hv, n_rows = n_here * H;
      const bool normed = side < 2 && ((a.norm >> side) & 1);
      for (int base = 0; base < n_rows; base += kRowsPerPass) {
        const int r = base + sub, rc = min(r, n_rows - 1);
        const bool on = r < n_rows && l.live;
        const int tok = rc / H, head = rc - tok * H;
        uint4 g0 = make_uint4(0, 0, 0, 0), g1 = g0, x0 = g0, x1 = g0;
        if (on) {
          const T *gp = row_ptr<const T>(a.g[side], tok0 + tok, head);
          g0 = __ldcs(reinterpret_cast<const uint4 *>(gp + l.c0));
          g1 = __ldcs(reinterpret_cast<const uint4 *>(gp + l.c1));
          if (normed) {
            const T *xp = row_ptr<const T>(a.x[side], tok0 + tok, head);
            x0 = __ldcs(reinterpret_cast<const uint4 *>(xp + l.c0));
            x1 = __ldcs(reinterpret_cast<const uint4 *>(xp + l.c1));
          }
        }
        if (side < 2) {
          float f0[CE], f1[CE];
          Elem<T>::unpack(g0, f0);
          Elem<T>::unpack(g1, f1);
          if (l.rot) {
            float2 cs[CE];
            load_cs<CE, TPR>(s_cs + tok * CE * TPR, j, cs);
            rotate<CE>(f0, f1, cs, a.rope.interleaved != 0, -1.f);
          }
          if (normed) {
            float u0[CE], u1[CE], w0[CE], w1[CE];
            Elem<T>::unpack(x0, u0);
            Elem<T>::unpack(x1, u1);
            load_w<CE, TPR>(s_w + side * 2 * CE * TPR, j, w0, w1);
            // sum x^2 and sum (w g) x in one pass: the mean of w g u is r times the latter's
            float ss = 0.f, gx = 0.f;
#pragma unroll
            for (int e = 0; e < CE; ++e) {
              ss = fmaf(u0[e], u0[e], ss);
              ss = fmaf(u1[e], u1[e], ss);
            }
            const float rr = rsqrtf(row_sum<TPR>(ss) * a.inv_d + a.eps);
#pragma unroll
            for (int e = 0; e < CE; ++e) {
              u0[e] *= rr; u1[e] *= rr;
              dw[side][e] = fmaf(f0[e], u0[e], dw[side][e]);
              dw[side][CE + e] = fmaf(f1[e], u1[e], dw[side][CE + e]);
              f0[e] *= w0[e]; f1[e] *= w1[e];
              gx = fmaf(f0[e], u0[e], gx);
              gx = fmaf(f1[e], u1[e], gx);
            }
            const float mean = row_sum<TPR>(gx) * a.inv_d;
#pragma unroll
            for (int e = 0; e < CE; ++e) {
              f0[e] = rr * (f0[e] - u0[e] * mean);
              f1[e] = rr * (f1[e] - u1[e] * mean);
            }
          }
          g0 = Elem<T>::pack(f0);
          g1 = Elem<T>::pack(f1);
        }
        if (on) {
          T *dst = row_ptr<T>(a.y[side], tok0 + tok, head);
          *reinterpret_cast<uint4 *>(dst + l.c0) = g0;
          *reinterpret_cast<uint4 *>(dst + l.c1) = g1;
        }
      }
    }
  }
  if (!a.part) return;
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 2 * CE; ++e) {
      float v = dw[side][e];
#pragma unroll
      for (int o = TPR; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
      if (lane < TPR) s_dw[(warp * 2 * CE + e) * TPR + j] = v;
    }
    __syncthreads();
    for (int x = threadIdx.x; x < 2 * CE * TPR; x += kRowThreads) {
      const int e = x / TPR, jj = x % TPR;
      const LaneChunks ll = lane_chunks<CE>(a, jj);
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) v += s_dw[(w * 2 * CE + e) * TPR + jj];
      if (ll.live) a.part[((size_t)blockIdx.x * 2 + side) * a.D + (e < CE ? ll.c0 + e : ll.c1 + e - CE)] = v;
    }
  }
}

// Sums the blocks' partial weight gradients, in a fixed order: grid (D / 16, 2 sides), 256 threads = 16 columns x 16 slices.
__global__ void __launch_bounds__(256) norm_weight_grad_kernel(const float *part, int n_blocks, int D, float *dwq, float *dwk) {
  __shared__ float s[16][17];
  const int col = blockIdx.x * 16 + (threadIdx.x & 15), slice = threadIdx.x >> 4, side = blockIdx.y;
  pdl_wait();
  float v = 0.f;
  for (int b = slice; b < n_blocks; b += 16) v += part[((size_t)b * 2 + side) * D + col];
  s[slice][threadIdx.x & 15] = v;
  __syncthreads();
  if (threadIdx.x < 16) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) t += s[i][threadIdx.x];
    float *out = side ? dwk : dwq;
    if (out) out[col] = t;
  }
}

static int elem_bytes(int dtype) { return dtype == SPKV_F32 ? 4 : 2; }

static int check_rows(const spkv_rows_t *r, int heads, int n_tok, int dtype) {
  if (heads == 0) return SPKV_OK;
  if (!r || !r->ptr) return SPKV_E_INVALID;
  const int64_t per16 = 16 / elem_bytes(dtype);
  if (((uintptr_t)r->ptr & 15) || r->head_stride % per16 || r->token_stride % per16) return SPKV_E_INVALID;
  (void)n_tok;
  return SPKV_OK;
}

static int check_norm_rope(const spkv_qk_norm_t *n, const spkv_rope_t *rope, int n_tok, const int32_t *d_pos) {
  if (!n || !rope || n_tok < 0) return SPKV_E_INVALID;
  if (n->dtype < SPKV_BF16 || n->dtype > SPKV_F32 || n->weight_dtype < SPKV_BF16 || n->weight_dtype > SPKV_F32)
    return SPKV_E_INVALID;
  if (n->head_dim < 16 || n->head_dim > SPKV_MAX_ROW_DIM || n->head_dim % 16) return SPKV_E_UNSUPPORTED;
  if (n->n_q_heads < 0 || n->n_kv_heads < 0 || n->n_q_heads > 4096 || n->n_kv_heads > 4096) return SPKV_E_INVALID;
  if (n->norm < 0 || n->norm > (SPKV_NORM_Q | SPKV_NORM_K)) return SPKV_E_INVALID;
  if (n->norm && !(n->eps >= 0.f && isfinite(n->eps))) return SPKV_E_INVALID;
  if (rope->rot_dim < 0 || rope->rot_dim % 16 || rope->rot_dim > n->head_dim) return SPKV_E_INVALID;
  if (rope->rot_dim && (rope->n_axes < 1 || rope->n_axes > SPKV_MAX_AXES || !isfinite(rope->scale))) return SPKV_E_INVALID;
  for (int p = 0; p < rope->rot_dim / 2; ++p)
    if (rope->axis[p] >= rope->n_axes) return SPKV_E_INVALID;
  if (rope->rot_dim && n_tok && !d_pos) return SPKV_E_INVALID;
  return SPKV_OK;
}

static RowArgs row_args(const spkv_qk_norm_t *n, const spkv_rope_t *rope, int n_tok, const int32_t *d_pos, bool has_v) {
  RowArgs a = {};
  a.rope = *rope;
  a.n_tok = n_tok; a.Hq = n->n_q_heads; a.Hkv = n->n_kv_heads; a.Hv = has_v ? n->n_kv_heads : 0; a.D = n->head_dim;
  a.norm = n->norm;
  a.w_dtype = n->weight_dtype;
  a.eps = n->eps; a.inv_d = 1.f / n->head_dim;
  a.wq = n->d_wq; a.wk = n->d_wk;
  a.pos = d_pos;
  return a;
}

static int device_sms(int *sms) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return SPKV_E_CUDA;
  return check_stream_error(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev));
}

template <class T, int TPR>
static int launch_rows(RowArgs &a, bool backward, int grid, float *dwq, float *dwk, cudaStream_t s) {
  constexpr int CE = Elem<T>::kChunk;
  const size_t smem = (size_t)a.tile * CE * TPR * 8 + 2 * 2 * CE * TPR * 4 +
                      (backward ? (size_t)(kRowThreads / 32) * 2 * CE * TPR * 4 : 0);
  if (!backward) {
    norm_rope_kernel<T, TPR><<<grid, kRowThreads, smem, s>>>(a);
    return check_stream_error(cudaGetLastError());
  }
  if (grid) norm_rope_backward_kernel<T, TPR><<<grid, kRowThreads, smem, s>>>(a);
  if (cudaGetLastError() != cudaSuccess) return SPKV_E_CUDA;
  if (!a.part) return SPKV_OK;
  if (!grid) {   // no rows: the sums are zero
    norm_weight_grad_kernel<<<dim3(a.D / 16, 2), 256, 0, s>>>(a.part, 0, a.D, dwq, dwk);
    return check_stream_error(cudaGetLastError());
  }
  return check_stream_error(launch_overlapped(norm_weight_grad_kernel, dim3(a.D / 16, 2), dim3(256), 0, s, a.part, grid,
                                              a.D, dwq, dwk));
}

// lanes per row: two 16-byte chunks each, rounded up to a power of two
static int dispatch_rows(RowArgs &a, int dtype, bool backward, int grid, float *dwq, float *dwk, cudaStream_t s) {
  const int lanes = a.D * elem_bytes(dtype) / 32;
#define SPKV_ROWS(T)                                                                            if (lanes <= 4) return launch_rows<T, 4>(a, backward, grid, dwq, dwk, s);                      if (lanes <= 8) return launch_rows<T, 8>(a, backward, grid, dwq, dwk, s);                      if (lanes <= 16) return launch_rows<T, 16>(a, backward, grid, dwq, dwk, s);
  if (dtype == SPKV_F32) {
    SPKV_ROWS(float)
    return launch_rows<float, 32>(a, backward, grid, dwq, dwk, s);
  }
  if (dtype == SPKV_F16) {
    SPKV_ROWS(__half)
  } else {
    SPKV_ROWS(__nv_bfloat16)
  }
#undef SPKV_ROWS
  return SPKV_E_UNSUPPORTED;
}

}  // namespace spkv

using namespace spkv;

extern "C" int spkv_rope_init(spkv_rope_t *rope, int32_t rot_dim, int32_t interleaved, int32_t n_axes, float scale,
                              const double *h_inv_freq, const uint8_t *h_axis) {
  if (!rope || rot_dim < 0 || rot_dim % 16 || rot_dim > SPKV_MAX_ROW_DIM || n_axes < 1 || n_axes > SPKV_MAX_AXES ||
      !isfinite(scale) || (rot_dim && !h_inv_freq))
    return SPKV_E_INVALID;
  spkv_rope_t r = {};
  r.rot_dim = rot_dim;
  r.interleaved = interleaved ? 1 : 0;
  r.n_axes = n_axes;
  r.scale = scale;
  for (int p = 0; p < rot_dim / 2; ++p) {
    const double f = h_inv_freq[p];
    if (!isfinite(f) || (h_axis && h_axis[p] >= n_axes)) return SPKV_E_INVALID;
    // turns per position, modulo one, in units of 2^-64 (long double: 64 significant bits)
    const long double t = (long double)f * 0.159154943091895335768883763372514362L;
    long double frac = t - floorl(t);
    const long double scaled = ldexpl(frac, 64);
    r.turn[p] = scaled >= 18446744073709551615.0L ? 0 : (uint64_t)scaled;
    r.axis[p] = h_axis ? h_axis[p] : 0;
  }
  *rope = r;
  return SPKV_OK;
}

extern "C" int spkv_norm_rope(const spkv_qk_norm_t *norm, const spkv_rope_t *rope, int32_t n_tok, const int32_t *d_pos,
                              const spkv_rows_t *q, const spkv_rows_t *k, const spkv_rows_t *v,
                              const spkv_rows_t *q_out, const spkv_rows_t *k_out, const spkv_rows_t *v_out,
                              spkv_stream_t stream) {
  int rc = check_norm_rope(norm, rope, n_tok, d_pos);
  if (rc) return rc;
  const bool has_v = v != nullptr;
  if (has_v != (v_out != nullptr)) return SPKV_E_INVALID;
  if (n_tok == 0) return SPKV_OK;
  RowArgs a = row_args(norm, rope, n_tok, d_pos, has_v);
  if (a.Hq + a.Hkv == 0) return SPKV_OK;
  const spkv_rows_t *in[3] = {q, k, v}, *out[3] = {q_out, k_out, v_out};
  const int heads[3] = {a.Hq, a.Hkv, a.Hv};
  for (int i = 0; i < 3; ++i) {
    if ((rc = check_rows(in[i], heads[i], n_tok, norm->dtype)) || (rc = check_rows(out[i], heads[i], n_tok, norm->dtype)))
      return rc;
    if (heads[i]) { a.x[i] = *in[i]; a.y[i] = *out[i]; }
  }
  int sms = 0;
  if ((rc = device_sms(&sms))) return rc;
  // tokens per block: enough blocks to fill the GPU four times over first, then fewer tables of angles
  a.tile = std::max(1, std::min(kMaxTile, n_tok / (4 * sms)));
  return dispatch_rows(a, norm->dtype, false, (int)(((int64_t)n_tok + a.tile - 1) / a.tile), nullptr, nullptr, as_stream(stream));
}

extern "C" size_t spkv_norm_rope_workspace_bytes(const spkv_qk_norm_t *norm) {
  if (!norm || norm->head_dim < 1 || norm->head_dim > SPKV_MAX_ROW_DIM) return 0;
  return (size_t)kMaxBwdBlocks * 2 * norm->head_dim * 4;
}

extern "C" int spkv_norm_rope_backward(const spkv_qk_norm_t *norm, const spkv_rope_t *rope, int32_t n_tok,
                                       const int32_t *d_pos, const spkv_rows_t *q, const spkv_rows_t *k,
                                       const spkv_rows_t *q_grad, const spkv_rows_t *k_grad, const spkv_rows_t *v_grad,
                                       const spkv_rows_t *dq, const spkv_rows_t *dk, const spkv_rows_t *dv,
                                       float *d_dwq, float *d_dwk, void *d_workspace, size_t workspace_bytes,
                                       spkv_stream_t stream) {
  int rc = check_norm_rope(norm, rope, n_tok, d_pos);
  if (rc) return rc;
  const bool has_v = v_grad != nullptr;
  if (has_v != (dv != nullptr)) return SPKV_E_INVALID;
  if ((d_dwq && !(norm->norm & SPKV_NORM_Q)) || (d_dwk && !(norm->norm & SPKV_NORM_K))) return SPKV_E_INVALID;
  RowArgs a = row_args(norm, rope, n_tok, d_pos, has_v);
  const bool weights = d_dwq || d_dwk;
  if (weights && (!d_workspace || ((uintptr_t)d_workspace & 15) || workspace_bytes < spkv_norm_rope_workspace_bytes(norm)))
    return SPKV_E_WORKSPACE;
  const bool rows = n_tok > 0 && a.Hq + a.Hkv > 0;
  if (!rows && !weights) return SPKV_OK;
  const spkv_rows_t *x[3] = {q, k, nullptr}, *g[3] = {q_grad, k_grad, v_grad}, *y[3] = {dq, dk, dv};
  const int heads[3] = {a.Hq, a.Hkv, a.Hv};
  for (int i = 0; rows && i < 3; ++i) {
    const bool normed = i < 2 && ((a.norm >> i) & 1);
    if ((rc = check_rows(g[i], heads[i], n_tok, norm->dtype)) || (rc = check_rows(y[i], heads[i], n_tok, norm->dtype)) ||
        (rc = check_rows(x[i], normed ? heads[i] : 0, n_tok, norm->dtype)))
      return rc;
    if (heads[i]) { a.g[i] = *g[i]; a.y[i] = *y[i]; }
    if (heads[i] && normed) a.x[i] = *x[i];
  }
  int sms = 0;
  if ((rc = device_sms(&sms))) return rc;
  a.tile = std::max(1, std::min(kMaxTile, n_tok / (4 * sms)));
  a.part = weights ? static_cast<float *>(d_workspace) : nullptr;
  const int n_tiles = (int)(((int64_t)n_tok + a.tile - 1) / a.tile);
  const int grid = rows ? std::min(n_tiles, std::min(kMaxBwdBlocks, 4 * sms)) : 0;
  return dispatch_rows(a, norm->dtype, true, grid, d_dwq, d_dwk, as_stream(stream));
}
