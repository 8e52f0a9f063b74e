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
// A row of head_dim elements belongs to TPR neighbouring lanes; a lane holds two 16-byte chunks of it, chosen so
// that both halves of every rotated pair are in the same lane: with pairs (i, i + rot/2) chunks j and j + rot/2,
// with pairs (2i, 2i + 1) chunks that hold whole pairs.  The row is read once, its sum of squares goes
// through log2(TPR) shuffles, everything else stays in registers, all in fp32 (two elements per
// instruction), and is rounded once on the way out.
//
// Angles.  A frequency is held as a fraction of a turn per position in 64-bit fixed point, so that
// position * frequency modulo one turn is one integer product without rounding; the upper 32 bits of that turn go
// through sincospif as a float.  That float's rounding, 2^-25 of a half turn or 9.4e-8 rad, is the angle's error at every
// position; the fraction's own (2^-64 turn, for |inv_freq| > 2 pi that many times more) times 2^31 positions and the bits
// cut off add 3e-9 (in fp32 a position of 10^6 is 0.06 rad off).  A warp
// computes the sines and cosines of a token once, through shared memory, for all its heads: no table
// in memory, no position limit.
//
// What bounds it: bytes; each row is read and written once.  B200, device time: 8192 tokens of 32/8 heads, bf16, 201 MB:
// 37.4 us = 5.4 TB/s (0.84 of the measured copy rate); backward of 32768 tokens, 1.14 GB: 185 us = 6.2 TB/s
// (0.96).  With rows held in registers on their way 50 and 271 us: too few bytes in flight.  One token: 2.9 us,
// a launch and three trips to memory.
#include <math.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include <cuda_fp16.h>

#include "spkv_internal.cuh"

namespace spkv {

constexpr int kRowThreads = 256, kRowWarps = kRowThreads / 32;
constexpr int kFwdBlocks = 2, kBwdBlocks = 2;   // blocks per SM (registers)
constexpr int kFewBlocks = 4;                   // blocks per SM up to which the kernel for few tokens is the faster one
constexpr int kMaxBwdBlocks = 512;              // partial sums of the weight gradients the workspace holds

struct RowArgs {
  spkv_rope_t rope;
  int n_tok, Hq, Hkv, Hv, D;
  int wpt;                     // warps per token: 1, 2, 4 or 8
  int norm;                    // bit 0: queries, bit 1: keys
  int w_dtype;
  float eps, inv_d;
  const void *wq, *wk;         // null = ones
  const int32_t *pos;          // [n_axes][n_tok]
  spkv_rows_t x[3], g[3], y[3];   // q, k, v: inputs, (backward) upstream gradients, results
  float *part;                 // backward: [gridDim.x][2][D] partial sums of g u, or null
};

// ---- two floats per instruction (packed fp32 arithmetic of sm_100), in one 64-bit register pair
typedef uint64_t f2;
__device__ inline f2 pk(float a, float b) {
  f2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ inline float2 up(f2 r) {
  float2 v;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(r));
  return v;
}
__device__ inline f2 mul(f2 a, f2 b) {
  f2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ inline f2 fma(f2 a, f2 b, f2 c) {
  f2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ inline f2 sub(f2 a, f2 b) {
  f2 r;
  asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// A 16-byte chunk as pairs of neighbouring elements.
template <class T> struct Elem;
template <> struct Elem<__nv_bfloat16> {
  static constexpr int kChunk = 8;
  static __device__ inline f2 pair(uint32_t w) { return pk(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
  static __device__ inline uint32_t word(f2 v) {
    const float2 f = up(v);
    const __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t *>(&h);
  }
};
template <> struct Elem<__half> {
  static constexpr int kChunk = 8;
  static __device__ inline f2 pair(uint32_t w) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w));
    return pk(f.x, f.y);
  }
  static __device__ inline uint32_t word(f2 v) {
    const float2 f = up(v);
    const __half2 h = __floats2half2_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t *>(&h);
  }
};
template <> struct Elem<float> {
  static constexpr int kChunk = 4;
};
template <class T>
__device__ inline void unpack(const uint4 &v, f2 (&f)[Elem<T>::kChunk / 2]) {
  if constexpr (Elem<T>::kChunk == 4) {
    f[0] = pk(__uint_as_float(v.x), __uint_as_float(v.y));
    f[1] = pk(__uint_as_float(v.z), __uint_as_float(v.w));
  } else {
    f[0] = Elem<T>::pair(v.x); f[1] = Elem<T>::pair(v.y); f[2] = Elem<T>::pair(v.z); f[3] = Elem<T>::pair(v.w);
  }
}
template <class T>
__device__ inline uint4 pack(const f2 (&f)[Elem<T>::kChunk / 2]) {
  if constexpr (Elem<T>::kChunk == 4) {
    const float2 a = up(f[0]), b = up(f[1]);
    return make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
  } else {
    return make_uint4(Elem<T>::word(f[0]), Elem<T>::word(f[1]), Elem<T>::word(f[2]), Elem<T>::word(f[3]));
  }
}

__device__ inline float load_weight(const void *w, int dtype, int i) {
  if (!w) return 1.f;
  if (dtype == SPKV_BF16) return __bfloat162float(static_cast<const __nv_bfloat16 *>(w)[i]);
  if (dtype == SPKV_F16) return __half2float(static_cast<const __half *>(w)[i]);
  return static_cast<const float *>(w)[i];
}

// Where lane j of a row finds its two chunks (element offsets).  Neighbouring lanes always read neighbouring chunks
// (a lane with two chunks side by side would make every 32-byte sector two requests).  Pairs (i, i + rot/2):
// chunks j and j + rot/2 of the rotated dims, the others in two halves likewise, not rotated; adjacent
// pairs lie within a chunk, the row goes in two halves.  A chunk is rotated as a whole or not at all (rot_dim is a
// multiple of 16), and what is not rotated is not touched: times (1, 0) an infinity would reach its neighbour as NaN.
struct LaneChunks { int c0, c1; bool live, rot0, rot1; };   // rot0, rot1: is the chunk rotated
template <int CE>
__device__ inline LaneChunks lane_chunks(const RowArgs &a, int j) {
  LaneChunks l;
  const int lanes = a.D / (2 * CE), n_rot = a.rope.interleaved ? lanes : a.rope.rot_dim / (2 * CE);
  l.live = j < lanes;
  if (j < n_rot) { l.c0 = j * CE; l.c1 = l.c0 + n_rot * CE; }
  else { l.c0 = (n_rot + j) * CE; l.c1 = l.c0 + (lanes - n_rot) * CE; }
  l.rot0 = l.c0 < a.rope.rot_dim;
  l.rot1 = l.c1 < a.rope.rot_dim;
  return l;
}
// Place of pair p in a token's table of (cos, sin): pair e of lane j at ((e / 2) TPR + j) 2 + e % 2.
template <int CE, int TPR, bool kAdjacent>
__device__ inline int pair_slot(const RowArgs &a, int p) {
  int j, e;
  if (kAdjacent) {
    const int chunk = p / (CE / 2), lanes = a.D / (2 * CE);
    j = chunk < lanes ? chunk : chunk - lanes;
    e = p % (CE / 2) + (chunk < lanes ? 0 : CE / 2);
  } else {
    j = p / CE;
    e = p % CE;
  }
  return ((e >> 1) * TPR + j) * 2 + (e & 1);
}
// A lane's CE pairs: pair e is (f0[e], f1[e]), or with adjacent pairs the two elements of f2 number e of chunk 0,
// then of chunk 1.  Angles as the rotation wants them: cosines c and sines s of pairs (2i, 2i + 1), or
// with adjacent pairs of pair i alone (c = (cos, cos), s = (sin, sin)).
template <int CE, bool kAdjacent> struct Angles { f2 c[kAdjacent ? CE : CE / 2], s[kAdjacent ? CE : CE / 2]; };

// Rotates the pairs of a lane's rotated chunks in place; kBack: by the opposite angle (the transpose); kAll: every
// dim of the head is rotated, nothing to select (timed in turn on the device: 8192 tokens of 32/8 heads 37.7 us, half of the
// dims rotated 42.0, of which the selects take 2.6; with a branch in their place the same, but 1001 fp32 tokens 10.1, not 9.9).
template <int CE, bool kAdjacent, bool kBack, bool kAll>
__device__ inline void rotate(f2 (&f0)[CE / 2], f2 (&f1)[CE / 2], const Angles<CE, kAdjacent> &a, const LaneChunks &l) {
  if constexpr (!kAdjacent) {
#pragma unroll
    for (int i = 0; i < CE / 2; ++i) {
      const f2 lo = f0[i], hi = f1[i];
      const f2 x = kBack ? fma(lo, a.c[i], mul(hi, a.s[i])) : sub(mul(lo, a.c[i]), mul(hi, a.s[i]));
      const f2 y = kBack ? sub(mul(hi, a.c[i]), mul(lo, a.s[i])) : fma(hi, a.c[i], mul(lo, a.s[i]));
      f0[i] = kAll || l.rot0 ? x : lo;   // (rot0 as rot1: the two chunks are each other's halves)
      f1[i] = kAll || l.rot0 ? y : hi;
    }
  } else {
    auto turn = [](f2 v, f2 c, f2 s) {   // (lo, hi) -> (lo c - hi s, hi c + lo s)
      const float2 x = up(v), cc = up(c), ss = up(s);
      const float sn = kBack ? -ss.x : ss.x;
      return pk(x.x * cc.x - x.y * sn, x.y * cc.x + x.x * sn);
    };
    if (kAll || l.rot0) {
#pragma unroll
      for (int i = 0; i < CE / 2; ++i) f0[i] = turn(f0[i], a.c[i], a.s[i]);
    }
    if (kAll || l.rot1) {
#pragma unroll
      for (int i = 0; i < CE / 2; ++i) f1[i] = turn(f1[i], a.c[CE / 2 + i], a.s[CE / 2 + i]);
    }
  }
}

// ---- shared memory of a block: the frequencies, the two weights as floats, and a table of (cos, sin) per warp.
// Weights and angles are ordered so that the lanes of a row read neighbouring 16-byte vectors.
template <int CE, int TPR>
struct Tables {
  uint64_t turn[SPKV_MAX_ROW_DIM / 2];
  int32_t axis[SPKV_MAX_ROW_DIM / 2];
  alignas(16) float w[2][2 * CE * TPR];             // element e of lane j at ((e / 4) TPR + j) 4 + e % 4
  alignas(16) float2 cs[kRowWarps][CE * TPR];       // pair e of lane j at ((e / 2) TPR + j) 2 + e % 2
};
template <int CE, int TPR>
__device__ inline void fill_weights(const RowArgs &a, float (&w)[2][2 * CE * TPR]) {
  for (int x = threadIdx.x; x < 2 * 2 * CE * TPR; x += kRowThreads) {
    const int side = x / (2 * CE * TPR), r = x % (2 * CE * TPR), j = r / (2 * CE), e = r % (2 * CE);
    const LaneChunks l = lane_chunks<CE>(a, j);
    const int d = e < CE ? l.c0 + e : l.c1 + e - CE;
    w[side][((e >> 2) * TPR + j) * 4 + (e & 3)] = l.live ? load_weight(side ? a.wk : a.wq, a.w_dtype, d) : 0.f;
  }
}
template <int CE, int TPR>
__device__ inline void fill_tables(const RowArgs &a, Tables<CE, TPR> &t) {   // the whole block; ends with a barrier
  for (int p = threadIdx.x; p < a.rope.rot_dim / 2; p += kRowThreads) {
    t.turn[p] = a.rope.turn[p];
    t.axis[p] = a.rope.axis[p];
  }
  if (a.norm) fill_weights<CE, TPR>(a, t.w);
  __syncthreads();
}
// (cos, sin) of one pair: turns modulo one as a 64-bit fixed-point product, its upper 32 bits as half turns in [-1, 1)
__device__ inline float2 pair_angle(const RowArgs &a, int pos, uint64_t turn) {
  const uint64_t turns = (uint64_t)(int64_t)pos * turn;
  float sn, cn;
  sincospif((float)(int32_t)(turns >> 32) * 4.656612873077393e-10f, &sn, &cn);
  return make_float2(cn * a.rope.scale, sn * a.rope.scale);
}
// A lane's share of a token's table (of its rotated chunks; the table holds no other pairs).
template <int CE, int TPR, bool kAdjacent>
__device__ inline void lane_angles(const float2 *tab, int j, const LaneChunks &l, Angles<CE, kAdjacent> &out) {
#pragma unroll
  for (int i = 0; i < CE / 2; ++i) {
    float4 v = make_float4(1.f, 0.f, 1.f, 0.f);
    if (!kAdjacent || i < CE / 4 ? l.rot0 : l.rot1) v = *reinterpret_cast<const float4 *>(tab + (i * TPR + j) * 2);
    if constexpr (kAdjacent) {
      out.c[2 * i] = pk(v.x, v.x); out.s[2 * i] = pk(v.y, v.y);
      out.c[2 * i + 1] = pk(v.z, v.z); out.s[2 * i + 1] = pk(v.w, v.w);
    } else {
      out.c[i] = pk(v.x, v.z);
      out.s[i] = pk(v.y, v.w);
    }
  }
}
// Sines and cosines of one token, by one warp, and this lane's share of them.
template <int CE, int TPR, bool kAdjacent>
__device__ inline void token_angles(const RowArgs &a, Tables<CE, TPR> &t, int tok, const LaneChunks &l, Angles<CE, kAdjacent> &out) {
  const int lane = threadIdx.x & 31, j = threadIdx.x % TPR;
  float2 *tab = t.cs[threadIdx.x >> 5];
  __syncwarp();    // the previous token's angles have been read
  for (int p = lane; p < a.rope.rot_dim / 2; p += 32)
    tab[pair_slot<CE, TPR, kAdjacent>(a, p)] = pair_angle(a, __ldg(&a.pos[(size_t)t.axis[p] * a.n_tok + tok]), t.turn[p]);
  __syncwarp();
  lane_angles<CE, TPR, kAdjacent>(tab, j, l, out);
}
template <int CE, int TPR>
__device__ inline void lane_weights(const float *w, int j, f2 (&w0)[CE / 2], f2 (&w1)[CE / 2]) {
#pragma unroll
  for (int i = 0; i < CE / 4; ++i) {
    const float4 v = *reinterpret_cast<const float4 *>(w + (i * TPR + j) * 4);
    w0[2 * i] = pk(v.x, v.y); w0[2 * i + 1] = pk(v.z, v.w);
    const float4 u = *reinterpret_cast<const float4 *>(w + ((i + CE / 4) * TPR + j) * 4);
    w1[2 * i] = pk(u.x, u.y); w1[2 * i + 1] = pk(u.z, u.w);
  }
}

template <int TPR>
__device__ inline float row_sum(float v) {
#pragma unroll
  for (int o = TPR / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// sum over a lane's elements of a * b
template <int CE>
__device__ inline float dot(const f2 (&a0)[CE / 2], const f2 (&b0)[CE / 2], const f2 (&a1)[CE / 2], const f2 (&b1)[CE / 2]) {
  f2 s = mul(a0[0], b0[0]), t = mul(a1[0], b1[0]);
#pragma unroll
  for (int i = 1; i < CE / 2; ++i) { s = fma(a0[i], b0[i], s); t = fma(a1[i], b1[i], t); }
  const float2 x = up(s), y = up(t);
  return (x.x + x.y) + (y.x + y.y);
}

template <class T>
__device__ inline T *row_ptr(const spkv_rows_t &v, int64_t tok, int head) {
  return static_cast<T *>(v.ptr) + tok * v.token_stride + (int64_t)head * v.head_stride;
}
template <class T>
__device__ inline void load_row(uint4 (&r)[2], const T *p, const LaneChunks &l, bool on) {
  r[0] = r[1] = make_uint4(0, 0, 0, 0);
  if (on) {
    r[0] = __ldcs(reinterpret_cast<const uint4 *>(p + l.c0));
    r[1] = __ldcs(reinterpret_cast<const uint4 *>(p + l.c1));
  }
}
template <class T>
__device__ inline void store_row(T *p, const LaneChunks &l, bool on, const uint4 &r0, const uint4 &r1) {
  if (on) {
    *reinterpret_cast<uint4 *>(p + l.c0) = r0;
    *reinterpret_cast<uint4 *>(p + l.c1) = r1;
  }
}

// Work split.  A token belongs to one warp, or to 2, 4 or 8 of a block's warps (split_rows); a warp's lanes take 32 / TPR heads at a time.  The token's sines and cosines
// stay in registers for all its heads, a row costs no index arithmetic but an addition, and the next rows
// are loaded before the current ones are worked on.
template <int TPR> struct WarpWork {
  int first, stride, head0, step;   // first token, tokens between two of this warp; first head, heads per pass
  __device__ WarpWork(const RowArgs &a) {
    const int w = blockIdx.x * kRowWarps + (threadIdx.x >> 5), part = w & (a.wpt - 1), rows = 32 / TPR;
    first = w / a.wpt;
    stride = gridDim.x * kRowWarps / a.wpt;
    head0 = part * rows;
    step = a.wpt * rows;
  }
};

// A warp's rows are one stream -- token after token, query, key and value heads, `step` heads a pass -- that runs
// kDepth passes ahead through shared memory: a lane copies its own 32 bytes of a pass there
// asynchronously and reads them back, so that what is on its way costs no registers (a warp's 2 KB in registers
// left memory waiting: 40 us for 8192 tokens of 32/8 heads, 37.3 this way).
template <class T, int TPR, int kStreams>
struct RowStream {
  static constexpr int kDepth = 4 / kStreams;
  const RowArgs &a;
  const WarpWork<TPR> &work;
  const LaneChunks &l;
  uint4 *ring;                  // this lane's first chunk of pass 0; chunk k of stream s of pass d at ((d kStreams + s) 2 + k) 32
  int64_t tok;                  // next pass to ask for
  int pass, slot;               // ... of the token; ring slot of the next pass to take (= to ask for, once the ring is full)
  int n_pass[3];                // passes of the warp per side
  __device__ RowStream(const RowArgs &a_, const WarpWork<TPR> &w, const LaneChunks &l_, uint4 *warp_ring, int first_side,
                       int last_side)
      : a(a_), work(w), l(l_), ring(warp_ring + (threadIdx.x & 31)), tok(w.first), pass(0), slot(0) {
    const int H[3] = {a.Hq, a.Hkv, a.Hv};
#pragma unroll
    for (int s = 0; s < 3; ++s)
      n_pass[s] = s < first_side || s > last_side || H[s] <= w.head0 ? 0 : (H[s] - w.head0 + w.step - 1) / w.step;
  }
  __device__ bool any() const { return n_pass[0] + n_pass[1] + n_pass[2] > 0; }
  // asks for the next pass, into the current slot
  __device__ void ask() {
    if (tok < a.n_tok && any()) {
      const int side = (pass >= n_pass[0]) + (pass >= n_pass[0] + n_pass[1]);
      const int i = pass - (side ? n_pass[0] : 0) - (side == 2 ? n_pass[1] : 0);
      const int h = work.head0 + i * work.step + (threadIdx.x & 31) / TPR;
      const bool on = l.live && h < (side ? a.Hkv : a.Hq);
#pragma unroll
      for (int s = 0; s < kStreams; ++s) {
        // stream 0 of the backward pass: upstream gradients; stream 1: the inputs of a normed side
        const spkv_rows_t &v = kStreams == 1 ? (side == 0 ? a.x[0] : side == 1 ? a.x[1] : a.x[2])
                               : s == 0      ? (side == 0 ? a.g[0] : side == 1 ? a.g[1] : a.g[2])
                                             : (side == 0 ? a.x[0] : a.x[1]);
        const bool use = on && (s == 0 || (side < 2 && ((a.norm >> side) & 1)));
        const T *src = use ? row_ptr<const T>(v, tok, h) : static_cast<const T *>(v.ptr);
        uint4 *dst = ring + (slot * kStreams + s) * 64;
        copy16(dst, src + l.c0, use);
        copy16(dst + 32, src + l.c1, use);
      }
      if (++pass == n_pass[0] + n_pass[1] + n_pass[2]) {
        pass = 0;
        tok += work.stride;
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  static __device__ void copy16(uint4 *dst, const T *src, bool on) {   // zeros where a lane has no row
    if (!on) { *dst = make_uint4(0, 0, 0, 0); return; }
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;"
                 ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(dst))), "l"(src) : "memory");
  }
  __device__ void start() {
#pragma unroll
    for (int d = 0; d < kDepth; ++d) {
      slot = d;
      ask();
    }
    slot = 0;
  }
  // the oldest pass; then asks for one more
  __device__ void take(uint4 (&r)[kStreams][2]) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory");
#pragma unroll
    for (int s = 0; s < kStreams; ++s) {
      r[s][0] = ring[(slot * kStreams + s) * 64];
      r[s][1] = ring[(slot * kStreams + s) * 64 + 32];
    }
    ask();
    slot = slot + 1 == kDepth ? 0 : slot + 1;
  }
};

// One side's heads of a warp's token.
template <class T, int TPR, bool kAdjacent, bool kCopy>
__device__ inline void forward_side(const RowArgs &a, const spkv_rows_t &y, int H, int n_pass, bool normed, const float *s_w,
                                    const Angles<Elem<T>::kChunk, kAdjacent> &ang, int64_t tok, const WarpWork<TPR> &work,
                                    const LaneChunks &l, RowStream<T, TPR, 1> &stream) {
  constexpr int CE = Elem<T>::kChunk;
  if (n_pass == 0) return;   // (warp-uniform, as is the loop: all lanes shuffle)
  const int sub = (threadIdx.x & 31) / TPR, j = threadIdx.x % TPR;
  f2 w0[CE / 2], w1[CE / 2];
  if (!kCopy && normed) lane_weights<CE, TPR>(s_w, j, w0, w1);
  T *dst = row_ptr<T>(y, tok, work.head0 + sub);
  const int64_t out_step = work.step * y.head_stride;
  int h = work.head0 + sub;
  auto passes = [&](auto all) {
#pragma unroll 2
    for (int i = 0; i < n_pass; ++i, h += work.step, dst += out_step) {
      uint4 cur[1][2];
      stream.take(cur);
      if (!kCopy) {
        f2 f0[CE / 2], f1[CE / 2];
        unpack<T>(cur[0][0], f0);
        unpack<T>(cur[0][1], f1);
        if (normed) {
          const float r = rsqrtf(row_sum<TPR>(dot<CE>(f0, f0, f1, f1)) * a.inv_d + a.eps);
          const f2 rr = pk(r, r);
#pragma unroll
          for (int e = 0; e < CE / 2; ++e) { f0[e] = mul(f0[e], mul(rr, w0[e])); f1[e] = mul(f1[e], mul(rr, w1[e])); }
        }
        rotate<CE, kAdjacent, false, decltype(all)::value>(f0, f1, ang, l);
        cur[0][0] = pack<T>(f0);
        cur[0][1] = pack<T>(f1);
      }
      store_row(dst, l, l.live && h < H, cur[0][0], cur[0][1]);
    }
  };
  if (kCopy || a.rope.rot_dim == a.D) passes(std::true_type()); else passes(std::false_type());
}

template <class T, int TPR, bool kAdjacent>
__global__ void __launch_bounds__(kRowThreads, kFwdBlocks) norm_rope_kernel(const __grid_constant__ RowArgs a) {
  constexpr int CE = Elem<T>::kChunk;
  __shared__ Tables<CE, TPR> tables;
  __shared__ uint4 s_ring[kRowWarps][RowStream<T, TPR, 1>::kDepth * 64];
  pdl_trigger();
  const WarpWork<TPR> work(a);
  const LaneChunks l = lane_chunks<CE>(a, threadIdx.x % TPR);
  RowStream<T, TPR, 1> stream(a, work, l, s_ring[threadIdx.x >> 5], 0, 2);
  stream.start();
  fill_tables<CE, TPR>(a, tables);
  for (int64_t tok = work.first; tok < a.n_tok; tok += work.stride) {
    Angles<CE, kAdjacent> ang;
    token_angles<CE, TPR, kAdjacent>(a, tables, (int)tok, l, ang);
    forward_side<T, TPR, kAdjacent, false>(a, a.y[0], a.Hq, stream.n_pass[0], a.norm & 1, tables.w[0], ang, tok, work, l, stream);
    forward_side<T, TPR, kAdjacent, false>(a, a.y[1], a.Hkv, stream.n_pass[1], (a.norm >> 1) & 1, tables.w[1], ang, tok, work, l, stream);
    forward_side<T, TPR, kAdjacent, true>(a, a.y[2], a.Hv, stream.n_pass[2], false, tables.w[0], ang, tok, work, l, stream);
  }
}

// Forward for few tokens (a decode step): a block per token, or several that share its rows (gridDim.y) while there
// is room for them; the rows of all sides in one short loop.  Such a launch is a chain of waits -- instructions,
// positions and weights, rows -- so the code is small (the kernel above spends more on fetching its
// instructions than on a token) and the first rows are on their way while the angles are computed.  One token of
// 32/8 heads 3.0 us a launch (4.3 above; 2.9 and 5.1 with 24/24 fp32 heads), 592 tokens 5.7 (6.3).
template <class T, int TPR, bool kAdjacent>
__global__ void __launch_bounds__(kRowThreads, kFewBlocks) norm_rope_few_kernel(const __grid_constant__ RowArgs a) {
  constexpr int CE = Elem<T>::kChunk, kRows = kRowThreads / TPR;
  __shared__ alignas(16) float2 s_cs[CE * TPR];
  __shared__ alignas(16) float s_w[2][2 * CE * TPR];
  pdl_trigger();
  const int tok = blockIdx.x, j = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  const LaneChunks l = lane_chunks<CE>(a, j);
  const int n_rows = a.Hq + a.Hkv + a.Hv;
  // row r of the token: side and head (a warp's rows may lie on several sides)
  auto side_of = [&](int r) { return (r >= a.Hq) + (r >= a.Hq + a.Hkv); };
  auto head_of = [&](int r, int side) { return r - (side ? a.Hq : 0) - (side == 2 ? a.Hkv : 0); };
  uint4 nxt[2];
  auto fetch = [&](int r) {
    const bool on = l.live && r < n_rows;
    const int side = on ? side_of(r) : 0;
    load_row(nxt, row_ptr<const T>(side == 0 ? a.x[0] : side == 1 ? a.x[1] : a.x[2], tok, on ? head_of(r, side) : 0), l, on);
  };
  const int first = blockIdx.y * kRows + sub, step = gridDim.y * kRows;
  fetch(first);
  for (int p = threadIdx.x; p < a.rope.rot_dim / 2; p += kRowThreads)
    s_cs[pair_slot<CE, TPR, kAdjacent>(a, p)] = pair_angle(a, __ldg(&a.pos[(size_t)a.rope.axis[p] * a.n_tok + tok]), a.rope.turn[p]);
  if (a.norm) fill_weights<CE, TPR>(a, s_w);
  __syncthreads();
  Angles<CE, kAdjacent> ang;
  lane_angles<CE, TPR, kAdjacent>(s_cs, j, l, ang);
#pragma unroll 1
  for (int r = first; r - sub < n_rows; r += step) {   // (the same passes for all lanes: they shuffle)
    const int side = side_of(r);
    uint4 cur[2] = {nxt[0], nxt[1]};
    fetch(r + step);
    if (__any_sync(0xffffffffu, side < 2)) {
      f2 f0[CE / 2], f1[CE / 2];
      unpack<T>(cur[0], f0);
      unpack<T>(cur[1], f1);
      if (a.norm) {
        const float q = rsqrtf(row_sum<TPR>(dot<CE>(f0, f0, f1, f1)) * a.inv_d + a.eps);
        if (side < 2 && ((a.norm >> side) & 1)) {
          f2 w0[CE / 2], w1[CE / 2];
          lane_weights<CE, TPR>(s_w[side], j, w0, w1);
          const f2 rr = pk(q, q);
#pragma unroll
          for (int i = 0; i < CE / 2; ++i) { f0[i] = mul(f0[i], mul(rr, w0[i])); f1[i] = mul(f1[i], mul(rr, w1[i])); }
        }
      }
      if (side < 2) {
        rotate<CE, kAdjacent, false, false>(f0, f1, ang, l);
        cur[0] = pack<T>(f0);
        cur[1] = pack<T>(f1);
      }
    }
    const bool on = l.live && r < n_rows;
    store_row(row_ptr<T>(side == 0 ? a.y[0] : side == 1 ? a.y[1] : a.y[2], tok, on ? head_of(r, side) : 0), l, on, cur[0], cur[1]);
  }
}

// One side's heads of a warp's token, backward: dx rows out, this lane's columns of g u added to dw.
template <class T, int TPR, bool kAdjacent, bool kCopy>
__device__ inline void backward_side(const RowArgs &a, const spkv_rows_t &y, int H, int n_pass, bool normed, const float *s_w,
                                     const Angles<Elem<T>::kChunk, kAdjacent> &ang, int64_t tok, const WarpWork<TPR> &work,
                                     const LaneChunks &l, RowStream<T, TPR, 2> &stream, f2 (&dw0)[Elem<T>::kChunk / 2],
                                     f2 (&dw1)[Elem<T>::kChunk / 2]) {
  constexpr int CE = Elem<T>::kChunk;
  if (n_pass == 0) return;
  const int sub = (threadIdx.x & 31) / TPR, j = threadIdx.x % TPR;
  T *dst = row_ptr<T>(y, tok, work.head0 + sub);
  const int64_t out_step = work.step * y.head_stride;
  int h = work.head0 + sub;
  auto passes = [&](auto all) {
    for (int i = 0; i < n_pass; ++i, h += work.step, dst += out_step) {
      uint4 cur[2][2];   // upstream gradients, inputs
      stream.take(cur);
      if (!kCopy) {
        f2 f0[CE / 2], f1[CE / 2];
        unpack<T>(cur[0][0], f0);
        unpack<T>(cur[0][1], f1);
        rotate<CE, kAdjacent, true, decltype(all)::value>(f0, f1, ang, l);
        if (normed) {
          f2 u0[CE / 2], u1[CE / 2], w0[CE / 2], w1[CE / 2];
          unpack<T>(cur[1][0], u0);
          unpack<T>(cur[1][1], u1);
          lane_weights<CE, TPR>(s_w, j, w0, w1);
          const float r0 = rsqrtf(row_sum<TPR>(dot<CE>(u0, u0, u1, u1)) * a.inv_d + a.eps);
          const float r = h < H ? r0 : 0.f;   // (lanes without a row hold zeros: with eps = 0 infinity times zero in dw)
          const f2 rr = pk(r, r);
#pragma unroll
          for (int e = 0; e < CE / 2; ++e) {
            u0[e] = mul(u0[e], rr);
            u1[e] = mul(u1[e], rr);
            dw0[e] = fma(f0[e], u0[e], dw0[e]);
            dw1[e] = fma(f1[e], u1[e], dw1[e]);
            f0[e] = mul(f0[e], w0[e]);
            f1[e] = mul(f1[e], w1[e]);
          }
          const float m = -row_sum<TPR>(dot<CE>(f0, u0, f1, u1)) * a.inv_d;
          const f2 mean = pk(m, m);
#pragma unroll
          for (int e = 0; e < CE / 2; ++e) { f0[e] = mul(rr, fma(u0[e], mean, f0[e])); f1[e] = mul(rr, fma(u1[e], mean, f1[e])); }
        }
        cur[0][0] = pack<T>(f0);
        cur[0][1] = pack<T>(f1);
      }
      store_row(dst, l, l.live && h < H, cur[0][0], cur[0][1]);
    }
  };
  if (kCopy || a.rope.rot_dim == a.D) passes(std::true_type()); else passes(std::false_type());
}

// Backward.  A warp goes over its tokens once for the queries and once for keys and values, so that the sums of one
// side's weight gradient are all a lane has to keep.  Which rows a lane adds up is fixed by the launch
// alone: the result is the same every time.  Lanes that share columns are added up at the end, first
// through shuffles, then through shared memory in warp order.
template <class T, int TPR, bool kAdjacent>
__global__ void __launch_bounds__(kRowThreads, kBwdBlocks) norm_rope_backward_kernel(const __grid_constant__ RowArgs a) {
  constexpr int CE = Elem<T>::kChunk;
  __shared__ Tables<CE, TPR> tables;
  __shared__ uint4 s_ring[kRowWarps][RowStream<T, TPR, 2>::kDepth * 128];
  // a side's sums at its end, [warp][2 CE * TPR], over the angles (nobody needs them then)
  float *s_dw = reinterpret_cast<float *>(tables.cs);
  static_assert(sizeof(tables.cs) >= kRowWarps * 2 * CE * TPR * 4, "room for the sums");
  pdl_trigger();
  const WarpWork<TPR> work(a);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = threadIdx.x % TPR;
  const LaneChunks l = lane_chunks<CE>(a, j);
  f2 dw0[CE / 2], dw1[CE / 2];
  auto walk = [&](auto side_c, RowStream<T, TPR, 2> &stream) {
    constexpr int side = decltype(side_c)::value;
#pragma unroll
    for (int i = 0; i < CE / 2; ++i) dw0[i] = dw1[i] = pk(0.f, 0.f);
    if (!stream.any()) return;
    for (int64_t tok = work.first; tok < a.n_tok; tok += work.stride) {
      Angles<CE, kAdjacent> ang;
      token_angles<CE, TPR, kAdjacent>(a, tables, (int)tok, l, ang);
      backward_side<T, TPR, kAdjacent, false>(a, a.y[side], side ? a.Hkv : a.Hq, stream.n_pass[side], (a.norm >> side) & 1,
                                              tables.w[side], ang, tok, work, l, stream, dw0, dw1);
      if (side == 1)
        backward_side<T, TPR, kAdjacent, true>(a, a.y[2], a.Hv, stream.n_pass[2], false, tables.w[0], ang, tok, work, l, stream,
                                               dw0, dw1);
    }
  };
  auto sum = [&](int side) {
    if (!a.part) return;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < CE; ++i) {
      float2 v = up(i < CE / 2 ? dw0[i % (CE / 2)] : dw1[i % (CE / 2)]);
#pragma unroll
      for (int o = TPR; o < 32; o <<= 1) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
      }
      if (lane < TPR) {
        s_dw[(warp * 2 * CE + 2 * i) * TPR + j] = v.x;
        s_dw[(warp * 2 * CE + 2 * i + 1) * TPR + j] = v.y;
      }
    }
    __syncthreads();
    for (int x = threadIdx.x; x < 2 * CE * TPR; x += kRowThreads) {
      const int e = x / TPR, jj = x % TPR;
      const LaneChunks ll = lane_chunks<CE>(a, jj);
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < kRowWarps; ++w) v += s_dw[(w * 2 * CE + e) * TPR + jj];
      if (ll.live) a.part[((size_t)blockIdx.x * 2 + side) * a.D + (e < CE ? ll.c0 + e : ll.c1 + e - CE)] = v;
    }
    __syncthreads();
  };
  // each side's first rows are on their way while the tables are filled, or the other side's sums made
  RowStream<T, TPR, 2> queries(a, work, l, s_ring[warp], 0, 0);
  queries.start();
  fill_tables<CE, TPR>(a, tables);
  walk(std::integral_constant<int, 0>(), queries);
  RowStream<T, TPR, 2> keys_values(a, work, l, s_ring[warp], 1, 2);
  keys_values.start();
  sum(0);
  walk(std::integral_constant<int, 1>(), keys_values);
  sum(1);
}

// Sums the blocks' partial weight gradients, in a fixed order: grid (D / 16, 2 sides), 512 threads = 16 columns x 32
// slices of the blocks.
constexpr int kGradSlices = 32;
__global__ void __launch_bounds__(16 * kGradSlices) norm_weight_grad_kernel(const float *part, int n_blocks, int D, float *dwq,
                                                                           float *dwk) {
  __shared__ float s[kGradSlices][17];
  const int col = blockIdx.x * 16 + (threadIdx.x & 15), slice = threadIdx.x >> 4, side = blockIdx.y;
  pdl_wait();
  float v = 0.f;
#pragma unroll 8
  for (int b = slice; b < n_blocks; b += kGradSlices) v += __ldcg(&part[((size_t)b * 2 + side) * D + col]);
  s[slice][threadIdx.x & 15] = v;
  __syncthreads();
  if (threadIdx.x < 16) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < kGradSlices; ++i) t += s[i][threadIdx.x];
    float *out = side ? dwk : dwq;
    if (out) out[col] = t;
  }
}

static int elem_bytes(int dtype) { return dtype == SPKV_F32 ? 4 : 2; }

static int check_rows(const spkv_rows_t *r, int heads, int dtype) {
  if (heads == 0) return SPKV_OK;
  if (!r || !r->ptr) return SPKV_E_INVALID;
  const int64_t per16 = 16 / elem_bytes(dtype);
  if (((uintptr_t)r->ptr & 15) || r->head_stride % per16 || r->token_stride % per16) return SPKV_E_INVALID;
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

// SMs of the current device, asked for once per device.
static int device_sms(int *sms) {
  static std::atomic<int> known[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return SPKV_E_CUDA;
  if (dev < 64 && (*sms = known[dev].load(std::memory_order_relaxed)) > 0) return SPKV_OK;
  if (cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return SPKV_E_CUDA;
  if (dev < 64) known[dev].store(*sms, std::memory_order_relaxed);
  return SPKV_OK;
}

// Warps per token, and blocks.  A launch lasts as many rounds as its busiest warp has tokens (or parts of tokens), and
// a round lasts as many passes over heads as a part has, plus about two for the token's angles: the split
// with the smallest product.  Measured against the fewest warps that fill the GPU, every split timed at 14
// lengths: 2400 tokens of 24/24 heads, fp32, 39.9 -> 32.4 us; 1001 tokens of 8/2 heads 7.1 -> 5.0 us; no worse than
// the best of the four by more than 5 % (backward pass: 10 %).
static int split_rows(RowArgs &a, int sms, int blocks_per_sm, int rows_per_pass, bool backward) {
  const int64_t warps = (int64_t)sms * blocks_per_sm * kRowWarps;
  const int heads[3] = {a.Hq, a.Hkv, a.Hv};
  int64_t least = 0;
  for (int w = 1; w <= kRowWarps; w *= 2) {
    int passes = backward ? 2 * 2 : 2;   // (the backward pass takes a token up twice)
    for (int h : heads) passes += (h + w * rows_per_pass - 1) / (w * rows_per_pass);
    const int64_t cost = (a.n_tok * (int64_t)w + warps - 1) / warps * passes;
    if (w == 1 || cost < least) { least = cost; a.wpt = w; }
  }
  return (int)std::min<int64_t>((int64_t)sms * blocks_per_sm, ((int64_t)a.n_tok * a.wpt + kRowWarps - 1) / kRowWarps);
}

template <class T, int TPR>
static int launch_rows(RowArgs &a, bool backward, int sms, float *dwq, float *dwk, cudaStream_t s) {
  const bool adjacent = a.rope.interleaved != 0;
  if (!backward && a.n_tok <= kFewBlocks * sms) {
    const int passes = ((a.Hq + a.Hkv + a.Hv) * TPR + kRowThreads - 1) / kRowThreads;
    const dim3 grid(a.n_tok, std::max(1, std::min(passes, kFewBlocks * sms / a.n_tok)));
    if (adjacent) norm_rope_few_kernel<T, TPR, true><<<grid, kRowThreads, 0, s>>>(a);
    else norm_rope_few_kernel<T, TPR, false><<<grid, kRowThreads, 0, s>>>(a);
    return check_stream_error(cudaGetLastError());
  }
  if (!backward) {
    const int grid = split_rows(a, sms, kFwdBlocks, 32 / TPR, false);
    if (adjacent) norm_rope_kernel<T, TPR, true><<<grid, kRowThreads, 0, s>>>(a);
    else norm_rope_kernel<T, TPR, false><<<grid, kRowThreads, 0, s>>>(a);
    return check_stream_error(cudaGetLastError());
  }
  const int grid = a.Hq + a.Hkv ? std::min(kMaxBwdBlocks, split_rows(a, sms, kBwdBlocks, 32 / TPR, true)) : 0;
  if (grid) {
    if (adjacent) norm_rope_backward_kernel<T, TPR, true><<<grid, kRowThreads, 0, s>>>(a);
    else norm_rope_backward_kernel<T, TPR, false><<<grid, kRowThreads, 0, s>>>(a);
    if (cudaGetLastError() != cudaSuccess) return SPKV_E_CUDA;
  }
  if (!a.part) return SPKV_OK;
  if (!grid) {   // no rows: the sums are zero
    norm_weight_grad_kernel<<<dim3(a.D / 16, 2), 16 * kGradSlices, 0, s>>>(a.part, 0, a.D, dwq, dwk);
    return check_stream_error(cudaGetLastError());
  }
  return check_stream_error(launch_overlapped(norm_weight_grad_kernel, dim3(a.D / 16, 2), dim3(16 * kGradSlices), 0, s, a.part, grid,
                                              a.D, dwq, dwk));
}

// lanes per row: two 16-byte chunks each, rounded up to a power of two
static int dispatch_rows(RowArgs &a, int dtype, bool backward, int sms, float *dwq, float *dwk, cudaStream_t s) {
  const int lanes = a.D * elem_bytes(dtype) / 32;
#define SPKV_ROWS(T)                                                       \
  if (lanes <= 4) return launch_rows<T, 4>(a, backward, sms, dwq, dwk, s); \
  if (lanes <= 8) return launch_rows<T, 8>(a, backward, sms, dwq, dwk, s); \
  if (lanes <= 16) return launch_rows<T, 16>(a, backward, sms, dwq, dwk, s);
  if (dtype == SPKV_F32) {
    SPKV_ROWS(float)
    return launch_rows<float, 32>(a, backward, sms, dwq, dwk, s);
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
    if ((rc = check_rows(in[i], heads[i], norm->dtype)) || (rc = check_rows(out[i], heads[i], norm->dtype)))
      return rc;
    if (heads[i]) { a.x[i] = *in[i]; a.y[i] = *out[i]; }
  }
  int sms = 0;
  if ((rc = device_sms(&sms))) return rc;
  note_cacheless_call();
  return dispatch_rows(a, norm->dtype, false, sms, nullptr, nullptr, as_stream(stream));
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
    if ((rc = check_rows(g[i], heads[i], norm->dtype)) || (rc = check_rows(y[i], heads[i], norm->dtype)) ||
        (rc = check_rows(x[i], normed ? heads[i] : 0, norm->dtype)))
      return rc;
    if (heads[i]) { a.g[i] = *g[i]; a.y[i] = *y[i]; }
    if (heads[i] && normed) a.x[i] = *x[i];
  }
  int sms = 0;
  if ((rc = device_sms(&sms))) return rc;
  a.part = weights ? static_cast<float *>(d_workspace) : nullptr;
  if (!rows) a.Hq = a.Hkv = a.Hv = 0;
  note_cacheless_call();
  return dispatch_rows(a, norm->dtype, true, sms, d_dwq, d_dwk, as_stream(stream));
}
