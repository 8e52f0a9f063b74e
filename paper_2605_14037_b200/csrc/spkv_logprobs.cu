// What rows of logits say (spkv_token_logprobs): log sum of exponentials, entropy, log probabilities of given tokens, and
// the largest logits.
//
// One pass over the logits.  A row is cut into chunks of 2 KB (the first takes the elements before the first
// 16-byte boundary as well); a warp holds a chunk in registers and asks for its next one meanwhile.  With c = scale log2 e, M
// a reference of the lane's own near its maximum (log2 domain) and t = c x - M
//     S = sum 2^t,   A = sum 2^t t,      lse = ln 2 (M + log2 S),   entropy = ln 2 (log2 S - A / S),
// of a warp's chunks of a row, and the chunk's maximum goes to memory, where a top list is wanted.  The n_top largest elements of a row lie in the n_top
// chunks with the largest maxima (of equal ones those with the lower index), so a second, small kernel -- a
// block per row, which also joins the row's sums -- looks into those chunks only, and the first pays nothing for the list.
//
// Elements below kFloor count as kFloor: 0 times -infinity has no place in A.  Their weight is 0, unless the
// whole row lies that low (masked by a low value throughout) or the scale is so small that kFloor is near.  M is c x rounded, so
// that t is off by up to 2^-24 |M|, a weight by 2 to that power: where the row's M is 2^24 or more in size it would count, from 2^31
// on S itself leaves float32.  Such rows, and those whose sums are not finite for another reason (a product of c that has left
// float32), are summed up again, about their own maximum, by the second kernel.
// What bounds it: 768 rows of 128256 bf16 logits, top 1: 43.5 us on the device, 4.5 TB/s (30 us at the copy rate).  37 of them are the
// first kernel, at 8 instructions an element (maxima and floor take two elements an instruction in the type itself) and 57 % of the
// issue slots; the other 6.5 are the second, which cannot begin before all rows are summed.  5 rows of 50257 fp32, top 5: 9.6 us, two
// launches with four trips to memory between them.
#include <cuda_fp16.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "spkv_internal.cuh"
#include "spkv_tc5.cuh"

namespace spkv {

namespace lp {
constexpr int kChunkBytes = 2048, kWarps = 8, kThreads = 32 * kWarps;
template <class T> constexpr int kChunk = kChunkBytes / (int)sizeof(T);   // elements
constexpr int kBlocksPerSm = 4;      // 64 registers a thread: a chunk and the next one (4 KB chunks spill: 67 against 47 us at the time for 768 rows of 128256)
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
}  // namespace lp

struct LogprobArgs {
  const void *x;
  int64_t stride;
  int n_rows, vocab, n_given, n_top, max_chunks, per, pitch;   // per: chunks a warp takes, of all rows' in one line; pitch: parts a row has at most
  float scale;
  const int32_t *given;
  float *lse, *entropy, *logp, *top_logp;
  int32_t *top_ids;
  float4 *part;        // [n_rows][pitch] {M, S, A, a NaN was among them}: what a warp holds of a row
  uint32_t *chunk_key; // [n_rows][max_chunks], n_top > 0 only
};

// Order of logits as unsigned integers: descending values are descending keys, NaN stands above all, and the two zeros
// are one value.
__device__ inline uint32_t value_key(float x) {
  if (x != x) return 0xffffffffu;
  const uint32_t b = __float_as_uint(x == 0.f ? 0.f : x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline float key_value(uint32_t k) {
  return k == 0xffffffffu ? NAN : __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
template <class T> __device__ inline float as_float(T x);
template <> __device__ inline float as_float(float x) { return x; }
template <> __device__ inline float as_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ inline float as_float(__half x) { return __half2float(x); }

// elements before the row's first 16-byte boundary
template <class T> __device__ inline int row_head(const T *row, int vocab) {
  return min(vocab, (int)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(T));
}
template <class T> __device__ inline int row_chunks(int head, int vocab) { return max(1, (vocab - head + lp::kChunk<T> - 1) / lp::kChunk<T>); }

// 16 bytes as floats
template <class T, int kN = 16 / sizeof(T)> __device__ inline void unpack(const uint4 &v, float (&f)[kN]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      f[i] = __uint_as_float(w[i]);
    } else if constexpr (std::is_same<T, __nv_bfloat16>::value) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    } else {
      const float2 p = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
      f[2 * i] = p.x;
      f[2 * i + 1] = p.y;
    }
  }
}

// Pairs of a type's elements: floor and maximum (NaN if there is one) without unpacking.  The floor lies where c x is still
// exact to a small fraction of 1 (an M far below -2^24 is not: its rounding alone would be a large exponent).
template <class T> struct Low;
template <> struct Low<__nv_bfloat16> {
  static constexpr float kFloor = -0x1p+20f;                       // 0xc980
  static __device__ inline uint32_t floor2(uint32_t x) {
    const __nv_bfloat162 f = __halves2bfloat162(__ushort_as_bfloat16(0xc980), __ushort_as_bfloat16(0xc980));
    const __nv_bfloat162 r = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162 *>(&x), f);
    return *reinterpret_cast<const uint32_t *>(&r);
  }
  static __device__ inline uint32_t max2(uint32_t x, uint32_t y) {
    const __nv_bfloat162 r = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162 *>(&x), *reinterpret_cast<const __nv_bfloat162 *>(&y));
    return *reinterpret_cast<const uint32_t *>(&r);
  }
};
template <> struct Low<__half> {
  static constexpr float kFloor = -65504.f;                        // 0xfbff: only -infinity lies below
  static __device__ inline uint32_t floor2(uint32_t x) {
    const __half2 f = __halves2half2(__ushort_as_half(0xfbff), __ushort_as_half(0xfbff));
    const __half2 r = __hmax2_nan(*reinterpret_cast<const __half2 *>(&x), f);
    return *reinterpret_cast<const uint32_t *>(&r);
  }
  static __device__ inline uint32_t max2(uint32_t x, uint32_t y) {
    const __half2 r = __hmax2_nan(*reinterpret_cast<const __half2 *>(&x), *reinterpret_cast<const __half2 *>(&y));
    return *reinterpret_cast<const uint32_t *>(&r);
  }
};
template <> struct Low<float> {
  static constexpr float kFloor = -0x1p+20f;
  static __device__ inline uint32_t floor2(uint32_t x) { return __float_as_uint(__uint_as_float(x) < kFloor ? kFloor : __uint_as_float(x)); }
  static __device__ inline uint32_t max2(uint32_t x, uint32_t y) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(__uint_as_float(x)), "f"(__uint_as_float(y)));
    return __float_as_uint(r);
  }
};

template <class T> __device__ inline void unpack2_of(uint32_t w, float (&f)[2]) {
  if constexpr (std::is_same<T, __nv_bfloat16>::value) {
    f[0] = __uint_as_float(w << 16);
    f[1] = __uint_as_float(w & 0xffff0000u);
  } else {
    const float2 p = __half22float2(*reinterpret_cast<const __half2 *>(&w));
    f[0] = p.x;
    f[1] = p.y;
  }
}

// Running (M, S, A) of one lane.  M grows only when a maximum outgrows it by 2^16, so that a row's chunks hardly ever
// rescale; the exponentials then reach 2^16, far from the type's end.
struct Sums {
  float M = -INFINITY, S = 0.f, A = 0.f;
  __device__ inline void raise(float to) {      // (NaN: stays)
    if (to > M + 16.f) {
      if (S > 0.f) {
        const float d = M - to, f = exp2f(d);
        A = f > 0.f ? f * fmaf(S, d, A) : 0.f;
        S = f > 0.f ? S * f : 0.f;   // (S about a far lower M may be infinite: see the head)
      }
      M = to;
    }
  }
};

// one element
template <class T> __device__ inline void one(T x, float c, Sums &s, float &top, bool &nan) {
  const float f = as_float(x);
  top = fmaxf(top, f);
  nan = nan || f != f;
  if (!(f > Low<T>::kFloor)) return;
  s.raise(f * c);
  const float t = fmaf(f, c, -s.M), e = fast_exp2(t);
  s.S += e;
  s.A = fmaf(e, t, s.A);
}

// 16-byte words of a chunk that lies inside the row: lane l holds words l, l + 32, ...
constexpr int kWords = lp::kChunkBytes / 512;
template <class T> __device__ inline void load_chunk(const T *p, uint4 (&v)[kWords]) {
#pragma unroll
  for (int i = 0; i < kWords; ++i) v[i] = __ldcs(reinterpret_cast<const uint4 *>(p) + (threadIdx.x & 31) + 32 * i);
}
// ... into a lane's sums; top: the lane's maximum, nan: is a NaN among its elements
template <class T>
__device__ inline void add_chunk(const uint4 (&v)[kWords], float c, Sums &s, float &top, bool &nan) {
  using namespace tc5;
  constexpr int kPer = 16 / sizeof(T);
  uint32_t mx = v[0].x;
#pragma unroll
  for (int i = 0; i < kWords; ++i) {
    mx = Low<T>::max2(mx, v[i].x); mx = Low<T>::max2(mx, v[i].y); mx = Low<T>::max2(mx, v[i].z); mx = Low<T>::max2(mx, v[i].w);
  }
  if constexpr (sizeof(T) == 4) {
    top = __uint_as_float(mx);
  } else {
    float f[2];
    unpack2_of<T>(mx, f);
    top = f[0] != f[0] || f[0] > f[1] ? f[0] : f[1];
  }
  if (top <= Low<T>::kFloor) return;   // nothing that counts
  s.raise(top * c);
  const float2 nM2 = make_float2(-s.M, -s.M), c2 = make_float2(c, c);
  float2 S2 = make_float2(0.f, 0.f), A2 = S2;
#pragma unroll
  for (int i = 0; i < kWords; ++i) {
    float f[kPer];
    unpack<T>(make_uint4(Low<T>::floor2(v[i].x), Low<T>::floor2(v[i].y), Low<T>::floor2(v[i].z), Low<T>::floor2(v[i].w)), f);
#pragma unroll
    for (int x = 0; x < kPer; x += 2) {
      const float2 t = __ffma2_rn(make_float2(f[x], f[x + 1]), c2, nM2);
      const float2 e = make_float2(fast_exp2(t.x), fast_exp2(t.y));
      S2 = __fadd2_rn(S2, e);
      A2 = __ffma2_rn(e, t, A2);
    }
  }
  const float add = S2.x + S2.y;
  s.S += add;
  s.A += A2.x + A2.y;
  if (add != add) {   // a NaN among the elements, or an infinity less itself
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      float f[kPer];
      unpack<T>(v[i], f);
#pragma unroll
      for (int x = 0; x < kPer; ++x) nan = nan || f[x] != f[x];
    }
  }
}

// {M, S, A, a NaN was among them} of two sets of elements together
__device__ inline float4 no_part() { return make_float4(-INFINITY, 0.f, 0.f, 0.f); }
__device__ inline float4 join(float4 p, float4 q) {
  const float M = fmaxf(p.x, q.x);
  auto weigh = [&](float4 &s) {
    if (s.y > 0.f && s.x < M) {
      const float d = s.x - M, f = exp2f(d);
      s.z = f > 0.f ? f * fmaf(s.y, d, s.z) : 0.f;
      s.y = f > 0.f ? s.y * f : 0.f;
    }
  };
  weigh(p);
  weigh(q);
  return make_float4(M, p.y + q.y, p.z + q.z, fmaxf(p.w, q.w));
}
__device__ inline float4 join_lanes(float4 p) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    p = join(p, make_float4(__shfl_xor_sync(0xffffffffu, p.x, o), __shfl_xor_sync(0xffffffffu, p.y, o),
                            __shfl_xor_sync(0xffffffffu, p.z, o), __shfl_xor_sync(0xffffffffu, p.w, o)));
  return p;
}

template <class T>
__global__ void __launch_bounds__(lp::kThreads, lp::kBlocksPerSm) logprob_sums_kernel(LogprobArgs a) {
  using namespace lp;
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const long long warp = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5), all = (long long)a.n_rows * a.max_chunks;
  const float c = a.scale * kLog2e;
  for (long long g = warp * a.per, to = min(g + a.per, all); g < to;) {
    const int row = (int)(g / a.max_chunks), first = (int)(g - (long long)row * a.max_chunks);
    const T *x = static_cast<const T *>(a.x) + (int64_t)row * a.stride;
    const int head = row_head(x, a.vocab);
    // this warp's chunks of the row: first ... < end; `full` of the row's chunks have all their elements
    const int last = (int)min((long long)a.max_chunks, first + (to - g)), end = min(last, row_chunks<T>(head, a.vocab));
    const int stop = min(end, (a.vocab - head) / kChunk<T>);
    g += last - first;
    Sums s;
    bool nan = false;
    auto key = [&](int ch, float top, bool odd) {
      const uint32_t k = __reduce_max_sync(0xffffffffu, odd ? 0xffffffffu : value_key(top));
      if (lane == 0) a.chunk_key[(size_t)row * a.max_chunks + ch] = k;
    };
    uint4 v[2][kWords];
    int ch = first;
    if (ch < stop) load_chunk(x + head + (int64_t)ch * kChunk<T>, v[0]);
    auto round = [&](const uint4 (&now)[kWords], uint4 (&next)[kWords]) {   // ... and ask for the next chunk first
      if (ch + 1 < stop) load_chunk(x + head + (int64_t)(ch + 1) * kChunk<T>, next);
      float top;
      bool odd = false;
      add_chunk<T>(now, c, s, top, odd);
      if (ch == 0 && lane < head) one<T>(x[lane], c, s, top, odd);   // the elements before the boundary belong to it
      if (a.n_top > 0) key(ch, top, odd);
      nan = nan || odd;
      ++ch;
    };
    while (ch < stop) {
      round(v[0], v[1]);
      if (ch < stop) round(v[1], v[0]);
    }
    if (ch < end) {   // the row's last chunk, in part
      float top = -INFINITY;
      bool odd = false;
      for (int i = head + ch * kChunk<T> + lane; i < a.vocab; i += 32) one<T>(x[i], c, s, top, odd);
      if (ch == 0 && lane < head) one<T>(x[lane], c, s, top, odd);
      if (a.n_top > 0) key(ch, top, odd);
      nan = nan || odd;
    }
    const float4 w = join_lanes(make_float4(s.M, s.S, s.A, nan ? 1.f : 0.f));
    if (lane == 0) a.part[(size_t)row * a.pitch + (warp - (long long)row * a.max_chunks / a.per)] = w;
  }
}

// A warp's list of the 32 largest keys so far, lane i holding the i-th largest; of a key the upper half is a logit's
// value_key, the lower 2^32 - 1 - index, 0 is no entry.
struct TopList {
  uint64_t mine = 0, over = 0;   // only keys above `over` are of use
  // A key of every lane (0: none), the largest first: after a list's worth of them the others are below `over`.
  __device__ inline void offer(uint64_t key, int n) {
    const int lane = threadIdx.x & 31;
    while (__any_sync(0xffffffffu, key > over)) {
      const uint32_t hi = __reduce_max_sync(0xffffffffu, key > over ? (uint32_t)(key >> 32) : 0u);
      const uint32_t lo = __reduce_max_sync(0xffffffffu, key > over && (uint32_t)(key >> 32) == hi ? (uint32_t)key : 0u);
      const uint64_t best = (uint64_t)hi << 32 | lo;
      if (key == best) key = 0;
      const uint64_t left = __shfl_up_sync(0xffffffffu, mine, 1);
      const bool below = mine < best;
      const unsigned first = __ballot_sync(0xffffffffu, below);
      if (below) mine = lane == __ffs(first) - 1 ? best : left;
      const uint64_t last = __shfl_sync(0xffffffffu, mine, n - 1);
      if (last > over) over = last;
    }
  }
};

// (six blocks an SM: 888 rows run at once; 768 rows 43.5 us together with the sums, 45.9 with five)
// One block per row: its parts joined, and its largest logits out of the chunks with the largest maxima.
template <class T>
__global__ void __launch_bounds__(lp::kThreads, 6) logprob_rows_kernel(LogprobArgs a) {
  using namespace lp;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, row = blockIdx.x;
  const T *x = static_cast<const T *>(a.x) + (int64_t)row * a.stride;
  const int head = row_head(x, a.vocab), n_chunks = row_chunks<T>(head, a.vocab);
  const float c = a.scale * kLog2e;
  __shared__ float s_base, s_log2;       // a logit's log probability is ln 2 ((c x - s_base) - s_log2), or, if the row was summed again,
  __shared__ int s_again;                // scale (x - s_base) - ln 2 s_log2
  // scale (x - y), also where the difference alone leaves float32
  auto scaled = [&](float x, float y) {
    const float d = x - y;
    return d == -INFINITY && x > -INFINITY ? (0.5f * x - 0.5f * y) * a.scale * 2.f : d * a.scale;
  };
  __shared__ int s_chunk[SPKV_MAX_TOP];
  __shared__ uint32_t s_bound;           // value_key that every wanted element reaches
  __shared__ uint64_t s_list[kWarps][32];
  __shared__ float4 s_part[kWarps];
  pdl_wait();
  if (warp == 0) {
    float4 p = no_part();
    const long long from = (long long)row * a.max_chunks;   // (the row's first and last warp: by their chunks)
    const int parts = (int)((from + a.max_chunks - 1) / a.per - from / a.per) + 1;
    for (int i0 = lane; i0 < parts; i0 += 128) {
      float4 q[4];
#pragma unroll
      for (int y = 0; y < 4; ++y) q[y] = i0 + 32 * y < parts ? __ldcg(&a.part[(size_t)row * a.pitch + i0 + 32 * y]) : no_part();
#pragma unroll
      for (int y = 0; y < 4; ++y) p = join(p, q[y]);
    }
    p = join_lanes(p);
    if (lane == 0) {
      const float M = p.x, l2 = log2f(p.y);
      const bool nan = p.w != 0.f;
      s_again = !nan && !(M > Low<T>::kFloor * c + 200.f && fabsf(M) < 0x1p+24f && isfinite(p.y) && isfinite(p.z));
      s_base = nan ? NAN : M;
      s_log2 = l2;
      if (a.lse) a.lse[row] = nan ? NAN : kLn2 * (M + l2);
      if (a.entropy) a.entropy[row] = nan ? NAN : kLn2 * (l2 - p.z / p.y);
    }
  } else if (warp == 1 && a.n_top > 0) {
    TopList list;
    const uint32_t *keys = a.chunk_key + (size_t)row * a.max_chunks;
    for (int i0 = lane; i0 - lane < n_chunks; i0 += 128) {
      uint32_t k[4];
#pragma unroll
      for (int y = 0; y < 4; ++y) k[y] = i0 + 32 * y < n_chunks ? __ldcg(&keys[i0 + 32 * y]) : 0;
#pragma unroll
      for (int y = 0; y < 4; ++y)
        list.offer(i0 + 32 * y < n_chunks ? (uint64_t)k[y] << 32 | (0xffffffffu - (uint32_t)(i0 + 32 * y)) : 0, a.n_top);
    }
    if (lane < a.n_top) s_chunk[lane] = list.mine ? (int)(0xffffffffu - (uint32_t)list.mine) : -1;
    if (lane == a.n_top - 1) s_bound = (uint32_t)(list.mine >> 32);
  }
  __syncthreads();
  if (s_again) {   // (no NaN in the row)
    float m = -INFINITY;
    for (int i = threadIdx.x; i < a.vocab; i += kThreads) m = fmaxf(m, as_float(x[i]));
    const uint32_t k = __reduce_max_sync(0xffffffffu, value_key(m));
    if (lane == 0) s_part[warp].x = key_value(k);
    __syncthreads();
    for (int w = 0; w < kWarps; ++w) m = fmaxf(m, s_part[w].x);
    __syncthreads();
    float4 p = make_float4(0.f, 0.f, 0.f, 0.f);
    if (m > -INFINITY && m < INFINITY)
      for (int i = threadIdx.x; i < a.vocab; i += kThreads) {
        const float t = scaled(as_float(x[i]), m), e = fast_exp2(t * kLog2e);   // (c may have left float32)
        p.y += e;
        p.z = fmaf(e, fmaxf(t, -300.f), p.z);
      }
    p = join_lanes(p);
    if (lane == 0) s_part[warp] = p;
    __syncthreads();
    if (threadIdx.x == 0) {
      p = s_part[0];
      for (int w = 1; w < kWarps; ++w) p = join(p, s_part[w]);
      const bool inf = m == INFINITY;
      const float l2 = log2f(p.y);   // (a row of -infinities: m and l2 are -infinity, the results NaN but for lse)
      s_base = inf ? 0.f : m;
      s_log2 = inf ? INFINITY : l2;
      if (a.lse) a.lse[row] = inf ? INFINITY : fmaf(m, a.scale, kLn2 * l2);
      if (a.entropy) a.entropy[row] = inf ? NAN : kLn2 * l2 - p.z / p.y;
    }
    __syncthreads();
  }
  auto log_probability = [&](float f) {
    const float d = fmaf(f, c, -s_base);
    if (s_again) return scaled(f, s_base) - kLn2 * s_log2;
    return d == -INFINITY ? f * a.scale : kLn2 * (d - s_log2);   // (c f may leave the type where scale f does not)
  };
  for (int j = threadIdx.x; j < a.n_given; j += kThreads) {
    const int tok = a.given[(size_t)row * a.n_given + j];
    a.logp[(size_t)row * a.n_given + j] = tok >= 0 && tok < a.vocab ? log_probability(as_float(x[tok])) : NAN;
  }
  if (a.n_top <= 0) return;
  TopList list;
  if (s_bound) list.over = ((uint64_t)s_bound << 32) - 1;
  // few chunks are looked through by several warps each: a warp takes every pieces-th 256 elements
  const int pieces = a.n_top == 1 ? 8 : a.n_top == 2 ? 4 : a.n_top <= 4 ? 2 : 1;
  for (int j = warp; j < a.n_top * pieces; j += kWarps) {
    const int ch = s_chunk[j / pieces];
    if (ch < 0) break;
    const int i0 = ch ? head + ch * kChunk<T> : 0, i1 = min(a.vocab, head + (ch + 1) * kChunk<T>);
    for (int b = i0 + j % pieces * 256; b < i1; b += 256 * pieces) {
      float f[8];
#pragma unroll
      for (int y = 0; y < 8; ++y) {
        const int i = b + 32 * y + lane;
        f[y] = i < i1 ? as_float(x[i]) : 0.f;
      }
#pragma unroll
      for (int y = 0; y < 8; ++y) {
        const int i = b + 32 * y + lane;
        list.offer(i < i1 ? (uint64_t)value_key(f[y]) << 32 | (0xffffffffu - (uint32_t)i) : 0, a.n_top);
      }
    }
  }
  s_list[warp][lane] = list.mine;
  __syncthreads();
  if (warp) return;
  for (int w = 1; w < kWarps; ++w) list.offer(s_list[w][lane], a.n_top);
  if (lane < a.n_top) {
    const size_t at = (size_t)row * a.n_top + lane;
    const bool have = list.mine != 0;
    if (a.top_ids) a.top_ids[at] = have ? (int)(0xffffffffu - (uint32_t)list.mine) : -1;
    if (a.top_logp) a.top_logp[at] = have ? log_probability(key_value((uint32_t)(list.mine >> 32))) : NAN;
  }
}

struct LogprobWs { size_t off_key, total; int max_chunks; };
static LogprobWs logprob_ws(int n_rows, int vocab, int n_top, int elem_bytes) {
  LogprobWs w;
  w.max_chunks = std::max(1, (int)(((int64_t)vocab * elem_bytes + lp::kChunkBytes - 1) / lp::kChunkBytes));
  w.off_key = (size_t)n_rows * w.max_chunks * sizeof(float4);   // (at most a part for every chunk)
  w.total = w.off_key + (n_top > 0 ? ((size_t)n_rows * w.max_chunks * 4 + 15) / 16 * 16 : 0);
  return w;
}

template <class T> static int launch_logprobs(LogprobArgs &a, cudaStream_t s) {
  const int64_t warps = ((int64_t)a.n_rows * a.max_chunks + a.per - 1) / a.per;
  logprob_sums_kernel<T><<<(unsigned)((warps + lp::kWarps - 1) / lp::kWarps), lp::kThreads, 0, s>>>(a);
  if (cudaGetLastError() != cudaSuccess) return SPKV_E_CUDA;
  return check_stream_error(launch_overlapped(logprob_rows_kernel<T>, dim3(a.n_rows), dim3(lp::kThreads), 0, s, a));
}

}  // namespace spkv

using namespace spkv;

extern "C" size_t spkv_logprobs_workspace_bytes(int32_t n_rows, int32_t vocab, int32_t n_top) {
  if (n_rows < 0 || vocab < 1 || n_top < 0 || n_top > SPKV_MAX_TOP) return 0;
  return std::max<size_t>(16, logprob_ws(n_rows, vocab, n_top, 4).total);
}

extern "C" int spkv_token_logprobs(int32_t dtype, int32_t n_rows, int32_t vocab, const void *d_logits, int64_t row_stride,
                                   float scale, const int32_t *d_given, int32_t n_given, int32_t n_top, float *d_lse,
                                   float *d_entropy, float *d_logp, int32_t *d_top_ids, float *d_top_logp, void *d_workspace,
                                   size_t workspace_bytes, spkv_stream_t stream) {
  if (dtype < SPKV_BF16 || dtype > SPKV_F32 || n_rows < 0 || vocab < 1 || n_given < 0 || n_top < 0) return SPKV_E_INVALID;
  if (n_top > SPKV_MAX_TOP) return SPKV_E_UNSUPPORTED;
  if (!(scale > 0.f) || !isfinite(scale)) return SPKV_E_INVALID;
  if ((int64_t)n_rows * n_given > INT32_MAX || (int64_t)n_rows * n_top > INT32_MAX) return SPKV_E_UNSUPPORTED;
  if (vocab > INT32_MAX - 2 * lp::kChunkBytes) return SPKV_E_UNSUPPORTED;
  if (n_rows == 0) return SPKV_OK;
  const int bytes = dtype == SPKV_F32 ? 4 : 2;
  if (!d_logits || ((uintptr_t)d_logits & (bytes - 1))) return SPKV_E_INVALID;
  if (!d_logp) n_given = 0;
  if (!d_top_ids && !d_top_logp) n_top = 0;
  if (n_given && !d_given) return SPKV_E_INVALID;
  if (!d_workspace || ((uintptr_t)d_workspace & 15) || workspace_bytes < spkv_logprobs_workspace_bytes(n_rows, vocab, n_top)) return SPKV_E_WORKSPACE;
  const LogprobWs w = logprob_ws(n_rows, vocab, n_top, bytes);
  int dev = -1, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return SPKV_E_CUDA;
  LogprobArgs a = {};
  a.x = d_logits; a.stride = row_stride; a.n_rows = n_rows; a.vocab = vocab; a.n_given = n_given; a.n_top = n_top; a.scale = scale;
  a.given = d_given; a.lse = d_lse; a.entropy = d_entropy; a.logp = d_logp; a.top_ids = d_top_ids; a.top_logp = d_top_logp;
  a.part = static_cast<float4 *>(d_workspace);
  a.chunk_key = reinterpret_cast<uint32_t *>(static_cast<char *>(d_workspace) + w.off_key);
  a.max_chunks = w.max_chunks;
  // All rows' chunks in one line, cut into as many equal pieces as the SMs hold warps (or one chunk each, if there are fewer): all
  // blocks start and end together, also where the rows are no multiple of them.
  const int64_t warps = (int64_t)sms * lp::kBlocksPerSm * lp::kWarps, per = ((int64_t)n_rows * w.max_chunks + warps - 1) / warps;
  if (per > INT32_MAX) return SPKV_E_UNSUPPORTED;
  a.per = (int)per;
  a.pitch = std::min(w.max_chunks, (int)((w.max_chunks + per - 1) / per) + 1);
  note_cacheless_call();
  cudaStream_t s = as_stream(stream);
  return dtype == SPKV_BF16 ? launch_logprobs<__nv_bfloat16>(a, s) : dtype == SPKV_F16 ? launch_logprobs<__half>(a, s)
                                                                                     : launch_logprobs<float>(a, s);
}
