// What rows of logits say (spkv_token_logprobs): log sum of exponentials, entropy, log probabilities of given tokens, and
// the largest logits.
//
// One pass over the logits.  A row is cut into chunks of 1024 elements (the first takes the elements before the first
// 16-byte boundary as well), a warp takes a chunk at a time: its maximum m in one round over the registers that hold
// it, then with t = (x - m) scale log2 e
//     S = sum 2^t,   A = sum 2^t t,      lse = scale m + ln S,   entropy = ln 2 (log2 S - A / S),
// and the chunk's maximum to memory, where a top list is wanted.  The n_top largest elements of a row lie in the n_top
// chunks with the largest maxima (of equal ones those with the lower index), so a second, small kernel -- a
// block per row, which also joins the row's sums -- looks into those chunks only, and the first pays nothing for the list.
// What bounds it: memory (2 or 4 bytes an element).  The first kernel's arithmetic is 5.5 instructions an element of the
// 11 that the SMs could issue while bf16 rows arrive at the copy rate.
#include <math.h>

#include <algorithm>

#include <cuda_fp16.h>

#include <type_traits>

#include "spkv_internal.cuh"
#include "spkv_tc5.cuh"

namespace spkv {

namespace lp {
constexpr int kChunk = 1024, kWarps = 8, kThreads = 32 * kWarps;
constexpr int kBlocksPerSm = 6;      // 40 registers a thread; a warp has 2 KB (bf16) or 4 KB of its chunk in flight
constexpr int kMaxRounds = 4;        // chunks a warp takes at most
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
}  // namespace lp

struct LogprobArgs {
  const void *x;
  int64_t stride;
  int n_rows, vocab, n_given, n_top, parts, rounds, max_chunks;
  float scale;
  const int32_t *given;
  float *lse, *entropy, *logp, *top_logp;
  int32_t *top_ids;
  float4 *part;        // [n_rows][parts] {m, S, A, a NaN was among them}
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
__device__ inline int row_chunks(int head, int vocab) { return max(1, (vocab - head + lp::kChunk - 1) / lp::kChunk); }

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

// Running (m, S, A) of one lane.  m grows only when a maximum outgrows it by 2^16, so that a row's chunks hardly ever
// rescale; the exponentials then reach 2^16, far from the type's end.
struct Sums {
  float m = -INFINITY, S = 0.f, A = 0.f;
  __device__ inline void raise(float to, float c) {      // (NaN: stays)
    if (to > m && !((to - m) * c <= 16.f)) {
      if (S > 0.f) {
        const float d = (m - to) * c, f = exp2f(d);
        A = f > 0.f ? f * fmaf(S, d, A) : 0.f;
        S *= f;
      }
      m = to;
    }
  }
  __device__ inline float base() const { return m == -INFINITY ? 0.f : m; }
};

// {m, S, A, a NaN was among them} of two sets of elements together
__device__ inline float4 no_part() { return make_float4(-INFINITY, 0.f, 0.f, 0.f); }
__device__ inline float4 join(float4 p, float4 q, float c) {
  const float M = fmaxf(p.x, q.x);
  auto weigh = [&](float4 &s) {
    if (s.y > 0.f && s.x < M) {
      const float d = (s.x - M) * c, f = exp2f(d);
      s.z = f > 0.f ? f * fmaf(s.y, d, s.z) : 0.f;
      s.y *= f;
    }
  };
  weigh(p);
  weigh(q);
  return make_float4(M, p.y + q.y, p.z + q.z, fmaxf(p.w, q.w));
}
__device__ inline float4 join_lanes(float4 p, float c) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    p = join(p, make_float4(__shfl_xor_sync(0xffffffffu, p.x, o), __shfl_xor_sync(0xffffffffu, p.y, o),
                            __shfl_xor_sync(0xffffffffu, p.z, o), __shfl_xor_sync(0xffffffffu, p.w, o)), c);
  return p;
}

// One warp's chunk, all of it inside the row: lane l holds vectors l, l + 32, ...
template <class T>
__device__ inline void full_chunk(const T *p, float c, Sums &s, float &top, bool &nan) {
  using namespace tc5;
  constexpr int kPer = 16 / sizeof(T), kVec = lp::kChunk / 32 / kPer;
  const int lane = threadIdx.x & 31;
  uint4 v[kVec];
#pragma unroll
  for (int i = 0; i < kVec; ++i) v[i] = __ldcs(reinterpret_cast<const uint4 *>(p) + lane + 32 * i);
  float mx = -INFINITY;
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    float f[kPer];
    unpack<T>(v[i], f);
#pragma unroll
    for (int x = 0; x < kPer; x += 2) mx = max3(mx, f[x], f[x + 1]);
  }
  s.raise(mx, c);
  const float b = s.base();
  const uint64_t nb2 = pack2(-b, -b), c2 = pack2(c, c);
  uint64_t S2 = pack2(0.f, 0.f), A2 = S2;
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    float f[kPer];
    unpack<T>(v[i], f);
#pragma unroll
    for (int x = 0; x < kPer; x += 2) {
      float t0, t1;
      unpack2(mul2(add2(pack2(f[x], f[x + 1]), nb2), c2), t0, t1);
      const uint64_t e2 = pack2(fast_exp2(t0), fast_exp2(t1));
      S2 = add2(S2, e2);
      A2 = fma2(e2, pack2(fmaxf(t0, -300.f), fmaxf(t1, -300.f)), A2);   // (0 times -infinity is not wanted)
    }
  }
  float a0, a1;
  unpack2(S2, a0, a1);
  const float add = a0 + a1;
  s.S += add;
  unpack2(A2, a0, a1);
  s.A += a0 + a1;
  top = mx;
  if (add != add) {   // a NaN among the elements, or an infinity less itself
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      float f[kPer];
      unpack<T>(v[i], f);
#pragma unroll
      for (int x = 0; x < kPer; ++x) nan = nan || f[x] != f[x];
    }
  }
}

template <class T>
__global__ void __launch_bounds__(lp::kThreads, lp::kBlocksPerSm) logprob_sums_kernel(LogprobArgs a) {
  using namespace lp;
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int row = blockIdx.x / a.parts, part = blockIdx.x - row * a.parts;
  const T *x = static_cast<const T *>(a.x) + (int64_t)row * a.stride;
  const int head = row_head(x, a.vocab), n_chunks = row_chunks(head, a.vocab);
  const float c = a.scale * kLog2e;
  Sums s;
  bool nan = false;
  auto one = [&](float f) {
    s.raise(f, c);
    const float t = (f - s.base()) * c, e = fast_exp2(t);
    s.S += e;
    s.A = fmaf(e, fmaxf(t, -300.f), s.A);
    nan = nan || f != f;
  };
  for (int r = 0; r < a.rounds; ++r) {
    const int ch = (part * a.rounds + r) * kWarps + warp;
    if (ch >= n_chunks) break;
    const int i0 = head + ch * kChunk;
    float top = -INFINITY;
    const bool before = nan;
    nan = false;
    if (i0 + kChunk <= a.vocab) {
      full_chunk(x + i0, c, s, top, nan);
    } else {
      for (int i = i0 + lane; i < a.vocab; i += 32) {
        const float f = as_float(x[i]);
        one(f);
        top = fmaxf(top, f);
      }
    }
    if (ch == 0 && lane < head) {
      const float f = as_float(x[lane]);
      one(f);
      top = fmaxf(top, f);
    }
    if (a.n_top > 0) {
      const uint32_t key = __reduce_max_sync(0xffffffffu, nan ? 0xffffffffu : value_key(top));
      if (lane == 0) a.chunk_key[(size_t)row * a.max_chunks + ch] = key;
    }
    nan = nan || before;
  }
  // ---- the block's sums: lanes, then warps, in a fixed order
  __shared__ float4 s_part[kWarps];
  const float4 w = join_lanes(make_float4(s.m, s.S, s.A, nan ? 1.f : 0.f), c);
  if (lane == 0) s_part[warp] = w;
  __syncthreads();
  if (warp == 0) {
    const float4 all = join_lanes(lane < kWarps ? s_part[lane] : no_part(), c);
    if (lane == 0) a.part[(size_t)row * a.parts + part] = all;
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

// One block per row: its parts joined, and its largest logits out of the chunks with the largest maxima.
template <class T>
__global__ void __launch_bounds__(lp::kThreads) logprob_rows_kernel(LogprobArgs a) {
  using namespace lp;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, row = blockIdx.x;
  const T *x = static_cast<const T *>(a.x) + (int64_t)row * a.stride;
  const int head = row_head(x, a.vocab), n_chunks = row_chunks(head, a.vocab);
  const float c = a.scale * kLog2e;
  __shared__ float s_m, s_ln;            // a logit's log probability is (x - s_m) scale - s_ln
  __shared__ int s_chunk[SPKV_MAX_TOP];
  __shared__ uint32_t s_bound;           // value_key that every wanted element reaches
  __shared__ uint64_t s_list[kWarps][32];
  pdl_wait();
  if (warp == 0) {
    float4 p = no_part();
    for (int i = lane; i < a.parts; i += 32) p = join(p, a.part[(size_t)row * a.parts + i], c);
    p = join_lanes(p, c);
    if (lane == 0) {
      const float M = p.x, S = p.y;
      const bool nan = p.w != 0.f, inf = M == INFINITY;
      s_m = nan ? NAN : inf ? 0.f : M;
      s_ln = inf ? INFINITY : logf(S);
      if (a.lse) a.lse[row] = nan ? NAN : inf ? INFINITY : fmaf(M, a.scale, logf(S));
      if (a.entropy) a.entropy[row] = nan || inf ? NAN : logf(S) - kLn2 * (p.z / S);
    }
  } else if (warp == 1 && a.n_top > 0) {
    TopList list;
    for (int i0 = 0; i0 < n_chunks; i0 += 32) {
      const int i = i0 + lane;
      list.offer(i < n_chunks ? (uint64_t)a.chunk_key[(size_t)row * a.max_chunks + i] << 32 | (0xffffffffu - (uint32_t)i) : 0, a.n_top);
    }
    if (lane < a.n_top) s_chunk[lane] = list.mine ? (int)(0xffffffffu - (uint32_t)list.mine) : -1;
    if (lane == a.n_top - 1) s_bound = (uint32_t)(list.mine >> 32);
  }
  __syncthreads();
  for (int j = threadIdx.x; j < a.n_given; j += kThreads) {
    const int tok = a.given[(size_t)row * a.n_given + j];
    a.logp[(size_t)row * a.n_given + j] =
        tok >= 0 && tok < a.vocab ? fmaf(as_float(x[tok]) - s_m, a.scale, -s_ln) : NAN;
  }
  if (a.n_top <= 0) return;
  TopList list;
  if (s_bound) list.over = ((uint64_t)s_bound << 32) - 1;
  for (int j = warp; j < a.n_top; j += kWarps) {
    const int ch = s_chunk[j];
    if (ch < 0) break;
    const int i0 = ch ? head + ch * kChunk : 0, i1 = min(a.vocab, head + (ch + 1) * kChunk);
    for (int b = i0; b < i1; b += 8 * 32) {
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
    if (a.top_logp) a.top_logp[at] = have ? fmaf(key_value((uint32_t)(list.mine >> 32)) - s_m, a.scale, -s_ln) : NAN;
  }
}

struct LogprobWs { size_t off_key, total; int max_chunks, max_parts; };
static LogprobWs logprob_ws(int n_rows, int vocab, int n_top) {
  LogprobWs w;
  w.max_chunks = std::max(1, (int)(((int64_t)vocab + lp::kChunk - 1) / lp::kChunk));
  w.max_parts = (w.max_chunks + lp::kWarps - 1) / lp::kWarps;
  w.off_key = (size_t)n_rows * w.max_parts * sizeof(float4);
  w.total = w.off_key + (n_top > 0 ? ((size_t)n_rows * w.max_chunks * 4 + 15) / 16 * 16 : 0);
  return w;
}

template <class T> static int launch_logprobs(LogprobArgs &a, cudaStream_t s) {
  logprob_sums_kernel<T><<<(unsigned)((int64_t)a.n_rows * a.parts), lp::kThreads, 0, s>>>(a);
  if (cudaGetLastError() != cudaSuccess) return SPKV_E_CUDA;
  return check_stream_error(launch_overlapped(logprob_rows_kernel<T>, dim3(a.n_rows), dim3(lp::kThreads), 0, s, a));
}

}  // namespace spkv

using namespace spkv;

extern "C" size_t spkv_logprobs_workspace_bytes(int32_t n_rows, int32_t vocab, int32_t n_top) {
  if (n_rows < 0 || vocab < 1 || n_top < 0 || n_top > SPKV_MAX_TOP) return 0;
  return std::max<size_t>(16, logprob_ws(n_rows, vocab, n_top).total);
}

extern "C" int spkv_token_logprobs(int32_t dtype, int32_t n_rows, int32_t vocab, const void *d_logits, int64_t row_stride,
                                   float scale, const int32_t *d_given, int32_t n_given, int32_t n_top, float *d_lse,
                                   float *d_entropy, float *d_logp, int32_t *d_top_ids, float *d_top_logp, void *d_workspace,
                                   size_t workspace_bytes, spkv_stream_t stream) {
  if (dtype < SPKV_BF16 || dtype > SPKV_F32 || n_rows < 0 || vocab < 1 || n_given < 0 || n_top < 0) return SPKV_E_INVALID;
  if (n_top > SPKV_MAX_TOP) return SPKV_E_UNSUPPORTED;
  if (!(scale > 0.f) || !isfinite(scale)) return SPKV_E_INVALID;
  if ((int64_t)n_rows * n_given > INT32_MAX || (int64_t)n_rows * n_top > INT32_MAX) return SPKV_E_UNSUPPORTED;
  if (vocab > INT32_MAX - 2 * lp::kChunk) return SPKV_E_UNSUPPORTED;
  if (n_rows == 0) return SPKV_OK;
  const int bytes = dtype == SPKV_F32 ? 4 : 2;
  if (!d_logits || ((uintptr_t)d_logits & (bytes - 1))) return SPKV_E_INVALID;
  if (!d_logp) n_given = 0;
  if (!d_top_ids && !d_top_logp) n_top = 0;
  if (n_given && !d_given) return SPKV_E_INVALID;
  const LogprobWs w = logprob_ws(n_rows, vocab, n_top);
  if (!d_workspace || ((uintptr_t)d_workspace & 15) || workspace_bytes < w.total) return SPKV_E_WORKSPACE;
  int dev = -1, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return SPKV_E_CUDA;
  LogprobArgs a = {};
  a.x = d_logits; a.stride = row_stride; a.n_rows = n_rows; a.vocab = vocab; a.n_given = n_given; a.n_top = n_top; a.scale = scale;
  a.given = d_given; a.lse = d_lse; a.entropy = d_entropy; a.logp = d_logp; a.top_ids = d_top_ids; a.top_logp = d_top_logp;
  a.part = static_cast<float4 *>(d_workspace);
  a.chunk_key = reinterpret_cast<uint32_t *>(static_cast<char *>(d_workspace) + w.off_key);
  a.max_chunks = w.max_chunks;
  // chunks a warp takes: one while there are fewer blocks than three fill the SMs, then up to kMaxRounds
  const int64_t blocks = (int64_t)n_rows * w.max_parts;
  a.rounds = (int)std::max<int64_t>(1, std::min<int64_t>(lp::kMaxRounds, blocks / ((int64_t)sms * lp::kBlocksPerSm * 3)));
  a.parts = (w.max_parts + a.rounds - 1) / a.rounds;
  if ((int64_t)n_rows * a.parts > INT32_MAX) return SPKV_E_UNSUPPORTED;
  note_cacheless_call();
  cudaStream_t s = as_stream(stream);
  return dtype == SPKV_BF16 ? launch_logprobs<__nv_bfloat16>(a, s) : dtype == SPKV_F16 ? launch_logprobs<__half>(a, s)
                                                                                     : launch_logprobs<float>(a, s);
}
