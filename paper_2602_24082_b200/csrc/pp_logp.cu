// Log-probabilities of the tokens of a packed batch from its logits, and the gradient of the logits.
//
// The packed row [x | y^1 | ... | y^K] (paper Sec. 3.2) stands for K sequences (x, y^k), so the row of
// logits that predicts a token is not always the one before it: a response's first token is
// predicted by the LAST PROMPT row, which all K responses share.  Row r predicts
//   r + 1                          inside a response,
//   the K responses' first tokens  at the end of a prompt,
//   nothing                        elsewhere (in a prompt before its end, at a response's end).
// With x = logits[r] / temperature, m = max x, l = log sum_v exp(x_v - m):
//   log p(y) = (x_y - m) - l
//   d logits[r][v] = sum_k g_k (1[v = y_k] - exp(x_v - m - l)) / temperature.
// Rows that predict nothing are not read; their gradient is zero.
//
// Both passes are bound by HBM: the forward reads a predicting row once, with the running maximum and sum of a
// softmax, the backward reads and writes it once.  9241 rows of 128256 bf16 columns, 4935 of which predict something:
// 1.27 GB in 195 us (6.5 TB/s, as a copy), the gradient 3.64 GB in 552 - 576 (6.6 - 6.3, from one B200 to another).
// What keeps the forward at the memory's rate is one exponential per element and little else: bf16 at 6.5 TB/s are
// 11.7 elements per clock and SM, of 16 that the special function unit makes (measured busy for 79 %).  The
// exponential is 2^(c x - K), c = log2(e) / temperature, with a whole number K for reference: K is exact in fp32, so
// nothing of c x is lost to the rounding of a reference (c m rounded would be off by 2^-24 |c m|, the same for the
// whole row), and sums of different references are joined by exact powers of two.  K comes from a thread's first
// elements and stays unless one is 2^8 times as large: a new reference with every new maximum was a branch that some
// lane of a warp took in nearly every step (with it, and a look at the row's end for every vector, 128 instead of 105
// million instructions; under the power limit of a long run, at 1.7 GHz, 219 us instead of 210).  An exponent of up to
// 8 is rounded to 2^-22; up to 64 it was 2^-19, which of a certain token's log-probability is the whole, and no faster
// (195 us and 210, both).  A thread has four 16-byte vectors on their way while it sums up four (without that 252 us).
// Rows whose values are beyond +-2^19 (a mask of the type's lowest value over everything, say)
// go through a second pass over exp(x - m).
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "pp_seg.cuh"

namespace pp {
namespace {

constexpr float kFar = 524288.f;   // |c m| up to which ceil(c m) is at most 1 above c m
constexpr float kFarOther = 512.f;  // the same in the gradient of fp32 logits at a temperature
constexpr int kMostK = 1 << 20;
constexpr float kSlack = 8.f;      // powers up to 2^8 are summed up: 2^38 with the longest row
constexpr int kOwn = 4;            // columns of a lane whose gradients it adds up at a time
constexpr float kLn2 = 0.693147180559945309f;
constexpr double kLog2e = 1.4426950408889634074;

struct LogpArgs {
  const int32_t* header;
  const int32_t* seg_start;
  const int32_t* key_end;
  int nseg, T;
  const void* logits;
  long long row_stride;   // elements
  int V;
  const void* ids;
  int ids_64;
  float temperature, c;   // c = log2(e) / temperature
};

// ---------------------------------------------------------------- 16 bytes of a row
template <typename X> struct Row;
template <> struct Row<__nv_bfloat16> {
  static constexpr int kN = 8;
  static constexpr uint32_t kLeast = 0xff80ff80u;   // -inf, twice
  static __device__ __forceinline__ float one(const __nv_bfloat16& x) { return __bfloat162float(x); }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
  static __device__ __forceinline__ float round(float x) { return __bfloat162float(__float2bfloat16_rn(x)); }
  static __device__ __forceinline__ void pair(uint32_t w, float& a, float& b) {
    a = __uint_as_float(w << 16);
    b = __uint_as_float(w & 0xffff0000u);
  }
  static __device__ __forceinline__ uint32_t word(float a, float b) { return pack_bf16(a, b); }
  static __device__ __forceinline__ uint32_t max_word(uint32_t a, uint32_t b) {
    const __nv_bfloat162 r = __hmax2(reinterpret_cast<__nv_bfloat162&>(a), reinterpret_cast<__nv_bfloat162&>(b));
    return reinterpret_cast<const uint32_t&>(r);
  }
  static __device__ __forceinline__ float max_of(uint32_t w) {
    float a, b;
    pair(w, a, b);
    return fmaxf(a, b);
  }
};
template <> struct Row<__half> {
  static constexpr int kN = 8;
  static constexpr uint32_t kLeast = 0xfc00fc00u;
  static __device__ __forceinline__ float one(const __half& x) { return __half2float(x); }
  static __device__ __forceinline__ void store(__half* p, float x) { *p = __float2half_rn(x); }
  static __device__ __forceinline__ float round(float x) { return __half2float(__float2half_rn(x)); }
  static __device__ __forceinline__ void pair(uint32_t w, float& a, float& b) {
    const float2 f = __half22float2(reinterpret_cast<const __half2&>(w));
    a = f.x;
    b = f.y;
  }
  static __device__ __forceinline__ uint32_t word(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return reinterpret_cast<const uint32_t&>(h);
  }
  static __device__ __forceinline__ uint32_t max_word(uint32_t a, uint32_t b) {
    const __half2 r = __hmax2(reinterpret_cast<__half2&>(a), reinterpret_cast<__half2&>(b));
    return reinterpret_cast<const uint32_t&>(r);
  }
  static __device__ __forceinline__ float max_of(uint32_t w) {
    float a, b;
    pair(w, a, b);
    return fmaxf(a, b);
  }
};
template <> struct Row<float> {
  static constexpr int kN = 4;
  static constexpr uint32_t kLeast = 0xff800000u;
  static __device__ __forceinline__ float one(const float& x) { return x; }
  static __device__ __forceinline__ void store(float* p, float x) { *p = x; }
  static __device__ __forceinline__ uint32_t max_word(uint32_t a, uint32_t b) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  }
  static __device__ __forceinline__ float max_of(uint32_t w) { return __uint_as_float(w); }
};
// f(a, b) over a vector's elements by twos
template <typename X, typename F>
__device__ __forceinline__ void for_pairs(const uint4& v, F f) {
  if constexpr (Row<X>::kN == 8) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a, b;
      Row<X>::pair(w[i], a, b);
      f(a, b);
    }
  } else {
    f(__uint_as_float(v.x), __uint_as_float(v.y));
    f(__uint_as_float(v.z), __uint_as_float(v.w));
  }
}
// a row passes through once and by far exceeds L1
__device__ __forceinline__ uint4 load_row(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p)
               : "memory");
  return v;
}

// ---------------------------------------------------------------- what a row predicts
struct Predicts {
  int r;         // the row
  int n;         // tokens; 0 = nothing
  int seg;       // n == 1: token r + 1.  Otherwise the responses' first tokens: starts of segments seg + 1 .. seg + n
  int id;        // n == 1: the token's id, -1 for any negative one and INT_MAX for any beyond
  bool prompt;
};
__device__ __forceinline__ int id_of(const LogpArgs& p, int t) {
  if (!p.ids_64) return static_cast<const int32_t*>(p.ids)[t];
  const long long y = static_cast<const long long*>(p.ids)[t];
  return y < 0 ? -1 : y > INT_MAX ? INT_MAX : int(y);
}
// (By a whole warp.  The loads are few and mostly side by side: in small calls, and for short rows, this chain is what
// counts.  A plan that was refused leaves searches that end, on whatever its tables hold.)
__device__ __forceinline__ Predicts predicts_of(const LogpArgs& p, int r, bool& fine) {
  const int status = p.header[0], seen = p.key_end[r];   // seen: where the keys of a prompt's tokens, or of a response's, end
  Predicts u;
  u.r = r;
  u.id = id_of(p, min(r + 1, p.T - 1));
  u.seg = warp_upper(p.seg_start, p.nseg, r);
  // where the next segments start: this one's end, and perhaps the group's
  const int start = p.seg_start[min(u.seg + 1 + int(threadIdx.x & 31), p.nseg)];
  const int e = __shfl_sync(0xffffffffu, start, 0);
  fine = status == kStatusOk;
  u.prompt = seen > e;   // (behind the group)
  u.n = 0;
  if (!fine) return u;
  if (!u.prompt) {
    u.n = r + 1 < e;
  } else if (r + 1 == e) {   // as many as there are segments up to the group's end
    const unsigned at = __ballot_sync(0xffffffffu, start == seen);
    u.n = at ? __ffs(at) - 1 : warp_upper(p.seg_start, p.nseg, seen - 1) - u.seg;
  }
  return u;
}
__device__ __forceinline__ int token_of(const LogpArgs& p, const Predicts& u, int k) {
  return u.n == 1 ? u.r + 1 : p.seg_start[u.seg + 1 + k];
}

// The part of a row that 2^lg_parts blocks share: vectors [v0, v1) from the first boundary of kAlign bytes on; the
// `edge` elements before it and the `tail` ones behind the last whole vector go to the first block and the last.
struct Span {
  int head, v0, v1, tail0;   // elements in front; vectors; first element behind the vectors
  int edge, tail;
};
template <int kAlign, typename X>
__device__ __forceinline__ Span span_of(const X* row, int V, int part, int lg_parts) {
  constexpr int kN = Row<X>::kN;
  Span s;
  s.head = min(V, int(((kAlign - (reinterpret_cast<uintptr_t>(row) & (kAlign - 1))) & (kAlign - 1)) / sizeof(X)));
  const int nv = (V - s.head) / kN, per = (nv + (1 << lg_parts) - 1) >> lg_parts;
  s.v0 = min(nv, part * per);
  s.v1 = min(nv, s.v0 + per);
  s.tail0 = s.head + nv * kN;
  s.edge = part == 0 ? s.head : 0;
  s.tail = part + 1 == 1 << lg_parts ? V - s.tail0 : 0;
  return s;
}

// Running maximum and sum of 2^(c x - K), K a whole number.
struct Running {
  float m = -INFINITY, s = 0.f;
  int K = -kMostK;
};
// K of a maximum m; where that is beyond +-2^20, the row goes through the second pass anyway
__device__ __forceinline__ int whole(float cm) { return int(fminf(fmaxf(ceilf(cm), float(-kMostK)), float(kMostK))); }
__device__ __forceinline__ float power(int from, int to) {   // 2^(from - to), from <= to: exact, and 0 far below
  return __int_as_float(max(127 + from - to, 0) << 23);
}
__device__ __forceinline__ float power2(int n) {   // 2^n, |n| < 127
  return __int_as_float((127 + n) << 23);
}
// floats in the order of signed whole numbers, and back
__device__ __forceinline__ int ordered(float x) {
  const int i = __float_as_int(x);
  return i ^ ((i >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float from_ordered(int i) { return __int_as_float(i ^ ((i >> 31) & 0x7fffffff)); }
template <int kWarps>
__device__ __forceinline__ void row_sync() {
  if constexpr (kWarps == 1) __syncwarp(); else __syncthreads();
}
// over the first kLanes lanes of a warp; all get the result
template <int kLanes>
__device__ __forceinline__ Running join_lanes(Running a) {
  const int K = __reduce_max_sync(0xffffffffu, a.K);
  a.s *= power(a.K, K);
  a.K = K;
  a.m = from_ordered(__reduce_max_sync(0xffffffffu, ordered(a.m)));
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
  return a;
}

// the maximum of a row's threads; after it, all of them have come here
template <int kWarps>
__device__ __forceinline__ float row_max(float m) {
  int top = __reduce_max_sync(0xffffffffu, ordered(m));
  if constexpr (kWarps > 1) {
    __shared__ int warp_top[kWarps];
    if ((threadIdx.x & 31) == 0) warp_top[threadIdx.x >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) top = max(top, warp_top[w]);
  } else {
    __syncwarp();
  }
  return from_ordered(top);
}

struct JoinSpace {
  Running warp[8], part[8];
};
// All threads of the row get the whole row's values.
template <int kWarps>
__device__ __forceinline__ Running join_row(Running a, JoinSpace* space, int parts, bool first) {
  a = join_lanes<32>(a);
  if constexpr (kWarps > 1) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (lane == 0) space->warp[warp] = a;
    __syncthreads();
    a = lane < kWarps ? space->warp[lane] : Running();
    a = join_lanes<32>(a);
    if (parts > 1) {
      auto cluster = cooperative_groups::this_cluster();
      if (first) cluster.barrier_wait();   // (all blocks have started: their arrival is before the row's loads)
      if (warp == 0 && lane < parts) *cluster.map_shared_rank(&space->part[cluster.block_rank()], lane) = a;
      cluster.sync();
      a = lane < parts ? space->part[lane] : Running();
      a = join_lanes<32>(a);
    }
  }
  return a;
}

constexpr int kMaxLgParts = 3;
template <int kWarps> constexpr int block_threads() { return kWarps == 1 ? 128 : kWarps * 32; }
template <int kWarps, int kUnroll> constexpr int blocks_per_sm() { return kWarps > 1 ? 32 / kWarps : kUnroll > 2 ? 8 : 12; }
// A row's team: a warp (four to a block), a block, or a cluster of 2^lg_parts blocks.
template <int kWarps> __device__ __forceinline__ int team_of(int lg_parts) {
  return kWarps == 1 ? blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x >> lg_parts;
}

// Whether one of a row's tokens counts; the log-probabilities and statistics of a row that is not read.
__device__ __forceinline__ bool row_used(const LogpArgs& p, const Predicts& u, bool writes, float* logp, float2* stats) {
  const int lane = threadIdx.x & 31;
  if (u.prompt && writes && lane == 0) logp[u.r] = 0.f;
  bool any = u.n == 1 && u.id >= 0;
  if (u.n > 1) {
    for (int k = lane; k < u.n; k += 32) any |= id_of(p, token_of(p, u, k)) >= 0;
    any = __any_sync(0xffffffffu, any);
  }
  if (!any && writes) {
    if (lane == 0) stats[u.r] = make_float2(0.f, 0.f);
    for (int k = lane; k < u.n; k += 32) logp[token_of(p, u, k)] = 0.f;
  }
  return any;
}

template <typename X, int kWarps, int kUnroll>
__device__ __forceinline__ void token_logp_row(const LogpArgs& p, const Predicts& u, int part, int lg_parts,
                                               JoinSpace* space, float* logp, float2* stats) {
  constexpr int kN = Row<X>::kN, kThreads = kWarps * 32, kStep = kUnroll * kThreads;
  const int tid = kWarps == 1 ? threadIdx.x & 31 : threadIdx.x;
  const X* row = static_cast<const X*>(p.logits) + (long long)u.r * p.row_stride;
  const Span sp = span_of<16>(row, p.V, part, lg_parts);
  const uint4* vec = reinterpret_cast<const uint4*>(row + sp.head);
  const float c = p.c;
  const uint64_t c2 = pack2(c, c);
  uint4 va[kUnroll], vb[kUnroll];
  auto load = [&](uint4 (&v)[kUnroll], int at) {
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
      v[i] = make_uint4(Row<X>::kLeast, Row<X>::kLeast, Row<X>::kLeast, Row<X>::kLeast);
      if (at + i * kThreads < sp.v1) v[i] = load_row(vec + at + i * kThreads);
    }
  };
  load(va, sp.v0 + tid);
  // the first tokens' own logits
  float own = 0.f;
  if (part == 0 && tid < u.n) {
    const int y = u.n == 1 ? u.id : id_of(p, token_of(p, u, tid));
    if (y >= 0 && y < p.V) own = Row<X>::one(row[y]);
  }
  Running run;
  uint64_t sum = pack2(0.f, 0.f);
  float k = float(kMostK);   // -K
  auto raise = [&](float bm) {
    run.m = fmaxf(run.m, bm);
    if (fmaf(bm, c, k) > kSlack) {
      const int K = whole(bm * c);
      const float f = power(run.K, K);
      sum = mul2(sum, pack2(f, f));
      run.K = K;
      k = -float(K);
    }
  };
  auto take = [&](const uint4 (&v)[kUnroll], int n) {   // (n: vectors that some thread has)
    uint32_t w = Row<X>::max_word(Row<X>::max_word(v[0].x, v[0].y), Row<X>::max_word(v[0].z, v[0].w));
#pragma unroll
    for (int i = 1; i < kUnroll; ++i)
      if (kWarps > 1 || i < n)
        w = Row<X>::max_word(w, Row<X>::max_word(Row<X>::max_word(v[i].x, v[i].y), Row<X>::max_word(v[i].z, v[i].w)));
    raise(Row<X>::max_of(w));
    const uint64_t k2 = pack2(k, k);
#pragma unroll
    for (int i = 0; i < kUnroll; ++i)
      if (kWarps > 1 || i < n)
        for_pairs<X>(v[i], [&](float a, float b) {
          float y, z;
          unpack2(fma2(pack2(a, b), c2, k2), y, z);
          sum = add2(sum, pack2(ex2(y), ex2(z)));
        });
  };
  // elements in front of the first boundary and behind the last, one per thread
  for (int i = tid; i < sp.edge + sp.tail; i += kThreads) {
    const float x = Row<X>::one(row[i < sp.edge ? i : sp.tail0 + i - sp.edge]);
    raise(x);
    sum = add2(sum, pack2(ex2(fmaf(x, c, k)), 0.f));
  }
  // one batch of vectors is on its way while the one before it is summed up; of a long row, while there are whole
  // ones, without a look at where it ends
  int at = sp.v0;
  if constexpr (kWarps > 1) {
    auto load_whole = [&](uint4 (&v)[kUnroll], int at) {
#pragma unroll
      for (int i = 0; i < kUnroll; ++i) v[i] = load_row(vec + at + i * kThreads);
    };
    for (; at + 3 * kStep <= sp.v1; at += 2 * kStep) {
      load_whole(vb, at + tid + kStep);
      take(va, kUnroll);
      load_whole(va, at + tid + 2 * kStep);
      take(vb, kUnroll);
    }
  }
  for (; at < sp.v1; at += 2 * kStep) {
    load(vb, at + tid + kStep);
    take(va, (sp.v1 - at + kThreads - 1) / kThreads);
    load(va, at + tid + 2 * kStep);
    if (at + kStep < sp.v1) take(vb, (sp.v1 - at - kStep + kThreads - 1) / kThreads);
  }
  float lo, hi;
  unpack2(sum, lo, hi);
  run.s = lo + hi;
  run = join_row<kWarps>(run, &space[0], 1 << lg_parts, true);
  float l;
  if (fabsf(run.m * c) < kFar) {
    const int K = whole(run.m * c);
    l = fmaf(fmaf(run.m, -c, float(K)), kLn2, logf(run.s * power2(run.K - K)));
  } else {
    // the whole row is far from zero (or infinite): once more, relative to the maximum
    Running far;
    far.K = 0;
    const int first = sp.head + sp.v0 * kN, n = (sp.v1 - sp.v0) * kN;
    for (int i = tid; i < n + sp.edge + sp.tail; i += kThreads) {
      const int e = i < sp.edge ? i : i - sp.edge < n ? first + i - sp.edge : sp.tail0 + i - sp.edge - n;
      far.s += exp2f((Row<X>::one(row[e]) - run.m) * c);
    }
    l = logf(join_row<kWarps>(far, &space[1], 1 << lg_parts, false).s);
  }
  if (l < 0.f) l = 0.f;   // (the maximum is one of the terms)
  if (part == 0) {
    if (tid == 0) stats[u.r] = make_float2(run.m / p.temperature, l);
    for (int k = tid; k < u.n; k += kThreads) {
      const int t = token_of(p, u, k);
      const int y = u.n == 1 ? u.id : id_of(p, t);
      logp[t] = y < 0 ? 0.f : y >= p.V ? NAN : ((k < kThreads ? own : Row<X>::one(row[y])) - run.m) / p.temperature - l;
    }
  }
}

// `rows`: what a block of eight warps looks over at once (with lg_parts == 0).
template <typename X, int kWarps, int kUnroll>
__global__ void __launch_bounds__(block_threads<kWarps>(), blocks_per_sm<kWarps, kUnroll>())
token_logp_kernel(LogpArgs p, int lg_parts, int rows, float* logp, float2* stats) {
  __shared__ JoinSpace space[2];
  __shared__ Predicts found[kWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int part = kWarps == 1 ? 0 : blockIdx.x & ((1 << lg_parts) - 1), r = team_of<kWarps>(lg_parts);
  if (kWarps == 1 && r >= p.T) return;
  dependency_wait();
  bool fine;
  if (kWarps < 8 || rows == 1) {
    const Predicts u = predicts_of(p, r, fine);
    if (!fine || !row_used(p, u, part == 0 && (kWarps == 1 || warp == 0), logp, stats)) return;
    if (kWarps > 1 && lg_parts) cooperative_groups::this_cluster().barrier_arrive();
    token_logp_row<X, kWarps, kUnroll>(p, u, part, kWarps == 1 ? 0 : lg_parts, space, logp, stats);
    return;
  }
  // a warp looks over a row, then the block takes those that predict something
  const long long mine = r + (long long)warp * gridDim.x;   // (of neighbours mostly all predict something or none)
  if (warp < rows) {
    Predicts u;
    u.n = 0;
    if (mine < p.T) {
      u = predicts_of(p, int(mine), fine);
      if (!fine || !row_used(p, u, true, logp, stats)) u.n = 0;
    }
    if (lane == 0) found[warp] = u;
  }
  __syncthreads();
  for (int i = 0; i < rows; ++i) {
    const Predicts u = found[i];
    if (!u.n) continue;
    token_logp_row<X, kWarps, kUnroll>(p, u, 0, 0, space, logp, stats);
    __syncthreads();   // (the space of the sums is used again)
  }
}

// ---------------------------------------------------------------- backward
struct LogpBwdArgs {
  const float* logp;
  const float2* stats;
  const float* grad;
  void* d_logits;
  long long d_stride;
};

// of a token's own column, from its log-probability: 1 - p without cancellation.  same: sum of the gradients of the
// tokens with its id, rest: of the others
__device__ __forceinline__ float own_gradient(const LogpArgs& p, float same, float rest, float lp) {
  return (-same * expm1f(lp) - rest * expf(lp)) / p.temperature;
}

// The own columns [first, last) of many responses' first tokens, by a row's team.  A look at all the others by each token
// would take the square of their number (8192 responses of 1000 columns: 99 ms and more, here 1.3); instead
// every warp goes over them once for each range of its columns, four to a lane, and adds their gradients up in their order.
template <typename X, int kWarps>
__device__ __forceinline__ void own_columns_of_many(const LogpArgs& p, const LogpBwdArgs& b, const Predicts& u, X* out,
                                                 int first, int last, double total) {
  constexpr int kUnroll = 4;
  const int lane = threadIdx.x & 31, warp = kWarps == 1 ? 0 : threadIdx.x >> 5;
  for (int from = first + warp * 32 * kOwn; from < last; from += kWarps * 32 * kOwn) {
    double sum[kOwn];
    float lp[kOwn];
    bool mine[kOwn];
#pragma unroll
    for (int c = 0; c < kOwn; ++c) {
      sum[c] = 0;
      mine[c] = false;
    }
    for (int k0 = 0; k0 < u.n; k0 += 32 * kUnroll) {
      int t[kUnroll], y[kUnroll];
#pragma unroll
      for (int i = 0; i < kUnroll; ++i) t[i] = token_of(p, u, min(k0 + 32 * i + lane, u.n - 1));
#pragma unroll
      for (int i = 0; i < kUnroll; ++i) y[i] = id_of(p, t[i]);
#pragma unroll
      for (int i = 0; i < kUnroll; ++i) {
        const bool in = k0 + 32 * i + lane < u.n && y[i] >= from && y[i] < last && y[i] - from < 32 * kOwn;
        const float g = in ? b.grad[t[i]] : 0.f, l = in ? b.logp[t[i]] : 0.f;
        for (unsigned at = __ballot_sync(0xffffffffu, in); at; at &= at - 1) {
          const int src = __ffs(at) - 1, column = __shfl_sync(0xffffffffu, y[i], src) - from;
          const float add = __shfl_sync(0xffffffffu, g, src), of = __shfl_sync(0xffffffffu, l, src);
#pragma unroll
          for (int c = 0; c < kOwn; ++c) {
            if (column != 32 * c + lane) continue;
            sum[c] += add;
            lp[c] = of;
            mine[c] = true;
          }
        }
      }
    }
#pragma unroll
    for (int c = 0; c < kOwn; ++c)
      if (mine[c]) Row<X>::store(out + from + 32 * c + lane, own_gradient(p, float(sum[c]), float(total - sum[c]), lp[c]));
  }
}

// kVec: rows of logits and of the gradient lie alike to 16 bytes.
template <typename X, int kWarps, bool kVec>
__global__ void __launch_bounds__(block_threads<kWarps>(), kWarps == 1 ? 10 : blocks_per_sm<kWarps, 4>())
token_logp_bwd_kernel(LogpArgs p, LogpBwdArgs b, int lg_parts) {
  constexpr int kN = Row<X>::kN, kThreads = kWarps * 32, kUnroll = 4, kStep = kUnroll * kThreads;
  if (kWarps == 1) lg_parts = 0;
  const int tid = kWarps == 1 ? threadIdx.x & 31 : threadIdx.x, lane = threadIdx.x & 31;
  const int part = blockIdx.x & ((1 << lg_parts) - 1), r = team_of<kWarps>(lg_parts);
  if (r >= p.T) return;
  dependency_wait();
  const float next = b.grad[min(r + 1, p.T - 1)], next_logp = b.logp[min(r + 1, p.T - 1)];
  const float2 st = b.stats[r];
  bool fine;
  const Predicts u = predicts_of(p, r, fine);
  if (!fine) return;
  // the sum of the gradients of the tokens that the row predicts
  double total = 0;
  bool any = false;
  if (u.n == 1) {
    if (u.id >= 0) {
      total = next;
      any = next != 0.f;
    }
  } else if (u.n > 1) {
    for (int k = lane; k < u.n; k += 32) {
      const int t = token_of(p, u, k);
      if (id_of(p, t) >= 0) {
        const float g = b.grad[t];
        any |= g != 0.f;
        total += g;
      }
    }
    any = __any_sync(0xffffffffu, any);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  }

  const X* row = static_cast<const X*>(p.logits) + (long long)r * p.row_stride;
  X* out = static_cast<X*>(b.d_logits) + (long long)r * b.d_stride;
  Span sp = span_of<128>(out, p.V, part, lg_parts);
  uint4* dst = reinterpret_cast<uint4*>(out + sp.head);
  if (!any) {
    for (int i = tid; i < sp.edge + sp.tail; i += kThreads)
      Row<X>::store(out + (i < sp.edge ? i : sp.tail0 + i - sp.edge), 0.f);
    for (int at = sp.v0 + tid; at < sp.v1; at += kThreads) dst[at] = make_uint4(0, 0, 0, 0);
    return;
  }
  // p_v = 2^(c x_v - K) 2^-f with K + f = c m + l log2(e) (m as it was before the temperature, c as it is in fp32),
  // K whole: 2^-f goes into the row's factor.  row_stats hold m / temperature, rounded to fp32.  That times the temperature
  // is within 2^-23 of m, which rounded to 16 bits is m itself, and m without a temperature.  Of other fp32
  // rows all probabilities have a factor of up to 1 + 2^-24 |m| / temperature, so that they pass for far ones early.
  double m_of = double(st.x) * double(p.temperature), near = kFar;
  if constexpr (sizeof(X) == 2) m_of = Row<X>::round(float(m_of));
  else if (p.temperature != 1.f) near = kFarOther;
  const double lse2 = m_of * double(p.c) + double(st.y) * kLog2e;
  const double whole = rint(lse2);
  const bool far = !(fabs(lse2) < near);
  const float scale = -float(total) / p.temperature, c = p.c;
  const uint4* vec = reinterpret_cast<const uint4*>(row + sp.head);
  // the gradient as `one` has it of an element
  auto write = [&](auto one) {
    for (int i = tid; i < sp.edge + sp.tail; i += kThreads) {
      const int e = i < sp.edge ? i : sp.tail0 + i - sp.edge;
      Row<X>::store(out + e, one(Row<X>::one(row[e])));
    }
    if (!kVec) {
      for (int e = sp.head + sp.v0 * kN + tid; e < sp.head + sp.v1 * kN; e += kThreads)
        Row<X>::store(out + e, one(Row<X>::one(row[e])));
      return;
    }
    auto take = [&](uint4 v) {
      uint32_t w[4];
      int i = 0;
      for_pairs<X>(v, [&](float x, float y) {
        x = one(x);
        y = one(y);
        if constexpr (kN == 8) {
          w[i++] = Row<X>::word(x, y);
        } else {
          w[i++] = __float_as_uint(x);
          w[i++] = __float_as_uint(y);
        }
      });
      return make_uint4(w[0], w[1], w[2], w[3]);
    };
    for (int at = sp.v0 + tid; at < sp.v1; at += kStep) {
      uint4 v[kUnroll];
#pragma unroll
      for (int i = 0; i < kUnroll; ++i)
        if (at + i * kThreads < sp.v1) v[i] = load_row(vec + at + i * kThreads);
#pragma unroll
      for (int i = 0; i < kUnroll; ++i)
        if (at + i * kThreads < sp.v1) dst[at + i * kThreads] = take(v[i]);
    }
  };
  if (!far) {
    const float coef = scale * exp2f(float(whole - lse2)), K = float(whole);
    write([&](float x) { return ex2(fmaf(x, c, -K)) * coef; });
  } else {
    // Far from zero c x loses its digits, and m / temperature itself may have passed fp32's range, so that
    // row_stats do not tell m: it is read again, and everything is relative to it as in the forward.  By one block
    // for the whole row: in place, other blocks would find theirs overwritten.  (3001 rows of 50257 fp32 around
    // 1000 at a temperature of 0.7: 221 us, around 0 167; 24 of 140000 42 and 13)
    if (part > 0) return;
    lg_parts = 0;
    sp = span_of<128>(out, p.V, 0, 0);
    float m = -INFINITY;   // (with a NaN, or no finite maximum, l is one)
    for (int e = tid; e < p.V; e += kThreads) m = fmaxf(m, Row<X>::one(row[e]));
    m = row_max<kWarps>(m);
    const float coef = scale * expf(-st.y);
    write([&](float x) { return ex2((x - m) * c) * coef; });
  }
  // the tokens' own columns.  The same id may be that of several responses: each writes the sum over all of them
  row_sync<kWarps>();
  const int first = part == 0 ? 0 : sp.head + sp.v0 * kN;
  const int last = part + 1 == 1 << lg_parts ? p.V : sp.head + sp.v1 * kN;
  // (us, looks at each other and ranges: 256 responses of 300 columns 21 and 14, of 32000 20 and 46; 1024 of 32000 186 and
  // 162, of 128256 248 and 191; 2048 of 1000 4384 and 269)
  if (u.n > 128 && 8 * ((u.n + kThreads - 1) / kThreads) > (last - first) / (kWarps * 32 * kOwn)) {
    own_columns_of_many<X, kWarps>(p, b, u, out, first, last, total);
    return;
  }
  for (int k = tid; k < u.n; k += kThreads) {
    const int t = token_of(p, u, k);
    const int y = u.n == 1 ? u.id : id_of(p, t);
    if (y < first || y >= last) continue;
    float same = float(total), rest = 0.f, lp = next_logp;
    if (u.n > 1) {
      double sum = 0;
      for (int j = 0; j < u.n; ++j) {
        const int tj = token_of(p, u, j);
        if (id_of(p, tj) == y) sum += b.grad[tj];
      }
      same = float(sum);
      rest = float(total - sum);
      lp = b.logp[t];
    }
    Row<X>::store(out + y, own_gradient(p, same, rest, lp));
  }
}

LogpArgs logp_args(const pp_plan* plan, const void* logits, long long row_stride, int V, const void* ids, int ids_64,
                   float temperature) {
  LogpArgs a;
  a.header = reinterpret_cast<const int32_t*>(plan->ws + plan->lay.header);
  a.seg_start = reinterpret_cast<const int32_t*>(plan->ws + plan->lay.seg_start);
  a.key_end = reinterpret_cast<const int32_t*>(plan->ws + plan->lay.key_end);
  a.nseg = plan->nseg;
  a.T = plan->prob.total_tokens;
  a.logits = logits;
  a.row_stride = row_stride;
  a.V = V;
  a.ids = ids;
  a.ids_64 = ids_64;
  a.temperature = temperature;
  a.c = float(kLog2e / double(temperature));
  return a;
}

// How the rows are dealt out: warps of a row's team, blocks that share a row, rows that a block looks over,
// vectors of a thread that are on their way at a time.  us on one B200, bf16, by T rows of V columns, half of which predict
// something where it is not said otherwise:
//  - a warp where there are rows enough: V 600, T 60000 26 (4 warps 106); 12000, 20000 45 and 56; 25000, 20000 85 and 91;
//    but 25000, 6000 41 and 32; 3001, 700 5.1 and 4.3.  Two vectors at a time of many short rows: 600, 60000 26 (four:
//    30), but 1500, 6000 7.2 and 6.7, 12000, 20000 49 and 45.
//  - 4 warps, then 8: 25000, 6000 32 (8 warps 41); 60000, 6000 61 and 64, with one row in nine 26 and 27; 25000, 700 8.8 and
//    8.5; fp32, 50257, 3001 57 and 55.  Backward 12000, 2000 16 and 17; 25000, 6000 76 and 77, with one in nine 61 and 57.
//  - forward, blocks that share a long row, where rows are few: 140000, 60 16 (8 warps), 10 (two blocks), 7.9 (four);
//    60000, 60 7.0, 6.2 and 6.0; 140000, 700 27, 24 and 28; but 60000, 700 14.5, 15 and 19: clusters start slowly, those of
//    rows that predict nothing too.
//  - backward, parts of 64 to 112 KB: 128256, 9241 573 (one), 567 (two), 555 (four); smaller ones where rows are
//    few: 140000, 60 35 (one), 13 (four), 8.1 (eight); 12000, 200 5.2, 4.5 (two) and 4.3 (four).
//  - forward, rows that a block looks over, with sixteen waves of blocks or more: 128256, 65536, one in nine 378 (one),
//    306 (eight); 20000, one in nine 116 and 97; but 140000, 2000, half 49 (one) and 55 (two).
struct RowShape {
  int warps, lg_parts, rows, unroll;
};
RowShape row_shape(const pp_plan* plan, size_t row_bytes, int num_sms, bool fwd) {
  const long long T = plan->prob.total_tokens, sms = num_sms;
  RowShape s{8, 0, 1, 4};
  const size_t one_warp = fwd ? (T > 64 * sms ? 65536 : T > 32 * sms ? 16384 : T > 8 * sms ? 8192 : 0)
                              : (T > 32 * sms ? 16384 : T > 8 * sms ? 2048 : 0);
  if (row_bytes <= one_warp) {
    s.warps = 1;
    if (row_bytes <= 8192 && T > 64 * sms) s.unroll = 2;
    return s;
  }
  if (fwd) {
    if (row_bytes <= (T > 32 * sms ? 131072 : T > 8 * sms ? 65536 : 32768)) {
      s.warps = 4;
    } else {
      auto share = [&](int lg) {
        const size_t part = row_bytes >> lg;
        return (T << lg) <= (part >= 122880 ? 10 : part >= 49152 ? 7 : part >= 14336 && row_bytes >= 98304 ? 3 : 0) * sms;
      };
      while (s.lg_parts < kMaxLgParts && share(s.lg_parts + 1)) ++s.lg_parts;
      // rows that predict something: all but the last of a response, and one of a prompt
      const long long used = plan->resp_tokens - plan->prob.num_responses + plan->prob.num_groups, waves = T / (4 * sms);
      if (waves >= 16) s.rows = int(std::min(8ll, std::max(waves / 16, plan->resp_tokens ? T / std::max(used, 1ll) : 1)));
    }
  } else {
    if (row_bytes <= (T > 8 * sms ? 32768 : 2 * T > 3 * sms ? 8192 : 0)) {
      s.warps = 4;
    } else {
      auto share = [&](int lg) {
        const size_t part = row_bytes >> lg;
        return row_bytes >> (lg - 1) > 114688 || (T << lg) <= (part >= 8192 ? 6 : part >= 2048 ? 3 : 0) * sms;
      };
      while (s.lg_parts < kMaxLgParts && share(s.lg_parts + 1)) ++s.lg_parts;
    }
  }
  return s;
}
dim3 blocks_of(int T, RowShape s) {
  const int rows = s.warps == 1 ? 4 : s.rows;
  return dim3(unsigned((T + rows - 1ll) / rows) << s.lg_parts);
}
dim3 threads_of(RowShape s) { return dim3(s.warps == 1 ? 128 : s.warps * 32); }

template <typename X>
cudaError_t launch_fwd_of(const LogpArgs& a, RowShape s, float* logp, float2* stats, cudaStream_t stream) {
  auto kernel = s.warps == 8    ? token_logp_kernel<X, 8, 4>
                : s.warps == 4  ? token_logp_kernel<X, 4, 4>
                : s.unroll == 4 ? token_logp_kernel<X, 1, 4>
                                : token_logp_kernel<X, 1, 2>;
  return launch_clusters(1 << s.lg_parts, kernel, blocks_of(a.T, s), threads_of(s), 0, stream, a, s.lg_parts, s.rows,
                         logp, stats);
}

template <typename X, bool kVec>
cudaError_t launch_bwd_of(const LogpArgs& a, RowShape s, const LogpBwdArgs& b, cudaStream_t stream) {
  auto kernel = s.warps == 8   ? token_logp_bwd_kernel<X, 8, kVec>
                : s.warps == 4 ? token_logp_bwd_kernel<X, 4, kVec>
                               : token_logp_bwd_kernel<X, 1, kVec>;
  return launch_kernel(true, kernel, blocks_of(a.T, s), threads_of(s), 0, stream, a, b, s.lg_parts);
}

size_t size_of(int type) { return type == PP_FP32 ? 4 : 2; }

}  // namespace

cudaError_t launch_token_logp(const pp_plan* plan, const void* logits, int type, long long row_stride, int V,
                              const void* ids, int ids_64, float temperature, float* logp, float* stats,
                              cudaStream_t stream) {
  static DeviceSetup setup[kMaxDevices];
  const DeviceSetup* dev = device_setup(setup);
  if (!dev) return cudaErrorInvalidDevice;
  const LogpArgs a = logp_args(plan, logits, row_stride, V, ids, ids_64, temperature);
  const RowShape s = row_shape(plan, size_t(V) * size_of(type), dev->num_sms, true);
  float2* st = reinterpret_cast<float2*>(stats);
  return type == PP_BF16   ? launch_fwd_of<__nv_bfloat16>(a, s, logp, st, stream)
         : type == PP_FP16 ? launch_fwd_of<__half>(a, s, logp, st, stream)
                           : launch_fwd_of<float>(a, s, logp, st, stream);
}

cudaError_t launch_token_logp_bwd(const pp_plan* plan, const void* logits, int type, long long row_stride, int V,
                                  const void* ids, int ids_64, float temperature, const float* logp,
                                  const float* stats, const float* grad, void* d_logits, long long d_stride,
                                  cudaStream_t stream) {
  static DeviceSetup setup[kMaxDevices];
  const DeviceSetup* dev = device_setup(setup);
  if (!dev) return cudaErrorInvalidDevice;
  const LogpArgs a = logp_args(plan, logits, row_stride, V, ids, ids_64, temperature);
  const LogpBwdArgs b{logp, reinterpret_cast<const float2*>(stats), grad, d_logits, d_stride};
  const RowShape s = row_shape(plan, size_t(V) * size_of(type), dev->num_sms, false);
  const long long apart = reinterpret_cast<const char*>(logits) - static_cast<char*>(d_logits);
  const bool vec = apart % 16 == 0 && (row_stride - d_stride) * (long long)size_of(type) % 16 == 0;
  auto go = [&](auto x) {
    using X = decltype(x);
    return vec ? launch_bwd_of<X, true>(a, s, b, stream) : launch_bwd_of<X, false>(a, s, b, stream);
  };
  return type == PP_BF16 ? go(__nv_bfloat16()) : type == PP_FP16 ? go(__half()) : go(float());
}

}  // namespace pp
