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
// softmax, the backward reads and writes it once.  What keeps the forward at the memory's rate
// is one exponential per element and little else: 128 K columns of bf16 at 6.5 TB/s are 11.7 elements per clock
// and SM, of 16 that the special function unit makes.  The exponential is 2^(c x - K), c = log2(e) /
// temperature, with a whole number K >= c max(x) for reference: K is exact in fp32, so nothing of c x is
// lost to the rounding of a reference (c m rounded would be off by 2^-24 |c m|, the same for the whole
// row), sums of different references are joined by exact powers of two, and a larger element than those
// seen so far costs one multiplication, rarely.  A thread takes four 16-byte vectors at a time.
// Rows whose values are beyond +-2^19 (a mask of the type's lowest value over everything, say)
// go through a second pass over exp(x - m).
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include "pp_seg.cuh"

namespace pp {
namespace {

constexpr float kFar = 524288.f;   // |c m| up to which K is a whole number apart from c m by less than 1.1
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
  static __device__ __forceinline__ float one(const __nv_bfloat16& x) { return __bfloat162float(x); }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
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
  static __device__ __forceinline__ float one(const __half& x) { return __half2float(x); }
  static __device__ __forceinline__ void store(__half* p, float x) { *p = __float2half_rn(x); }
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
  int n;       // tokens; 0 = nothing
  int token;   // n == 1: the token.  Otherwise the responses' first tokens: starts of segments
  int seg;     //   seg + 1 .. seg + n
  bool prompt;
};
// (by a whole warp)
__device__ __forceinline__ Predicts predicts_of(const LogpArgs& p, int r) {
  Predicts u;
  u.seg = warp_upper(p.seg_start, p.nseg, r);
  const int a = p.seg_start[u.seg], e = p.seg_start[u.seg + 1];
  const int seen = p.key_end[a];       // behind the group for a prompt's keys, behind the response for its own
  u.prompt = seen > e;
  u.n = 0;
  u.token = r + 1;
  if (!u.prompt) u.n = r + 1 < e;
  else if (r + 1 == e) u.n = warp_upper(p.seg_start, p.nseg, seen - 1) - u.seg;
  return u;
}
__device__ __forceinline__ int token_of(const LogpArgs& p, const Predicts& u, int k) {
  return u.n == 1 ? u.token : p.seg_start[u.seg + 1 + k];
}
__device__ __forceinline__ long long id_of(const LogpArgs& p, int t) {
  return p.ids_64 ? static_cast<const long long*>(p.ids)[t] : (long long)static_cast<const int32_t*>(p.ids)[t];
}

// The part of a row that `parts` blocks share: vectors [v0, v1) from the first 16-byte boundary on; the
// elements before it (head) and behind the last whole vector (tail) go to the first block and the last.
struct Span {
  int head, v0, v1, tail0;   // elements in front; vectors; first element behind the vectors
};
template <typename X>
__device__ __forceinline__ Span span_of(const X* row, int V, int part, int parts) {
  constexpr int kN = Row<X>::kN;
  Span s;
  s.head = min(V, int(((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / sizeof(X)));
  const int nv = (V - s.head) / kN, per = (nv + parts - 1) / parts;
  s.v0 = min(nv, part * per);
  s.v1 = min(nv, s.v0 + per);
  s.tail0 = s.head + nv * kN;
  return s;
}

// Running maximum and sum of 2^(c x - K), K a whole number (or -inf before anything finite).
struct Running {
  float m = -INFINITY, K = -INFINITY, s = 0.f;
};
__device__ __forceinline__ float rescale(float from, float to) {   // 2^(from - to), from <= to
  return from == to ? 1.f : exp2f(from - to);
}
__device__ __forceinline__ void join(Running& a, float m, float K, float s) {
  a.m = fmaxf(a.m, m);
  const float top = fmaxf(a.K, K);
  a.s = a.s * rescale(a.K, top) + s * rescale(K, top);
  a.K = top;
}
template <int kWarps>
__device__ __forceinline__ void row_sync() {
  if constexpr (kWarps == 1) __syncwarp(); else __syncthreads();
}

// All threads of the row get the whole row's values.
template <int kWarps>
__device__ __forceinline__ Running join_row(Running a, float (*part_of)[4], float (*warp_of)[4], int parts, bool first) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    join(a, __shfl_xor_sync(0xffffffffu, a.m, o), __shfl_xor_sync(0xffffffffu, a.K, o),
         __shfl_xor_sync(0xffffffffu, a.s, o));
  if constexpr (kWarps > 1) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (lane == 0) {
      warp_of[warp][0] = a.m;
      warp_of[warp][1] = a.K;
      warp_of[warp][2] = a.s;
    }
    __syncthreads();
    a = Running();
    if (lane < kWarps) {
      a.m = warp_of[lane][0];
      a.K = warp_of[lane][1];
      a.s = warp_of[lane][2];
    }
#pragma unroll
    for (int o = kWarps / 2; o > 0; o >>= 1)
      join(a, __shfl_xor_sync(0xffffffffu, a.m, o), __shfl_xor_sync(0xffffffffu, a.K, o),
           __shfl_xor_sync(0xffffffffu, a.s, o));
    if (parts > 1) {
      auto cluster = cooperative_groups::this_cluster();
      if (first) cluster.barrier_wait();   // (all blocks have started: their arrival is before the row's loads)
      const int me = int(cluster.block_rank());
      if (warp == 0 && lane < 3) {
        const float v = lane == 0 ? a.m : lane == 1 ? a.K : a.s;
        for (int b = 0; b < parts; ++b) cluster.map_shared_rank(&part_of[me][0], b)[lane] = v;
      }
      cluster.sync();
      a = Running();
      for (int b = 0; b < parts; ++b) join(a, part_of[b][0], part_of[b][1], part_of[b][2]);
    }
  }
  // (every thread of the last lanes may hold nothing: all take what lane 0 has)
  a.m = __shfl_sync(0xffffffffu, a.m, 0);
  a.K = __shfl_sync(0xffffffffu, a.K, 0);
  a.s = __shfl_sync(0xffffffffu, a.s, 0);
  return a;
}

constexpr int kMaxParts = 8;
template <int kWarps> constexpr int block_threads() { return kWarps == 1 ? 256 : kWarps * 32; }

template <typename X, int kWarps>
__global__ void __launch_bounds__(block_threads<kWarps>())
token_logp_kernel(LogpArgs p, int parts, float* logp, float2* stats) {
  constexpr int kN = Row<X>::kN, kThreads = kWarps * 32, kUnroll = 4;
  __shared__ float warp_of[2][kWarps][4];
  __shared__ float part_of[2][kMaxParts][4];
  dependency_wait();
  if (p.header[0] != kStatusOk) return;
  const int tid = kWarps == 1 ? threadIdx.x & 31 : threadIdx.x;
  const int r = kWarps == 1 ? blockIdx.x * 8 + (threadIdx.x >> 5) : blockIdx.x / parts;
  const int part = kWarps == 1 ? 0 : blockIdx.x % parts;
  if (r >= p.T) return;
  const Predicts u = predicts_of(p, r);
  const bool writes = part == 0;
  if (u.prompt && writes && tid == 0) logp[r] = 0.f;
  bool any = false;
  for (int k = tid & 31; k < u.n; k += 32) any |= id_of(p, token_of(p, u, k)) >= 0;
  if (!__any_sync(0xffffffffu, any)) {
    if (writes) {
      if (tid == 0) stats[r] = make_float2(0.f, 0.f);
      for (int k = tid; k < u.n; k += kThreads) logp[token_of(p, u, k)] = 0.f;
    }
    return;
  }
  if constexpr (kWarps > 1)
    if (parts > 1) cooperative_groups::this_cluster().barrier_arrive();
  const X* row = static_cast<const X*>(p.logits) + (long long)r * p.row_stride;
  const Span sp = span_of(row, p.V, part, parts);
  const uint4* vec = reinterpret_cast<const uint4*>(row + sp.head);
  const float c = p.c;
  const uint64_t c2 = pack2(c, c);

  Running run;
  uint64_t sum = pack2(0.f, 0.f);
  auto raise = [&](float bm) {
    const float K = ceilf(bm * c);
    run.m = fmaxf(run.m, bm);
    if (K > run.K) {
      const float f = exp2f(run.K - K);
      sum = mul2(sum, pack2(f, f));
      run.K = K;
    }
    return run.K == -INFINITY ? 0.f : -run.K;
  };
  // elements in front of the first boundary and behind the last, one per thread
  {
    const int edge = (part == 0 ? sp.head : 0), tail = part == parts - 1 ? p.V - sp.tail0 : 0;
    for (int i = tid; i < edge + tail; i += kThreads) {
      const float x = Row<X>::one(row[i < edge ? i : sp.tail0 + i - edge]);
      const float k = raise(x);
      sum = add2(sum, pack2(ex2(fmaf(x, c, k)), 0.f));
    }
  }
  auto take = [&](const uint4* v, int n) {
    uint32_t w = Row<X>::max_word(Row<X>::max_word(v[0].x, v[0].y), Row<X>::max_word(v[0].z, v[0].w));
#pragma unroll
    for (int i = 1; i < kUnroll; ++i)
      if (i < n)
        w = Row<X>::max_word(w, Row<X>::max_word(Row<X>::max_word(v[i].x, v[i].y), Row<X>::max_word(v[i].z, v[i].w)));
    const float k = raise(Row<X>::max_of(w));
    const uint64_t k2 = pack2(k, k);
#pragma unroll
    for (int i = 0; i < kUnroll; ++i)
      if (i < n)
        for_pairs<X>(v[i], [&](float a, float b) {
          float y, z;
          unpack2(fma2(pack2(a, b), c2, k2), y, z);
          sum = add2(sum, pack2(ex2(y), ex2(z)));
        });
  };
  int at = sp.v0 + tid;
  uint4 v[kUnroll];
  for (; at + (kUnroll - 1) * kThreads < sp.v1; at += kUnroll * kThreads) {
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) v[i] = load_row(vec + at + i * kThreads);
    take(v, kUnroll);
  }
  for (; at < sp.v1; at += kThreads) {
    v[0] = load_row(vec + at);
    take(v, 1);
  }
  float lo, hi;
  unpack2(sum, lo, hi);
  run.s = lo + hi;
  run = join_row<kWarps>(run, part_of[0], warp_of[0], parts, true);
  float l;
  if (fabsf(run.m * c) < kFar) {
    l = fmaf(fmaf(run.m, -c, run.K), kLn2, logf(run.s));
  } else {
    // the whole row is far from zero (or infinite): once more, relative to the maximum
    Running far;
    far.K = 0.f;
    const int first = sp.head + sp.v0 * kN, last = sp.head + sp.v1 * kN;
    const int edge = part == 0 ? sp.head : 0, tail = part == parts - 1 ? p.V - sp.tail0 : 0;
    for (int i = tid; i < last - first + edge + tail; i += kThreads) {
      const int e = i < edge ? i : i - edge < last - first ? first + i - edge : sp.tail0 + i - edge - (last - first);
      far.s += exp2f((Row<X>::one(row[e]) - run.m) * c);
    }
    l = logf(join_row<kWarps>(far, part_of[1], warp_of[1], parts, false).s);
  }
  if (l < 0.f) l = 0.f;   // (the maximum is one of the terms)
  if (writes) {
    if (tid == 0) stats[r] = make_float2(run.m / p.temperature, l);
    for (int k = tid; k < u.n; k += kThreads) {
      const int t = token_of(p, u, k);
      const long long y = id_of(p, t);
      logp[t] = y < 0 ? 0.f : y >= p.V ? NAN : (Row<X>::one(row[y]) - run.m) / p.temperature - l;
    }
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

// kVec: rows of logits and of the gradient lie alike to 16 bytes.
template <typename X, int kWarps, bool kVec>
__global__ void __launch_bounds__(block_threads<kWarps>())
token_logp_bwd_kernel(LogpArgs p, LogpBwdArgs b, int parts) {
  constexpr int kN = Row<X>::kN, kThreads = kWarps * 32, kUnroll = 4;
  dependency_wait();
  if (p.header[0] != kStatusOk) return;
  const int tid = kWarps == 1 ? threadIdx.x & 31 : threadIdx.x, lane = threadIdx.x & 31;
  const int r = kWarps == 1 ? blockIdx.x * 8 + (threadIdx.x >> 5) : blockIdx.x / parts;
  const int part = kWarps == 1 ? 0 : blockIdx.x % parts;
  if (r >= p.T) return;
  const Predicts u = predicts_of(p, r);
  // the sum of the gradients of the tokens that the row predicts
  double total = 0;
  bool any = false;
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

  const X* row = static_cast<const X*>(p.logits) + (long long)r * p.row_stride;
  X* out = static_cast<X*>(b.d_logits) + (long long)r * b.d_stride;
  const Span sp = span_of<X>(out, p.V, part, parts);
  uint4* dst = reinterpret_cast<uint4*>(out + sp.head);
  const int edge = part == 0 ? sp.head : 0, tail = part == parts - 1 ? p.V - sp.tail0 : 0;
  if (!any) {
    for (int i = tid; i < edge + tail; i += kThreads) Row<X>::store(out + (i < edge ? i : sp.tail0 + i - edge), 0.f);
    for (int at = sp.v0 + tid; at < sp.v1; at += kThreads) dst[at] = make_uint4(0, 0, 0, 0);
    return;
  }
  // p_v = 2^(c x_v - K) 2^-f with K + f = (m + l) log2(e), K whole: 2^-f goes into the row's factor
  const float2 st = b.stats[r];
  const double lse2 = (double(st.x) + double(st.y)) * kLog2e;
  const double whole = rint(lse2);
  const bool far = !(fabs(lse2) < double(kFar));
  const float scale = float(-total / double(p.temperature));
  const float coef = far ? scale : scale * exp2f(float(whole - lse2));
  const float K = float(whole), c = p.c;
  auto one = [&](float x) {
    return far ? scale * expf(x / p.temperature - st.x - st.y) : coef * ex2(fmaf(x, c, -K));
  };
  for (int i = tid; i < edge + tail; i += kThreads) {
    const int e = i < edge ? i : sp.tail0 + i - edge;
    Row<X>::store(out + e, one(Row<X>::one(row[e])));
  }
  if (kVec && !far) {
    const uint4* vec = reinterpret_cast<const uint4*>(row + sp.head);
    const uint64_t c2 = pack2(c, c), k2 = pack2(-K, -K), f2 = pack2(coef, coef);
    auto take = [&](uint4 v) {
      uint32_t w[4];
      int i = 0;
      for_pairs<X>(v, [&](float x, float y) {
        unpack2(fma2(pack2(x, y), c2, k2), x, y);
        unpack2(mul2(pack2(ex2(x), ex2(y)), f2), x, y);
        if constexpr (kN == 8) {
          w[i++] = Row<X>::word(x, y);
        } else {
          w[i++] = __float_as_uint(x);
          w[i++] = __float_as_uint(y);
        }
      });
      return make_uint4(w[0], w[1], w[2], w[3]);
    };
    int at = sp.v0 + tid;
    uint4 v[kUnroll];
    for (; at + (kUnroll - 1) * kThreads < sp.v1; at += kUnroll * kThreads) {
#pragma unroll
      for (int i = 0; i < kUnroll; ++i) v[i] = load_row(vec + at + i * kThreads);
#pragma unroll
      for (int i = 0; i < kUnroll; ++i) dst[at + i * kThreads] = take(v[i]);
    }
    for (; at < sp.v1; at += kThreads) dst[at] = take(load_row(vec + at));
  } else {
    for (int e = sp.head + sp.v0 * kN + tid; e < sp.head + sp.v1 * kN; e += kThreads)
      Row<X>::store(out + e, one(Row<X>::one(row[e])));
  }
  // the tokens' own columns, from their log-probabilities: 1 - p without cancellation.  The same id may be
  // that of several responses: each writes the sum over all of them.
  row_sync<kWarps>();
  const int first = part == 0 ? 0 : sp.head + sp.v0 * kN;
  const int last = part == parts - 1 ? p.V : sp.head + sp.v1 * kN;
  for (int k = tid; k < u.n; k += kThreads) {
    const int t = token_of(p, u, k);
    const long long y = id_of(p, t);
    if (y < first || y >= last) continue;
    double same = 0;
    if (u.n == 1) {
      same = total;
    } else {
      for (int j = 0; j < u.n; ++j) {
        const int tj = token_of(p, u, j);
        if (id_of(p, tj) == y) same += b.grad[tj];
      }
    }
    const float lp = b.logp[t];
    Row<X>::store(out + y, float((-same * double(expm1f(lp)) - (total - same) * double(expf(lp))) / double(p.temperature)));
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

// Warps per row and blocks per row.
struct RowShape {
  int warps, parts;
};
RowShape row_shape(int T, size_t row_bytes, int num_sms) {
  RowShape s{16, 1};
  if (row_bytes <= 8192) s.warps = 1;
  else if (row_bytes <= 65536 && T >= 4 * num_sms) s.warps = 4;
  if (s.warps == 16)
    while (s.parts < kMaxParts && (long long)T * s.parts < 4ll * num_sms && row_bytes / (2 * s.parts) >= 8192) s.parts *= 2;
  return s;
}

template <typename X>
cudaError_t launch_fwd_of(const LogpArgs& a, RowShape s, float* logp, float2* stats, cudaStream_t stream) {
  if (s.warps == 1)
    return launch_kernel(true, token_logp_kernel<X, 1>, dim3((a.T + 7) / 8), dim3(256), 0, stream, a, 1, logp, stats);
  if (s.warps == 4)
    return launch_kernel(true, token_logp_kernel<X, 4>, dim3(a.T), dim3(128), 0, stream, a, 1, logp, stats);
  return launch_clusters(s.parts, token_logp_kernel<X, 16>, dim3(unsigned(a.T) * s.parts), dim3(512), 0, stream, a,
                         s.parts, logp, stats);
}

template <typename X, bool kVec>
cudaError_t launch_bwd_of(const LogpArgs& a, RowShape s, const LogpBwdArgs& b, cudaStream_t stream) {
  if (s.warps == 1)
    return launch_kernel(true, token_logp_bwd_kernel<X, 1, kVec>, dim3((a.T + 7) / 8), dim3(256), 0, stream, a, b, 1);
  if (s.warps == 4)
    return launch_kernel(true, token_logp_bwd_kernel<X, 4, kVec>, dim3(a.T), dim3(128), 0, stream, a, b, 1);
  return launch_kernel(true, token_logp_bwd_kernel<X, 16, kVec>, dim3(unsigned(a.T) * s.parts), dim3(512), 0, stream, a,
                       b, s.parts);
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
  const RowShape s = row_shape(a.T, size_t(V) * size_of(type), dev->num_sms);
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
  const RowShape s = row_shape(a.T, size_t(V) * size_of(type), dev->num_sms);
  const long long apart = reinterpret_cast<const char*>(logits) - static_cast<char*>(d_logits);
  const bool vec = apart % 16 == 0 && (row_stride - d_stride) * (long long)size_of(type) % 16 == 0;
  auto go = [&](auto x) {
    using X = decltype(x);
    return vec ? launch_bwd_of<X, true>(a, s, b, stream) : launch_bwd_of<X, false>(a, s, b, stream);
  };
  return type == PP_BF16 ? go(__nv_bfloat16()) : type == PP_FP16 ? go(__half()) : go(float());
}

}  // namespace pp
