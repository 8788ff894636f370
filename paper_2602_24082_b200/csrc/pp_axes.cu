// Position ids with several axes (time, height, width) and the rotary embedding by them.
//
// The paper packs image prompts too (Sec. 4: llava on RLAIF-V).  Where the positions of an image's tokens
// have axes, a token of text has the running number n on all of them, a span of f x h x w image tokens
// that starts at n has (n + frame, n + row, n + column), and the text behind it goes on at n + max(f, h, w).
// In the packed layout every response goes on where the prompt has ended (Sec. 3.2).  So with S[i] = sum over
// the spans before span i of f h w - max(f, h, w), the number at a token is its index in its own unpacked sequence less the S
// of the spans of that sequence before it: a few look-ups per token, no chain.
//
// The rotary embedding is the rotate-half form of pp_rope.cu with the angle of frequency i taken from the axis that i
// belongs to.  The angle is pos * base^(-2i/D); in fp32 it is off by 2^-24 of itself, 0.008 at position 131072.
// Here the frequency is a 64-bit fraction of a turn, so pos times it modulo a whole turn is one integer
// product without rounding; sine and cosine get what is left, in [-pi, pi).
// One pass over Q and K, read once and written once (in place, from or into the buffer of a fused projection, or to
// others), bound by HBM; the inverse is the backward pass.
#include <math.h>

#include <algorithm>

#include "pp_seg.cuh"

namespace pp {
namespace {

// ---------------------------------------------------------------- position ids
struct AxesArgs {
  const int32_t* header;
  const int32_t* seg_start;
  const int32_t* grp_resp_off;
  int nseg, G, T;
  const int32_t* span_start;   // [I] ascending
  const int32_t* span_grid;    // [I][3]
  int I;
  int32_t* pos;                // [3][T]
  int32_t* status;             // [2]
};

__device__ __forceinline__ long long span_size(const int32_t* grid, int i) {
  const int f = grid[3 * i], h = grid[3 * i + 1], w = grid[3 * i + 2];
  if (f < 1 || h < 1 || w < 1) return 0;
  const long long hw = (long long)h * w;
  return hw > INT_MAX || hw * f > INT_MAX ? 0 : hw * f;
}
// spans in front of token t: the first index with start >= t
__device__ __forceinline__ int spans_before(const AxesArgs& p, int t) {
  int lo = 0, hi = p.I;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (p.span_start[mid] < t) lo = mid + 1; else hi = mid;
  }
  return lo;
}

constexpr int kPosThreads = 256, kPosChunk = 4 * kPosThreads;   // spans whose sums are at hand at a time

// The array, copied to shared memory by the block if it has the room.
template <int kRoom>
__device__ __forceinline__ const int32_t* held(int32_t* to, const int32_t* from, int n) {
  if (n > kRoom) return from;
  for (int i = threadIdx.x; i < n; i += kPosThreads) to[i] = from[i];
  return to;
}

__global__ void __launch_bounds__(kPosThreads) position_ids_axes_kernel(AxesArgs p) {
  constexpr int kHeld = 1024;
  __shared__ int32_t s_seg[kHeld], s_off[kHeld], s_span[kHeld];
  __shared__ uint32_t sums[kPosChunk];
  __shared__ uint32_t warp_sum[kPosThreads / 32];
  __shared__ int bad;
  __shared__ int range[2];
  dependency_wait();
  if (p.header[0] != kStatusOk) return;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // the tables that are searched, at hand: a look-up in L2 takes as long as twenty here
  p.seg_start = held<kHeld>(s_seg, p.seg_start, p.nseg + 1);
  p.grp_resp_off = held<kHeld>(s_off, p.grp_resp_off, p.G + 1);
  p.span_start = held<kHeld>(s_span, p.span_start, p.I);
  __syncthreads();
  if (blockIdx.x == gridDim.x - 1) {   // one block looks the spans over
    if (tid == 0) bad = INT_MAX;
    __syncthreads();
    for (int i = tid; i < p.I; i += kPosThreads) {
      const long long n = span_size(p.span_grid, i), s = p.span_start[i];
      bool ok = n > 0 && s >= 0 && s + n <= p.T;
      if (ok && i) ok = p.span_start[i - 1] + span_size(p.span_grid, i - 1) <= s && p.span_start[i - 1] < s;
      if (ok) ok = s + n <= p.seg_start[thread_upper(p.seg_start, p.nseg, int(s)) + 1];
      if (!ok) atomicMin(&bad, i);
    }
    __syncthreads();
    if (tid == 0) {
      p.status[0] = bad != INT_MAX;
      p.status[1] = bad != INT_MAX ? bad : 0;
    }
    return;
  }
  const int t = blockIdx.x * kPosThreads + tid;
  const bool in = t < p.T;
  // where the token's sequence begins, and which spans lie in front: [i_group, i_prompt) those of its prompt,
  // [i_seg, i_token) those of its segment
  int seg = 0, a = 0, group = 0, prompt_end = 0;
  int i_group = 0, i_prompt = 0, i_seg = 0, i_token = 0;
  int k = -1, f_h = 1, f_w = 1;      // index inside a span, its height and width
  if (in) {
    seg = thread_upper(p.seg_start, p.nseg, t);
    a = p.seg_start[seg];
    int g = 0;                       // its group: the largest g with g + grp_resp_off[g] <= seg
    for (int hi = p.G; hi - g > 1;) {
      const int mid = (g + hi) >> 1;
      if (mid + p.grp_resp_off[mid] <= seg) g = mid; else hi = mid;
    }
    const int sp = g + p.grp_resp_off[g];   // the group's prompt
    group = p.seg_start[sp];
    prompt_end = p.seg_start[sp + 1];
    i_seg = spans_before(p, a);
    i_token = spans_before(p, t);
    if (seg != sp) {
      i_group = spans_before(p, group);
      i_prompt = spans_before(p, prompt_end);
    }
    const int i = i_token < p.I && p.span_start[i_token] == t ? i_token : i_token - 1;
    if (i >= i_seg && i < p.I) {
      const long long n = span_size(p.span_grid, i), at = (long long)t - p.span_start[i];
      if (at >= 0 && at < n) {
        k = int(at);
        i_token = i;
        f_h = p.span_grid[3 * i + 1];
        f_w = p.span_grid[3 * i + 2];
      }
    }
  }
  // sums of the spans that some token of the block asks for
  if (tid == 0) range[0] = INT_MAX, range[1] = 0;
  __syncthreads();
  const bool prompt_too = in && i_group < i_prompt;
  const int from = prompt_too ? min(i_group, i_seg) : i_seg, to = prompt_too ? max(i_prompt, i_token) : i_token;
  if (in && from < to) {
    atomicMin(&range[0], from);
    atomicMax(&range[1], to);
  }
  __syncthreads();
  const int lo = range[0], hi = range[1];
  uint32_t less = 0, carry = 0;
  auto pick = [&](int i, int c0, int n, uint32_t sign) {   // sum of the spans [lo, i)
    if (i > c0 && i <= c0 + n) less += sign * sums[i - c0 - 1];
  };
  for (int c0 = lo; c0 < hi; c0 += kPosChunk) {
    const int n = min(kPosChunk, hi - c0);
    uint32_t d[4], mine = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = c0 + 4 * tid + j;
      d[j] = 0;
      if (4 * tid + j < n) {
        const int f = p.span_grid[3 * i], h = p.span_grid[3 * i + 1], w = p.span_grid[3 * i + 2];
        d[j] = uint32_t(span_size(p.span_grid, i)) - uint32_t(max(f, max(h, w)));
      }
      mine += d[j];
    }
    uint32_t upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += x;
    }
    if (lane == 31) warp_sum[warp] = upto;
    __syncthreads();
    uint32_t before = carry + upto - mine;
    for (int w = 0; w < kPosThreads / 32; ++w) {
      if (w < warp) before += warp_sum[w];
      carry += warp_sum[w];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      before += d[j];
      sums[4 * tid + j] = before;
    }
    __syncthreads();
    if (in) {
      pick(i_token, c0, n, 1u);
      pick(i_seg, c0, n, ~0u);
      if (prompt_too) {
        pick(i_prompt, c0, n, 1u);
        pick(i_group, c0, n, ~0u);
      }
    }
    __syncthreads();
  }
  if (!in) return;
  uint32_t number = uint32_t((k >= 0 ? t - k : t) - a) - less;
  if (a != group) number += uint32_t(prompt_end - group);
  int x = 0, y = 0, z = 0;
  if (k >= 0) {
    const int hw = f_h * f_w;
    x = k / hw;
    y = k % hw / f_w;
    z = k % f_w;
  }
  p.pos[t] = int32_t(number + x);
  p.pos[size_t(p.T) + t] = int32_t(number + y);
  p.pos[2 * size_t(p.T) + t] = int32_t(number + z);
}

// ---------------------------------------------------------------- rotary embedding
struct RopeTable {
  uint64_t turn[64];   // the frequencies as fractions of a turn, times 2^64
  uint8_t axis[64];
};
struct RopeArgs {
  const int32_t* header;
  int T, Hq, Hkv;
  const __nv_bfloat16 *q, *k;
  __nv_bfloat16 *q_out, *k_out;
  long long q_stride, k_stride, q_out_stride, k_out_stride;   // elements between tokens
  const int32_t* pos;                                         // [axes][T]
  float sign;                                                 // -1: the inverse
};

// A thread takes eight frequencies -- 16 bytes of a head's lower half and 16 of its upper -- of every
// `heads`-th head of a token, four heads in all: as many as it has on their way at once.  The block computes each token's
// sines and cosines once, in shared memory, under the first loads.  With more heads for a thread the batches follow each
// other, with fewer too little is on its way: 65536 tokens, 40 heads, D 128 197 us with four, 228 with eight, 220
// with two or three; 47325 tokens, 16 heads 62.5, 70 and 84; sines by every thread for its own eight frequencies
// 203 and 63 at best, with ten and eight heads.
constexpr int kRopeBatch = 4;
template <int D>
__host__ __device__ constexpr int rope_threads() { return D == 96 ? 192 : 256; }

template <int D>
__global__ void __launch_bounds__(rope_threads<D>(), 3)
rope_axes_kernel(RopeArgs p, const __grid_constant__ RopeTable table, int heads) {
  constexpr int kChunks = D / 16, kHalf = D / 2, kThreads = rope_threads<D>(), kSlots = kThreads / kChunks;
  constexpr int kBatch = kRopeBatch;
  // cosine and sine of two frequencies: [token][four pairs][chunk]
  __shared__ float4 turned[kSlots * 4 * kChunks];
  dependency_wait();
  if (p.header[0] != kStatusOk) return;
  const int per_block = kSlots / heads;
  const long long t0 = (long long)blockIdx.x * per_block;
  const int tokens = int(min((long long)per_block, p.T - t0));
  const int chunk = threadIdx.x % kChunks, slot = threadIdx.x / kChunks, token = slot / heads, H = p.Hq + p.Hkv;
  const long long t = t0 + token;
  // a batch of heads is loaded in front of its stores (the tensors may be the same), the first under the sines
  uint4 lo[kBatch], hi[kBatch];
  auto load = [&](int h0) {
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int h = h0 + j * heads;
      if (h < H) {
        const __nv_bfloat16* src = h < p.Hq ? p.q + t * p.q_stride + h * D : p.k + t * p.k_stride + (h - p.Hq) * D;
        lo[j] = reinterpret_cast<const uint4*>(src)[chunk];
        hi[j] = reinterpret_cast<const uint4*>(src + kHalf)[chunk];
      }
    }
  };
  int h0 = token < tokens ? slot % heads : H;
  load(h0);
  for (int i = threadIdx.x; i < tokens * kHalf; i += kThreads) {
    const int of = i / kHalf, f = i % kHalf;
    const long long at = p.pos[size_t(table.axis[f]) * p.T + t0 + of];
    const uint64_t turn = uint64_t(at) * table.turn[f];
    float c, s;
    sincospif(float(int32_t(turn >> 32)) * 4.656612873077393e-10f, &s, &c);   // (2^-31 half turns)
    reinterpret_cast<float2*>(turned)[((of * 4 + f % 8 / 2) * kChunks + f / 8) * 2 + f % 2] = make_float2(c, s * p.sign);
  }
  __syncthreads();
  if (token >= tokens) return;
  const float4* mine = turned + token * 4 * kChunks + chunk;
  for (; h0 < H; h0 += kBatch * heads) {
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int h = h0 + j * heads;
      if (h >= H) break;
      const uint32_t l[4] = {lo[j].x, lo[j].y, lo[j].z, lo[j].w}, u[4] = {hi[j].x, hi[j].y, hi[j].z, hi[j].w};
      uint32_t x[4], y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 cs = mine[i * kChunks];   // cosine and sine of the pair's first, of its second
        const float a0 = __uint_as_float(l[i] << 16), a1 = __uint_as_float(l[i] & 0xffff0000u);
        const float b0 = __uint_as_float(u[i] << 16), b1 = __uint_as_float(u[i] & 0xffff0000u);
        x[i] = pack_bf16(a0 * cs.x - b0 * cs.y, a1 * cs.z - b1 * cs.w);
        y[i] = pack_bf16(b0 * cs.x + a0 * cs.y, b1 * cs.z + a1 * cs.w);
      }
      __nv_bfloat16* dst =
          h < p.Hq ? p.q_out + t * p.q_out_stride + h * D : p.k_out + t * p.k_out_stride + (h - p.Hq) * D;
      reinterpret_cast<uint4*>(dst)[chunk] = make_uint4(x[0], x[1], x[2], x[3]);
      reinterpret_cast<uint4*>(dst + kHalf)[chunk] = make_uint4(y[0], y[1], y[2], y[3]);
    }
    load(h0 + kBatch * heads);
  }
}

template <int D>
cudaError_t launch_rope_of(const RopeArgs& p, const RopeTable& table, cudaStream_t stream) {
  constexpr int kSlots = rope_threads<D>() / (D / 16);
  const int H = p.Hq + p.Hkv;
  const int heads = std::min(kSlots, (H + kRopeBatch - 1) / kRopeBatch);
  const int per_block = kSlots / heads;
  return launch_kernel(true, rope_axes_kernel<D>, dim3(unsigned((p.T + (long long)per_block - 1) / per_block)),
                       dim3(rope_threads<D>()), 0, stream, p, table, heads);
}

}  // namespace

cudaError_t launch_position_ids_axes(const pp_plan* plan, int num_spans, const int32_t* span_start,
                                     const int32_t* span_grid, int32_t* pos, int32_t* status, cudaStream_t stream) {
  AxesArgs p;
  p.header = reinterpret_cast<const int32_t*>(plan->ws + plan->lay.header);
  p.seg_start = reinterpret_cast<const int32_t*>(plan->ws + plan->lay.seg_start);
  p.grp_resp_off = plan->prob.grp_resp_off;
  p.nseg = plan->nseg;
  p.G = plan->prob.num_groups;
  p.T = plan->prob.total_tokens;
  p.span_start = span_start;
  p.span_grid = span_grid;
  p.I = num_spans;
  p.pos = pos;
  p.status = status;
  const unsigned blocks = unsigned((p.T + (long long)kPosThreads - 1) / kPosThreads) + 1;
  return launch_kernel(true, position_ids_axes_kernel, dim3(blocks), dim3(kPosThreads), 0, stream, p);
}

cudaError_t launch_rope_axes(const pp_plan* plan, const void* q, long long q_stride, const void* k, long long k_stride,
                             void* q_out, long long q_out_stride, void* k_out, long long k_out_stride,
                             const int32_t* pos, const uint8_t* axis_of_freq, float base, bool inverse,
                             cudaStream_t stream) {
  const int D = plan->prob.head_dim;
  // base^(-2i/D) / (2 pi) turns per position, below 0.16: one power, and products with 64 bits
  RopeTable table = {};
  const long double ratio = powl((long double)base, -2.0L / D);
  long double turns = 0.159154943091895335768883763372514362L;
  for (int i = 0; i < D / 2; ++i, turns *= ratio) {
    table.turn[i] = uint64_t(ldexpl(turns, 64));
    table.axis[i] = axis_of_freq[i];
  }
  RopeArgs p;
  p.header = reinterpret_cast<const int32_t*>(plan->ws + plan->lay.header);
  p.T = plan->prob.total_tokens;
  p.Hq = plan->prob.num_q_heads;
  p.Hkv = plan->prob.num_kv_heads;
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.k = static_cast<const __nv_bfloat16*>(k);
  p.q_out = static_cast<__nv_bfloat16*>(q_out);
  p.k_out = static_cast<__nv_bfloat16*>(k_out);
  p.q_stride = q_stride;
  p.k_stride = k_stride;
  p.q_out_stride = q_out_stride;
  p.k_out_stride = k_out_stride;
  p.pos = pos;
  p.sign = inverse ? -1.f : 1.f;
  return D == 128  ? launch_rope_of<128>(p, table, stream)
         : D == 96 ? launch_rope_of<96>(p, table, stream)
                   : launch_rope_of<64>(p, table, stream);
}

}  // namespace pp
