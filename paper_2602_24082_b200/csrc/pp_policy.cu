// Clipped policy loss with a KL term over the responses of a packed batch, and its gradient.
//
// The packed groups (paper Sec. 3.1: a prompt and its K responses) are what policy training samples; the paper
// itself trains on pairwise losses, of which this is the sibling for rewards.  Per response k of a group:
//   A_k    = its reward as given, less the group's mean, or that over the group's standard deviation
//            (n - 1 in the denominator; 0 for one response) + eps; or one value per token
//   rho_t  = exp(logp_t - old_t)                          (1 without old log-probabilities)
//   l_t    = -min(rho_t A, clip(rho_t, 1 - lo, 1 + hi) A) + kl (exp(d) - d - 1),   d = ref_t - logp_t
//   loss_k = w_k sum_t l_t over the tokens that the mask leaves, w_k = scale / n_k or scale
//   d logp = w_k ((rho A where rho A <= clip(rho) A, else 0) (-1) + kl (1 - exp(d)))
// Everything per token is in 64 bits: ratio and border decide whether a token has a gradient at all,
// and exp(d) - d - 1 is the small difference of large terms near d = 0.  That costs nothing: 16
// bytes per token make this a kernel of latencies.  So one launch does it all: a team
// of 1, 2, 4 or 8 warps takes a response, as many as its tokens ask for, or a cluster of up to 8 blocks
// that add up their sums through distributed shared memory, in the order of their ranks.
// A prompt's tokens have no gradient; the zeros are written by its responses' teams.
#include <cooperative_groups.h>

#include "pp_seg.cuh"

namespace pp {
namespace {

struct PolicyArgs {
  const int32_t* header;
  const int32_t* seg_start;
  const int32_t* grp_resp_off;
  int G, N;
  const float *logp, *old, *ref, *reward;
  const uint8_t* mask;
  pp_policy o;
  float *advantage, *loss, *kl, *clipped, *d_logp;
};

constexpr int kThreads = 256, kMaxParts = 8;

// What a team adds up.
struct Sums {
  double loss, kl;
  int clipped, used;
  __device__ __forceinline__ void add(const Sums& x) {
    loss += x.loss;
    kl += x.kl;
    clipped += x.clipped;
    used += x.used;
  }
};
// ... over kTeam threads of a block, or over all blocks of a cluster (which have started).  (kCount: `used` alone)
template <int kTeam, bool kCount>
__device__ __forceinline__ Sums team_sum(Sums x, Sums* warp_of, Sums* part_of, int parts) {
  x.used = __reduce_add_sync(0xffffffffu, x.used);
  if constexpr (!kCount) {
    x.clipped = __reduce_add_sync(0xffffffffu, x.clipped);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      x.loss += __shfl_xor_sync(0xffffffffu, x.loss, o);
      x.kl += __shfl_xor_sync(0xffffffffu, x.kl, o);
    }
  }
  if constexpr (kTeam > 32) {
    const int warp = threadIdx.x >> 5, first = warp / (kTeam / 32) * (kTeam / 32);
    if ((threadIdx.x & 31) == 0) warp_of[warp] = x;
    if constexpr (kTeam == kThreads) __syncthreads();
    else named_barrier_sync(1 + threadIdx.x / kTeam, kTeam);
    x = warp_of[first];
#pragma unroll
    for (int w = 1; w < kTeam / 32; ++w) x.add(warp_of[first + w]);
  }
  if constexpr (kTeam == kThreads) {
    if (parts > 1) {
      auto cluster = cooperative_groups::this_cluster();
      if (threadIdx.x < parts) *cluster.map_shared_rank(part_of + cluster.block_rank(), int(threadIdx.x)) = x;
      cluster.sync();
      x = part_of[0];
      for (int b = 1; b < parts; ++b) x.add(part_of[b]);
    }
  }
  return x;
}

template <int kTeam>
__global__ void __launch_bounds__(kThreads) policy_loss_kernel(PolicyArgs p, int parts) {
  __shared__ Sums warp_of[2][kThreads / 32], part_of[2][kMaxParts];
  dependency_wait();
  const int lane = threadIdx.x & 31, in_team = threadIdx.x % kTeam;
  const int x = kTeam == kThreads ? blockIdx.x / parts : blockIdx.x * (kThreads / kTeam) + threadIdx.x / kTeam;
  const int part = kTeam == kThreads ? blockIdx.x % parts : 0;
  if (x >= p.N) return;
  if (kTeam == kThreads && parts > 1) cooperative_groups::this_cluster().barrier_arrive();
  const int status = p.header[0];
  const int g = warp_upper(p.grp_resp_off, p.G, x);
  if (status != kStatusOk) {   // (a refused plan's offsets may point anywhere)
    // who has arrived waits, too.  (Arriving behind this look at the status is 0.2 us later, of 6.9)
    if (kTeam == kThreads && parts > 1) cooperative_groups::this_cluster().barrier_wait();
    return;
  }
  const int seg = g + 1 + x;
  const int a = p.seg_start[seg], b = p.seg_start[seg + 1];
  const int x0 = p.grp_resp_off[g], n = p.grp_resp_off[g + 1] - x0, sp = g + x0;
  const int p0 = p.seg_start[sp], p1 = p.seg_start[sp + 1];
  const int stride = kTeam * parts, first = a + part * kTeam + in_team;
  const bool per_token = p.o.advantage_mode == PP_ADVANTAGE_TOKEN;
  // what a token needs; that of a thread's first is on its way while the advantage and the count are found
  struct Token {
    float lp, old, ref, adv;
    bool use;
  };
  auto load = [&](int t) {
    Token k{};
    if (t < b) {
      k.use = !p.mask || p.mask[t];
      k.lp = p.logp[t];
      if (p.old) k.old = p.old[t];
      if (p.ref) k.ref = p.ref[t];
      if (per_token) k.adv = p.reward[t];
    }
    return k;
  };
  Token k = load(first);
  if (p.d_logp) {   // this response's share of the prompt's zeros
    const int len = p1 - p0, j = x - x0;
    const int lo = p0 + int((long long)len * j / n), hi = p0 + int((long long)len * (j + 1) / n);
    for (int t = lo + part * kTeam + in_team; t < hi; t += stride) p.d_logp[t] = 0.f;
  }
  // the advantage, by every warp for itself
  double A = 0;
  if (!per_token) {
    A = p.reward[x];
    if (p.o.advantage_mode != PP_ADVANTAGE_GIVEN) {
      const double inv_n = 1.0 / n, inv_n1 = n > 1 ? 1.0 / (n - 1) : 0.0;   // (under the loads)
      const double mine = lane < n ? p.reward[x0 + lane] : 0.f;
      double sum = mine;
      for (int j = lane + 32; j < n; j += 32) sum += p.reward[x0 + j];
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      // the quotient as a division rounds it: equal rewards have to have themselves for mean, and no advantage
      const double q = sum * inv_n, mean = fma(fma(-q, double(n), sum), inv_n, q);
      A -= mean;
      if (p.o.advantage_mode == PP_ADVANTAGE_NORMALIZED) {
        double sq = lane < n ? (mine - mean) * (mine - mean) : 0.0;
        for (int j = lane + 32; j < n; j += 32) {
          const double d = p.reward[x0 + j] - mean;
          sq += d * d;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
        A = n > 1 ? A / (sqrt(sq * inv_n1) + p.o.eps) : 0.0;
      }
    }
    if (p.advantage && part == 0 && in_team == 0) p.advantage[x] = float(A);
  }
  if (kTeam == kThreads && parts > 1) cooperative_groups::this_cluster().barrier_wait();
  // tokens that count: found first where the gradient has to be divided by their number
  double w = p.o.scale;
  if (p.o.reduction == PP_REDUCE_RESPONSE) {
    double count = b - a;
    if (p.mask) {
      int c = k.use;
#pragma unroll 4
      for (int t = first + stride; t < b; t += stride) c += p.mask[t] != 0;
      count = team_sum<kTeam, true>(Sums{0, 0, 0, c}, warp_of[0], part_of[0], parts).used;
    }
    w = count > 0 ? p.o.scale / count : 0.0;
  }
  const double low = 1.0 - p.o.clip_low, high = 1.0 + p.o.clip_high;
  Sums sum{0, 0, 0, 0};
  for (int t = first; t < b; t += stride) {
    const Token now = k;
    k = load(t + stride);
    float d = 0.f;
    if (now.use) {
      const double lp = now.lp, At = per_token ? double(now.adv) : A;
      const double rho = p.old ? exp(lp - double(now.old)) : 1.0;
      // (comparisons, which keep a ratio that is no number)
      const double u = rho * At, v = (rho < low ? low : rho > high ? high : rho) * At;
      const bool cut = v < u;
      double term = cut ? -v : -u, slope = cut ? 0.0 : -u;
      sum.clipped += cut;
      ++sum.used;
      if (p.ref) {
        const double delta = double(now.ref) - lp, e = expm1(delta);
        sum.kl += e - delta;
        term += p.o.kl_coef * (e - delta);
        slope -= p.o.kl_coef * e;
      }
      sum.loss += term;
      d = float(w * slope);
    }
    if (p.d_logp) p.d_logp[t] = d;
  }
  sum = team_sum<kTeam, false>(sum, warp_of[1], part_of[1], parts);
  if (part == 0 && in_team == 0) {
    const double inv = sum.used ? 1.0 / sum.used : 0.0;
    p.loss[x] = float(w * sum.loss);
    p.kl[x] = float(inv * sum.kl);
    p.clipped[x] = float(inv * sum.clipped);
  }
}

}  // namespace

cudaError_t launch_policy_loss(const pp_plan* plan, const pp_policy& o, const float* logp, const float* old,
                               const float* ref, const float* reward, const uint8_t* mask, float* advantage,
                               float* loss, float* kl, float* clipped, float* d_logp, cudaStream_t stream) {
  static DeviceSetup setup[kMaxDevices];
  const DeviceSetup* dev = device_setup(setup);
  if (!dev) return cudaErrorInvalidDevice;
  PolicyArgs p;
  p.header = reinterpret_cast<const int32_t*>(plan->ws + plan->lay.header);
  p.seg_start = reinterpret_cast<const int32_t*>(plan->ws + plan->lay.seg_start);
  p.grp_resp_off = plan->prob.grp_resp_off;
  p.G = plan->prob.num_groups;
  p.N = plan->prob.num_responses;
  p.logp = logp;
  p.old = old;
  p.ref = ref;
  p.reward = reward;
  p.mask = mask;
  p.o = o;
  p.advantage = advantage;
  p.loss = loss;
  p.kl = kl;
  p.clipped = clipped;
  p.d_logp = d_logp;
  // A team has up to four threads for a token of a mean segment, while all of them fit the chip, and a
  // cluster of blocks where segments are long.  us, by tokens of a mean segment and responses: 18, 1880 5.1 (32
  // threads), 5.2 (64), 12.5 (256); 94, 376 8.1, 6.0, 5.0; 100, 20 7.7, 5.8, 4.3; 307, 104 19, 11, 6.2, blocks by twos 6.8, by
  // fours 6.4; 809, 72 8.9 (256), 8.5 (two blocks), 7.1 (four), 8.4 (eight); 2427, 18 16, 13, 9.5, 7.8.
  const long long N = p.N, mean = plan->prob.total_tokens / plan->nseg, most = 2048ll * dev->num_sms;
  if (32 * 2 > 4 * mean || N * 64 > most)
    return launch_kernel(true, policy_loss_kernel<32>, dim3(unsigned((N + 7) / 8)), dim3(kThreads), 0, stream, p, 1);
  if (64 * 2 > 4 * mean || N * 128 > most)
    return launch_kernel(true, policy_loss_kernel<64>, dim3(unsigned((N + 3) / 4)), dim3(kThreads), 0, stream, p, 1);
  if (128 * 2 > 4 * mean || N * 256 > most)
    return launch_kernel(true, policy_loss_kernel<128>, dim3(unsigned((N + 1) / 2)), dim3(kThreads), 0, stream, p, 1);
  int parts = mean > 1536 ? 8 : mean > 400 ? 4 : 1;
  if (N * parts > 4ll * dev->num_sms) parts = N * 4 > 4ll * dev->num_sms ? 1 : 4;
  return launch_clusters(parts, policy_loss_kernel<kThreads>, dim3(unsigned(N) * parts), dim3(kThreads), 0, stream, p,
                         parts);
}

}  // namespace pp
