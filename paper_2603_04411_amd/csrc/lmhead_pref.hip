// Preference loss: one pass over the log-probabilities for the sums of the responses, one over the gradient, whose last workgroup adds up
// loss and statistics; of few tokens both in one workgroup.  A token is 4 bytes in (8 with a reference) and 4 out, its arithmetic two
// additions: up to a million tokens what it takes is launches and the latency of their first loads, so
//  - a response's pairs are looked at by one wavefront, which counts by ballots and meets the others at one barrier;
//  - loads leave before the length that they are masked by has arrived, padding's too (4 x 4 x 262144 full 25.1 us, with 2000 tokens 23.9).
#include "train_common.h"

namespace lmhead {

namespace {

__device__ inline double wave_sum(double x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
  return x;
}
__device__ inline int wave_sum(int x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

struct PrefArgs {
  const float* lp;
  const float* lr;
  const float* reward;
  const int32_t* len;
  int P, G, T, nb, ns;   // nb: blocks of slots in a response, ns: sums that the gradient's launch finds for one
  lmhead_preference q;
  double2* sums;       // [response][block]{log-ratio, log-probability}
  double2* totals;     // [response], the same of all its blocks; with one sum to a response the same memory
  int2* rank;          // [response]{pairs in which it is preferred, best | worst << 1}
  double* part;        // [response, or four short ones]{loss, u > 0, beta s_a, beta s_b, pairs} where it is preferred
  int32_t* done;       // workgroups that have left theirs
  int32_t* pairs;      // pairs of all prompts, where pref_count_kernel has added them up
  float* loss;
  float* g;
  float* ratio;
  float* stats;
};

__device__ inline int length(const PrefArgs& a, int r) { return min(max(a.len[r], 0), a.T); }
__device__ inline double per_token(const PrefArgs& a, int r) {
  const int n = length(a, r);
  return n > 0 ? 1.0 / n : 0.0;
}

// Sums of thread t's share (t, t + step, ..) of slots t0 .. t0 + U * step of response r.
template <int U>
__device__ inline double2 slot_sums(const PrefArgs& a, int r, int n, int t0, int t, int step) {
  const float* lp = a.lp + (int64_t)r * a.T;
  const float* lr = a.lr ? a.lr + (int64_t)r * a.T : nullptr;
  float x[U], y[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = t0 + u * step + t;
    x[u] = i < a.T ? lp[i] : 0.f;
    y[u] = lr && i < a.T ? lr[i] : 0.f;
  }
  double2 s = {0.0, 0.0};
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (t0 + u * step + t < n) {
      s.x += (double)x[u] - (double)y[u];
      s.y += (double)x[u];
    }
  return s;
}

// Where r stands among its prompt's rewards; one wavefront.
__device__ inline int2 rank_of(const PrefArgs& a, int r, int lane) {
  const int first = r / a.G * a.G;
  const float mine = a.reward[r];
  int less = 0, before = 0, after = 0;   // how many have less, come before r as the best, come before r as the worst
  for (int c0 = 0; c0 < a.G; c0 += 64) {
    const int c = first + c0 + lane;
    const bool have = c0 + lane < a.G;
    const float x = have ? a.reward[c] : 0.f;
    less += __popcll(__ballot(have && x < mine));
    before += __popcll(__ballot(have && (x > mine || (x == mine && c < r))));
    after += __popcll(__ballot(have && (x < mine || (x == mine && c < r))));
  }
  const bool number = mine == mine;
  const int best = number && before == 0, worst = number && after == 0;
  return {a.q.pairs == LMHEAD_PAIRS_ALL ? less : best && less > 0, best | worst << 1};
}

// What the pairs with r come to: w times the slope of its log-ratio, and of those in which it is preferred the number, how often u > 0,
// the loss and the sum of the others' log-ratios.  One wavefront; `total`: pairs of all prompts (weights = 1).
struct Outcome {
  double w, slope, loss, other;
  int won, hit;
};
template <typename Ratio, typename Rank>
__device__ inline Outcome outcome(const PrefArgs& a, int r, double sr, int lane, Ratio&& ratio, Rank&& rank, int64_t total) {
  const lmhead_preference& q = a.q;
  const int first = r / a.G * a.G;
  const bool all = q.pairs == LMHEAD_PAIRS_ALL;
  const double beta = q.beta, smooth = q.smoothing;
  const float mine = a.reward[r];
  const int place = rank(r).y;
  double du = 0.0, l = 0.0, other = 0.0;
  int won = 0, hit = 0;
  int pairs = 0;
  for (int c0 = 0; c0 < a.G; c0 += 64) {
    const int c = first + c0 + lane;
    const bool have = c0 + lane < a.G;
    const float x = have ? a.reward[c] : mine;
    const int2 k = have ? rank(c) : int2{0, 0};
    pairs += k.x;
    const bool up = mine > x && (all || ((place & 1) && (k.y & 2))), down = x > mine && (all || ((k.y & 1) && (place & 2)));
    const double sc = have ? ratio(c) : 0.0, u = up ? sr - sc : sc - sr;   // (asked for without waiting for the rewards)
    if (up || down) {
      double h = beta * u - q.margin;
      if (q.margin_scale != 0.f) h -= (double)q.margin_scale * (up ? (double)mine - x : (double)x - mine);
      double each, d;
      if (q.loss == LMHEAD_PREF_LOGISTIC) {
        // e^-|h| once: log(1 + e^-|h|) for both logarithms, and sigma(-h) from it without overflow.  A term whose factor is 0 is left
        // out: at h = -inf or +inf one of the logarithms is infinite.
        const double e = exp(-fabs(h)), soft = log1p(e), small = e / (1.0 + e);
        each = smooth != 1.0 ? (1.0 - smooth) * (fmax(-h, 0.0) + soft) : 0.0;
        if (smooth != 0.0) each += smooth * (fmax(h, 0.0) + soft);
        d = beta * (smooth - (h > 0.0 ? small : 1.0 - small));
      } else if (q.loss == LMHEAD_PREF_HINGE) {
        each = h >= 1.0 ? 0.0 : 1.0 - h;     // NaN stays
        d = h < 1.0 ? -beta : 0.0;
      } else {
        const double e = h / beta - 0.5 / beta;
        each = e * e;
        d = 2.0 * e;
      }
      du += up ? d : -d;
      if (up) {
        l += each;
        other += sc;
      }
    }
    won += __popcll(__ballot(up));
    hit += __popcll(__ballot(up && u > 0.0));
  }
  const int64_t m = q.weights ? total : (int64_t)wave_sum(pairs) * a.P;
  const double w = m > 0 ? 1.0 / (double)m : 0.0;
  return {w, w * wave_sum(du), wave_sum(l), wave_sum(other), won, hit};
}

// dloss/dlogp of every slot of r.
__device__ inline float slot_gradient(const PrefArgs& a, int r, const Outcome& o) {
  const double each = per_token(a, r);
  double g = o.slope * (a.q.mean ? each : 1.0);
  if (a.q.nll_coef != 0.f) g -= o.w * o.won * a.q.nll_coef * each;
  return (float)g;
}

// What r adds to loss and stats.
constexpr int kParts = 5;
__device__ inline void contribution(const PrefArgs& a, int r, const Outcome& o, double ratio, double logp_sum, double (&p)[kParts]) {
  double l = o.loss;
  if (a.q.nll_coef != 0.f && o.won > 0) l -= o.won * (double)a.q.nll_coef * (logp_sum * per_token(a, r));
  p[0] = o.w * l;
  p[1] = o.hit;
  p[2] = o.won > 0 ? a.q.beta * ratio * o.won : 0.0;
  p[3] = (double)a.q.beta * o.other;
  p[4] = o.won;
}

__device__ inline void put_results(const PrefArgs& a, const double (&v)[kParts]) {
  a.loss[0] = (float)v[0];
  if (!a.stats) return;
  const double pairs = v[4], inv = pairs > 0.0 ? 1.0 / pairs : 0.0;
#pragma unroll
  for (int k = 1; k < 4; ++k) a.stats[k - 1] = (float)(v[k] * inv);
  a.stats[3] = (float)pairs;
}

// Long responses: block (r, b) sums its slots of response r; b = 0 also places r among its prompt's rewards.
__global__ __launch_bounds__(256) void pref_sum_kernel(PrefArgs a) {
  __shared__ double2 sh[4];
  const int r = blockIdx.x / a.nb, b = blockIdx.x % a.nb, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.done = 0;
  double2 s = slot_sums<kLossSlotsPerBlock / 256>(a, r, length(a, r), b * kLossSlotsPerBlock, threadIdx.x, 256);
  if (b == 0 && w == 3) {
    const int2 k = rank_of(a, r, lane);
    if (lane == 0) a.rank[r] = k;
  }
  s.x = wave_sum(s.x);
  s.y = wave_sum(s.y);
  if (lane == 0) sh[w] = s;
  __syncthreads();
  if (threadIdx.x == 0)
    a.sums[(int64_t)r * a.nb + b] = {(sh[0].x + sh[1].x) + (sh[2].x + sh[3].x), (sh[0].y + sh[1].y) + (sh[2].y + sh[3].y)};
}

// Of very long responses a workgroup adds up the blocks of one, which in the gradient's launch each block would do again.
__global__ __launch_bounds__(1024) void pref_join_kernel(PrefArgs a) {
  constexpr int U = 4;
  __shared__ double2 sh[16];
  const double2* from = a.sums + (int64_t)blockIdx.x * a.nb;
  double2 s = {0.0, 0.0};
  for (int b0 = threadIdx.x; b0 < a.nb; b0 += 1024 * U) {
    double2 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = b0 + u * 1024 < a.nb ? from[b0 + u * 1024] : double2{0.0, 0.0};
#pragma unroll
    for (int u = 0; u < U; ++u) {
      s.x += x[u].x;
      s.y += x[u].y;
    }
  }
  s.x = wave_sum(s.x);
  s.y = wave_sum(s.y);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int k = 1; k < 16; ++k) {
    s.x += sh[k].x;
    s.y += sh[k].y;
  }
  a.totals[blockIdx.x] = s;
}

// Sums of all slots of response r; one wavefront.
__device__ inline double2 response_sums(const PrefArgs& a, int r, int lane) {
  constexpr int U = 8;
  const int n = length(a, r);
  double2 s = {0.0, 0.0};
  for (int t0 = 0; t0 < a.T; t0 += 64 * U) {
    const double2 x = slot_sums<U>(a, r, n, t0, lane, 64);
    s.x += x.x;
    s.y += x.y;
  }
  return {wave_sum(s.x), wave_sum(s.y)};
}

// Short ones: a wavefront per response.
__global__ __launch_bounds__(256) void pref_sum_short_kernel(PrefArgs a) {
  const int r = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.done = 0;
  if (r >= a.P * a.G) return;
  const double2 s = response_sums(a, r, lane);
  const int2 k = rank_of(a, r, lane);
  if (lane == 0) {
    a.sums[r] = s;
    a.rank[r] = k;
  }
}

__global__ __launch_bounds__(1024) void pref_count_kernel(PrefArgs a) {
  __shared__ int sh[16];
  int m = 0;
  for (int c = threadIdx.x; c < a.P * a.G; c += 1024) m += a.rank[c].x;
  m = wave_sum(m);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = m;
  __syncthreads();
  if (threadIdx.x == 0) {
    m = 0;
    for (int k = 0; k < 16; ++k) m += sh[k];
    *a.pairs = m;
  }
}

// Loss and statistics from the n parts that all have left, this launch's (kSame: past the caches) or another's; one workgroup of up
// to 16 wavefronts.
template <bool kSame>
__device__ inline void add_up(const PrefArgs& a, int n) {
  __shared__ double sh[16][kParts];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  double v[kParts] = {};
  for (int c = threadIdx.x; c < n; c += blockDim.x)
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
      const double* p = a.part + (int64_t)c * kParts + k;
      v[k] += kSame ? __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : *p;
    }
#pragma unroll
  for (int k = 0; k < kParts; ++k) v[k] = wave_sum(v[k]);
  if (lane == 0)
    for (int k = 0; k < kParts; ++k) sh[w][k] = v[k];
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int q = 1; q < (int)blockDim.x >> 6; ++q)
    for (int k = 0; k < kParts; ++k) v[k] += sh[q][k];
  put_results(a, v);
}

__global__ __launch_bounds__(1024) void pref_final_kernel(PrefArgs a, int n) { add_up<false>(a, n); }

// dloss/dlogp.  kLong: block (r, b) writes its slots of response r, one wavefront looks at r's pairs, and b = 0 leaves what they add to
// loss and stats; otherwise a wavefront per response does all that, and the block leaves the sum of its four.  ticket: the last block to
// leave something adds it all up.
template <bool kLong>
__global__ __launch_bounds__(256) void pref_grad_kernel(PrefArgs a, bool counted, bool ticket) {
  __shared__ float gs;
  __shared__ int last;
  __shared__ double four[4][kParts];
  const int R = a.P * a.G, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int r = kLong ? blockIdx.x / a.nb : blockIdx.x * 4 + w, b = kLong ? blockIdx.x % a.nb : 0;
  const bool have = r < R;
  const int n = have ? length(a, r) : 0;
  auto sums = [&](int c) {
    double2 s = {0.0, 0.0};
    for (int k0 = 0; k0 < a.ns; k0 += 4) {
      double2 x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = a.totals[(int64_t)c * a.ns + min(k0 + k, a.ns - 1)];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k0 + k < a.ns) {
          s.x += x[k].x;
          s.y += x[k].y;
        }
    }
    return s;
  };
  auto ratio = [&](int c) { return sums(c).x * (a.q.mean ? per_token(a, c) : 1.0); };
  float g = 0.f;
  if (have && (!kLong || w == 0)) {
    const double2 mine = sums(r);
    const double sr = mine.x * (a.q.mean ? per_token(a, r) : 1.0);
    int64_t total = 0;
    if (a.q.weights && counted) {
      total = *a.pairs;
    } else if (a.q.weights) {
      int m = 0;
      for (int c = lane; c < R; c += 64) m += a.rank[c].x;
      total = wave_sum(m);
    }
    const Outcome o = outcome(a, r, sr, lane, ratio, [&](int c) { return a.rank[c]; }, total);
    if (b == 0) {
      double p[kParts];
      contribution(a, r, o, sr, mine.y, p);
      if (lane == 0) {
        for (int k = 0; k < kParts; ++k) four[w][k] = p[k];
        if (a.ratio) a.ratio[r] = (float)sr;
      }
    }
    g = slot_gradient(a, r, o);
    if (kLong && lane == 0) gs = g;
  }
  __syncthreads();
  // What all have left is added up by the last one here, or by a launch of its own.  It goes past the caches (a release fence would
  // first write back all of g_logp that L2 holds: 20 us), and has arrived when the count goes up.
  if (b == 0 && w == 0) {
    if (lane < kParts) {
      double p = four[0][lane];
      for (int q = 1; !kLong && q < 4 && (int)blockIdx.x * 4 + q < R; ++q) p += four[q][lane];
      __hip_atomic_store(a.part + (int64_t)(kLong ? r : (int)blockIdx.x) * kParts + lane, p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (ticket) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      if (lane == 0) last = __hip_atomic_fetch_add(a.done, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (kLong ? R : (R + 3) / 4) - 1;
    }
  }
  if (a.g && have) {
    if (kLong) g = gs;
    const int t0 = b * kLossSlotsPerBlock, slots = kLong ? block_slots(t0, a.T) : a.T;
    float* out = a.g + (int64_t)r * a.T + t0;
    for (int k = kLong ? (int)threadIdx.x : lane; k < slots; k += kLong ? 256 : 64) out[k] = t0 + k < n ? g : 0.f;
  }
  if (!ticket || b != 0) return;
  __syncthreads();
  if (last) add_up<true>(a, kLong ? R : (R + 3) / 4);
}

// Few responses of few tokens: one workgroup, a wavefront per response.
__global__ __launch_bounds__(1024) void pref_few_kernel(PrefArgs a) {
  __shared__ double2 sums[kPrefFewResponses];
  __shared__ int2 rank[kPrefFewResponses];
  __shared__ double part[kPrefFewResponses][kParts];
  const int R = a.P * a.G, lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int r = w; r < R; r += 16) {
    const double2 s = response_sums(a, r, lane);
    const int2 k = rank_of(a, r, lane);
    if (lane == 0) {
      sums[r] = s;
      rank[r] = k;
    }
  }
  __syncthreads();
  int m = 0;
  for (int c = lane; c < R; c += 64) m += rank[c].x;
  m = wave_sum(m);
  auto ratio = [&](int c) { return sums[c].x * (a.q.mean ? per_token(a, c) : 1.0); };
  for (int r = w; r < R; r += 16) {
    const double sr = ratio(r);
    const Outcome o = outcome(a, r, sr, lane, ratio, [&](int c) { return rank[c]; }, m);
    const float g = slot_gradient(a, r, o);
    const int n = length(a, r);
    if (a.g)
      for (int t = lane; t < a.T; t += 64) a.g[(int64_t)r * a.T + t] = t < n ? g : 0.f;
    if (lane == 0) {
      double p[kParts];
      contribution(a, r, o, sr, sums[r].y, p);
      for (int k = 0; k < kParts; ++k) part[r][k] = p[k];
      if (a.ratio) a.ratio[r] = (float)sr;
    }
  }
  __syncthreads();
  if (w != 0) return;
  double v[kParts] = {};
  for (int c = lane; c < R; c += 64)
    for (int k = 0; k < 4; ++k) v[k] += part[c][k];
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = wave_sum(v[k]);
  v[4] = m;
  if (lane == 0) put_results(a, v);
}

}  // namespace

hipError_t launch_preference(const lmhead_preference& q, const float* lp, const float* lr, const float* reward, const int32_t* len,
                             int P, int G, int T, float* loss, float* g, float* ratio, float* stats, char* ws, hipStream_t s) {
  const PrefLayout L = pref_layout(P, G, T);
  PrefArgs a{lp, lr, reward, len, P, G, T, (int)L.nb, (int)L.nb, q};
  a.sums = a.totals = reinterpret_cast<double2*>(ws + L.sums);
  a.rank = reinterpret_cast<int2*>(ws + L.rank);
  a.part = reinterpret_cast<double*>(ws + L.part);
  a.done = reinterpret_cast<int32_t*>(ws + L.done);
  a.pairs = a.done + 1;
  a.loss = loss;
  a.g = g;
  a.ratio = ratio;
  a.stats = stats;
  if (L.R <= kPrefFewResponses && L.R * T <= kPrefFewSlots) {
    hipLaunchKernelGGL(pref_few_kernel, dim3(1), dim3(1024), 0, s, a);
    return hipGetLastError();
  }
  // few responses, or long ones, are spread over workgroups; many short ones are a wavefront each
  const bool shorts = T <= kPrefShort && L.R > kPrefTickets;
  const int parts = (int)(shorts ? (L.R + 3) / 4 : L.R);
  const dim3 grid((unsigned)(shorts ? parts : L.R * L.nb));
  if (shorts) hipLaunchKernelGGL(pref_sum_short_kernel, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(pref_sum_kernel, grid, dim3(256), 0, s, a);
  if (L.nb > kPrefBlocks) {
    a.totals = reinterpret_cast<double2*>(ws + L.totals);
    a.ns = 1;
    hipLaunchKernelGGL(pref_join_kernel, dim3((unsigned)L.R), dim3(1024), 0, s, a);
  }
  // every workgroup adds up the pairs of few prompts itself
  const bool counted = q.weights && L.R > kPrefCounted;
  if (counted) hipLaunchKernelGGL(pref_count_kernel, dim3(1), dim3(1024), 0, s, a);
  // counts that meet on one word cost some 20 ns each: a launch is quicker than many
  const bool ticket = parts <= kPrefTickets;
  if (shorts) hipLaunchKernelGGL(pref_grad_kernel<false>, grid, dim3(256), 0, s, a, counted, ticket);
  else hipLaunchKernelGGL(pref_grad_kernel<true>, grid, dim3(256), 0, s, a, counted, ticket);
  if (!ticket) hipLaunchKernelGGL(pref_final_kernel, dim3(1), dim3(1024), 0, s, a, parts);
  return hipGetLastError();
}

}  // namespace lmhead
