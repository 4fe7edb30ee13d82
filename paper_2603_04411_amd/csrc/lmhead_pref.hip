// Preference loss: one pass over the log-probabilities for the sums of the responses, one over the gradient.
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

// Sum over a 256-thread block, valid in every thread; sh[4] is free again after the next barrier.
template <typename T>
__device__ inline T block_sum(T x, T* sh) {
  x = wave_sum(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
  __syncthreads();
  return (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

struct PrefArgs {
  const float* lp;
  const float* lr;
  const float* reward;
  const int32_t* len;
  int P, G, T, nb;
  lmhead_preference q;
  double* sums;
  int32_t* rank;
  double* part;
  int32_t* done;
  float* loss;
  float* g;
  float* ratio;
  float* stats;
};

// Block (r, b): sums over its slots of response r; b = 0 also places r among its prompt's rewards.
__global__ __launch_bounds__(256) void pref_sum_kernel(PrefArgs a) {
  __shared__ double sh[4];
  __shared__ int shi[4];
  const int r = blockIdx.x / a.nb, b = blockIdx.x % a.nb;
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.done = 0;
  const int n = min(max(a.len[r], 0), a.T);
  double s = 0.0, l = 0.0;
  const int t0 = b * kLossSlotsPerBlock;
  for (int t = t0 + threadIdx.x; t < min(t0 + kLossSlotsPerBlock, n); t += 256) {
    const int64_t i = (int64_t)r * a.T + t;
    const double x = a.lp[i];
    l += x;
    s += a.lr ? x - (double)a.lr[i] : x;
  }
  s = block_sum(s, sh);
  l = block_sum(l, sh);
  if (threadIdx.x == 0) {
    a.sums[((int64_t)r * a.nb + b) * 2] = s;
    a.sums[((int64_t)r * a.nb + b) * 2 + 1] = l;
  }
  if (b != 0) return;
  const int first = r / a.G * a.G;
  const float mine = a.reward[r];
  int less = 0, before = 0, after = 0;   // how many have less, come before r as the best, come before r as the worst
  for (int c = first + threadIdx.x; c < first + a.G; c += 256) {
    const float x = a.reward[c];
    less += x < mine;
    before += x > mine || (x == mine && c < r);
    after += x < mine || (x == mine && c < r);
  }
  less = block_sum(less, shi);
  before = block_sum(before, shi);
  after = block_sum(after, shi);
  if (threadIdx.x == 0) {
    const bool number = mine == mine;
    const int best = number && before == 0, worst = number && after == 0;
    a.rank[2 * r] = a.q.pairs == LMHEAD_PAIRS_ALL ? less : (best && less > 0);
    a.rank[2 * r + 1] = best | worst << 1;
  }
}

// Block (r, b): dloss/dlogp on its slots of response r; b = 0 also what the pairs with r preferred add to loss and stats, and
// the last block sums those.
__global__ __launch_bounds__(256) void pref_grad_kernel(PrefArgs a) {
  __shared__ double sh[4];
  __shared__ long long shl[4];
  __shared__ int last;
  const lmhead_preference q = a.q;
  const int r = blockIdx.x / a.nb, b = blockIdx.x % a.nb, R = a.P * a.G;
  const int first = r / a.G * a.G;
  auto response = [&](int c, int which) {
    double s = 0.0;
    for (int k = 0; k < a.nb; ++k) s += a.sums[((int64_t)c * a.nb + k) * 2 + which];
    return s;
  };
  auto per_token = [&](int c) {
    const int n = min(max(a.len[c], 0), a.T);
    return n > 0 ? 1.0 / n : 0.0;
  };
  // pairs: of the prompt, or of all prompts
  double pairs = 0.0;
  for (int c = (q.weights ? 0 : first) + (int)threadIdx.x; c < (q.weights ? R : first + a.G); c += 256) pairs += a.rank[2 * c];
  pairs = block_sum(pairs, sh);
  const double w = pairs > 0.0 ? 1.0 / (q.weights ? pairs : pairs * a.P) : 0.0;

  const double sr = response(r, 0) * (q.mean ? per_token(r) : 1.0), like = response(r, 1) * per_token(r);
  const double beta = q.beta, smooth = q.smoothing;
  const float mine = a.reward[r];
  const int best_r = a.rank[2 * r + 1];
  double du = 0.0, won = 0.0, l = 0.0, hit = 0.0, other = 0.0;
  for (int c = first + threadIdx.x; c < first + a.G; c += 256) {
    const float x = a.reward[c];
    const int best_c = a.rank[2 * c + 1];
    const bool up = mine > x && (q.pairs == LMHEAD_PAIRS_ALL || ((best_r & 1) && (best_c & 2)));
    const bool down = x > mine && (q.pairs == LMHEAD_PAIRS_ALL || ((best_c & 1) && (best_r & 2)));
    if (!up && !down) continue;
    const double sc = response(c, 0) * (q.mean ? per_token(c) : 1.0);
    const double u = up ? sr - sc : sc - sr;
    double h = beta * u - q.margin;
    if (q.margin_scale != 0.f) h -= (double)q.margin_scale * (up ? (double)mine - x : (double)x - mine);
    double each, d;
    if (q.loss == LMHEAD_PREF_LOGISTIC) {
      // e^-|h| once: log(1 + e^-|h|) for both logarithms, and sigma(-h) from it without overflow
      const double e = exp(-fabs(h)), soft = log1p(e), small = e / (1.0 + e);
      each = (1.0 - smooth) * (fmax(-h, 0.0) + soft);
      if (smooth != 0.0) each += smooth * (fmax(h, 0.0) + soft);
      d = beta * (smooth - (h > 0.0 ? small : 1.0 - small));
    } else if (q.loss == LMHEAD_PREF_HINGE) {
      each = h >= 1.0 ? 0.0 : 1.0 - h;     // NaN stays
      d = h >= 1.0 ? 0.0 : -beta;
    } else {
      const double e = h / beta - 0.5 / beta;
      each = e * e;
      d = 2.0 * e;
    }
    du += up ? d : -d;
    if (up) {
      won += 1.0;
      l += each;
      hit += u > 0.0 ? 1.0 : 0.0;
      other += sc;
    }
  }
  du = block_sum(du, sh);
  won = block_sum(won, sh);
  if (a.g) {
    double g = w * du * (q.mean ? per_token(r) : 1.0);
    if (q.nll_coef != 0.f) g -= w * won * q.nll_coef * per_token(r);
    const float gf = (float)g;
    const int n = min(max(a.len[r], 0), a.T), t0 = b * kLossSlotsPerBlock;
    for (int t = t0 + threadIdx.x; t < min(t0 + kLossSlotsPerBlock, a.T); t += 256) a.g[(int64_t)r * a.T + t] = t < n ? gf : 0.f;
  }
  if (b != 0) return;
  l = block_sum(l, sh);
  hit = block_sum(hit, sh);
  other = block_sum(other, sh);
  if (threadIdx.x == 0) {
    if (q.nll_coef != 0.f && won > 0.0) l -= won * q.nll_coef * like;
    double* p = a.part + (int64_t)r * 4;
    p[0] = w * l;
    p[1] = hit;
    p[2] = won > 0.0 ? beta * sr * won : 0.0;
    p[3] = beta * other;
    if (a.ratio) a.ratio[r] = (float)sr;
  }
}

__global__ __launch_bounds__(256) void pref_final_kernel(PrefArgs a) {
  __shared__ double sh[4];
  const int R = a.P * a.G;
  double v[4] = {}, m = 0.0;
  for (int r = threadIdx.x; r < R; r += 256) {
    for (int c = 0; c < 4; ++c) v[c] += a.part[(int64_t)r * 4 + c];
    m += a.rank[2 * r];
  }
  for (int c = 0; c < 4; ++c) v[c] = block_sum(v[c], sh);
  m = block_sum(m, sh);
  if (threadIdx.x != 0) return;
  a.loss[0] = (float)v[0];
  if (!a.stats) return;
  const double inv = m > 0.0 ? 1.0 / m : 0.0;
  for (int c = 1; c < 4; ++c) a.stats[c - 1] = (float)(v[c] * inv);
  a.stats[3] = (float)m;
}

}  // namespace

hipError_t launch_preference(const lmhead_preference& q, const float* lp, const float* lr, const float* reward, const int32_t* len,
                             int P, int G, int T, float* loss, float* g, float* ratio, float* stats, char* ws, hipStream_t s) {
  const PrefLayout L = pref_layout(P, G, T);
  PrefArgs a{lp, lr, reward, len, P, G, T, (int)L.nb, q};
  a.sums = reinterpret_cast<double*>(ws + L.sums);
  a.rank = reinterpret_cast<int32_t*>(ws + L.rank);
  a.part = reinterpret_cast<double*>(ws + L.part);
  a.done = reinterpret_cast<int32_t*>(ws + L.done);
  a.loss = loss;
  a.g = g;
  a.ratio = ratio;
  a.stats = stats;
  const dim3 grid((unsigned)(L.R * L.nb));
  hipLaunchKernelGGL(pref_sum_kernel, grid, dim3(256), 0, s, a);
  hipLaunchKernelGGL(pref_grad_kernel, grid, dim3(256), 0, s, a);
  hipLaunchKernelGGL(pref_final_kernel, dim3(1), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace lmhead
