// The norm over many gradients and their clipping: one pass for the sum of squares, one that scales.  Nothing is computed, so both are
// bound by memory; a large set is read twice, since the factor is known only at the end of the first pass.
//  - Squares and sums are fp64: no square of an fp32 number overflows or vanishes there, and the sum does not depend on the sizes.
//  - The table of tensors travels in a launch's arguments (nothing is uploaded, a captured call holds it); of more than kGradTensors
//    tensors parts of it are first copied into the workspace, so that each pass stays one launch.
#include "train_common.h"

namespace lmhead {

namespace {

template <typename T, int N>
struct Vec {
  typedef __attribute__((ext_vector_type(N))) T type;
};

__device__ inline double wave_sum(double x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

// Sum over a workgroup of up to 16 wavefronts, valid in every thread.
__device__ inline double block_sum(double x) {
  __shared__ double sh[16];
  x = wave_sum(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
  __syncthreads();
  double s = 0.0;
  for (int i = 0; i < (int)blockDim.x >> 6; ++i) s += sh[i];
  return s;
}

enum { kBf16In = 1, kBf16Out = 2, kAligned = 4 };

// A tensor, and the number of its first chunk among those of all.
struct GradEntry {
  const void* in;
  void* out;
  int64_t n;
  uint32_t first, how;
};
static_assert(sizeof(GradEntry) == kGradEntryBytes, "workspace");

struct ArgTable {
  GradEntry e[kGradTensors];
  int count;
  uint32_t chunks;
  __device__ inline const GradEntry& at(int i) const { return e[i]; }
};
static_assert(sizeof(ArgTable) <= 3200, "kernel arguments");
struct WsTable {
  const GradEntry* e;
  int count;
  uint32_t chunks;
  __device__ inline const GradEntry& at(int i) const { return e[i]; }
};

// A part of a table on its way into the workspace: as many tensors as arguments hold (4 KB), their first chunks counted on arrival.
constexpr int kUpload = 164;
struct Upload {
  const void* in[kUpload];
  void* out[kUpload];
  uint64_t n_how[kUpload];   // elements, and how << 60
  int count;
  uint32_t base;             // chunks before these
};
static_assert(sizeof(Upload) <= 4000 && (kGradMost >> 60) == 0, "kernel arguments");
__global__ __launch_bounds__(256) void grad_table_kernel(Upload t, GradEntry* to) {
  __shared__ uint32_t sums[4];
  const int i = threadIdx.x, lane = i & 63, w = i >> 6;
  const uint64_t nh = i < t.count ? t.n_how[i] : 0;
  const int64_t n = (int64_t)(nh & ((1ull << 60) - 1));
  const uint32_t mine = (uint32_t)((n + kGradChunk - 1) / kGradChunk);
  uint32_t s = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t y = __shfl_up(s, o);
    if (lane >= o) s += y;
  }
  if (lane == 63) sums[w] = s;
  __syncthreads();
  for (int k = 0; k < w; ++k) s += sums[k];
  if (i < t.count) to[i] = GradEntry{t.in[i], t.out[i], n, t.base + s - mine, (uint32_t)(nh >> 60)};
}

// Tensor that chunk c lies in, one of lo .. hi - 1: first of lo <= c, and of hi (were there one more) > c.
template <typename Table>
__device__ inline int tensor_of(const Table& t, uint32_t c, int lo, int hi) {
  while (hi - lo > 1) {
    const int m = (lo + hi) >> 1;
    if (t.at(m).first <= c) lo = m;
    else hi = m;
  }
  return lo;
}

// Squares of p[0 .. n) by `threads` threads, this one being number t.
template <typename T>
__device__ inline double squares(const T* p, int n, bool aligned, int t, int threads) {
  constexpr int E = 16 / (int)sizeof(T), U = 8;
  typedef typename Vec<T, E>::type vec;
  double s = 0.0;
  int i = 0;
  if (aligned) {
    const int whole = n / E * E;
    for (i = t * E; i < whole; i += threads * E * U) {
      vec x[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i + u * threads * E < whole) x[u] = __builtin_nontemporal_load(reinterpret_cast<const vec*>(p + i + u * threads * E));
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i + u * threads * E < whole) {
#pragma unroll
          for (int k = 0; k < E; ++k) {
            const double y = (double)(float)x[u][k];
            s = fma(y, y, s);
          }
        }
    }
    i = whole;
  }
  for (i += t; i < n; i += threads) {
    const double y = (double)(float)p[i];
    s = fma(y, y, s);
  }
  return s;
}

__device__ inline double squares_of(const GradEntry& e, int64_t at, int most, int t, int threads) {
  const int n = (int)(e.n - at < most ? e.n - at : most);
  if (e.how & kBf16In) return squares(static_cast<const __bf16*>(e.in) + at, n, e.how & kAligned, t, threads);
  return squares(static_cast<const float*>(e.in) + at, n, e.how & kAligned, t, threads);
}

// Workgroup b takes chunks b * each .. and leaves the tensor in which they begin, where the second pass starts to look.
// 3.0 GB (the head's dW beside a few layers) in 435 us: 6.9 TB/s, a bare loop of loads 7.0; through the caches 6.0.
template <typename Table>
__global__ __launch_bounds__(256) void grad_norm_kernel(Table t, uint32_t each, double* part, int32_t* begins) {
  double s = 0.0;
  const uint32_t lo = blockIdx.x * each, hi = lo + each < t.chunks ? lo + each : t.chunks;
  if (lo < hi) {
    int i = tensor_of(t, lo, 0, t.count);
    if (threadIdx.x == 0) begins[blockIdx.x] = i;
    for (uint32_t c = lo; c < hi; ++c) {
      while (i + 1 < t.count && t.at(i + 1).first <= c) ++i;
      s += squares_of(t.at(i), (int64_t)(c - t.at(i).first) * kGradChunk, kGradChunk, threadIdx.x, 256);
    }
  }
  s = block_sum(s);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

struct Clip {
  float max_norm, eps;
  float* norm;       // norm[0], norm[1] of the caller
};

__device__ inline float factor(double n, const Clip& k) {
  const double ratio = (double)k.max_norm / (n + (double)k.eps);
  return (float)(ratio >= 1.0 ? 1.0 : ratio);     // NaN stays
}

__device__ inline double norm_of(const double* part, int parts) {
  double s = 0.0;
  for (int i = threadIdx.x; i < parts; i += blockDim.x) s += part[i];
  return sqrt(block_sum(s));
}

// The norm, and with `clip` the factor.
__global__ __launch_bounds__(1024) void grad_final_kernel(const double* part, int parts, Clip k, bool clip) {
  const double n = norm_of(part, parts);
  if (threadIdx.x != 0) return;
  k.norm[0] = (float)n;
  if (clip) k.norm[1] = factor(n, k);
}

template <typename TI, typename TO>
__device__ inline void scaled(const TI* p, TO* q, int n, bool aligned, float c, int t, int threads) {
  constexpr int E = 16 / (int)(sizeof(TI) < sizeof(TO) ? sizeof(TO) : sizeof(TI)), U = 4;
  typedef typename Vec<TI, E>::type veci;
  typedef typename Vec<TO, E>::type veco;
  int i = 0;
  if (aligned) {
    const int whole = n / E * E;
    for (i = t * E; i < whole; i += threads * E * U) {
      veci x[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i + u * threads * E < whole) x[u] = __builtin_nontemporal_load(reinterpret_cast<const veci*>(p + i + u * threads * E));
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i + u * threads * E < whole) {
          veco y;
#pragma unroll
          for (int k = 0; k < E; ++k) y[k] = (TO)((float)x[u][k] * c);
          __builtin_nontemporal_store(y, reinterpret_cast<veco*>(q + i + u * threads * E));
        }
    }
    i = whole;
  }
  for (i += t; i < n; i += threads) q[i] = (TO)((float)p[i] * c);
}

__device__ inline void scaled_of(const GradEntry& e, int64_t at, int most, float c, int t, int threads) {
  if (at >= e.n || (c == 1.f && e.in == e.out)) return;
  const int n = (int)(e.n - at < most ? e.n - at : most);
  const bool al = e.how & kAligned;
  const float* pf = static_cast<const float*>(e.in) + at;
  const __bf16* pb = static_cast<const __bf16*>(e.in) + at;
  float* qf = static_cast<float*>(e.out) + at;
  __bf16* qb = static_cast<__bf16*>(e.out) + at;
  switch (e.how & (kBf16In | kBf16Out)) {
    case 0: scaled(pf, qf, n, al, c, t, threads); break;
    case kBf16In: scaled(pb, qf, n, al, c, t, threads); break;
    case kBf16Out: scaled(pf, qb, n, al, c, t, threads); break;
    default: scaled(pb, qb, n, al, c, t, threads); break;
  }
}

// A part of a chunk per workgroup: two vectors a thread.  790 million elements in 1007 us, 6.1 TB/s, a bare copy of
// one vector a thread 6.6; whole chunks 1090, halves 1065, eighths as quarters, but slower where tensors are many.  Looking the tensor up
// from the first pass's place on instead of among all: 290 tensors 270 -> 209 us.
// shared: each workgroup derives the factor from the partial sums, and the first one writes
// the norm; otherwise grad_final_kernel has done both.
template <typename Table>
__global__ __launch_bounds__(256) void grad_clip_kernel(Table t, uint32_t each, const double* part, const int32_t* begins, int parts,
                                                        bool shared, Clip k) {
  const uint32_t wg = grid_wg(), chunk = wg / kClipParts, b = chunk / each;
  if (chunk >= t.chunks) return;
  const GradEntry& e = t.at(tensor_of(t, chunk, begins[b], (b + 1 < (uint32_t)parts ? begins[b + 1] : t.count - 1) + 1));
  float c;
  if (shared) {
    const double n = norm_of(part, parts);
    c = factor(n, k);
    if (wg == 0 && threadIdx.x == 0) {
      k.norm[0] = (float)n;
      k.norm[1] = c;
    }
  } else {
    c = k.norm[1];
  }
  scaled_of(e, (int64_t)(chunk - e.first) * kGradChunk + wg % kClipParts * (kGradChunk / kClipParts), kGradChunk / kClipParts, c,
            threadIdx.x, 256);
}

// A small set in one launch: a wavefront per chunk, sixteen of them.
__global__ __launch_bounds__(1024) void grad_few_kernel(ArgTable t, Clip k, bool clip) {
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  double s = 0.0;
  for (uint32_t c = w; c < t.chunks; c += 16) {
    const GradEntry& e = t.at(tensor_of(t, c, 0, t.count));
    s += squares_of(e, (int64_t)(c - e.first) * kFewChunk, kFewChunk, lane, 64);
  }
  const double n = sqrt(block_sum(s));
  const float f = clip ? factor(n, k) : 1.f;
  if (threadIdx.x == 0) {
    k.norm[0] = (float)n;
    if (clip) k.norm[1] = f;
  }
  if (!clip) return;
  for (uint32_t c = w; c < t.chunks; c += 16) {
    const GradEntry& e = t.at(tensor_of(t, c, 0, t.count));
    scaled_of(e, (int64_t)(c - e.first) * kFewChunk, kFewChunk, f, lane, 64);
  }
}

}  // namespace

hipError_t launch_grads(const lmhead_tensor* g, const lmhead_tensor* out, int count, bool clip, float max_norm, float eps, float* norm,
                        char* ws, hipStream_t s) {
  const Clip k{max_norm, eps, norm};
  GradEntry* const table = reinterpret_cast<GradEntry*>(ws);
  double* const part = reinterpret_cast<double*>(ws + grad_table_bytes());
  int32_t* const begins = reinterpret_cast<int32_t*>(part + kGradParts);
  const bool args = count <= kGradTensors;
  int64_t small = 0;
  for (int i = 0; args && i < count && small <= kGradFew; ++i) small += (g[i].n + kFewChunk - 1) / kFewChunk;
  const bool few = args && small <= kGradFew;
  const int64_t size = few ? kFewChunk : kGradChunk;
  uint32_t chunks = 0;
  auto entry = [&](int i) {
    const lmhead_tensor& o = out ? out[i] : g[i];
    const bool aligned = ((reinterpret_cast<uintptr_t>(g[i].data) | (clip ? reinterpret_cast<uintptr_t>(o.data) : 0)) & 15) == 0;
    const GradEntry e{g[i].data, o.data, g[i].n, chunks,
                      (g[i].dtype == LMHEAD_BF16 ? kBf16In : 0u) | (o.dtype == LMHEAD_BF16 ? kBf16Out : 0u) | (aligned ? kAligned : 0u)};
    chunks += (uint32_t)((g[i].n + size - 1) / size);
    return e;
  };
  ArgTable t;
  t.count = 0;
  if (args) {
    while (t.count < count) {
      t.e[t.count] = entry(t.count);
      ++t.count;
    }
  } else {
    for (int at = 0; at < count;) {
      Upload u;
      u.base = chunks;
      GradEntry* const to = table + at;
      for (u.count = 0; at < count && u.count < kUpload; ++at, ++u.count) {
        const GradEntry e = entry(at);
        u.in[u.count] = e.in;
        u.out[u.count] = e.out;
        u.n_how[u.count] = (uint64_t)e.n | (uint64_t)e.how << 60;
      }
      hipLaunchKernelGGL(grad_table_kernel, dim3(1), dim3(256), 0, s, u, to);
    }
  }
  t.chunks = chunks;
  if (few || chunks == 0) {
    hipLaunchKernelGGL(grad_few_kernel, dim3(1), dim3(1024), 0, s, t, k, clip);
    return hipGetLastError();
  }
  const WsTable wt{table, count, chunks};
  uint32_t each = chunks / kGradSpread;
  each = each < 1 ? 1 : each > kGradEach ? kGradEach : each;
  if ((chunks + each - 1) / each > kGradParts) each = (chunks + kGradParts - 1) / kGradParts;
  const int parts = (int)((chunks + each - 1) / each);
  if (args) hipLaunchKernelGGL(grad_norm_kernel<ArgTable>, dim3((unsigned)parts), dim3(256), 0, s, t, each, part, begins);
  else hipLaunchKernelGGL(grad_norm_kernel<WsTable>, dim3((unsigned)parts), dim3(256), 0, s, wt, each, part, begins);
  const bool shared = clip && parts <= kGradShared;
  if (!shared) hipLaunchKernelGGL(grad_final_kernel, dim3(1), dim3(1024), 0, s, part, parts, k, clip);
  if (!clip) return hipGetLastError();
  const dim3 grid = grid_of((int64_t)chunks * kClipParts);
  if (args) hipLaunchKernelGGL(grad_clip_kernel<ArgTable>, grid, dim3(256), 0, s, t, each, part, begins, parts, shared, k);
  else hipLaunchKernelGGL(grad_clip_kernel<WsTable>, grid, dim3(256), 0, s, wt, each, part, begins, parts, shared, k);
  return hipGetLastError();
}

}  // namespace lmhead
