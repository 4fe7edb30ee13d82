// The norm over many gradients and their clipping.  One pass for the sum of squares, one that scales; the second derives the norm from the
// first one's partial sums itself.  The table of tensors travels in the launch's arguments: nothing is uploaded, and a captured call
// holds it.
#include "train_common.h"

namespace lmhead {

namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;

constexpr int kChunk = 8192;   // elements of a tensor that a workgroup takes at a time

__device__ inline double wave_sum(double x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
  return x;
}
__device__ inline double block_sum(double x, double* sh) {
  x = wave_sum(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
  __syncthreads();
  return (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

enum { kBf16In = 1, kBf16Out = 2, kAligned = 4 };
struct GradTable {
  const void* in[kGradTensors];
  void* out[kGradTensors];
  int64_t n[kGradTensors];
  int32_t first[kGradTensors + 1];   // number of its first chunk among those of this launch
  uint8_t how[kGradTensors];
  int count;
};
static_assert(sizeof(GradTable) < 3500, "kernel arguments");

// Tensor that chunk c lies in.
__device__ inline int tensor_of(const GradTable& t, int c) {
  int lo = 0, hi = t.count;      // first[lo] <= c < first[hi]
  while (hi - lo > 1) {
    const int m = (lo + hi) >> 1;
    if (t.first[m] <= c) lo = m;
    else hi = m;
  }
  return lo;
}

template <typename T>
__device__ inline double squares(const T* p, int n, bool aligned) {
  constexpr int E = 16 / (int)sizeof(T);
  typedef __attribute__((ext_vector_type(E))) T vec;
  double s = 0.0;
  int i = 0;
  if (aligned) {
    for (i = threadIdx.x * E; i + E <= n; i += 256 * E) {
      const vec x = *reinterpret_cast<const vec*>(p + i);
#pragma unroll
      for (int k = 0; k < E; ++k) {
        const double y = (double)(float)x[k];
        s = fma(y, y, s);
      }
    }
    i = n / E * E;
  }
  for (i += threadIdx.x; i < n; i += 256) {
    const double y = (double)(float)p[i];
    s = fma(y, y, s);
  }
  return s;
}

__global__ __launch_bounds__(256) void grad_norm_kernel(GradTable t, double* part) {
  __shared__ double sh[4];
  const int chunks = t.first[t.count];
  double s = 0.0;
  for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int i = tensor_of(t, c);
    const int64_t at = (int64_t)(c - t.first[i]) * kChunk;
    const int n = (int)(t.n[i] - at < kChunk ? t.n[i] - at : kChunk);
    if (t.how[i] & kBf16In) s += squares(static_cast<const __bf16*>(t.in[i]) + at, n, t.how[i] & kAligned);
    else s += squares(static_cast<const float*>(t.in[i]) + at, n, t.how[i] & kAligned);
  }
  s = block_sum(s, sh);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__device__ inline double norm_of(const double* part, int parts, double* sh) {
  double s = 0.0;
  for (int i = threadIdx.x; i < parts; i += 256) s += part[i];
  return sqrt(block_sum(s, sh));
}

__global__ __launch_bounds__(256) void grad_final_kernel(const double* part, int parts, float* norm) {
  __shared__ double sh[4];
  const double n = norm_of(part, parts, sh);
  if (threadIdx.x == 0) norm[0] = (float)n;
}

template <typename TI, typename TO>
__device__ inline void scaled(const TI* p, TO* q, int n, bool aligned, float c) {
  constexpr int E = 16 / (int)(sizeof(TI) < sizeof(TO) ? sizeof(TO) : sizeof(TI));
  typedef __attribute__((ext_vector_type(E))) TI veci;
  typedef __attribute__((ext_vector_type(E))) TO veco;
  int i = 0;
  if (aligned) {
    for (i = threadIdx.x * E; i + E <= n; i += 256 * E) {
      const veci x = *reinterpret_cast<const veci*>(p + i);
      veco y;
#pragma unroll
      for (int k = 0; k < E; ++k) y[k] = (TO)((float)x[k] * c);
      *reinterpret_cast<veco*>(q + i) = y;
    }
    i = n / E * E;
  }
  for (i += threadIdx.x; i < n; i += 256) q[i] = (TO)((float)p[i] * c);
}

__global__ __launch_bounds__(256) void grad_clip_kernel(GradTable t, const double* part, int parts, float max_norm, float eps,
                                                        float* norm) {
  __shared__ double sh[4];
  const double n = norm_of(part, parts, sh);
  const double ratio = (double)max_norm / (n + (double)eps);
  const float c = (float)(ratio >= 1.0 ? 1.0 : ratio);     // NaN stays
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) {
    norm[0] = (float)n;
    norm[1] = c;
  }
  const int chunks = t.first[t.count];
  for (int k = blockIdx.x; k < chunks; k += gridDim.x) {
    const int i = tensor_of(t, k);
    if (c == 1.f && t.in[i] == t.out[i]) continue;
    const int64_t at = (int64_t)(k - t.first[i]) * kChunk;
    const int m = (int)(t.n[i] - at < kChunk ? t.n[i] - at : kChunk);
    const bool al = t.how[i] & kAligned;
    const float* pf = static_cast<const float*>(t.in[i]) + at;
    const __bf16* pb = static_cast<const __bf16*>(t.in[i]) + at;
    float* qf = static_cast<float*>(t.out[i]) + at;
    __bf16* qb = static_cast<__bf16*>(t.out[i]) + at;
    switch (t.how[i] & (kBf16In | kBf16Out)) {
      case 0: scaled(pf, qf, m, al, c); break;
      case kBf16In: scaled(pb, qf, m, al, c); break;
      case kBf16Out: scaled(pf, qb, m, al, c); break;
      default: scaled(pb, qb, m, al, c); break;
    }
  }
}

}  // namespace

hipError_t launch_grads(const lmhead_tensor* g, const lmhead_tensor* out, int count, bool clip, float max_norm, float eps, float* norm,
                        char* ws, hipStream_t s) {
  double* part = reinterpret_cast<double*>(ws);
  int64_t total = 0;
  for (int i = 0; i < count; ++i) total += (g[i].n + kChunk - 1) / kChunk;
  int parts = 0;
  // both passes go through the tensors in the same launches
  for (int pass = 0; pass < (clip ? 2 : 1); ++pass) {
    for (int at = 0; at < count;) {
      GradTable t;
      int64_t chunks = 0;
      int k = 0;
      for (; at < count && k < kGradTensors; ++at) {
        const int64_t c = (g[at].n + kChunk - 1) / kChunk;
        const lmhead_tensor& o = out ? out[at] : g[at];
        t.in[k] = g[at].data;
        t.out[k] = o.data;
        t.n[k] = g[at].n;
        t.first[k] = (int32_t)chunks;
        const bool aligned = ((reinterpret_cast<uintptr_t>(g[at].data) | (pass ? reinterpret_cast<uintptr_t>(o.data) : 0)) & 15) == 0;
        t.how[k] = (uint8_t)((g[at].dtype == LMHEAD_BF16 ? kBf16In : 0) | (o.dtype == LMHEAD_BF16 ? kBf16Out : 0) | (aligned ? kAligned : 0));
        chunks += c;
        ++k;
      }
      t.first[k] = (int32_t)chunks;
      t.count = k;
      if (pass == 0) {
        int wgs = (int)(chunks * kGradParts / (total > kGradParts ? total : kGradParts));
        if (wgs < 1) wgs = 1;
        hipLaunchKernelGGL(grad_norm_kernel, dim3(wgs), dim3(256), 0, s, t, part + parts);
        parts += wgs;
      } else {
        int64_t wgs = chunks < 4096 ? chunks : 4096;
        if (wgs < 1) wgs = 1;
        hipLaunchKernelGGL(grad_clip_kernel, dim3((unsigned)wgs), dim3(256), 0, s, t, part, parts, max_norm, eps,
                           at == count ? norm : nullptr);
      }
    }
  }
  if (!clip) hipLaunchKernelGGL(grad_final_kernel, dim3(1), dim3(256), 0, s, part, parts, norm);
  return hipGetLastError();
}

}  // namespace lmhead
