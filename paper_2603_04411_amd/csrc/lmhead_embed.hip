// Rows of a matrix by token id, and the gradient of that matrix.
//
// The gradient is a sum over the slots of each id.  Atomic additions would make its rounding depend on their order, and meet on the few
// ids that make up most of a text; instead the slots are sorted by (id, slot) - a stable radix sort of N keys, small next to the N rows -
// and the rows of an id, then neighbours, are summed in registers.
#include "train_common.h"

namespace lmhead {

namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;

// Eight neighbouring values of a row, in fp32.
template <typename T>
struct Row8;
template <>
struct Row8<float> {
  f32x4 a, b;
  __device__ inline void load(const float* p) {
    a = *reinterpret_cast<const f32x4*>(p);
    b = *reinterpret_cast<const f32x4*>(p + 4);
  }
  __device__ inline void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
  }
  __device__ static inline void store(float* p, const float (&v)[8]) {
    *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
  }
};
template <>
struct Row8<__bf16> {
  bf16x8 a;
  __device__ inline void load(const __bf16* p) { a = *reinterpret_cast<const bf16x8*>(p); }
  __device__ inline void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)a[i];
  }
  __device__ static inline void store(__bf16* p, const float (&v)[8]) {
    bf16x8 t;
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = (__bf16)v[i];
    *reinterpret_cast<bf16x8*>(p) = t;
  }
};

struct Batch {
  const int32_t* tok;
  const int32_t* len;   // or null: every slot counts
  int R, T, V;
};

// Id of a slot, V where it does not count; error bits of what it met.
__device__ inline uint32_t id_of(const Batch& b, int64_t i, int& err) {
  const int r = (int)((uint32_t)i / (uint32_t)b.T), t = (int)((uint32_t)i % (uint32_t)b.T);
  int n = b.T;
  if (b.len) {
    n = b.len[r];
    if (n < 0 || n > b.T) err |= kErrLen;
  }
  if (t >= n) return b.V;
  const int v = b.tok[i];
  if (v < 0 || v >= b.V) {
    err |= kErrTok;
    return b.V;
  }
  return v;
}

__global__ void embed_clear_kernel(EmbedHeader* hdr) {
  hdr->err = 0;
  hdr->nlong = 0;
}

// A wavefront per row.
template <typename TW, typename TX>
__global__ __launch_bounds__(256) void embed_fwd_kernel(Batch b, const TW* __restrict__ W, int64_t ldW, int d, float scale,
                                                        TX* __restrict__ X, int64_t ldX, EmbedHeader* hdr) {
  const int lane = threadIdx.x & 63;
  const int64_t N = (int64_t)b.R * b.T;
  for (int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); i < N; i += (int64_t)gridDim.x * 4) {
    int err = 0;
    const uint32_t v = id_of(b, i, err);
    if (err && lane == 0) atomicOr(&hdr->err, err);
    for (int c = lane * 8; c < d; c += 512) {
      float x[8] = {};
      if (v < (uint32_t)b.V) {
        Row8<TW> w;
        w.load(W + v * ldW + c);
        w.get(x);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] *= scale;
      }
      Row8<TX>::store(X + i * ldX + c, x);
    }
  }
}

// ---- the sort --------------------------------------------------------------------------

struct SortArgs {
  Batch b;                 // first pass: keys come from here
  bool first;
  const uint32_t* key;
  const uint32_t* slot;
  uint32_t* key_out;
  uint32_t* slot_out;
  uint32_t* hist;          // [digit value][tile]: counts, then where the tile's slots of that value begin among all of that value
  uint32_t* totals;        // [digit value]
  int64_t N;
  int tiles, shift, digit;
  EmbedHeader* hdr;
};

__device__ inline uint32_t sort_key(const SortArgs& a, int64_t i, int& err) {
  return a.first ? id_of(a.b, i, err) : a.key[i];
}

__global__ __launch_bounds__(256) void sort_count_kernel(SortArgs a) {
  __shared__ uint32_t h[1 << kSortBits];
  const int D = 1 << a.digit;
  for (int i = threadIdx.x; i < D; i += 256) h[i] = 0;
  __syncthreads();
  const int64_t base = (int64_t)blockIdx.x * kSortTile;
  int err = 0;
  for (int j = threadIdx.x; j < kSortTile; j += 256)
    if (base + j < a.N) atomicAdd(&h[sort_key(a, base + j, err) >> a.shift & (D - 1)], 1u);
  if (a.first && err) atomicOr(&a.hdr->err, err);
  __syncthreads();
  for (int i = threadIdx.x; i < D; i += 256) a.hist[(int64_t)i * a.tiles + blockIdx.x] = h[i];
}

// A wavefront per digit value: exclusive sums over the tiles, and the total.
__global__ __launch_bounds__(64) void sort_scan_kernel(SortArgs a) {
  const int lane = threadIdx.x;
  uint32_t* h = a.hist + (int64_t)blockIdx.x * a.tiles;
  uint32_t sum = 0;
  for (int t0 = 0; t0 < a.tiles; t0 += 64) {
    const uint32_t x = t0 + lane < a.tiles ? h[t0 + lane] : 0;
    uint32_t s = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t y = __shfl_up(s, o);
      if (lane >= o) s += y;
    }
    if (t0 + lane < a.tiles) h[t0 + lane] = sum + s - x;
    sum += __shfl(s, 63);
  }
  if (lane == 0) a.totals[blockIdx.x] = sum;
}

// Slots to their places: stable, since wavefront w owns the w-th quarter of the tile and goes through it in order.
__global__ __launch_bounds__(256) void sort_place_kernel(SortArgs a) {
  __shared__ uint32_t at[4][1 << kSortBits];
  __shared__ uint32_t wsum[4];
  const int D = 1 << a.digit, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t base = (int64_t)blockIdx.x * kSortTile + w * (kSortTile / 4);
  for (int i = threadIdx.x; i < 4 * (1 << kSortBits); i += 256) (&at[0][0])[i] = 0;
  __syncthreads();
  int err = 0;
  uint32_t key[kSortTile / 256];
#pragma unroll
  for (int j = 0; j < kSortTile / 256; ++j) {
    const int64_t i = base + j * 64 + lane;
    key[j] = i < a.N ? sort_key(a, i, err) : 0;
    if (i < a.N) atomicAdd(&at[w][key[j] >> a.shift & (D - 1)], 1u);
  }
  // first place of each digit value: two neighbouring values per thread
  uint32_t tot[2], s = 0;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int v = threadIdx.x * 2 + k;
    tot[k] = v < D ? a.totals[v] : 0;
    s += tot[k];
  }
  const uint32_t own = s;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t y = __shfl_up(s, o);
    if (lane >= o) s += y;
  }
  if (lane == 63) wsum[w] = s;
  __syncthreads();
  uint32_t begin = s - own;
  for (int k = 0; k < w; ++k) begin += wsum[k];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int v = threadIdx.x * 2 + k;
    if (v < D) {
      uint32_t p = begin + a.hist[(int64_t)v * a.tiles + blockIdx.x];
      for (int q = 0; q < 4; ++q) {
        const uint32_t c = at[q][v];
        at[q][v] = p;
        p += c;
      }
    }
    begin += tot[k];
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kSortTile / 256; ++j) {
    const int64_t i = base + j * 64 + lane;
    const bool have = i < a.N;
    const uint32_t v = key[j] >> a.shift & (D - 1);
    uint64_t same = __ballot(have);
    for (int bit = 0; bit < a.digit; ++bit) {
      const uint64_t m = __ballot(v >> bit & 1);
      same &= v >> bit & 1 ? m : ~m;
    }
    if (!have) same = 0;
    const int lead = have ? __ffsll((unsigned long long)same) - 1 : lane;
    uint32_t p = 0;
    if (have && lane == lead) p = atomicAdd(&at[w][v], (uint32_t)__popcll(same));
    p = __shfl(p, lead) + __popcll(same & ((1ull << lane) - 1));
    if (have) {
      a.key_out[p] = key[j];
      a.slot_out[p] = a.first ? (uint32_t)i : a.slot[i];
    }
  }
}

// ---- the sums --------------------------------------------------------------------------

struct SumArgs {
  const uint32_t* key;     // sorted; V at the end where slots do not count
  const uint32_t* slot;
  int64_t N, chunks;
  int V, d;
  int64_t ldX;
  float scale;
  float* dW;
  bool add;
  float* part;
  int32_t* list;
  EmbedHeader* hdr;
};

__device__ inline uint32_t key_at(const SumArgs& a, int64_t p) { return p >= 0 && p < a.N ? a.key[p] : 0xffffffffu; }

template <typename T>
__device__ inline void put_row(const SumArgs& a, uint32_t v, int c, const float (&s)[8]) {
  float* p = a.dW + (int64_t)v * a.d + c;
  float x[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) x[k] = s[k] * a.scale;
  if (a.add) {
    Row8<float> old;
    old.load(p);
    float o[8];
    old.get(o);
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] += o[k];
  }
  Row8<float>::store(p, x);
}

// A wavefront per chunk of sorted slots and 512 columns.  An id belongs to the chunk in which its first slot lies, which reads on
// into the next chunk where the id ends there.  An id that ends later still is long: every chunk that it touches
// leaves a partial sum, and embed_join_kernel adds them up.
template <typename T>
__global__ __launch_bounds__(64) void embed_sum_kernel(SumArgs a, const T* __restrict__ gX) {
  constexpr int C = kEmbedChunk, U = 8;
  const int lane = threadIdx.x;
  const int64_t chunk = blockIdx.x, p0 = chunk * C;
  const int c = blockIdx.y * 512 + lane * 8;
  const bool in = c < a.d;
  const int c_load = in ? c : a.d - 8;             // lanes past the row read its end along
  const uint32_t V = (uint32_t)a.V;
  const uint32_t k0 = p0 + lane < a.N ? a.key[p0 + lane] : V;
  const uint32_t s0 = p0 + lane < a.N ? a.slot[p0 + lane] : 0;
  const int n = __popcll(__ballot(k0 < V));        // slots that count come first
  if (n == 0) return;
  auto rows = [&](uint32_t slots, int from, int to, uint32_t keys, uint32_t& cur, float (&s)[8], bool flush) {
    for (int i = from; i < to; i += U) {
      Row8<T> x[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i + u < to) x[u].load(gX + (int64_t)(uint32_t)__builtin_amdgcn_readlane(slots, i + u) * a.ldX + c_load);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i + u < to) {
          const uint32_t v = __builtin_amdgcn_readlane(keys, i + u);
          if (flush && v != cur) {
            if (cur != V && in) put_row<T>(a, cur, c, s);
#pragma unroll
            for (int k = 0; k < 8; ++k) s[k] = 0.f;
            cur = v;
          }
          float y[8];
          x[u].get(y);
#pragma unroll
          for (int k = 0; k < 8; ++k) s[k] += y[k];
        }
    }
  };
  auto partial = [&](int which, const float (&s)[8]) {
    if (in) Row8<float>::store(a.part + (chunk * 2 + which) * a.d + c, s);
  };
  // an id that began in an earlier chunk
  const uint32_t before = key_at(a, p0 - 1);
  const int lead = __popcll(__ballot(lane < n && k0 == before));
  if (lead > 0) {
    const bool on = lead == C && key_at(a, p0 + C) == before;
    if (on || key_at(a, p0 - C - 1) == before) {
      float s[8] = {};
      uint32_t cur = before;
      rows(s0, 0, lead, k0, cur, s, false);
      partial(0, s);
    }
  }
  if (lead == n) return;
  // the others; the last one may go on
  const uint32_t tail = __builtin_amdgcn_readlane(k0, n - 1);
  const bool goes_on = n == C && key_at(a, p0 + C) == tail;
  const bool is_long = goes_on && key_at(a, p0 + 2 * C) == tail;
  int end = n;
  if (is_long) end = n - __popcll(__ballot(lane < n && k0 == tail));
  float s[8] = {};
  uint32_t cur = V;
  rows(s0, lead, end, k0, cur, s, true);
  if (goes_on && !is_long) {
    const uint32_t k1 = key_at(a, p0 + C + lane);
    const uint32_t s1 = p0 + C + lane < a.N ? a.slot[p0 + C + lane] : 0;
    rows(s1, 0, __popcll(__ballot(k1 == tail)), k1, cur, s, false);
  }
  if (cur != V && in) put_row<T>(a, cur, c, s);
  if (is_long) {
#pragma unroll
    for (int k = 0; k < 8; ++k) s[k] = 0.f;
    rows(s0, end, n, k0, cur, s, false);
    partial(1, s);
    if (blockIdx.y == 0 && lane == 0) a.list[atomicAdd(&a.hdr->nlong, 1)] = (int32_t)chunk;
  }
}

// The long ids: partial sums in the order of their chunks.
__global__ __launch_bounds__(64) void embed_join_kernel(SumArgs a) {
  constexpr int C = kEmbedChunk;
  const int lane = threadIdx.x, c = blockIdx.y * 512 + lane * 8;
  const int nlong = a.hdr->nlong;
  for (int i = blockIdx.x; i < nlong; i += gridDim.x) {
    const int64_t chunk = a.list[i];
    const uint32_t v = a.key[chunk * C + C - 1];
    if (c >= a.d) continue;
    float s[8];
    Row8<float> x;
    x.load(a.part + (chunk * 2 + 1) * a.d + c);
    x.get(s);
    for (int64_t q = chunk + 1; q < a.chunks && a.key[q * C] == v; ++q) {
      x.load(a.part + q * 2 * a.d + c);
      float y[8];
      x.get(y);
#pragma unroll
      for (int k = 0; k < 8; ++k) s[k] += y[k];
    }
    put_row<float>(a, v, c, s);
  }
}

// Zeros to the rows of ids that do not occur: a wavefront looks for 64 ids at a time, then fills.
__global__ __launch_bounds__(256) void embed_zero_kernel(SumArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t v0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * 64, v = v0 + lane;
  if (v0 >= a.V) return;
  bool absent = false;
  if (v < a.V) {
    int64_t lo = 0, hi = a.N;     // first position whose key is v or more
    while (lo < hi) {
      const int64_t m = (lo + hi) >> 1;
      if (a.key[m] < (uint32_t)v) lo = m + 1;
      else hi = m;
    }
    absent = key_at(a, lo) != (uint32_t)v;
  }
  uint64_t todo = __ballot(absent);
  while (todo) {
    const int k = __ffsll((unsigned long long)todo) - 1;
    todo &= todo - 1;
    float* p = a.dW + (v0 + k) * a.d;
    for (int c = lane * 4; c < a.d; c += 256) *reinterpret_cast<f32x4*>(p + c) = f32x4{0.f, 0.f, 0.f, 0.f};
  }
}

template <typename TW, typename TX>
void run_fwd(const lmhead_embed_desc& d, const Batch& b, const void* W, float scale, void* X, EmbedHeader* hdr, hipStream_t s) {
  const int64_t N = (int64_t)d.R * d.T, wgs = (N + 3) / 4;
  hipLaunchKernelGGL((embed_fwd_kernel<TW, TX>), dim3((unsigned)(wgs < 65536 ? wgs : 65536)), dim3(256), 0, s, b,
                     static_cast<const TW*>(W), d.ldW, d.d, scale, static_cast<TX*>(X), d.ldX, hdr);
}

}  // namespace

hipError_t launch_embed_fwd(const lmhead_embed_desc& d, const void* W, const int32_t* tok, const int32_t* len, float scale, void* X,
                            EmbedHeader* hdr, hipStream_t s) {
  const Batch b{tok, len, d.R, d.T, d.V};
  hipLaunchKernelGGL(embed_clear_kernel, dim3(1), dim3(1), 0, s, hdr);
  if (d.dtype == LMHEAD_BF16 && d.rows == LMHEAD_BF16) run_fwd<__bf16, __bf16>(d, b, W, scale, X, hdr, s);
  else if (d.dtype == LMHEAD_BF16) run_fwd<__bf16, float>(d, b, W, scale, X, hdr, s);
  else if (d.rows == LMHEAD_BF16) run_fwd<float, __bf16>(d, b, W, scale, X, hdr, s);
  else run_fwd<float, float>(d, b, W, scale, X, hdr, s);
  return hipGetLastError();
}

hipError_t launch_embed_bwd(const lmhead_embed_desc& d, const void* gX, const int32_t* tok, const int32_t* len, float scale, float* dW,
                            char* ws, hipStream_t s) {
  const EmbedLayout L = embed_layout(&d);
  EmbedHeader* hdr = reinterpret_cast<EmbedHeader*>(ws + L.hdr);
  auto u32 = [&](size_t off) { return reinterpret_cast<uint32_t*>(ws + off); };
  hipLaunchKernelGGL(embed_clear_kernel, dim3(1), dim3(1), 0, s, hdr);
  SortArgs so{};
  so.b = Batch{tok, len, d.R, d.T, d.V};
  so.N = L.N;
  so.tiles = (int)L.tiles;
  so.digit = L.digit;
  so.hist = u32(L.hist);
  so.totals = so.hist + ((int64_t)L.tiles << L.digit);
  so.hdr = hdr;
  for (int p = 0; p < L.passes; ++p) {
    so.first = p == 0;
    so.key = u32(L.key[(p + 1) & 1]);
    so.slot = u32(L.slot[(p + 1) & 1]);
    so.key_out = u32(L.key[p & 1]);
    so.slot_out = u32(L.slot[p & 1]);
    so.shift = p * L.digit;
    hipLaunchKernelGGL(sort_count_kernel, dim3((unsigned)L.tiles), dim3(256), 0, s, so);
    hipLaunchKernelGGL(sort_scan_kernel, dim3(1u << L.digit), dim3(64), 0, s, so);
    hipLaunchKernelGGL(sort_place_kernel, dim3((unsigned)L.tiles), dim3(256), 0, s, so);
  }
  SumArgs a{};
  a.key = so.key_out;
  a.slot = so.slot_out;
  a.N = L.N;
  a.chunks = L.chunks;
  a.V = d.V;
  a.d = d.d;
  a.ldX = d.ldX;
  a.scale = scale;
  a.dW = dW;
  a.add = (d.flags & LMHEAD_FLAG_ACCUM_DW) != 0;
  a.part = reinterpret_cast<float*>(ws + L.part);
  a.list = reinterpret_cast<int32_t*>(ws + L.list);
  a.hdr = hdr;
  const unsigned cols = (unsigned)((d.d + 511) / 512);
  if (!a.add) hipLaunchKernelGGL(embed_zero_kernel, dim3((unsigned)(((int64_t)d.V + 255) / 256)), dim3(256), 0, s, a);
  if (d.rows == LMHEAD_BF16)
    hipLaunchKernelGGL(embed_sum_kernel<__bf16>, dim3((unsigned)L.chunks, cols), dim3(64), 0, s, a, static_cast<const __bf16*>(gX));
  else
    hipLaunchKernelGGL(embed_sum_kernel<float>, dim3((unsigned)L.chunks, cols), dim3(64), 0, s, a, static_cast<const float*>(gX));
  hipLaunchKernelGGL(embed_join_kernel, dim3((unsigned)(L.chunks < 256 ? L.chunks : 256), cols), dim3(64), 0, s, a);
  return hipGetLastError();
}

}  // namespace lmhead
