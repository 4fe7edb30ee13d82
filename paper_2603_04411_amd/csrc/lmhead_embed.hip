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
  __device__ inline void load_once(const float* p) {
    a = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p));
    b = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p + 4));
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
  __device__ inline void load_once(const __bf16* p) { a = __builtin_nontemporal_load(reinterpret_cast<const bf16x8*>(p)); }
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
__device__ inline uint32_t id_of(const Batch& b, uint32_t i, int& err) {
  // both loads leave before either result is looked at
  const uint32_t r = i / (uint32_t)b.T, v = (uint32_t)b.tok[i];
  const int n = b.len ? b.len[r] : b.T, t = (int)(i - r * (uint32_t)b.T);
  const bool counts = t < n, known = v < (uint32_t)b.V;
  err |= ((uint32_t)n > (uint32_t)b.T ? kErrLen : 0) | (counts && !known ? kErrTok : 0);
  return counts && known ? v : (uint32_t)b.V;
}

__device__ inline int wave_or(int x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x |= __shfl_xor(x, o);
  return x;
}

// Error bits of all slots, by one workgroup of 256 threads, into the header.
__device__ inline void report_all(const Batch& b, EmbedHeader* hdr) {
  __shared__ int bits[4];
  int err = 0;
  for (uint32_t i = threadIdx.x; i < (uint32_t)b.R * (uint32_t)b.T; i += 256) id_of(b, i, err);
  err = wave_or(err);
  if ((threadIdx.x & 63) == 0) bits[threadIdx.x >> 6] = err;
  __syncthreads();
  if (threadIdx.x == 0) hdr->err = bits[0] | bits[1] | bits[2] | bits[3];
}

__global__ void embed_clear_kernel(EmbedHeader* hdr) { hdr->err = 0; }

// Units of 256 threads and 16 bytes each of X, in the order of the addresses; a workgroup has kLookup of them in flight, so that
// the wait for an id and then for its row is shared.  Long rows: `parts` units to a row, and the id is the same for all
// threads; short ones: 2^lanes neighbouring threads to a row.
// Bound by memory: 524288 slots x 4096 bf16 write 4.3 GB and fetch 1.2 GB of W past L2 (41000 different rows are 0.34), in 805 us: 6.8 TB/s.
// One unit 1290 us, two 1020, eight as four; X through the caches 923 (it pushes W out of them; what reads X next is not slower for it
// from 8 MB to 540 MB of X).
// Of a batch of few slots the last workgroup reports for all (`reports`); otherwise the header has been cleared, and whoever meets
// an error adds it.
constexpr int kLookup = 4;
template <typename TW, typename TX, bool kLong>
__global__ __launch_bounds__(256) void embed_fwd_kernel(Batch b, const TW* __restrict__ W, int64_t ldW, int d, float scale,
                                                        TX* __restrict__ X, int64_t ldX, EmbedHeader* hdr, int lanes, uint32_t parts,
                                                        bool reports) {
  constexpr int E = 16 / (int)sizeof(TX), U = kLookup;
  typedef __attribute__((ext_vector_type(E))) TW in_t;
  typedef __attribute__((ext_vector_type(E))) TX out_t;
  if (reports && blockIdx.x == gridDim.x - 1) return report_all(b, hdr);
  const uint32_t N = (uint32_t)b.R * (uint32_t)b.T;
  const uint64_t u0 = (uint64_t)grid_wg() * U;
  int64_t i[U];
  int c[U];
  uint32_t v[U];
  int err = 0;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (kLong) {
      i[u] = (int64_t)((u0 + u) / parts);
      c[u] = ((int)((u0 + u) % parts) * 256 + (int)threadIdx.x) * E;
    } else {
      i[u] = (int64_t)(((u0 + u) << (8 - lanes)) + (threadIdx.x >> lanes));
      c[u] = (int)(threadIdx.x & ((1u << lanes) - 1)) * E;
    }
    v[u] = i[u] < N ? id_of(b, (uint32_t)i[u], err) : 0;
  }
  if (!reports && err) atomicOr(&hdr->err, err);
  in_t x[U];
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (i[u] < N && c[u] < d && v[u] < (uint32_t)b.V) x[u] = *reinterpret_cast<const in_t*>(W + (int64_t)v[u] * ldW + c[u]);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    out_t y;
#pragma unroll
    for (int k = 0; k < E; ++k) y[k] = v[u] < (uint32_t)b.V ? (TX)((float)x[u][k] * scale) : (TX)0.f;
    if (i[u] < N && c[u] < d) __builtin_nontemporal_store(y, reinterpret_cast<out_t*>(X + i[u] * ldX + c[u]));
  }
}

// ---- the gradient's rows -----------------------------------------------------------------

struct Rows {
  const void* g;
  int64_t ld;
  float* dW;
  int d;
  float scale;
  bool add;
};

__device__ inline void put_row(const Rows& a, uint32_t v, int c, const float (&s)[8]) {
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

template <typename T>
__device__ inline void add_to(float (&s)[8], const Row8<T>& x) {
  float y[8];
  x.get(y);
#pragma unroll
  for (int k = 0; k < 8; ++k) s[k] += y[k];
}

__device__ inline void clear(float (&s)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) s[k] = 0.f;
}

// ---- few slots: one launch, no sort -------------------------------------------------------

// The first `owners` workgroups take four slots and 512 columns each, a wavefront per slot.  The first slot of an id lists the
// id's slots (every workgroup holds all ids in LDS: at most kFewSlots) and sums their rows; an id of more than kShared rows is shared by
// the four wavefronts, whose sums are joined in order.  The other workgroups write zeros to the rows of their `rows_each` ids
// that do not occur.  All slots pass through every workgroup, so the first one can report errors without a cleared header.
constexpr int kShared = 32;
template <typename T>
__global__ __launch_bounds__(256) void embed_few_kernel(Batch b, Rows a, EmbedHeader* hdr, int owners, int cols, int rows_each) {
  constexpr int U = 8;
  __shared__ uint32_t id[kFewSlots];
  __shared__ uint16_t list[4][kFewSlots];
  __shared__ int count[4];
  __shared__ uint32_t whose[4];
  __shared__ float sums[4][512];
  __shared__ int bits[4];
  const int N = b.R * b.T, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const uint32_t V = (uint32_t)b.V;
  int err = 0;
  for (int i = threadIdx.x; i < N; i += 256) id[i] = id_of(b, i, err);
  if (grid_wg() == 0) {
    err = wave_or(err);
    if (lane == 0) bits[w] = err;
  }
  const uint32_t wg = grid_wg();
  if (wg >= (uint32_t)owners) {
    // at most 64 ids: bit k of `present`, gathered by the four wavefronts
    __shared__ uint64_t present;
    if (threadIdx.x == 0) present = 0;
    __syncthreads();
    const uint32_t v0 = (wg - owners) * (uint32_t)rows_each;
    for (int i = threadIdx.x; i < N; i += 256)
      if (id[i] - v0 < (uint32_t)rows_each) atomicOr(reinterpret_cast<unsigned long long*>(&present), 1ull << (id[i] - v0));
    __syncthreads();
    const uint64_t have = present;
    for (int k = 0; k < rows_each && v0 + k < V; ++k) {
      if (have >> k & 1) continue;
      float* p = a.dW + (int64_t)(v0 + k) * a.d;
      for (int c = threadIdx.x * 4; c < a.d; c += 1024) *reinterpret_cast<f32x4*>(p + c) = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    return;
  }
  __syncthreads();
  if (wg == 0 && threadIdx.x == 0) hdr->err = bits[0] | bits[1] | bits[2] | bits[3];
  const int slot = (int)wg / cols * 4 + w;
  const uint32_t mine = slot < N ? id[slot] : V;
  int n = 0;
  if (mine < V) {
    for (int i0 = 0; i0 < N; i0 += 64) {
      const bool hit = i0 + lane < N && id[i0 + lane] == mine;
      const uint64_t m = __ballot(hit);
      if (i0 <= slot && (m & (slot - i0 >= 64 ? ~0ull : (1ull << (slot - i0)) - 1))) {
        n = 0;      // an earlier slot has this id
        break;
      }
      if (hit) list[w][n + __popcll(m & ((1ull << lane) - 1))] = (uint16_t)(i0 + lane);
      n += __popcll(m);
    }
  }
  if (lane == 0) {
    count[w] = n;
    whose[w] = mine;
  }
  const int c = (int)wg % cols * 512 + lane * 8;
  const bool in = c < a.d;
  const T* g = static_cast<const T*>(a.g) + (in ? c : a.d - 8);
  auto sum = [&](const uint16_t* l, int from, int to, float (&s)[8]) {
    for (int i = from; i < to; i += U) {
      Row8<T> x[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i + u < to) x[u].load(g + (int64_t)__builtin_amdgcn_readfirstlane(l[i + u]) * a.ld);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i + u < to) add_to(s, x[u]);
    }
  };
  __syncthreads();
  if (n > 0 && n <= kShared) {
    float s[8] = {};
    sum(list[w], 0, n, s);
    if (in) put_row(a, mine, c, s);
  }
  for (int q = 0; q < 4; ++q) {
    const int m = count[q];
    if (m <= kShared) continue;
    float s[8] = {};
    sum(list[q], m * w / 4, m * (w + 1) / 4, s);
    Row8<float>::store(&sums[w][lane * 8], s);
    __syncthreads();
    if (w == q) {
      clear(s);
      for (int k = 0; k < 4; ++k) {
        Row8<float> x;
        x.load(&sums[k][lane * 8]);
        add_to(s, x);
      }
      if (in) put_row(a, whose[q], c, s);
    }
    __syncthreads();
  }
}

// ---- the sort --------------------------------------------------------------------------

// Zeros for [lo, hi) of dW, by workgroups that ride along in the launches of the sort.
struct Fill {
  float* p;
  int64_t lo, hi;
};
template <int kThreads = 256>
__device__ inline void fill(const Fill& f, int64_t block) {
  const int64_t i = f.lo + (block * kThreads + threadIdx.x) * 4;    // one store per thread: 6.9 TB/s, in a loop 5.5
  if (i < f.hi) *reinterpret_cast<f32x4*>(f.p + i) = f32x4{0.f, 0.f, 0.f, 0.f};
}

// A radix sort, least digit first, in tiles of 1024 slots: counts, their sums, places.  Launches and latency: of 524288 slots 7, 4.8 and 9 us
// a digit, of which 152064 ids have two.  (Tiles of 4096 slots: places alone 20, sixteen rounds of ballots one after the other.)
struct SortArgs {
  Batch b;                 // first pass: keys come from here
  bool first;
  bool scanned;            // hist is [digit value][tile] and goes through sort_scan_kernel, or [tile][digit value]
  const uint32_t* key;
  const uint32_t* slot;
  uint32_t* key_out;
  uint32_t* slot_out;
  uint32_t* hist;          // counts; scanned: then where the tile's slots of that value begin among all of that value
  uint32_t* totals;        // scanned: [digit value]
  uint32_t N;
  int tiles, shift, digit;
  EmbedHeader* hdr;
  Fill f;
};

__device__ inline uint32_t sort_key(const SortArgs& a, uint32_t i, int& err) {
  return a.first ? id_of(a.b, i, err) : a.key[i];
}

__global__ __launch_bounds__(256) void sort_count_kernel(SortArgs a) {
  __shared__ uint32_t h[1 << kSortBits];
  if (grid_wg() >= (uint32_t)a.tiles) return fill(a.f, grid_wg() - a.tiles);
  const int D = 1 << a.digit;
  for (int i = threadIdx.x; i < D; i += 256) h[i] = 0;
  if (a.first && blockIdx.x == 0 && threadIdx.x == 0) {
    a.hdr->err = 0;
    a.hdr->nlong = 0;
  }
  __syncthreads();
  int err = 0;      // reported by sort_place_kernel, after the header has been cleared
#pragma unroll
  for (int j = 0; j < kSortTile / 256; ++j) {
    const uint32_t i = blockIdx.x * (uint32_t)kSortTile + j * 256 + threadIdx.x;
    if (i < a.N) atomicAdd(&h[sort_key(a, i, err) >> a.shift & (D - 1)], 1u);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < D; i += 256) a.hist[a.scanned ? (int64_t)i * a.tiles + blockIdx.x : (int64_t)blockIdx.x * D + i] = h[i];
}

// A wavefront per digit value: exclusive sums over the tiles, and the total.  Eight segments of 64 tiles are asked for at once (16.7
// million rows of 64 columns 1444 us, with one segment after the other 1546).
__global__ __launch_bounds__(256) void sort_scan_kernel(SortArgs a) {
  constexpr int U = 8;
  const int D = 1 << a.digit, groups = (D + 3) / 4;
  if (grid_wg() >= (uint32_t)groups) return fill(a.f, grid_wg() - groups);
  const int lane = threadIdx.x & 63, v = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (v >= D) return;
  uint32_t* h = a.hist + (int64_t)v * a.tiles;
  uint32_t sum = 0;
  for (int t0 = 0; t0 < a.tiles; t0 += 64 * U) {
    uint32_t x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = t0 + u * 64 + lane < a.tiles ? h[t0 + u * 64 + lane] : 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      uint32_t s = x[u];
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t y = __shfl_up(s, o);
        if (lane >= o) s += y;
      }
      if (t0 + u * 64 + lane < a.tiles) h[t0 + u * 64 + lane] = sum + s - x[u];
      sum += __shfl(s, 63);
    }
  }
  if (lane == 0) a.totals[v] = sum;
}

// Slots to their places: stable, since wavefront w owns the w-th quarter of the tile and goes through it in order.
__global__ __launch_bounds__(256) void sort_place_kernel(SortArgs a) {
  constexpr int K = kSortTile / 256;
  __shared__ uint32_t at[4][1 << kSortBits];
  __shared__ uint32_t wsum[4];
  if (grid_wg() >= (uint32_t)a.tiles) return fill(a.f, grid_wg() - a.tiles);
  const int D = 1 << a.digit, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const uint32_t base = blockIdx.x * (uint32_t)kSortTile + w * (kSortTile / 4) + lane;
  for (int i = threadIdx.x; i < 4 * (1 << kSortBits); i += 256) (&at[0][0])[i] = 0;
  int err = 0;
  uint32_t key[K], slot[K];
#pragma unroll
  for (int j = 0; j < K; ++j) {
    const uint32_t i = base + j * 64;
    key[j] = i < a.N ? sort_key(a, i, err) : 0;
    slot[j] = a.first ? i : i < a.N ? a.slot[i] : 0;
  }
  // two neighbouring digit values per thread: how many slots have them, in all tiles and in those before this one
  uint32_t tot[2] = {0, 0}, before[2] = {0, 0};
  const int v0 = threadIdx.x * 2;
  if (v0 < D) {
    if (a.scanned) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        tot[k] = a.totals[v0 + k];
        before[k] = a.hist[(int64_t)(v0 + k) * a.tiles + blockIdx.x];
      }
    } else {
#pragma unroll 8
      for (int q = 0; q < a.tiles; ++q) {
        const uint2 x = *reinterpret_cast<const uint2*>(a.hist + (int64_t)q * D + v0);
        tot[0] += x.x;
        tot[1] += x.y;
        if (q < (int)blockIdx.x) {
          before[0] += x.x;
          before[1] += x.y;
        }
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < K; ++j)
    if (base + j * 64 < a.N) atomicAdd(&at[w][key[j] >> a.shift & (D - 1)], 1u);
  uint32_t s = tot[0] + tot[1];
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
  if (v0 < D) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      uint32_t p = begin + before[k];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t c = at[q][v0 + k];
        at[q][v0 + k] = p;
        p += c;
      }
      begin += tot[k];
    }
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < K; ++j) {
    const bool have = base + j * 64 < a.N;
    const uint32_t v = key[j] >> a.shift & (D - 1);
    uint64_t same = __ballot(have);
#pragma unroll
    for (int bit = 0; bit < kSortBits; ++bit) {
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
      a.slot_out[p] = slot[j];
    }
  }
  if (a.first && err) atomicOr(&a.hdr->err, err);
}

// ---- the sort of a few tiles ---------------------------------------------------------------

// Up to kMergeTiles tiles take two launches instead of two per digit: each tile is sorted by itself, then each slot looks up how
// many slots of every other tile come before it.  The gradient of 3000 / 8192 / 16384 rows of 64, added to 152064 ids: 18 / 22 / 27 us, by
// digits 26 / 29 / 32; with twice the LDS 24000 rows take 39, by digits 36.

// A tile's values id << 10 | place in the tile, ascending; one value per thread.  Bitonic: exchanges over less than 64 places stay in a
// wavefront.
__global__ __launch_bounds__(kSortTile) void tile_sort_kernel(SortArgs a) {
  __shared__ uint32_t sh[kSortTile];
  __shared__ int bits[kSortTile / 64];
  if (grid_wg() >= (uint32_t)a.tiles) return fill<kSortTile>(a.f, grid_wg() - a.tiles);
  const uint32_t t = threadIdx.x, i = blockIdx.x * (uint32_t)kSortTile + t;
  int err = 0;
  uint32_t x = i < a.N ? id_of(a.b, i, err) << 10 | t : 0xffffffffu;
  err = wave_or(err);
  if ((t & 63) == 0) bits[t >> 6] = err;
#pragma unroll
  for (uint32_t size = 2; size <= kSortTile; size <<= 1) {
#pragma unroll
    for (uint32_t step = size >> 1; step > 0; step >>= 1) {
      uint32_t y;
      if (step >= 64) {
        __syncthreads();
        sh[t] = x;
        __syncthreads();
        y = sh[t ^ step];
      } else {
        y = __shfl_xor(x, step);
      }
      const bool low = ((t & step) == 0) == ((t & size) == 0);     // this place gets the smaller value
      x = low ? (x < y ? x : y) : (x < y ? y : x);
    }
  }
  if (i < a.N) a.key_out[i] = x;
  __syncthreads();
  if (t == 0) {
    err = 0;
    for (int k = 0; k < kSortTile / 64; ++k) err |= bits[k];
    a.hist[blockIdx.x] = err;
    if (blockIdx.x == 0) a.hdr->nlong = 0;
  }
}

// Each workgroup holds all tiles in LDS (eleven dependent steps through each of them would each wait for L2: 26 us for 16 tiles) and places
// 64 slots, each wavefront looking through a quarter of the tiles (256 slots, every wavefront through all: 11 us; 1024: 19).
__global__ __launch_bounds__(256) void tile_merge_kernel(SortArgs a) {
  constexpr int U = kMergeTiles / 4;
  extern __shared__ __align__(16) uint32_t all[];
  __shared__ uint32_t parts[4][64];
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    uint32_t err = 0;
    for (int q = 0; q < a.tiles; ++q) err |= a.hist[q];
    a.hdr->err = (int)err;
  }
  const uint32_t whole = a.N & ~3u;
  for (uint32_t i = threadIdx.x * 4; i < whole; i += 1024) *reinterpret_cast<uint4*>(all + i) = *reinterpret_cast<const uint4*>(a.key + i);
  if (threadIdx.x < (a.N & 3u)) all[whole + threadIdx.x] = a.key[whole + threadIdx.x];
  __syncthreads();
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, tile = (int)(blockIdx.x * 64 / kSortTile);
  const uint32_t i = blockIdx.x * 64u + lane, x = all[min(i, a.N - 1)], id = x >> 10;
  // slots of the same id come first where their tile does
  uint32_t below[U], n[U], at[U], k[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int q = u * 4 + w;
    k[u] = q < a.tiles ? (uint32_t)q * kSortTile : 0;
    n[u] = q >= a.tiles || q == tile ? 0 : q + 1 < a.tiles ? kSortTile : a.N - k[u];
    below[u] = (id + (q < tile)) << 10;
    at[u] = 0;
  }
#pragma unroll
  for (uint32_t step = kSortTile; step > 0; step >>= 1)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      // read whether it counts or not: a branch would wait for one of the U reads at a time
      const uint32_t to = at[u] + step, v = all[min(k[u] + to - 1, a.N - 1)];
      at[u] = ((to <= n[u]) & (v < below[u])) ? to : at[u];
    }
  uint32_t p = 0;
#pragma unroll
  for (int u = 0; u < U; ++u) p += at[u];
  parts[w][lane] = p;
  __syncthreads();
  if (w != 0 || i >= a.N) return;
  p = i % kSortTile + parts[0][lane] + parts[1][lane] + parts[2][lane] + parts[3][lane];
  a.key_out[p] = id;
  a.slot_out[p] = (uint32_t)tile * kSortTile + (x & 1023u);
}

// ---- the sums --------------------------------------------------------------------------

struct SumArgs {
  Rows r;
  const uint32_t* key;     // sorted; V at the end where slots do not count
  const uint32_t* slot;
  int64_t N, chunks;
  int C;                   // sorted slots of a chunk, at most 64
  int V;
  float* part;
  int64_t ld_part;
  int cols;                // workgroups that a chunk's columns are spread over
  struct LongId* list;
  EmbedHeader* hdr;
};

__device__ inline uint32_t key_at(const SumArgs& a, int64_t p) { return p >= 0 && p < a.N ? a.key[p] : 0xffffffffu; }

// What embed_join_kernel has to add up for an id: the partial sums of chunks first .. last.
struct LongId {
  uint32_t id;
  int32_t first, last, pad;
};
static_assert(sizeof(LongId) == kLongIdBytes, "workspace");

// A wavefront per chunk of sorted slots and 512 columns.  An id belongs to the chunk in which its first slot lies, which reads on
// into the next chunk where the id ends there.  An id that ends later still is long: every chunk that it touches leaves a partial
// sum, and embed_join_kernel adds them up.
// Bound by memory: 524288 slots x 4096 bf16 (327000 of them valid, 41000 ids) added to a dW move 4.1 GB, measured and needed, in 726 to 805 us
// by the card: 5.2 to 5.7 TB/s, as much as this card gives a mix of reads and scattered read-modify-writes (reads alone, 200 ids: 5.8).  Rows in the order
// of memory, 4 or 16 rows in flight, dW past the caches and workgroups of 4 or 8 wavefronts are within 2 % of it.
template <typename T>
__global__ __launch_bounds__(64) void embed_sum_kernel(SumArgs a) {
  constexpr int U = 8;
  const int lane = threadIdx.x, C = a.C, d = a.r.d;
  const int64_t chunk = blockIdx.x / a.cols, p0 = chunk * C;
  const int c = (int)(blockIdx.x % a.cols) * 512 + lane * 8;
  const bool in = c < d;
  const T* gX = static_cast<const T*>(a.r.g) + (in ? c : d - 8);     // lanes past the row read its end along
  const uint32_t V = (uint32_t)a.V;
  const bool mine = lane < C && p0 + lane < a.N;
  const uint32_t k0 = mine ? a.key[p0 + lane] : V;
  const uint32_t s0 = mine ? a.slot[p0 + lane] : 0;
  // the neighbours' ids that say what goes on beyond the chunk: asked for at once, not one after the other
  const uint32_t before = key_at(a, p0 - 1), long_before = key_at(a, p0 - C - 1), after = key_at(a, p0 + C), long_after = key_at(a, p0 + 2 * C);
  const int n = __popcll(__ballot(k0 < V));        // slots that count come first
  if (n == 0) return;
  auto rows = [&](uint32_t slots, int from, int to, uint32_t keys, uint32_t& cur, float (&s)[8], bool flush) {
    for (int i = from; i < to; i += U) {
      Row8<T> x[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i + u < to) x[u].load_once(gX + (int64_t)(uint32_t)__builtin_amdgcn_readlane(slots, i + u) * a.r.ld);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i + u < to) {
          const uint32_t v = __builtin_amdgcn_readlane(keys, i + u);
          if (flush && v != cur) {
            if (cur != V && in) put_row(a.r, cur, c, s);
            clear(s);
            cur = v;
          }
          add_to(s, x[u]);
        }
    }
  };
  auto partial = [&](int which, const float (&s)[8]) {
    if (in) Row8<float>::store(a.part + (chunk * 2 + which) * a.ld_part + c, s);
  };
  // an id that began in an earlier chunk
  const int lead = __popcll(__ballot(lane < n && k0 == before));
  if (lead > 0) {
    const bool on = lead == C && after == before;
    if (on || long_before == before) {
      float s[8] = {};
      uint32_t cur = before;
      rows(s0, 0, lead, k0, cur, s, false);
      partial(0, s);
      if (!on && c == lane * 8) {
        // it ends here: where it began, 64 probes at a time (chunks from hi on begin inside it, those below lo do not)
        int64_t lo = 1, hi = chunk;
        while (lo < hi) {
          const int64_t step = (hi - lo + 63) / 64, q = hi - 1 - lane * step;
          const int have = __popcll(__ballot(q >= lo && a.key[q * C] == before && a.key[q * C - 1] == before));
          if (have == 0) {
            lo = hi;
            break;
          }
          const int64_t below = hi - 1 - have * step;      // the first probe that was not inside, if there was one
          hi = hi - 1 - (have - 1) * step;
          lo = below + 1 > lo ? below + 1 : lo;
        }
        if (lane == 0) a.list[atomicAdd(&a.hdr->nlong, 1)] = LongId{before, (int32_t)(hi - 1), (int32_t)chunk, 0};
      }
    }
  }
  if (lead == n) return;
  // the others; the last one may go on
  const uint32_t tail = __builtin_amdgcn_readlane(k0, n - 1);
  const bool goes_on = n == C && after == tail;
  const bool is_long = goes_on && long_after == tail;
  int end = n;
  if (is_long) end = n - __popcll(__ballot(lane < n && k0 == tail));
  float s[8] = {};
  uint32_t cur = V;
  rows(s0, lead, end, k0, cur, s, true);
  if (goes_on && !is_long) {
    const uint32_t k1 = lane < C ? key_at(a, p0 + C + lane) : V;
    const uint32_t s1 = lane < C && p0 + C + lane < a.N ? a.slot[p0 + C + lane] : 0;
    rows(s1, 0, __popcll(__ballot(k1 == tail)), k1, cur, s, false);
  }
  if (cur != V && in) put_row(a.r, cur, c, s);
  if (is_long) {
    clear(s);
    rows(s0, end, n, k0, cur, s, false);
    partial(1, s);
  }
}

// The long ids: a workgroup per id and 256 columns, those of one id next to each other (a launch that went through all ids with the same
// columns first met on few memory channels: 60 us for the 3600 partial rows of 4096 that 330000 slots leave, now 34).  Wavefront w takes
// the w-th part of the id's partial sums in order, U at a time, and the W sums are added in order.
template <int W, int U>
__global__ __launch_bounds__(64 * W) void embed_join_kernel(SumArgs a) {
  __shared__ f32x4 sums[W][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), d = a.r.d;
  const int cols = (d + 255) / 256, c = (int)(blockIdx.x % cols) * 256 + lane * 4;
  const bool in = c < d;
  const float* part = a.part + (in ? c : d - 4);
  const int nlong = a.hdr->nlong;
  for (int i = blockIdx.x / cols; i < nlong; i += gridDim.x / cols) {
    const LongId l = a.list[i];
    const int n = l.last + 1 - l.first, from = l.first + (int)((int64_t)n * w / W), to = l.first + (int)((int64_t)n * (w + 1) / W);
    f32x4* p = reinterpret_cast<f32x4*>(a.r.dW + (int64_t)l.id * d + c);
    f32x4 s = {0.f, 0.f, 0.f, 0.f}, old = s;
    if (w == 0 && in && a.r.add) old = *p;
    for (int q = from; q < to; q += U) {
      f32x4 x[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (q + u < to) x[u] = *reinterpret_cast<const f32x4*>(part + ((int64_t)(q + u) * 2 + (q + u == l.first)) * a.ld_part);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (q + u < to) s += x[u];
    }
    sums[w][lane] = s;
    __syncthreads();
    if (w == 0 && in) {
      for (int k = 1; k < W; ++k) s += sums[k][lane];
      s *= a.r.scale;
      *p = a.r.add ? old + s : s;
    }
    __syncthreads();
  }
}

template <typename TW, typename TX>
void run_fwd(const lmhead_embed_desc& d, const Batch& b, const void* W, float scale, void* X, EmbedHeader* hdr, hipStream_t s) {
  const int64_t N = (int64_t)d.R * d.T;
  constexpr int E = 16 / (int)sizeof(TX);
  int lanes = 0;
  while (lanes < 8 && (E << lanes) < d.d) ++lanes;
  const int64_t parts = (d.d + E * 256 - 1) / (E * 256);
  const bool reports = N <= kReportSlots;
  const int64_t units = lanes == 8 ? N * parts : (N + (256 >> lanes) - 1) / (256 >> lanes), wgs = (units + kLookup - 1) / kLookup;
  if (!reports) hipLaunchKernelGGL(embed_clear_kernel, dim3(1), dim3(1), 0, s, hdr);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid_of(wgs + reports), dim3(256), 0, s, b, static_cast<const TW*>(W), d.ldW, d.d, scale,
                       static_cast<TX*>(X), d.ldX, hdr, lanes, (uint32_t)parts, reports);
  };
  if (lanes == 8) go(embed_fwd_kernel<TW, TX, true>);
  else go(embed_fwd_kernel<TW, TX, false>);
}

}  // namespace

hipError_t launch_embed_fwd(const lmhead_embed_desc& d, const void* W, const int32_t* tok, const int32_t* len, float scale, void* X,
                            EmbedHeader* hdr, hipStream_t s) {
  const Batch b{tok, len, d.R, d.T, d.V};
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
  const Batch b{tok, len, d.R, d.T, d.V};
  const bool add = (d.flags & LMHEAD_FLAG_ACCUM_DW) != 0, bf16 = d.rows == LMHEAD_BF16;
  const Rows r{gX, d.ldX, dW, d.d, scale, add};
  const int cols = (d.d + 511) / 512;
  if (L.N <= kFewSlots && L.N * L.N * cols <= kFewWork) {
    const int owners = (int)((L.N + 3) / 4) * cols;
    // 16 KB of zeros per workgroup, or 32 where it has many ids to look through (64 KB: 5.4 TB/s)
    int rows_each = (L.N <= 256 ? 4096 : 8192) / d.d;
    rows_each = rows_each < 1 ? 1 : rows_each > 64 ? 64 : rows_each;
    const int64_t fills = add ? 0 : ((int64_t)d.V + rows_each - 1) / rows_each;
    auto go = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, grid_of(owners + fills), dim3(256), 0, s, b, r, hdr, owners, cols, rows_each);
    };
    if (bf16) go(embed_few_kernel<__bf16>);
    else go(embed_few_kernel<float>);
    return hipGetLastError();
  }
  auto u32 = [&](size_t off) { return reinterpret_cast<uint32_t*>(ws + off); };
  SortArgs so{};
  so.b = b;
  so.N = (uint32_t)L.N;
  so.tiles = (int)L.tiles;
  so.scanned = L.tiles > kScanTiles;
  so.digit = L.digit;
  so.hist = u32(L.hist);
  so.totals = so.hist + ((int64_t)L.tiles << L.digit);
  so.hdr = hdr;
  const int64_t cells = add ? 0 : (int64_t)d.V * d.d;
  // Where many zeros are written they hide all launches of the sort by digits, but not tile_merge_kernel, whose LDS would leave them few
  // workgroups.  8192 rows of 1024: 64 MB of zeros 33 us, by digits 42; 125 MB 46 and 51; 594 MB 129 and 122.
  const bool merged = L.tiles <= kMergeTiles && d.V < (1 << 22) - 1 && cells <= kMergeCells;
  const int launches = merged ? 1 : L.passes * (so.scanned ? 3 : 2);
  int launch = 0;
  // one launch of the sort, with its share of the zeros
  auto go = [&](auto kernel, int64_t wgs, int threads = 256) {
    so.f = Fill{dW, cells / 8 * launch / launches * 8, cells / 8 * (launch + 1) / launches * 8};
    ++launch;
    hipLaunchKernelGGL(kernel, grid_of(wgs + (so.f.hi - so.f.lo + threads * 4 - 1) / (threads * 4)), dim3(threads), 0, s, so);
  };
  auto buffers = [&](int from) {
    so.key = u32(L.key[from]);
    so.slot = u32(L.slot[from]);
    so.key_out = u32(L.key[from ^ 1]);
    so.slot_out = u32(L.slot[from ^ 1]);
  };
  if (merged) {
    buffers(1);
    go(tile_sort_kernel, L.tiles, kSortTile);
    buffers(0);
    hipLaunchKernelGGL(tile_merge_kernel, dim3((unsigned)((L.N + 63) / 64)), dim3(256), (size_t)(L.N + 3) / 4 * 16, s, so);
  }
  for (int p = 0; !merged && p < L.passes; ++p) {
    so.first = p == 0;
    buffers((p & 1) ^ 1);
    so.shift = p * L.digit;
    go(sort_count_kernel, L.tiles);
    if (so.scanned) go(sort_scan_kernel, ((1 << L.digit) + 3) / 4);
    go(sort_place_kernel, L.tiles);
  }
  SumArgs a{};
  a.r = r;
  a.key = so.key_out;
  a.slot = so.slot_out;
  a.N = L.N;
  a.C = L.C;
  a.chunks = L.chunks;
  a.V = d.V;
  a.part = reinterpret_cast<float*>(ws + L.part);
  a.ld_part = L.ld_part;
  a.list = reinterpret_cast<LongId*>(ws + L.list);
  a.hdr = hdr;
  a.cols = cols;
  const dim3 grid((unsigned)(L.chunks * cols));
  if (bf16) hipLaunchKernelGGL(embed_sum_kernel<__bf16>, grid, dim3(64), 0, s, a);
  else hipLaunchKernelGGL(embed_sum_kernel<float>, grid, dim3(64), 0, s, a);
  // an id is long from two chunks' slots on
  const int64_t most = L.N / (2 * L.C) + 1;
  const dim3 joins((unsigned)(most < 512 ? most : 512) * ((d.d + 255) / 256));
  // Of many short rows the most frequent id decides: 65536 / 200000 x 64 54 / 76 us, with eight wavefronts 57 / 81; of 16384 27.4 and 26.8,
  // of 65536 x 1024 as much either way.
  if (d.d <= 512 && L.N > 32768) hipLaunchKernelGGL((embed_join_kernel<16, 16>), joins, dim3(1024), 0, s, a);
  else hipLaunchKernelGGL((embed_join_kernel<8, 8>), joins, dim3(512), 0, s, a);
  return hipGetLastError();
}

}  // namespace lmhead
