// The cache itself: rows quantised to 4 bits, and tokens that leave it.
#include <algorithm>

#include "attn_common.h"

namespace lmhead {

namespace {

struct StoreArgs {
  int B, Tq, Tk, Hkv, D, esz;
  AttnTensor x[2];
  uint8_t* codes[2];
  uint8_t* scales[2];
  const int32_t *len_q, *len_k;
  AttnHeader* hdr;
};

__device__ inline uint32_t e2m1(float y) {     // y = |x| / 2^e <= 6: between two steps the nearer one, half-way the even index
  return (y > 0.25f) + (y >= 0.75f) + (y > 1.25f) + (y >= 1.75f) + (y > 2.5f) + (y >= 3.5f) + (y > 5.f);
}

// Four lanes make a block of 32, eight values each: its maximum takes two exchanges, its codes are a word a lane.  A step's rows are few: it is
// the launch (4 us).  A prompt's are bound by their reading.
template <typename E>
__global__ __launch_bounds__(256) void kv4_store_kernel(StoreArgs a) {
  using El = AttnElem<E>;
  if (blockIdx.x == 0 && blockIdx.y == 0) {
    AttnArgs r{};
    r.B = a.B, r.Tq = a.Tq, r.Tk = a.Tk, r.len_q = a.len_q, r.len_k = a.len_k, r.hdr = a.hdr;
    report_lengths(r);
  }
  const int parts = a.D / 8;
  const int64_t rows = (int64_t)a.B * a.Tq * a.Hkv, id = ((int64_t)blockIdx.y * kAttnRow + blockIdx.x) * 256 + threadIdx.x;
  const int64_t row = id / parts;      // (which of k and v, b, i, h)
  const int part = (int)(id % parts);
  if (row >= 2 * rows) return;         // a whole block or none: a row is a multiple of four lanes
  const int which = row >= rows;
  const int64_t at = which ? row - rows : row;
  const int h = (int)(at % a.Hkv), i = (int)(at / a.Hkv % a.Tq), b = (int)(at / a.Hkv / a.Tq);
  const int lq = a.len_q ? min(max(a.len_q[b], 0), a.Tq) : a.Tq, lk = a.len_k ? min(max(a.len_k[b], 0), a.Tk) : a.Tk;
  const int slot = lk - lq + i;
  if (i >= lq || slot < 0) return;
  const AttnTensor& t = a.x[which];
  const typename El::Frag f = El::load(t.p + b * t.seq + (int64_t)i * t.slot + h * t.head + part * 8 * El::size);
  float x[8], top = 0.f;
  bool bad = false;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    x[j] = El::value(f, j);
    top = fmaxf(top, fabsf(x[j]));
    bad |= !(fabsf(x[j]) <= 3.402823466e38f);
  }
  int flag = bad;
#pragma unroll
  for (int s = 1; s < 4; s <<= 1) {
    top = fmaxf(top, __shfl_xor(top, s));
    flag |= __shfl_xor(flag, s);
  }
  // top = (1 + m / 2^23) 2^x: the smallest e with top <= 1.5 2^(e + 2)
  const uint32_t bits = __builtin_bit_cast(uint32_t, top);
  int e = (int)(bits >> 23) - 127 - 2 + ((bits & 0x7fffffu) > 0x400000u);
  e = e < -126 ? -126 : e > 125 ? 125 : e;      // (6 * 2^125 is the largest value that bf16 and fp32 hold)
  uint32_t code = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t c = e2m1(ldexpf(fabsf(x[j]), -e)) | (__builtin_bit_cast(uint32_t, x[j]) >> 31) << 3;
    code |= c << (4 * j);
  }
  const int64_t to = ((int64_t)b * a.Hkv + h) * a.Tk + slot;
  *reinterpret_cast<uint32_t*>(a.codes[which] + to * (a.D / 2) + part * 4) = flag ? 0u : code;
  if (part % 4 == 0) a.scales[which][to * (a.D / 32) + part / 4] = (uint8_t)(flag ? 255 : e + 127);
}

// ---- eviction ----

struct EvictArgs {
  int B, T, Hkv, keep, sinks, recent;
  float* weight;
  const int32_t* len;
  int32_t *len_out, *kept;
  AttnHeader* hdr;
};

// Weights as integers of the same order; a NaN is below all numbers, -0 equals 0.
__device__ inline uint32_t order_of(float x) {
  if (x != x) return 0;
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.f);
  return b >> 31 ? ~b : b | 0x80000000u;
}

// One workgroup finds what a key head keeps: the threshold by four passes over eight bits each, then the tokens above it and the first of
// those at it, in order.  kHold: values that a thread holds on to over the passes, so that the weights are read once (of more than
// 1024 * kHold tokens they are read again for each pass).
//
// A key head is one workgroup's, since a pass has to know the one before: bound by the chain of passes (a count of 256 bins each, their sum, the
// ranks), 7 us of 1024 tokens, 23 of 8192.
template <int kHold>
__global__ __launch_bounds__(1024) void evict_choose_kernel(EvictArgs a) {
  __shared__ uint32_t hist[4][256];      // of four wavefronts each: the frequent digits are few
  __shared__ uint32_t wave_sum[2][16];
  __shared__ uint32_t s_digit, s_need;
  const int tid = threadIdx.x, l = tid & 63, w = tid >> 6;
  const uint32_t row = blockIdx.y * kAttnRow + blockIdx.x;
  const int b = row / a.Hkv;
  if (row == 0) {
    int bad = 0;
    if (a.len)
      for (int i = tid; i < a.B; i += 1024) bad |= (uint32_t)a.len[i] > (uint32_t)a.T;
    bad = __syncthreads_or(bad);
    if (tid == 0) a.hdr->err = bad ? kErrLen : 0;
  }
  if (row >= (uint32_t)a.B * a.Hkv) return;
  const int n = clamp_len(a.len, b, a.T);
  int32_t* const kept = a.kept + (int64_t)row * a.keep;
  float* const weight = a.weight + (int64_t)row * a.T;
  if (row % a.Hkv == 0 && tid == 0) a.len_out[b] = min(n, a.keep);
  if (n <= a.keep) {
    for (int i = tid; i < a.keep; i += 1024) kept[i] = i < n ? i : -1;
    return;
  }
  const int lo = a.sinks, hi = n - a.recent;
  constexpr int HOLD = kHold ? kHold : 1;
  float held[HOLD];
  if constexpr (kHold > 0) {
#pragma unroll
    for (int u = 0; u < HOLD; ++u) held[u] = u * 1024 + tid < n ? weight[u * 1024 + tid] : 0.f;
  }
  const int rounds = (n + 1023) / 1024;
  auto value = [&](int u, int i) -> float {
    if constexpr (kHold > 0) return held[u];
    else return i < n ? weight[i] : 0.f;
  };
  uint32_t need = a.keep - a.sinks - a.recent, prefix = 0;     // of [lo, hi): more than `need` of them
  if (need) {
#pragma unroll 1
    for (int shift = 24; shift >= 0; shift -= 8) {
      hist[tid >> 8][tid & 255] = 0;
      __syncthreads();
      auto count = [&](int u) {
        const int i = u * 1024 + tid;
        const uint32_t o = order_of(value(u, i));
        if (i >= lo && i < hi && (shift == 24 || (o >> (shift + 8)) == (prefix >> (shift + 8)))) atomicAdd(&hist[w & 3][o >> shift & 255], 1u);
      };
      if constexpr (kHold > 0) {
#pragma unroll
        for (int u = 0; u < HOLD; ++u)
          if (u < rounds) count(u);
      } else {
        for (int u = 0; u < rounds; ++u) count(u);
      }
      __syncthreads();
      if (w == 0) {      // the highest digits first: lane l has digits 255 - 4 l .. 252 - 4 l
        uint32_t c[4], sum = 0;
        for (int j = 0; j < 4; ++j) {
          const int d = 255 - 4 * l - j;
          c[j] = hist[0][d] + hist[1][d] + hist[2][d] + hist[3][d];
          sum += c[j];
        }
        uint32_t before = sum;
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) {
          const uint32_t y = __shfl_up(before, x);
          before += l >= x ? y : 0;
        }
        before -= sum;
        for (int j = 0; j < 4; ++j) {
          if (before < need && need <= before + c[j]) {
            s_digit = 255 - 4 * l - j;
            s_need = need - before;
          }
          before += c[j];
        }
      }
      __syncthreads();
      prefix |= s_digit << shift;
      need = s_need;
    }
  }
  // `need` of those equal to `prefix` stay, the first ones.  (With need = 0 from the start: none of [lo, hi).)
  const bool any = a.keep > a.sinks + a.recent;
  uint32_t equal = 0, out = 0;      // so far
  auto place = [&](int u) {
    const int i = u * 1024 + tid;
    const float x = value(u, i);
    const uint32_t o = order_of(x);
    const bool fixed = i < n && (i < lo || i >= hi), open = i >= lo && i < hi && any;
    const bool above = open && o > prefix, same = open && o == prefix;
    const uint64_t below = (1ull << l) - 1, eq = __ballot(same);
    if (l == 0) wave_sum[0][w] = __popcll(eq);
    __syncthreads();
    uint32_t at = equal + __popcll(eq & below);
    // (a sum over sixteen wavefronts: every lane has one of them)
    const uint32_t e = wave_sum[0][l & 15];
    uint32_t prior = (l & 15) < w ? e : 0, all = e;
#pragma unroll
    for (int x2 = 1; x2 < 16; x2 <<= 1) prior += __shfl_xor(prior, x2), all += __shfl_xor(all, x2);
    at += prior;
    equal += all;
    const bool stays = fixed || above || (same && at < need);
    const uint64_t st = __ballot(stays);
    if (l == 0) wave_sum[1][w] = __popcll(st);
    __syncthreads();
    const uint32_t m = wave_sum[1][l & 15];
    prior = (l & 15) < w ? m : 0, all = m;
#pragma unroll
    for (int x2 = 1; x2 < 16; x2 <<= 1) prior += __shfl_xor(prior, x2), all += __shfl_xor(all, x2);
    // slots written here were read by this round or an earlier one (by all threads: a barrier lies between)
    if (stays) {
      const uint32_t pos = out + prior + __popcll(st & below);
      kept[pos] = i;
      weight[pos] = x;
    }
    out += all;
  };
  if constexpr (kHold > 0) {
#pragma unroll
    for (int u = 0; u < HOLD; ++u)
      if (u < rounds) place(u);
  } else {
    for (int u = 0; u < rounds; ++u) place(u);
  }
  for (int i = a.keep + tid; i < n; i += 1024) weight[i] = 0.f;
}

struct MoveArgs {
  int B, T, Hkv, keep;
  const int32_t *len, *kept;
  cache_plane plane[EVICT_PLANES];
  int slices, parts[EVICT_PLANES];      // column slices of a row in all planes, and in each
};

// Rows close up in place.  A workgroup takes rows in ascending order, and a row only moves towards the front: what a step reads lies at or
// behind everything that it and the steps before it write, so a step reads all of its rows, waits, and writes them.  Slices of the
// rows' columns are independent of each other and go to workgroups of their own.
//
// Bound by the rows that move, read and written once, and by the steps' waits where few workgroups have long columns.  32 sequences of 4096 to
// 8192 tokens, 8 heads, half of them kept: 225 us where they have to close up (482 MB read and 465 written, 4.2 TB/s), 45 to 65 where the kept rows lie
// in front already.
template <typename W>
__global__ __launch_bounds__(256) void evict_move_kernel(MoveArgs a) {
  constexpr int U = 8;      // units a thread and step
  const uint32_t id = blockIdx.y * kAttnRow + blockIdx.x, works = (uint32_t)a.B * a.Hkv * a.slices;
  if (id >= works) return;
  int slice = id % a.slices, which = 0;
  while (slice >= a.parts[which]) slice -= a.parts[which++];
  const uint32_t row = id / a.slices;
  const int b = row / a.Hkv, h = row % a.Hkv;
  const int n = clamp_len(a.len, b, a.T);
  if (n <= a.keep) return;
  const cache_plane& p = a.plane[which];
  const int all_words = (int)(p.bytes / (int)sizeof(W)), each = (all_words + a.parts[which] - 1) / a.parts[which];
  const int w0 = slice * each, words = min(each, all_words - w0);
  if (words <= 0) return;      // (41 units in ten slices of five)
  char* const base = static_cast<char*>(p.data) + b * p.seq + h * p.head + (int64_t)w0 * sizeof(W);
  const int32_t* const kept = a.kept + (int64_t)row * a.keep;
  const int64_t all = (int64_t)a.keep * words;
  // (a row's first unit and its place in the row, carried along: no division in the loop)
  int r[U], c[U];
  const int dr = 256 * U / words, dc = 256 * U % words;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = u * 256 + threadIdx.x;
    r[u] = i / words, c[u] = i % words;
  }
  for (int64_t s = 0; s < all; s += 256 * U) {
    W x[U];
    int from[U];
#pragma unroll
    for (int u = 0; u < U; ++u) from[u] = r[u] < a.keep ? kept[r[u]] : r[u];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (from[u] != r[u]) x[u] = *reinterpret_cast<const W*>(base + from[u] * p.slot + c[u] * (int64_t)sizeof(W));
    __builtin_amdgcn_s_waitcnt(kWaitVm0);
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (from[u] != r[u]) *reinterpret_cast<W*>(base + r[u] * p.slot + c[u] * (int64_t)sizeof(W)) = x[u];
      r[u] += dr, c[u] += dc;
      if (c[u] >= words) c[u] -= words, ++r[u];
    }
  }
}

}  // namespace

hipError_t launch_kv4_store(const attn_desc* d, const AttnArgs& a, uint8_t* const* cache, hipStream_t s) {
  StoreArgs t{};
  t.B = a.B, t.Tq = a.Tq, t.Tk = a.Tk, t.Hkv = a.Hkv, t.D = a.D;
  t.x[0] = a.k, t.x[1] = a.v;
  t.codes[0] = cache[0], t.scales[0] = cache[1], t.codes[1] = cache[2], t.scales[1] = cache[3];
  t.len_q = a.len_q, t.len_k = a.len_k, t.hdr = a.hdr;
  const int64_t threads = 2 * (int64_t)a.B * a.Tq * a.Hkv * (a.D / 8);
  const dim3 grid = attn_grid((threads + 255) / 256);
  if (d->dtype == LMHEAD_BF16) kv4_store_kernel<bf16_tag><<<grid, 256, 0, s>>>(t);
  else kv4_store_kernel<f32_tag><<<grid, 256, 0, s>>>(t);
  return hipGetLastError();
}

hipError_t launch_evict(const evict_desc& d, const cache_plane* planes, int count, float* weight, const int32_t* len, int32_t* len_out,
                        int32_t* kept, char* ws, hipStream_t s) {
  EvictArgs a{d.B, d.T, d.Hkv, d.keep, d.sinks, d.recent, weight, len, len_out, kept, reinterpret_cast<AttnHeader*>(ws)};
  const dim3 rows = attn_grid((int64_t)d.B * d.Hkv);
  if (d.T <= 1024) evict_choose_kernel<1><<<rows, 1024, 0, s>>>(a);
  else if (d.T <= 4096) evict_choose_kernel<4><<<rows, 1024, 0, s>>>(a);
  else if (d.T <= 16384) evict_choose_kernel<16><<<rows, 1024, 0, s>>>(a);
  else evict_choose_kernel<0><<<rows, 1024, 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  MoveArgs m{};
  m.B = d.B, m.T = d.T, m.Hkv = d.Hkv, m.keep = d.keep, m.len = len, m.kept = kept;
  bool wide = true;
  for (int i = 0; i < count; ++i) {
    const cache_plane& p = planes[i];
    m.plane[i] = p;
    wide = wide && (reinterpret_cast<uintptr_t>(p.data) | p.seq | p.slot | p.head | p.bytes) % 16 == 0;
  }
  // Slices of at least 64 bytes, as many as keep 1024 workgroups busy (2 sequences of 1024 tokens, 8 heads of 256 bytes in two planes: 5 us, in
  // one slice 20).
  const int64_t most = (1024 + (int64_t)d.B * d.Hkv * count - 1) / ((int64_t)d.B * d.Hkv * count);
  for (int i = 0; i < count; ++i) {
    m.parts[i] = (int)std::max<int64_t>(1, std::min<int64_t>(most, planes[i].bytes / 64));
    m.slices += m.parts[i];
  }
  const dim3 grid = attn_grid((int64_t)d.B * d.Hkv * m.slices);
  if (wide) evict_move_kernel<u32x4_t><<<grid, 256, 0, s>>>(m);
  else evict_move_kernel<uint32_t><<<grid, 256, 0, s>>>(m);
  return hipGetLastError();
}

}  // namespace lmhead
