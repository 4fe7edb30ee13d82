// Attention over a window and a few first tokens, and the join of its parts.
#include "attn_common.h"

namespace lmhead {

namespace {

// 32 values of a row from their codes, as four chunks (fp32: eight) of a tile's row.
template <typename Tile>
__device__ inline void put_block(char* lds, int r, int block, const u32x4_t& codes, uint32_t scale) {
  const float size = __builtin_bit_cast(float, scale << 23);
  const bool bad = scale == 255;
  typedef __attribute__((ext_vector_type(2))) float f32x2_t;
#pragma unroll
  for (int i = 0; i < 4; ++i) {        // eight values: a word of codes
    const f32x2_t x0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[i], size, 0), x1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[i], size, 1);
    const f32x2_t x2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[i], size, 2), x3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[i], size, 3);
    float x[8] = {x0[0], x0[1], x1[0], x1[1], x2[0], x2[1], x3[0], x3[1]};
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = bad ? NAN : x[j];
    if constexpr (Tile::El::size == 2) {
      *reinterpret_cast<u32x4_t*>(lds + Tile::at(r, block * 4 + i)) = Tile::El::of(x);
    } else {
      const auto f = Tile::El::of(x);
      *reinterpret_cast<f32x4_t*>(lds + Tile::at(r, block * 8 + 2 * i)) = f.x[0];
      *reinterpret_cast<f32x4_t*>(lds + Tile::at(r, block * 8 + 2 * i + 1)) = f.x[1];
    }
  }
}

// BK rows of the cache in 4 bits, the ones from `valid` on and the columns from D on as zeros.
template <typename Tile, int NW, int BK>
__device__ inline void load_cache(char* lds, const uint8_t* codes, const uint8_t* scales, int valid, int D, int w, int l) {
  constexpr int BLOCKS = Tile::KS / 2;      // blocks of 32 in a row
  for (int i = w * 64 + l; i < BK * BLOCKS; i += NW * 64) {
    const int r = i / BLOCKS, block = i % BLOCKS;
    const bool in = r < valid && block * 32 < D;
    const u32x4_t c = in ? *reinterpret_cast<const u32x4_t*>(codes + (int64_t)r * (D / 2) + block * 16) : u32x4_t{0, 0, 0, 0};
    put_block<Tile>(lds, r, block, c, in ? scales[(int64_t)r * (D / 32) + block] : 127u);
  }
}

// O = softmax(scale Q K^T) V in one pass over the keys, with the running maximum and sum of each row.
//
// One workgroup takes NW * 32 rows (query i, head g of the key head: row r = i G + g) of one key head and walks the keys that
// they see in tiles of BK: S^T = K Q^T with the keys along the accumulators' rows, so that a lane holds one query's logits and the
// softmax needs one exchange between lane halves; the exponentials are the second operand of O^T = V^T P^T as they lie.
//
// P is rounded to bf16 for its product, which leaves out of 8 x 2048 2.1e-3 off (relative to 64 bits; its own rounding alone 1.6e-3): a second
// part would be a product more beside the two.
//
// Bound by the matrix cores and the exponentials, whose instructions overlap only so far.  32 and 8 heads of 128, 4 sequences of 4096: 525 to 580 us
// as the clocks allow, 0.95 to 1.05 PFLOP/s over the pairs that are seen, matrix cores busy 60 % of the time and vector units 58 %; 8 of 512 to
// 2048: 145 to 195 us, by the lengths, 36 % and 50 % (of one draw 151, 263 with a key head's workgroups on all XCDs, 160 with the order of steps
// that the compiler chose, 158 with rows stored as they lie); 40 and 8 heads, 4 of 1024 to 8192 under a window of 1024: 400 to 720 us, by the lengths.
// The grid is a workgroup for 128 rows, the last ones (which see most) first; where that leaves compute units idle the keys are cut.
template <typename E, int DP, int NW, int BK, bool kCache>
__global__ __launch_bounds__(NW * 64, AttnElem<E>::size == 2 || DP == 64 ? 2 : 1) void attn_fwd_kernel(AttnArgs a) {
  using El = AttnElem<E>;
  using Frag = typename El::Frag;
  using Tile = AttnTile<E, DP, BK>;
  constexpr int KS = Tile::KS, KB = BK / 32, DB = DP / 32, ROWS = NW * 32;
  extern __shared__ char lds[];
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  report_lengths(a);
  Work work;
  if (!attn_work(a.B * a.Hkv, a.nblk * a.nsplit, work)) return;
  const int split = uniform(work.in % a.nsplit), blk = uniform(a.nblk - 1 - work.in / a.nsplit);
  const uint32_t bh = work.bh;
  const int hk = uniform(bh % a.Hkv), b = uniform(bh / a.Hkv);
  const int lq = clamp_len(a.len_q, b, a.Tq), lk = clamp_len(a.len_k, b, a.Tk);

  // this lane's row
  const uint32_t r = blk * ROWS + w * 32 + (l & 31);
  const int qi = r / (uint32_t)a.G, head = hk * a.G + r % (uint32_t)a.G;
  const bool in = qi < a.Tq;
  const int p = qi < lq ? lk - lq + qi : -1;     // below 0: sees nothing
  Frag q[KS];
  {
    const char* src = a.q.p + b * a.q.seq + (int64_t)qi * a.q.slot + head * a.q.head;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const int d = 16 * ks + 8 * (l >> 5);
      q[ks] = p >= 0 && d < a.D ? El::load(src + d * El::size) : El::zero();
    }
  }
  // positions of the block's rows, and of this wavefront's
  const uint32_t r0 = blk * ROWS;
  auto first = [&](uint32_t row) { const int i = uniform(row / (uint32_t)a.G); return i < lq ? max(0, lk - lq + i) : -1; };
  auto last = [&](uint32_t row) { const int i = uniform(row / (uint32_t)a.G); return lk - lq + (i < lq ? i : lq - 1); };
  const int bmin = first(r0), bmax = bmin < 0 ? -1 : last(r0 + ROWS - 1);
  const int wmin = first(r0 + w * 32), wmax = wmin < 0 ? -1 : last(r0 + w * 32 + 31);
  const int wlow = __any(p < 0) ? -1 : wmin;      // with a row that sees nothing no tile is seen whole
  KeyTiles kt = key_tiles<BK>(bmin < 0 ? 0 : bmin, bmax, a.window, a.sinks);
  if (bmax < 0) kt.n = 0;
  const int per = uniform((kt.n + a.nsplit - 1) / (uint32_t)a.nsplit), t0 = split * per, t1 = min(kt.n, t0 + per);

  const char* kbase = a.k.p + b * a.k.seq + hk * a.k.head;
  const char* vbase = a.v.p + b * a.v.seq + hk * a.v.head;
  // K and V have two tiles each in LDS: K runs one tile ahead
  auto load_k = [&](int t, int at) {
    char* const to = lds + at * Tile::BYTES;
    const int s = tile_start<BK>(kt, t), n = tile_end(kt, t) - s;
    if constexpr (kCache) {
      const int64_t row = (int64_t)bh * a.Tk + s;
      load_cache<Tile, NW, BK>(to, a.k_codes + row * (a.D / 2), a.k_scales + row * (a.D / 32), n, a.D, w, l);
    } else {
      Tile::template load<NW>(to, kbase + s * a.k.slot, (uint32_t)a.k.slot, n, a.D * El::size, w, l);
    }
  };
  auto load_v = [&](int t, int at) {
    char* const to = lds + (2 + at) * Tile::BYTES;
    const int s = tile_start<BK>(kt, t), n = tile_end(kt, t) - s;
    if constexpr (kCache) {
      const int64_t row = (int64_t)bh * a.Tk + s;
      load_cache<Tile, NW, BK>(to, a.v_codes + row * (a.D / 2), a.v_scales + row * (a.D / 32), n, a.D, w, l);
    } else {
      Tile::template load<NW>(to, vbase + s * a.v.slot, (uint32_t)a.v.slot, n, a.D * El::size, w, l);
    }
  };

  f32x16_t o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
  float m = -INFINITY, sum = 0.f;      // the maximum that the exponentials are taken against, see below
  using Logits = f32x16_t[KB];
  const uint32_t rbase = Tile::row_base(l), cbase = Tile::col_base(l);

  auto logits = [&](Logits& s, const char* k) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[kb][i] = 0.f;
#pragma unroll
    for (int x = 0; x < KS * KB; ++x) El::mma(s[x % KB], Tile::row_frag(k, rbase, x % KB, x / KB), q[x / KB]);
  };

  // One tile: the softmax of `s`, beside which the matrix cores form the next tile's logits, and the product with V.
  auto step = [&](int t, auto which, auto last, Logits& s, Logits& next) {
    constexpr int P = decltype(which)::value;      // where its K and V lie
    __builtin_amdgcn_s_waitcnt(kWaitVm0);
    __syncthreads();
    if constexpr (!decltype(last)::value)
      if (t + 2 < t1) load_k(t + 2, P);
    if constexpr (!decltype(last)::value) load_v(t + 1, 1 - P);
    const int s0 = tile_start<BK>(kt, t), n = min(BK, tile_end(kt, t) - s0);
    if (n < BK || !all_seen(s0, n, wlow, wmax, a.window, a.sinks)) {
      const Seen sees(s0, n, p, a.window, a.sinks, 4 * (l >> 5));
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = sees(kb * 32 + acc_row(i, 0)) ? s[kb][i] : -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[kb][i]);
    top = max_halves(top) * a.scale2;
    if (__any(top > m + kSlack)) {
      const float now = fmaxf(m, top), keep = __builtin_amdgcn_exp2f(m - (now == -INFINITY ? 0.f : now));
      m = now;
      sum *= keep;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] *= keep;
    }
    const float base = m == -INFINITY ? 0.f : m;
    const char* const k = lds + (1 - P) * Tile::BYTES;
    const char* const v = lds + (2 + P) * Tile::BYTES;
    // In this order, which the compiler keeps between the steps: a product of the next tile's logits, two exponentials of this one's, the
    // reads of LDS three products ahead.  (Left to itself it puts the exponentials before the products and each read before its product.)
    constexpr int M = KS * KB, N = 2 * KB * DB, A = 3, EACH = 16 * KB / M;      // products, reads ahead, exponentials a product
    constexpr bool kMore = !decltype(last)::value;
    Frag pf[2 * KB], kf[A + 1], vf[A + 1];
    float e[16 * KB], part[2] = {0.f, 0.f};
    // fma, exponential and sum of a logit are a step apart each, so that none waits for the one before
    auto weigh = [&](int x) {
#pragma unroll
      for (int y = x * EACH; y < (x + 1) * EACH; ++y)
        if (y < 16 * KB) e[y] = fmaf(s[y / 16][y % 16], a.scale2, -base);
#pragma unroll
      for (int y = (x - 1) * EACH; y < x * EACH; ++y)
        if (y >= 0 && y < 16 * KB) e[y] = __builtin_amdgcn_exp2f(e[y]);
#pragma unroll
      for (int y = (x - 2) * EACH; y < (x - 1) * EACH; ++y)
        if (y >= 0) {
          part[y & 1] += e[y];
          if (y % 8 == 7) pf[y / 8] = El::of(e + y - 7);
        }
    };
    auto row = [&](int x) {
      if (x < M) kf[x % (A + 1)] = Tile::row_frag(k, rbase, x % KB, x / KB);
    };
    auto col = [&](int x) {
      if (x < N) vf[x % (A + 1)] = Tile::col_frag(v, cbase, x % DB, x / DB);
    };
    if constexpr (kMore) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) next[kb][i] = 0.f;
#pragma unroll
      for (int x = 0; x < A; ++x) row(x);
    }
    // (of a unit's two wavefronts the one in these products goes first, so that they fall out of step: 566 -> 553 us of the full 4 x 4096)
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int x = 0; x < M; ++x) {
      if constexpr (kMore) {
        El::mma(next[x % KB], kf[x % (A + 1)], q[x / KB]);
        row(x + A);
      }
      if (x >= M - A) col(x - (M - A));
      weigh(x);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
    weigh(M);
    weigh(M + 1);
    sum += part[0] + part[1];
#pragma unroll
    for (int x = 0; x < N; ++x) {
      El::mma(o[x % DB], vf[x % (A + 1)], pf[x / DB]);
      col(x + A);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  if (t0 < t1) {
    Logits s[2];
    load_k(t0, 0);
    load_v(t0, 0);
    __builtin_amdgcn_s_waitcnt(kWaitVm0);
    __syncthreads();
    if (t0 + 1 < t1) load_k(t0 + 1, 1);
    logits(s[0], lds);
    const std::integral_constant<int, 0> even;
    const std::integral_constant<int, 1> odd;
    int t = t0;
    for (; t + 2 < t1; t += 2) {
      step(t, even, std::false_type{}, s[0], s[1]);
      step(t + 1, odd, std::false_type{}, s[1], s[0]);
    }
    if (t + 1 < t1) {
      step(t, even, std::false_type{}, s[0], s[1]);
      step(t + 1, odd, std::true_type{}, s[1], s[0]);
    } else {
      step(t, even, std::true_type{}, s[0], s[1]);
    }
  }
  sum = add_halves(sum);

  if (a.nsplit > 1) {
    float* const part = a.part + ((int64_t)(bh * a.nsplit + split) * (a.nblk * ROWS) + r) * (DP + 2);
    if (!in) return;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) part[db * 32 + acc_row(i, l)] = o[db][i];
    if (l < 32) {
      part[DP] = m;
      part[DP + 1] = sum;
    }
    return;
  }
  __syncthreads();      // the tiles are done with
  const uint32_t row0 = r0 + w * 32;
  store_rows<E, DP>(lds + w * AttnTile<E, DP, 32>::BYTES, o, sum == 0.f ? 0.f : 1.f / sum, a.D, a.past_out, l, [&](int row) -> char* {
    const uint32_t i = (row0 + row) / (uint32_t)a.G, g = (row0 + row) % (uint32_t)a.G;
    return (int)i < a.Tq ? a.o.p + b * a.o.seq + (int64_t)i * a.o.slot + (hk * a.G + g) * a.o.head : nullptr;
  });
  if (in && a.lse && l < 32) a.lse[((int64_t)b * a.Hq + head) * a.Tq + qi] = lse_of(m, sum);
}

// Joins the parts of a row, sums and maxima of which it reads once: a wavefront each.  (Of a launch that did not fill the card, so short.)
template <typename E, int DP>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a, int rows) {
  const int l = threadIdx.x & 63;
  const int64_t R = (int64_t)a.Tq * a.G, id = ((int64_t)blockIdx.y * kAttnRow + blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (id >= R * a.B * a.Hkv) return;
  const int64_t bh = id / R, r = id % R;
  const float* const part = a.part + (bh * a.nsplit * a.nblk * rows + r) * (DP + 2);
  const int64_t step = (int64_t)a.nblk * rows * (DP + 2);
  float m = -INFINITY;
  for (int s = l; s < a.nsplit; s += 64) m = fmaxf(m, part[s * step + DP]);
#pragma unroll
  for (int x = 32; x; x >>= 1) m = fmaxf(m, __shfl_xor(m, x));
  const float base = m == -INFINITY ? 0.f : m;
  float sum = 0.f, o[DP / 64] = {};
#pragma unroll 8
  for (int s = 0; s < a.nsplit; ++s) {
    const float f = __builtin_amdgcn_exp2f(part[s * step + DP] - base);
    sum += f * part[s * step + DP + 1];
#pragma unroll
    for (int i = 0; i < DP / 64; ++i) o[i] += f * part[s * step + i * 64 + l];
  }
  const int b = (int)(bh / a.Hkv), head = (int)(bh % a.Hkv) * a.G + (int)(r % a.G), qi = (int)(r / a.G);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  char* const out = a.o.p + b * a.o.seq + (int64_t)qi * a.o.slot + head * a.o.head;
#pragma unroll
  for (int i = 0; i < DP / 64; ++i) {
    const int d = i * 64 + l;
    if (d >= a.D) continue;
    if constexpr (AttnElem<E>::size == 2) reinterpret_cast<uint16_t*>(out)[d] = (uint16_t)pack_bf16(o[i] * inv, 0.f);
    else reinterpret_cast<float*>(out)[d] = o[i] * inv;
  }
  if (a.lse && l == 0) a.lse[((int64_t)b * a.Hq + head) * a.Tq + qi] = lse_of(m, sum);
}

// 128 keys from s0 on, a wavefront 32 of them: lane l holds key 32 w + l % 32.  Codes come through `lds`, which is free again afterwards.
template <typename Tile, bool kCache>
__device__ inline void load_keys(const AttnArgs& a, typename Tile::Frag (&k)[Tile::KS], char* lds, uint32_t bh, int b, int hk, int s0, int lk, int w, int l) {
  using El = typename Tile::El;
  if constexpr (kCache) {
    const uint32_t rbase = Tile::row_base(l);
    for (int y = 0; y < 4; ++y) {
      const int64_t row = (int64_t)bh * a.Tk + s0 + y * 32;
      __syncthreads();
      load_cache<Tile, 4, 32>(lds, a.k_codes + row * (a.D / 2), a.k_scales + row * (a.D / 32), lk - s0 - y * 32, a.D, w, l);
      __syncthreads();
      if (w == y) {
#pragma unroll
        for (int ks = 0; ks < Tile::KS; ++ks) k[ks] = Tile::row_frag(lds, rbase, 0, ks);
      }
    }
    __syncthreads();
  } else {
    const int key = s0 + w * 32 + (l & 31);
    const char* src = a.k.p + b * a.k.seq + (int64_t)key * a.k.slot + hk * a.k.head;
#pragma unroll
    for (int ks = 0; ks < Tile::KS; ++ks) {
      const int d = 16 * ks + 8 * (l >> 5);
      k[ks] = key < lk && d < a.D ? El::load(src + d * El::size) : El::zero();
    }
  }
}

__device__ inline void put_weight(const AttnArgs& a, uint32_t bh, int key, float sum) {
  float* const to = a.weight + (int64_t)bh * a.Tk + key;
  *to = a.decay == 0.f ? sum : fmaf(a.decay, *to, sum);
}

// Weight that the keys got: S = Q K^T with the queries along the accumulators' rows, so that a lane adds up one key's column.  A workgroup
// takes a block of 128 keys of a key head (a wavefront 32 of them, in registers) and a part of the queries that see it, head by head in tiles
// of 32, one tile ahead in LDS.  The queries behind the window that see a block's first tokens are parts of their own.
//
// Bound by the exponentials and the masks beside one product.  4 sequences of 8192 under a window of 1024 with 28 and 4 heads of 128: 410 us (a
// workgroup a block of keys, one tile at a time: 2440, as long as the block of the first tokens takes); 8 of 2048 without: 205 (546).
template <typename E, int DP, bool kCache>
__global__ __launch_bounds__(256) void attn_weight_kernel(AttnArgs a, int parts) {
  using El = AttnElem<E>;
  using Frag = typename El::Frag;
  using Tile = AttnTile<E, DP, kQueryTile>;
  constexpr int KS = Tile::KS;
  extern __shared__ char lds[];
  __shared__ __attribute__((aligned(16))) float ends[2][kQueryTile], lows[2][kQueryTile];
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Work work;
  if (!attn_work(a.B * a.Hkv, parts, work)) return;
  const uint32_t bh = work.bh;
  const int hk = uniform(bh % a.Hkv), b = uniform(bh / a.Hkv);
  const int lq = clamp_len(a.len_q, b, a.Tq), lk = clamp_len(a.len_k, b, a.Tk);
  const int behind = a.nsink * a.far;
  const bool far = (int)work.in < behind;
  const uint32_t x = far ? work.in : work.in - behind, cut = far ? a.far : a.main;
  const int blk = uniform(x / cut), part = uniform(x % cut);
  const int s0 = blk * kKeyBlock, k0 = s0 + w * 32, key = k0 + (l & 31);
  const uint32_t rbase = Tile::row_base(l);
  if (s0 >= lk) return;
  const KeyItem item = key_item(s0, lq, lk, a.window, a.sinks);
  // the part's tiles, of all heads
  const int run = far ? item.far : item.main, begin = far ? item.far0 : item.i0, end = far ? lq : item.far0;
  const int64_t all = (int64_t)run * a.G;
  const int t0 = uniform((int)(all * part / cut)), t1 = uniform((int)(all * (part + 1) / cut));
  float sum = 0.f;
  if (t0 < t1) {
    Frag k[KS];
    load_keys<Tile, kCache>(a, k, lds, bh, b, hk, s0, lk, w, l);
    const int offset = lk - lq;
    int head = hk * a.G + t0 / run, i = begin + t0 % run * kQueryTile;      // of the tile that is loaded next
    float lse = 0.f, run_sum = 0.f;
    auto load = [&](int at) {
      Tile::template load<4>(lds + at * Tile::BYTES, a.q.p + b * a.q.seq + head * a.q.head + i * a.q.slot, (uint32_t)a.q.slot, end - i,
                             a.D * El::size, w, l);
      if (threadIdx.x < kQueryTile) lse = i + (int)threadIdx.x < end ? a.lse[((int64_t)b * a.Hq + head) * a.Tq + i + threadIdx.x] : -INFINITY;
    };
    load(0);
    for (int t = t0; t < t1; ++t) {
      const int at = (t - t0) & 1, i0 = i;
      if (threadIdx.x < kQueryTile) {
        const Ends e(lse);
        ends[at][threadIdx.x] = e.a, lows[at][threadIdx.x] = e.b;
      }
      __builtin_amdgcn_s_waitcnt(kWaitVm0);
      __syncthreads();
      i += kQueryTile;
      if (i >= end) i = begin, ++head;
      if (t + 1 < t1) load(1 - at);
      const char* const q = lds + at * Tile::BYTES;
      f32x16_t s;
#pragma unroll
      for (int y = 0; y < 16; ++y) s[y] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) El::mma(s, Tile::row_frag(q, rbase, 0, ks), k[ks]);
      float e[16], some[2] = {0.f, 0.f};
#pragma unroll
      for (int y = 0; y < 16; y += 4) {
        const f32x4_t hi = *reinterpret_cast<const f32x4_t*>(&ends[at][acc_row(y, l)]), lo = *reinterpret_cast<const f32x4_t*>(&lows[at][acc_row(y, l)]);
#pragma unroll
        for (int z = 0; z < 4; ++z) e[y + z] = fmaf(s[y + z], a.scale2, -hi[z]) - lo[z];
      }
      // (sums of a tile, then of sixteen: over thousands of queries a third of the error of one running sum)
      const int p0 = offset + i0;
      if (i0 + kQueryTile <= end && all_seen(k0, 32, p0, p0 + kQueryTile - 1, a.window, a.sinks)) {
#pragma unroll
        for (int y = 0; y < 16; ++y) some[y & 1] += __builtin_amdgcn_exp2f(e[y]);
      } else {
#pragma unroll
        for (int y = 0; y < 16; ++y) {
          const int row = acc_row(y, l);
          const float v = __builtin_amdgcn_exp2f(e[y]);
          some[y & 1] += ((i0 + row < end) & seen(key, p0 + row, a.window, a.sinks)) ? v : 0.f;
        }
      }
      run_sum += some[0] + some[1];
      if ((t & 15) == 15) sum += run_sum, run_sum = 0.f;
    }
    sum += run_sum;
  }
  const float mine = add_halves(sum);
  if (l >= 32) return;
  if (a.sums) {
    a.sums[((int64_t)bh * parts + work.in) * kKeyBlock + w * 32 + l] = mine;
  } else if (key < lk) {
    put_weight(a, bh, key, mine);
  }
}

// The same of fewer queries than a tile has rows: the rows (query, head) of a key head are packed as in the forward, and a workgroup goes
// through all of them.  (9 x 7069 keys in 4 bits, two queries of five heads: 51 us with a tile for each head.)
template <typename E, int DP, bool kCache>
__global__ __launch_bounds__(256) void attn_weight_few_kernel(AttnArgs a, int nkey) {
  using El = AttnElem<E>;
  using Tile = AttnTile<E, DP, kQueryTile>;
  constexpr int KS = Tile::KS;
  extern __shared__ char lds[];
  __shared__ float ends[kQueryTile], lows[kQueryTile];
  __shared__ int positions[kQueryTile];
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Work work;
  if (!attn_work(a.B * a.Hkv, nkey, work)) return;
  const uint32_t bh = work.bh;
  const int hk = uniform(bh % a.Hkv), b = uniform(bh / a.Hkv);
  const int lq = clamp_len(a.len_q, b, a.Tq), lk = clamp_len(a.len_k, b, a.Tk);
  const int s0 = work.in * kKeyBlock, key = s0 + w * 32 + (l & 31), offset = lk - lq, rows = lq * a.G;
  if (s0 >= lk) return;
  float sum = 0.f;
  if (!none_seen(s0, kKeyBlock, offset, lk - 1, a.window, a.sinks)) {
    typename El::Frag k[KS];
    load_keys<Tile, kCache>(a, k, lds, bh, b, hk, s0, lk, w, l);
    const uint32_t rbase = Tile::row_base(l);
    for (int r0 = 0; r0 < rows; r0 += kQueryTile) {
      __syncthreads();
      for (int x = threadIdx.x; x < kQueryTile * Tile::CH; x += 256) {
        const uint32_t row = x / Tile::CH, r = r0 + row, c = x % Tile::CH, qi = r / (uint32_t)a.G;
        u32x4_t v = {0, 0, 0, 0};
        if ((int)r < rows && (int)c * 16 < a.D * El::size)
          v = *reinterpret_cast<const u32x4_t*>(a.q.p + b * a.q.seq + (int64_t)qi * a.q.slot + (hk * a.G + r % (uint32_t)a.G) * a.q.head + c * 16);
        *reinterpret_cast<u32x4_t*>(lds + Tile::at(row, c)) = v;
      }
      if (threadIdx.x < kQueryTile) {
        const uint32_t r = r0 + threadIdx.x, qi = r / (uint32_t)a.G;
        const bool in = (int)r < rows;
        const Ends e(in ? a.lse[((int64_t)b * a.Hq + hk * a.G + r % (uint32_t)a.G) * a.Tq + qi] : -INFINITY);
        ends[threadIdx.x] = e.a, lows[threadIdx.x] = e.b;
        positions[threadIdx.x] = in ? offset + (int)qi : -1;
      }
      __syncthreads();
      f32x16_t s;
#pragma unroll
      for (int x = 0; x < 16; ++x) s[x] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) El::mma(s, Tile::row_frag(lds, rbase, 0, ks), k[ks]);
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const int row = acc_row(x, l);
        const float e = __builtin_amdgcn_exp2f(fmaf(s[x], a.scale2, -ends[row]) - lows[row]);
        sum += seen(key, positions[row], a.window, a.sinks) ? e : 0.f;
      }
    }
    sum = add_halves(sum);
  }
  if (l < 32 && key < lk) put_weight(a, bh, key, sum);
}

// Adds up the parts of a block of keys, in order.
__global__ __launch_bounds__(kKeyBlock) void attn_weight_sum_kernel(AttnArgs a, int parts, int nkey) {
  const int64_t x = (int64_t)blockIdx.y * kAttnRow + blockIdx.x, bh = x / nkey;
  if (bh >= (int64_t)a.B * a.Hkv) return;
  const int blk = (int)(x % nkey), key = blk * kKeyBlock + threadIdx.x;
  if (key >= clamp_len(a.len_k, (int)(bh / a.Hkv), a.Tk)) return;
  const float* const from = a.sums + bh * parts * kKeyBlock + threadIdx.x;
  float sum = 0.f;
  if (blk < a.nsink)
    for (int y = 0; y < a.far; ++y) sum += from[((int64_t)blk * a.far + y) * kKeyBlock];
  for (int y = 0; y < a.main; ++y) sum += from[((int64_t)a.nsink * a.far + (int64_t)blk * a.main + y) * kKeyBlock];
  put_weight(a, (uint32_t)bh, key, sum);
}

template <typename E, int DP, int NW, int BK, bool kCache>
hipError_t fwd(const AttnArgs& a, hipStream_t s) {
  constexpr auto kernel = attn_fwd_kernel<E, DP, NW, BK, kCache>;
  const int bytes = 4 * AttnTile<E, DP, BK>::BYTES;
  hipError_t e = allow_lds<kernel>(bytes);
  if (e != hipSuccess) return e;
  kernel<<<attn_grid(attn_wgs((int64_t)a.B * a.Hkv, (int64_t)a.nblk * a.nsplit)), NW * 64, bytes, s>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess || a.nsplit == 1) return e;
  attn_join_kernel<E, DP><<<attn_grid(((int64_t)a.B * a.Hkv * a.Tq * a.G + 3) / 4), 256, 0, s>>>(a, NW * 32);
  return hipGetLastError();
}

template <typename E, int DP, bool kCache>
hipError_t fwd_rows(const AttnArgs& a, hipStream_t s) {
  constexpr int BK = AttnElem<E>::size == 2 ? 64 : 32;
  return fwd<E, DP, 4, BK, kCache>(a, s);
}

template <typename E, int DP, bool kCache>
hipError_t weight(const attn_desc* d, const AttnPlan& p, const AttnArgs& a, hipStream_t s) {
  constexpr auto kernel = attn_weight_kernel<E, DP, kCache>;
  const int bytes = 2 * AttnTile<E, DP, kQueryTile>::BYTES, nkey = (a.Tk + kKeyBlock - 1) / kKeyBlock;
  const int64_t heads = (int64_t)a.B * a.Hkv, parts = attn_weight_parts(d, p);
  if (d->Tq < kQueryTile) {
    attn_weight_few_kernel<E, DP, kCache><<<attn_grid(attn_wgs(heads, nkey)), 256, bytes / 2, s>>>(a, nkey);
    return hipGetLastError();
  }
  kernel<<<attn_grid(attn_wgs(heads, parts)), 256, bytes, s>>>(a, (int)parts);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.sums) return e;
  attn_weight_sum_kernel<<<attn_grid(heads * nkey), kKeyBlock, 0, s>>>(a, (int)parts, nkey);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_fwd(const attn_desc* d, const AttnPlan& p, AttnArgs& a, hipStream_t s) {
  const bool c = a.k_codes != nullptr;
  if (d->dtype == LMHEAD_BF16) {
    if (p.DP == 64) return c ? fwd_rows<bf16_tag, 64, true>(a, s) : fwd_rows<bf16_tag, 64, false>(a, s);
    return c ? fwd_rows<bf16_tag, 128, true>(a, s) : fwd_rows<bf16_tag, 128, false>(a, s);
  }
  if (p.DP == 64) return c ? fwd_rows<f32_tag, 64, true>(a, s) : fwd_rows<f32_tag, 64, false>(a, s);
  return c ? fwd_rows<f32_tag, 128, true>(a, s) : fwd_rows<f32_tag, 128, false>(a, s);
}

hipError_t launch_attn_weight(const attn_desc* d, const AttnPlan& p, AttnArgs& a, hipStream_t s) {
  const bool c = a.k_codes != nullptr;
  if (d->dtype == LMHEAD_BF16) {
    if (p.DP == 64) return c ? weight<bf16_tag, 64, true>(d, p, a, s) : weight<bf16_tag, 64, false>(d, p, a, s);
    return c ? weight<bf16_tag, 128, true>(d, p, a, s) : weight<bf16_tag, 128, false>(d, p, a, s);
  }
  if (p.DP == 64) return c ? weight<f32_tag, 64, true>(d, p, a, s) : weight<f32_tag, 64, false>(d, p, a, s);
  return c ? weight<f32_tag, 128, true>(d, p, a, s) : weight<f32_tag, 128, false>(d, p, a, s);
}

}  // namespace lmhead
