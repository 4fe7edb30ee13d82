// Backward of attention over a window and a few first tokens: dq by blocks of queries, then dk and dv by blocks of keys, each recomputing
// P from the logits and lse.  Seven products instead of the five that one pass over the pairs would take, and no atomics; with bf16 storage two
// more in dq (and one in dk of few queries), for what rounding dS and out would cost.
#include <algorithm>

#include "attn_common.h"

namespace lmhead {

namespace {

// How dk and dv are cut.  Items (KeyItem: a block of keys of a key head, and the queries that see it) differ in length, with the
// window, the sequences' lengths and the first tokens, so the workgroups (as many as are resident) take equal shares of the row of all tiles.  A
// share may begin and end inside an item: what it has of that item it leaves as fp32 sums, which attn_parts_kernel adds up in order.
// (Eight sequences of 1024 to 4096 under a window of 1024, 28 and 4 heads: a workgroup an item, with the queries behind in items of their own, 920 us.)

// Where up to so many queries of a head see a block of keys, dS goes into its dk with sixteen bits instead of eight: over many queries its rounding
// leaves dk 1.41 times as far off as the rounding of dk alone, whatever the input; over few it depends on the few that carry weight (1.7 seen).
// That is decided for each block, so that neither a batch's padding nor what lies outside the window changes what a key gets.
constexpr int kFineQueries = 512;

// Least tiles of a share, where there are fewer than the card takes: a tile is 2 us in bf16 and 7 in fp32, and a part that is cut off is 128 KB
// to write and to read again.  (2 sequences of 33, 8 heads of one key head of 96 in fp32: 70 us the whole step, with 8 tiles 120; 8 of 128, bf16
// heads of 128: 65 and 71; 8 of 512: 134, but 137 in shares of 4 or 5.  So shares of up to twice that are made fewer, down to kFirstShares.)
constexpr int kLeastShare = 4, kLeastShareF32 = 2, kFirstShares = 256;
constexpr int kSumGroups = 8;       // workgroups that add up a cut item: with 4 they take twice as long for short sequences

// How many workgroups there are, and whether each has one item (short ones are not cut).
struct KeyShares {
  int nkey, wgs, least;     // least: tiles of a share
  bool whole;
};
KeyShares key_shares(const attn_desc* d, int resident) {
  KeyShares k{};
  k.nkey = (d->Tk + kKeyBlock - 1) / kKeyBlock;
  const int64_t G = d->Hq / d->Hkv, each = ((int64_t)d->Tq + kQueryTile - 1) / kQueryTile + 1, items = (int64_t)d->B * d->Hkv * k.nkey;
  k.least = d->dtype == LMHEAD_BF16 ? kLeastShare : kLeastShareF32;
  k.whole = each * G <= k.least;
  // (tiles of fewer items than are resident: up to 2^34)
  const int64_t wgs = k.whole ? items : items >= resident ? resident : std::min<int64_t>(resident, (items * each * G + k.least - 1) / k.least);
  k.wgs = (int)((wgs + 7) / 8 * 8);
  return k;
}

// before[b * nkey + blk]: tiles of one head's items before this one, over sequences and blocks; the last entry: all.  By one workgroup.
__device__ inline void count_tiles(const AttnArgs& a, int nkey) {
  __shared__ int64_t s_wave[4];
  const int n = a.B * nkey, l = threadIdx.x & 63, w = threadIdx.x >> 6;
  int64_t sum = 0;
  for (int x = 0; x < n; x += 256) {
    const int at = x + threadIdx.x;
    int64_t mine = 0;
    if (at < n) {
      const int b = at / nkey;
      const int lq = a.len_q ? min(max(a.len_q[b], 0), a.Tq) : a.Tq, lk = a.len_k ? min(max(a.len_k[b], 0), a.Tk) : a.Tk;
      mine = key_item(at % nkey * kKeyBlock, lq, lk, a.window, a.sinks).tiles();
    }
    int64_t upto = mine;
#pragma unroll
    for (int y = 1; y < 64; y <<= 1) {
      const int64_t v = __shfl_up(upto, y);
      upto += l >= y ? v : 0;
    }
    if (l == 63) s_wave[w] = upto;
    __syncthreads();
    int64_t prior = sum;
    for (int y = 0; y < 4; ++y) {
      if (y < w) prior += s_wave[y];
      sum += s_wave[y];
    }
    if (at < n) a.before[at] = prior + upto - mine;
    __syncthreads();
  }
  if (threadIdx.x == 0) a.before[n] = sum;
}

// Part of an item that a workgroup does: tiles [from, to) of the item's `tiles` (all heads).
struct Share {
  int64_t at, end;       // of this workgroup, in the row of all tiles
  int hk, item, from, to, tiles;
};
// The share's piece that begins at x.at; false: none is left.
__device__ inline bool next_piece(const AttnArgs& a, int nkey, Share& x) {
  if (x.at >= x.end) return false;
  const int n = a.B * nkey;
  const int64_t all = a.before[n] * a.G;      // of a key head
  x.hk = uniform((int)(x.at / all));
  const int64_t in = x.at - x.hk * all;
  int lo = 0, hi = n - 1;      // the last item that begins at or before `in` and is not empty: the last one of equal beginnings
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.before[mid] * a.G <= in) lo = mid;
    else hi = mid - 1;
  }
  x.item = uniform(lo);
  const int64_t begin = a.before[x.item] * a.G, stop = a.before[x.item + 1] * a.G;
  x.tiles = uniform((int)(stop - begin));
  x.from = uniform((int)(in - begin));
  const int64_t left = x.end - x.at;
  x.to = uniform((int)min((int64_t)x.tiles, x.from + left));
  x.at += x.to - x.from;
  return true;
}
__device__ inline void share_of(const AttnArgs& a, const KeyShares& sh, int wg, Share& x) {
  const int64_t all = a.before[a.B * sh.nkey] * a.G * a.Hkv;
  int64_t each = (all + sh.wgs - 1) / sh.wgs;
  // a compute unit each first: longer shares leave fewer parts to add up
  each = max(each, min((int64_t)2 * sh.least, (all + kFirstShares - 1) / kFirstShares));
  if (each < sh.least) each = sh.least;
  x.at = min(all, each * wg);
  x.end = min(all, x.at + each);
}

// bf16: the fourth operand of the pairs' products (g beside q, v beside k) stays in LDS, a wavefront's rows read by itself, since registers hold
// the sums; fp32: 512 registers a lane hold it.
template <typename E>
constexpr bool kRowsInLds = AttnElem<E>::size == 2;

// Rows as in the forward: a lane holds one query's column of S^T, dP^T and dQ^T, so lse and delta are one value each.
//
// delta = <g, out> carries the rounding of out.  Where few keys hold the weight that error is not small beside dP - delta, and its part of dq,
// the error times sum_j P_j k_j, does not average out.  But sum_j dS_j = sum_j P_j dP_j - delta is exactly that error, so with bf16 storage
// sum_j P_j k_j is added up beside dq (the same fragments of K) and taken out at the end, and dk gets the better delta.  And dS, whose few
// large values carry dq, goes into it as a sum of two bf16 numbers.  dq of eight sequences of 4096, relative to 64 bits: 2.7e-3 off without
// either, 2.4e-3 with the first, 1.7e-3 with both; the rounding of dq itself is 1.7e-3.
//
// Five products of a pair, bound by them and the exponentials.  Eight sequences of 1024 to 4096 under a window of 1024, 28 and 4 heads of 128:
// 680 to 780 us, matrix cores busy 49 % of the time.
template <typename E, int DP, int BK>
__global__ __launch_bounds__(256, kRowsInLds<E> ? 2 : 1) void attn_dq_kernel(AttnArgs a, int nkey) {
  using El = AttnElem<E>;
  using Frag = typename El::Frag;
  using Tile = AttnTile<E, DP, BK>;
  using Rows = AttnTile<E, DP, 32>;
  constexpr bool kFix = El::size == 2;
  constexpr int KS = Tile::KS, KB = BK / 32, DB = DP / 32, ROWS = 128, STAGE = 2 * Tile::BYTES;
  extern __shared__ char lds[];
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t rbase = Tile::row_base(l), cbase = Tile::col_base(l);      // (of Rows too)
  char* const grows = lds + 2 * STAGE + w * Rows::BYTES;
  report_lengths(a);
  if (nkey && !(blockIdx.x | blockIdx.y)) count_tiles(a, nkey);      // for the kernel that follows
  Work work;
  if (!attn_work(a.B * a.Hkv, a.nblk, work)) return;
  const int blk = a.nblk - 1 - work.in;
  const uint32_t bh = work.bh;
  const int hk = uniform(bh % a.Hkv), b = uniform(bh / a.Hkv);
  const int lq = clamp_len(a.len_q, b, a.Tq), lk = clamp_len(a.len_k, b, a.Tk);
  const uint32_t r = blk * ROWS + w * 32 + (l & 31);
  const int qi = r / (uint32_t)a.G, head = hk * a.G + r % (uint32_t)a.G;
  const bool in = qi < a.Tq;
  const int p = qi < lq ? lk - lq + qi : -1;
  const float lse = p >= 0 ? a.lse[((int64_t)b * a.Hq + head) * a.Tq + qi] : -INFINITY;
  const Ends end(lse);
  Frag q[KS], g[kRowsInLds<E> ? 1 : KS];
  float delta = 0.f;
  {
    const char* qs = a.q.p + b * a.q.seq + (int64_t)qi * a.q.slot + head * a.q.head;
    const int64_t at = b * a.o.seq + (int64_t)qi * a.o.slot + head * a.o.head;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const int d = 16 * ks + 8 * (l >> 5);
      const bool has = p >= 0 && d < a.D;
      q[ks] = has ? El::load(qs + d * El::size) : El::zero();
      const Frag f = has ? El::load(a.g.p + at + d * El::size) : El::zero();
      const Frag o = has ? El::load(a.o.p + at + d * El::size) : El::zero();
#pragma unroll
      for (int j = 0; j < 8; ++j) delta = fmaf(El::value(f, j), El::value(o, j), delta);
      if constexpr (kRowsInLds<E>) Rows::put_row(grows, rbase, ks, f);
      else g[ks] = f;
    }
    delta = add_halves(delta);
  }
  const uint32_t r0 = blk * ROWS;
  auto first = [&](uint32_t row) { const int i = uniform(row / (uint32_t)a.G); return i < lq ? max(0, lk - lq + i) : -1; };
  auto last = [&](uint32_t row) { const int i = uniform(row / (uint32_t)a.G); return lk - lq + (i < lq ? i : lq - 1); };
  const int bmin = first(r0), bmax = bmin < 0 ? -1 : last(r0 + ROWS - 1);
  const int wmin = first(r0 + w * 32), wmax = wmin < 0 ? -1 : last(r0 + w * 32 + 31);
  const int wlow = __any(p < 0) ? -1 : wmin;      // with a row that sees nothing no tile is seen whole
  KeyTiles kt = key_tiles<BK>(bmin < 0 ? 0 : bmin, bmax, a.window, a.sinks);
  if (bmax < 0) kt.n = 0;

  const char* kbase = a.k.p + b * a.k.seq + hk * a.k.head;
  const char* vbase = a.v.p + b * a.v.seq + hk * a.v.head;
  auto load = [&](int t, char* to) {
    const int s = tile_start<BK>(kt, t), n = tile_end(kt, t) - s;
    Tile::template load<4>(to, kbase + s * a.k.slot, (uint32_t)a.k.slot, n, a.D * El::size, w, l);
    Tile::template load<4>(to + Tile::BYTES, vbase + s * a.v.slot, (uint32_t)a.v.slot, n, a.D * El::size, w, l);
  };
  f32x16_t dq[DB], mean[kFix ? DB : 1];
  float off = 0.f;      // sum of dS
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      dq[db][i] = 0.f;
      if constexpr (kFix) mean[db][i] = 0.f;
    }

  if (kt.n) load(0, lds);
  for (int t = 0; t < kt.n; ++t) {
    char* const cur = lds + (t & 1) * STAGE;
    __builtin_amdgcn_s_waitcnt(kWaitVm0);
    __syncthreads();
    if (t + 1 < kt.n) load(t + 1, lds + ((t + 1) & 1) * STAGE);
    const int s0 = tile_start<BK>(kt, t), n = min(BK, tile_end(kt, t) - s0);
    if (none_seen(s0, n, wmin, wmax, a.window, a.sinks)) continue;
    const bool part = n < BK || !all_seen(s0, n, wlow, wmax, a.window, a.sinks);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      f32x16_t s, dp;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = dp[i] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        El::mma(s, Tile::row_frag(cur, rbase, kb, ks), q[ks]);
        if constexpr (kRowsInLds<E>) El::mma(dp, Tile::row_frag(cur + Tile::BYTES, rbase, kb, ks), Rows::row_frag(grows, rbase, 0, ks));
        else El::mma(dp, Tile::row_frag(cur + Tile::BYTES, rbase, kb, ks), g[ks]);
      }
      float e[16], ds[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float x = fmaf(s[i], a.scale2, -end.a);
        if constexpr (El::size == 4) x -= end.b;
        e[i] = __builtin_amdgcn_exp2f(x);
        ds[i] = e[i] * (dp[i] - delta);
      }
      if (part) {
        const Seen sees(s0, n, p, a.window, a.sinks, 4 * (l >> 5));
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const bool yes = sees(kb * 32 + acc_row(i, 0));
          e[i] = yes ? e[i] : 0.f;
          ds[i] = yes ? ds[i] : 0.f;
        }
      }
      if constexpr (kFix) {
#pragma unroll
        for (int i = 0; i < 16; ++i) off += ds[i];
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        Frag f, low, pf;
        if constexpr (kFix) El::split(ds + 8 * h, f, low), pf = El::of(e + 8 * h);
        else f = El::of(ds + 8 * h);
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const Frag kf = Tile::col_frag(cur, cbase, db, kb * 2 + h);
          El::mma(dq[db], kf, f);
          if constexpr (kFix) El::mma(dq[db], kf, low), El::mma(mean[db], kf, pf);
        }
      }
    }
  }
  off = add_halves(off);
  if (in && l < 32) a.delta[((int64_t)b * a.Hq + head) * a.Tq + qi] = delta + off;
  if constexpr (kFix) {
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) dq[db][i] = fmaf(-off, mean[db][i], dq[db][i]);
  }
  __syncthreads();      // the tiles are done with
  const uint32_t row0 = r0 + w * 32;
  store_rows<E, DP>(lds + w * AttnTile<E, DP, 32>::BYTES, dq, a.scale, a.D, a.past_out, l, [&](int row) -> char* {
    const uint32_t i = (row0 + row) / (uint32_t)a.G, g = (row0 + row) % (uint32_t)a.G;
    return (int)i < a.Tq ? a.dq.p + b * a.dq.seq + (int64_t)i * a.dq.slot + (hk * a.G + g) * a.dq.head : nullptr;
  });
}

// A wavefront holds 32 keys and their values; the workgroup's four walk the queries that see them, head by head, in tiles of 32.  S and dP
// have the queries along the accumulators' rows, so P and dS are operands of dV^T = g^T P and dK^T = Q^T dS as they lie.
//
// P in dv, and dS in dk of many queries, are single bf16 numbers: a second part of each would be two products more beside the four, and the outputs of
// the step below are 2.3e-3 off together, where their own roundings leave 1.7e-3.
//
// Four products of a pair (five where few queries see the keys, see kFineQueries), bound by reads of LDS beside them (q and g are read along rows and
// across).  The sequences above: 720 to 940 us (2 to 4 % of the backward less with four throughout).
// (64 keys a wavefront, which halves those reads, takes 512 registers and one wavefront a unit, and was slower by a tenth.)
template <typename E, int DP>
__global__ __launch_bounds__(256, kRowsInLds<E> ? 2 : 1) void attn_dkv_kernel(AttnArgs a, KeyShares sh) {
  using El = AttnElem<E>;
  using Frag = typename El::Frag;
  constexpr int BQ = kQueryTile;
  using Tile = AttnTile<E, DP, BQ>;
  constexpr int KS = Tile::KS, DB = DP / 32, STAGE = 2 * Tile::BYTES + 3 * BQ * 4;
  constexpr bool kSplit = El::size == 2;
  extern __shared__ char lds[];
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t rbase = Tile::row_base(l), cbase = Tile::col_base(l);
  char* const vrows = lds + 2 * STAGE + w * Tile::BYTES;
  // consecutive shares go to one XCD
  const int id = blockIdx.y * kAttnRow + blockIdx.x, wg = (id % 8) * (sh.wgs / 8) + id / 8;
  if (id >= sh.wgs) return;
  Share x;
  if (sh.whole) {
    if (wg >= a.B * a.Hkv * sh.nkey) return;
    x.hk = wg % a.Hkv, x.item = wg / a.Hkv, x.from = 0, x.to = x.tiles = -1, x.at = x.end = 0;
  } else {
    share_of(a, sh, wg, x);
  }
  for (bool first = true;; first = false) {
    if (sh.whole ? !first : !next_piece(a, sh.nkey, x)) return;
    const int b = uniform(x.item / (uint32_t)sh.nkey), s0 = uniform(x.item % (uint32_t)sh.nkey) * kKeyBlock, hk = x.hk;
    const int lq = clamp_len(a.len_q, b, a.Tq), lk = clamp_len(a.len_k, b, a.Tk);
    const KeyItem item = key_item(s0, lq, lk, a.window, a.sinks);
    const int each = item.tiles(), from = x.from, n = sh.whole ? each * a.G : x.to - x.from;
    const int key0 = s0 + w * 32, key = key0 + (l & 31), offset = lk - lq;
    __syncthreads();      // the piece before is done with LDS
    Frag k[KS], v[kRowsInLds<E> ? 1 : KS];
    {
      const char* ks_ = a.k.p + b * a.k.seq + (int64_t)key * a.k.slot + hk * a.k.head;
      const char* vs_ = a.v.p + b * a.v.seq + (int64_t)key * a.v.slot + hk * a.v.head;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int d = 16 * ks + 8 * (l >> 5);
        k[ks] = key < lk && d < a.D ? El::load(ks_ + d * El::size) : El::zero();
        const Frag f = key < lk && d < a.D ? El::load(vs_ + d * El::size) : El::zero();
        if constexpr (kRowsInLds<E>) Tile::put_row(vrows, rbase, ks, f);
        else v[ks] = f;
      }
    }
    // The tile that is loaded next: its head, its first query and the end of its run of queries.
    int g = each ? uniform((uint32_t)from / (uint32_t)each) : 0, c = each ? uniform((uint32_t)from % (uint32_t)each) : 0, ni = 0, nend = 0;
    auto place = [&]() {
      const bool main = c < item.main;
      ni = main ? item.i0 + c * BQ : item.far0 + (c - item.main) * BQ;
      nend = main ? item.far0 : lq;
    };
    float end_next = 0.f, low_next = 0.f, delta_next = 0.f;      // of the tile that is loaded next: one query a thread
    auto load = [&](char* to) {
      const int head = hk * a.G + g;
      Tile::template load<4>(to, a.q.p + b * a.q.seq + head * a.q.head + ni * a.q.slot, (uint32_t)a.q.slot, nend - ni, a.D * El::size, w, l);
      Tile::template load<4>(to + Tile::BYTES, a.g.p + b * a.g.seq + head * a.g.head + ni * a.g.slot, (uint32_t)a.g.slot, nend - ni,
                             a.D * El::size, w, l);
      if (threadIdx.x < BQ) {
        const int qi = ni + threadIdx.x;
        const int64_t at = ((int64_t)b * a.Hq + head) * a.Tq + qi;
        const float lse = qi < nend ? a.lse[at] : -INFINITY;
        const Ends e(lse);
        end_next = e.a, low_next = e.b;
        delta_next = qi < nend ? a.delta[at] : 0.f;
      }
    };
    auto put = [&](char* to) {
      if (threadIdx.x < BQ) {
        float* const f = reinterpret_cast<float*>(to + 2 * Tile::BYTES);
        f[threadIdx.x] = end_next;
        f[BQ + threadIdx.x] = delta_next;
        if constexpr (El::size == 4) f[2 * BQ + threadIdx.x] = low_next;
      }
    };
    f32x16_t dk[DB], dv[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) dk[db][i] = dv[db][i] = 0.f;

    if (n) {
      place();
      load(lds);
      put(lds);
    }
    auto walk = [&](auto fine) {
      for (int t = 0; t < n; ++t) {
        char* const cur = lds + (t & 1) * STAGE;
        char* const next = lds + ((t + 1) & 1) * STAGE;
        __builtin_amdgcn_s_waitcnt(kWaitVm0);
        __syncthreads();
        // (hidden from the compiler, which would keep every address of the loop in a register of its own)
        uint32_t rb = rbase, cb = cbase;
        asm volatile("" : "+v"(rb), "+v"(cb));
        const int rows = min(BQ, nend - ni), pmin = offset + ni, pmax = pmin + rows - 1;
        if (t + 1 < n) {
          if (++c == each) c = 0, ++g;
          place();
          load(next);
        }
        const float* const end = reinterpret_cast<const float*>(cur + 2 * Tile::BYTES);
        const float* const delta = end + BQ;
        if (!none_seen(key0, 32, pmin, pmax, a.window, a.sinks)) {
          f32x16_t s, dp;
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = dp[i] = 0.f;
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            El::mma(s, Tile::row_frag(cur, rb, 0, ks), k[ks]);
            if constexpr (kRowsInLds<E>) El::mma(dp, Tile::row_frag(cur + Tile::BYTES, rb, 0, ks), Tile::row_frag(vrows, rb, 0, ks));
            else El::mma(dp, Tile::row_frag(cur + Tile::BYTES, rb, 0, ks), v[ks]);
          }
          float pr[16], ds[16];
          const f32x4_t* const ends = reinterpret_cast<const f32x4_t*>(end + 4 * (l >> 5));
          const f32x4_t* const deltas = reinterpret_cast<const f32x4_t*>(delta + 4 * (l >> 5));
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float x = fmaf(s[i], a.scale2, -ends[2 * (i >> 2)][i & 3]);
            if constexpr (El::size == 4) x -= end[2 * BQ + acc_row(i, l)];
            pr[i] = __builtin_amdgcn_exp2f(x);
            ds[i] = pr[i] * (dp[i] - deltas[2 * (i >> 2)][i & 3]);
          }
          if (rows < BQ || !all_seen(key0, 32, pmin, pmax, a.window, a.sinks)) {
            // row c sees the key from position pmin + c on, to the end or to the last one whose window reaches it
            const int lane = 4 * (l >> 5), low = key - pmin - lane;
            const int high = (key < a.sinks ? rows - 1 : min(rows - 1, key + a.window - 1 - pmin)) - lane;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int c = acc_row(i, 0);
              const bool yes = (c >= low) & (c <= high);
              pr[i] = yes ? pr[i] : 0.f;
              ds[i] = yes ? ds[i] : 0.f;
            }
          }
          const Frag pf[2] = {El::of(pr), El::of(pr + 8)};
          Frag sf[2], low[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if constexpr (kSplit) {
              if constexpr (decltype(fine)::value) El::split(ds + 8 * h, sf[h], low[h]);
              else sf[h] = El::of(ds + 8 * h);
            } else {
              sf[h] = El::of(ds + 8 * h);
            }
          }
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int db = 0; db < DB; ++db) {
              El::mma(dv[db], Tile::col_frag(cur + Tile::BYTES, cb, db, h), pf[h]);
              const Frag qf = Tile::col_frag(cur, cb, db, h);
              El::mma(dk[db], qf, sf[h]);
              if constexpr (decltype(fine)::value) El::mma(dk[db], qf, low[h]);
            }
        }
        if (t + 1 < n) put(next);
      }
    };
    const int seers = item.far0 - item.i0 + (item.far ? lq - item.far0 : 0);      // queries of a head that see the block
    if (kSplit && seers <= kFineQueries) walk(std::integral_constant<bool, kSplit>{});
    else walk(std::false_type{});
    if (!sh.whole && (x.from > 0 || x.to < x.tiles)) {
      // slot 0: the end of an item, or its middle; slot 1: the beginning of one
      float* const to = a.part + ((int64_t)(2 * wg + (x.from > 0 ? 0 : 1)) * kKeyBlock + w * 32 + (l & 31)) * (2 * DP);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const int d = db * 32 + acc_row(i, l);
          *reinterpret_cast<f32x4_t*>(to + d) = f32x4_t{dk[db][i], dk[db][i + 1], dk[db][i + 2], dk[db][i + 3]};
          *reinterpret_cast<f32x4_t*>(to + DP + d) = f32x4_t{dv[db][i], dv[db][i + 1], dv[db][i + 2], dv[db][i + 3]};
        }
      continue;
    }
    if (key >= a.Tk) continue;
    char* const ok = a.dk.p + b * a.dk.seq + (int64_t)key * a.dk.slot + hk * a.dk.head;
    char* const ov = a.dv.p + b * a.dv.seq + (int64_t)key * a.dv.slot + hk * a.dv.head;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int d = db * 32 + acc_row(i, l);
        if (d >= a.D) continue;
        El::store4(ok + d * El::size, dk[db][i] * a.scale, dk[db][i + 1] * a.scale, dk[db][i + 2] * a.scale, dk[db][i + 3] * a.scale);
        El::store4(ov + d * El::size, dv[db][i], dv[db][i + 1], dv[db][i + 2], dv[db][i + 3]);
      }
  }
}

// Items that were cut: the workgroup whose share has the beginning adds up the parts, which lie with the shares that follow.  And blocks of
// keys without any tile, which no share has, become zeros (workgroups from sh.wgs on, one for each block of a key head).  Bound by reading
// the parts, 128 KB each and at most two for each of 512 workgroups: 37 us (a workgroup an item: 110).
template <typename E, int DP>
__global__ __launch_bounds__(256) void attn_parts_kernel(AttnArgs a, KeyShares sh) {
  using El = AttnElem<E>;
  constexpr int UNITS = 2 * DP / 4;
  const uint32_t wid = blockIdx.y * kAttnRow + blockIdx.x;
  const int id = wid / kSumGroups;
  if (id >= sh.wgs) {
    const uint32_t x = wid - kSumGroups * sh.wgs;
    const int item = x / a.Hkv, hk = x % a.Hkv, b = item / sh.nkey, s0 = item % sh.nkey * kKeyBlock;
    if (item >= a.B * sh.nkey || a.before[item + 1] != a.before[item]) return;
    for (int y = threadIdx.x; y < kKeyBlock * UNITS; y += 256) {
      const int key = s0 + y / UNITS, c = y % UNITS * 4, d = c >= DP ? c - DP : c;
      if (key >= a.Tk || d >= a.D) continue;
      const AttnTensor& t = c >= DP ? a.dv : a.dk;
      El::store4(t.p + b * t.seq + (int64_t)key * t.slot + hk * t.head + d * El::size, 0.f, 0.f, 0.f, 0.f);
    }
    return;
  }
  // the last piece of this share
  Share x, y;
  share_of(a, sh, id, x);
  if (x.at >= x.end) return;
  y = x;
  y.at = x.end - 1;
  next_piece(a, sh.nkey, y);
  // the item's first tile is in this share, its last one is not
  const int64_t begin = x.end - 1 - y.from;
  if (begin < x.at || begin + y.tiles <= x.end) return;
  const int64_t each = x.end - x.at;      // of the shares that follow too, less the last one
  const int parts = (int)((begin + y.tiles - x.end + each - 1) / each);
  const int b = y.item / sh.nkey, s0 = y.item % sh.nkey * kKeyBlock;
  for (int u = wid % kSumGroups * (kKeyBlock / kSumGroups * UNITS) + threadIdx.x; u < (wid % kSumGroups + 1) * (kKeyBlock / kSumGroups * UNITS); u += 256) {
    const int key = s0 + u / UNITS, c = u % UNITS * 4, d = c >= DP ? c - DP : c;
    if (key >= a.Tk || d >= a.D) continue;
    const int64_t in = (int64_t)(u / UNITS) * (2 * DP) + c, slot = (int64_t)kKeyBlock * 2 * DP;
    f32x4_t sum = *reinterpret_cast<const f32x4_t*>(a.part + (2 * (int64_t)id + 1) * slot + in);
#pragma unroll 8
    for (int z = 1; z <= parts; ++z) sum += *reinterpret_cast<const f32x4_t*>(a.part + 2 * (int64_t)(id + z) * slot + in);
    if (c < DP) sum *= a.scale;
    const AttnTensor& t = c >= DP ? a.dv : a.dk;
    El::store4(t.p + b * t.seq + (int64_t)key * t.slot + y.hk * t.head + d * El::size, sum.x, sum.y, sum.z, sum.w);
  }
}

int resident(const attn_desc* d) { return device_compute_units() * (d->dtype == LMHEAD_BF16 ? 2 : 1); }

template <typename E, int DP>
hipError_t bwd(const KeyShares& sh, AttnArgs a, hipStream_t s) {
  constexpr int BK = 32, fixed = kRowsInLds<E> ? 4 * AttnTile<E, DP, 32>::BYTES : 0;
  constexpr auto dq = attn_dq_kernel<E, DP, BK>;
  constexpr auto dkv = attn_dkv_kernel<E, DP>;
  const int bytes = 4 * AttnTile<E, DP, BK>::BYTES + fixed, more = bytes + 6 * BK * 4;
  hipError_t e = allow_lds<dq>(bytes);
  if (e == hipSuccess) e = allow_lds<dkv>(more);
  if (e != hipSuccess) return e;
  a.nblk = (int)(((int64_t)a.Tq * a.G + 127) / 128);
  dq<<<attn_grid(attn_wgs((int64_t)a.B * a.Hkv, a.nblk)), 256, bytes, s>>>(a, sh.whole ? 0 : sh.nkey);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  dkv<<<attn_grid(sh.wgs), 256, more, s>>>(a, sh);
  e = hipGetLastError();
  if (e != hipSuccess || sh.whole) return e;
  attn_parts_kernel<E, DP><<<attn_grid((int64_t)kSumGroups * sh.wgs + (int64_t)a.B * a.Hkv * sh.nkey), 256, 0, s>>>(a, sh);
  return hipGetLastError();
}

}  // namespace

size_t attn_before_bytes(const attn_desc* d) {
  const KeyShares k = key_shares(d, resident(d));
  return k.whole ? 0 : round_up(((size_t)d->B * k.nkey + 1) * sizeof(int64_t), 256);
}
size_t attn_parts_bytes(const attn_desc* d) {
  const KeyShares k = key_shares(d, resident(d));
  return k.whole ? 0 : (size_t)k.wgs * 2 * kKeyBlock * 2 * (d->D <= 64 ? 64 : 128) * sizeof(float);
}

hipError_t launch_attn_bwd(const attn_desc* d, const AttnPlan& p, AttnArgs& a, hipStream_t s) {
  const KeyShares k = key_shares(d, resident(d));
  if (d->dtype == LMHEAD_BF16) return p.DP == 64 ? bwd<bf16_tag, 64>(k, a, s) : bwd<bf16_tag, 128>(k, a, s);
  return p.DP == 64 ? bwd<f32_tag, 64>(k, a, s) : bwd<f32_tag, 128>(k, a, s);
}

}  // namespace lmhead
