// Backward of attention over a window and a few first tokens: dq by blocks of queries, then dk and dv by blocks of keys, each recomputing
// P from the logits and lse.  Seven products (bf16: eight) instead of the five that one pass over the pairs would take, and no atomics.
#include "attn_common.h"

namespace lmhead {

namespace {

// bf16: the fourth operand of the pairs' products (g beside q, v beside k) stays in LDS, a wavefront's rows read by itself, since registers hold
// the sums; fp32: 512 registers a lane hold it.
template <typename E>
constexpr bool kRowsInLds = AttnElem<E>::size == 2;

// Rows as in the forward: a lane holds one query's column of S^T, dP^T and dQ^T, so lse and delta are one value each.
//
// delta = <g, out> carries the rounding of out.  Where few keys hold the weight that error is not small beside dP - delta, and its part of dq,
// the error times sum_j P_j k_j, does not average out.  But sum_j dS_j = sum_j P_j dP_j - delta is exactly that error, so with bf16 storage
// sum_j P_j k_j is added up beside dq (the same fragments of K) and taken out at the end, and dk gets the better delta: dq of eight sequences
// of 4096 was 2.7e-3 off without it, of which the rounding of dq itself is 1.7e-3.
template <typename E, int DP, int BK>
__global__ __launch_bounds__(256, kRowsInLds<E> ? 2 : 1) void attn_dq_kernel(AttnArgs a) {
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
  const float end = lse == -INFINITY ? INFINITY : lse * kLog2e;
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
        e[i] = __builtin_amdgcn_exp2f(fmaf(s[i], a.scale2, -end));
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
        const Frag f = El::of(ds + 8 * h);
        Frag pf;
        if constexpr (kFix) pf = El::of(e + 8 * h);
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const Frag kf = Tile::col_frag(cur, cbase, db, kb * 2 + h);
          El::mma(dq[db], kf, f);
          if constexpr (kFix) El::mma(mean[db], kf, pf);
        }
      }
    }
  }
  off = add_halves(off);
  if (!in) return;
  if (l < 32) a.delta[((int64_t)b * a.Hq + head) * a.Tq + qi] = delta + off;
  char* const out = a.dq.p + b * a.dq.seq + (int64_t)qi * a.dq.slot + head * a.dq.head;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const int d = db * 32 + acc_row(i, l);
      float x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[j] = dq[db][i + j];
        if constexpr (kFix) x[j] = fmaf(-off, mean[db][i + j], x[j]);
      }
      if (d < a.D) El::store4(out + d * El::size, x[0] * a.scale, x[1] * a.scale, x[2] * a.scale, x[3] * a.scale);
    }
}

// How dk and dv are cut: per key head the blocks of 128 keys, each with the queries that it reaches through its window, and for
// the first tokens, which all later queries see, chunks of the queries behind those.  The rows of the first tokens are then sums of parts.
struct KeyWork {
  int nkey, nfirst, nchunk, rows;      // blocks; those with first tokens; chunks of queries; first tokens of a block that have parts
  __host__ __device__ int items() const { return nkey + nfirst * nchunk; }
};
constexpr int kFarQueries = 512;

// A wavefront holds 32 keys and their values; the workgroup's four walk the queries that see them, head by head, in tiles of BQ.  S and dP
// have the queries along the accumulators' rows, so P and dS are operands of dV^T = g^T P and dK^T = Q^T dS as they lie.
template <typename E, int DP, int BQ>
__global__ __launch_bounds__(256, kRowsInLds<E> ? 2 : 1) void attn_dkv_kernel(AttnArgs a, KeyWork kw) {
  using El = AttnElem<E>;
  using Frag = typename El::Frag;
  using Tile = AttnTile<E, DP, BQ>;
  using Rows = AttnTile<E, DP, 32>;
  constexpr int KS = Tile::KS, QB = BQ / 32, DB = DP / 32, STAGE = 2 * Tile::BYTES + 2 * BQ * 4;
  extern __shared__ char lds[];
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t rbase = Tile::row_base(l), cbase = Tile::col_base(l);      // (of Rows too)
  char* const vrows = lds + 2 * STAGE + w * Rows::BYTES;
  Work work;
  if (!attn_work(a.B * a.Hkv, kw.items(), work)) return;
  const uint32_t bh = work.bh;
  const int item = work.in, hk = uniform(bh % a.Hkv), b = uniform(bh / a.Hkv);
  const bool far = item >= kw.nkey;
  const int blk = far ? uniform((item - kw.nkey) / (uint32_t)kw.nchunk) : item, chunk = far ? uniform((item - kw.nkey) % (uint32_t)kw.nchunk) : 0;
  const int lq = clamp_len(a.len_q, b, a.Tq), lk = clamp_len(a.len_k, b, a.Tk);
  const int s0 = blk * 128, key0 = s0 + w * 32, key = key0 + (l & 31);
  Frag k[KS], v[kRowsInLds<E> ? 1 : KS];
  {
    const char* ks_ = a.k.p + b * a.k.seq + (int64_t)key * a.k.slot + hk * a.k.head;
    const char* vs_ = a.v.p + b * a.v.seq + (int64_t)key * a.v.slot + hk * a.v.head;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const int d = 16 * ks + 8 * (l >> 5);
      k[ks] = key < lk && d < a.D ? El::load(ks_ + d * El::size) : El::zero();
      const Frag f = key < lk && d < a.D ? El::load(vs_ + d * El::size) : El::zero();
      if constexpr (kRowsInLds<E>) Rows::put_row(vrows, rbase, ks, f);
      else v[ks] = f;
    }
  }
  // queries from the first at the block's first key to the last whose window reaches its last one
  const int offset = lk - lq, end_key = min(lk, s0 + 128) - 1;
  int i0 = max(0, s0 - offset), i1 = (int)min((int64_t)lq, (int64_t)end_key + a.window - offset);
  if (far) {
    i0 = max(max(i0, i1), chunk * kFarQueries);
    i1 = min(lq, (chunk + 1) * kFarQueries);
  }
  const int tiles = s0 < lk && i1 > i0 ? (i1 - i0 + BQ - 1) / BQ : 0, n = tiles * a.G;

  float end_next = 0.f, delta_next = 0.f;      // of the tile that is loaded next: one query a thread
  auto load = [&](int t, char* to) {
    const int g = uniform((uint32_t)t / (uint32_t)tiles), i = i0 + uniform((uint32_t)t % (uint32_t)tiles) * BQ, head = hk * a.G + g;
    Tile::template load<4>(to, a.q.p + b * a.q.seq + head * a.q.head + i * a.q.slot, (uint32_t)a.q.slot, i1 - i, a.D * El::size, w, l);
    Tile::template load<4>(to + Tile::BYTES, a.g.p + b * a.g.seq + head * a.g.head + i * a.g.slot, (uint32_t)a.g.slot, i1 - i,
                           a.D * El::size, w, l);
    if (threadIdx.x < BQ) {
      const int qi = i + threadIdx.x;
      const int64_t at = ((int64_t)b * a.Hq + head) * a.Tq + qi;
      const float lse = qi < i1 ? a.lse[at] : -INFINITY;
      end_next = lse == -INFINITY ? INFINITY : lse * kLog2e;
      delta_next = qi < i1 ? a.delta[at] : 0.f;
    }
  };
  auto put = [&](char* to) {
    if (threadIdx.x < BQ) {
      float* const f = reinterpret_cast<float*>(to + 2 * Tile::BYTES);
      f[threadIdx.x] = end_next;
      f[BQ + threadIdx.x] = delta_next;
    }
  };
  f32x16_t dk[DB], dv[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) dk[db][i] = dv[db][i] = 0.f;

  if (n) {
    load(0, lds);
    put(lds);
  }
  for (int t = 0; t < n; ++t) {
    char* const cur = lds + (t & 1) * STAGE;
    char* const next = lds + ((t + 1) & 1) * STAGE;
    __builtin_amdgcn_s_waitcnt(kWaitVm0);
    __syncthreads();
    if (t + 1 < n) load(t + 1, next);
    const int i = i0 + uniform((uint32_t)t % (uint32_t)tiles) * BQ, rows = min(BQ, i1 - i);
    const float* const end = reinterpret_cast<const float*>(cur + 2 * Tile::BYTES);
    const float* const delta = end + BQ;
    const int pmin = offset + i, pmax = offset + i + rows - 1;
    if (!none_seen(key0, 32, pmin, pmax, a.window, a.sinks)) {
      const bool part = rows < BQ || !all_seen(key0, 32, pmin, pmax, a.window, a.sinks);
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        f32x16_t s, dp;
#pragma unroll
        for (int x = 0; x < 16; ++x) s[x] = dp[x] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          El::mma(s, Tile::row_frag(cur, rbase, qb, ks), k[ks]);
          if constexpr (kRowsInLds<E>) El::mma(dp, Tile::row_frag(cur + Tile::BYTES, rbase, qb, ks), Rows::row_frag(vrows, rbase, 0, ks));
          else El::mma(dp, Tile::row_frag(cur + Tile::BYTES, rbase, qb, ks), v[ks]);
        }
        float pr[16], ds[16];
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const int row = qb * 32 + acc_row(x, l);
          pr[x] = __builtin_amdgcn_exp2f(fmaf(s[x], a.scale2, -end[row]));
          ds[x] = pr[x] * (dp[x] - delta[row]);
        }
        if (part) {
          // row c sees the key from position pmin + c on, to the end or to the last one whose window reaches it
          const int lane = 4 * (l >> 5), from = key - pmin - lane;
          const int to = (key < a.sinks ? rows - 1 : min(rows - 1, key + a.window - 1 - pmin)) - lane;
#pragma unroll
          for (int x = 0; x < 16; ++x) {
            const int c = qb * 32 + acc_row(x, 0);
            const bool yes = (c >= from) & (c <= to);
            pr[x] = yes ? pr[x] : 0.f;
            ds[x] = yes ? ds[x] : 0.f;
          }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const Frag pf = El::of(pr + 8 * h), sf = El::of(ds + 8 * h);
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            El::mma(dv[db], Tile::col_frag(cur + Tile::BYTES, cbase, db, qb * 2 + h), pf);
            El::mma(dk[db], Tile::col_frag(cur, cbase, db, qb * 2 + h), sf);
          }
        }
      }
    }
    if (t + 1 < n) put(next);
  }
  if (key >= a.Tk) return;
  const bool parts = blk < kw.nfirst && key - s0 < kw.rows && key < a.sinks;
  if (far && !parts) return;
  if (parts) {
    float* const to = a.part + (((int64_t)(bh * kw.nfirst + blk) * (kw.nchunk + 1) + (far ? chunk + 1 : 0)) * kw.rows + (key - s0)) * (2 * DP);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int d = db * 32 + acc_row(i, l);
        *reinterpret_cast<f32x4_t*>(to + d) = f32x4_t{dk[db][i], dk[db][i + 1], dk[db][i + 2], dk[db][i + 3]};
        *reinterpret_cast<f32x4_t*>(to + DP + d) = f32x4_t{dv[db][i], dv[db][i + 1], dv[db][i + 2], dv[db][i + 3]};
      }
    return;
  }
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

// Rows of the first tokens: a thread adds up four channels of one row's parts, in order.
template <typename E, int DP>
__global__ __launch_bounds__(256) void attn_first_kernel(AttnArgs a, KeyWork kw) {
  using El = AttnElem<E>;
  constexpr int UNITS = 2 * DP / 4;
  const int64_t id = ((int64_t)blockIdx.y * kAttnRow + blockIdx.x) * 256 + threadIdx.x, row = id / UNITS;
  const int c = (int)(id % UNITS) * 4, keys = kw.nfirst * kw.rows;
  const int64_t bh = row / keys;
  if (bh >= (int64_t)a.B * a.Hkv) return;
  const int blk = (int)(row % keys) / kw.rows, in = (int)(row % keys) % kw.rows, key = blk * 128 + in;
  if (key >= a.sinks || key >= a.Tk) return;
  const float* at = a.part + ((bh * kw.nfirst + blk) * (kw.nchunk + 1) * kw.rows + in) * (2 * DP) + c;
  f32x4_t sum = f32x4_t{0, 0, 0, 0};
  for (int i = 0; i <= kw.nchunk; ++i, at += (int64_t)kw.rows * 2 * DP) sum += *reinterpret_cast<const f32x4_t*>(at);
  const bool value = c >= DP;
  const int d = value ? c - DP : c, b = (int)(bh / a.Hkv), hk = (int)(bh % a.Hkv);
  if (d >= a.D) return;
  if (!value) sum *= a.scale;
  const AttnTensor& t = value ? a.dv : a.dk;
  El::store4(t.p + b * t.seq + (int64_t)key * t.slot + hk * t.head + d * El::size, sum.x, sum.y, sum.z, sum.w);
}

KeyWork key_work(int Tq, int Tk, int window, int sinks) {
  KeyWork w{};
  w.nkey = (Tk + 127) / 128;
  if (window == 0 || window >= Tk || sinks == 0) return w;
  sinks = sinks < Tk ? sinks : Tk;
  w.nfirst = (sinks + 127) / 128;
  w.nchunk = (Tq + kFarQueries - 1) / kFarQueries;
  w.rows = sinks < 128 ? sinks : 128;
  return w;
}

template <typename E, int DP>
hipError_t bwd(const KeyWork& kw, AttnArgs a, hipStream_t s) {
  constexpr int BK = 32, fixed = kRowsInLds<E> ? 4 * AttnTile<E, DP, 32>::BYTES : 0;
  constexpr auto dq = attn_dq_kernel<E, DP, BK>;
  constexpr auto dkv = attn_dkv_kernel<E, DP, BK>;
  const int bytes = 4 * AttnTile<E, DP, BK>::BYTES + fixed, more = bytes + 4 * BK * 4;
  hipError_t e = allow_lds<dq>(bytes);
  if (e == hipSuccess) e = allow_lds<dkv>(more);
  if (e != hipSuccess) return e;
  a.nblk = (int)(((int64_t)a.Tq * a.G + 127) / 128);
  dq<<<attn_grid(attn_wgs((int64_t)a.B * a.Hkv, a.nblk)), 256, bytes, s>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  dkv<<<attn_grid(attn_wgs((int64_t)a.B * a.Hkv, kw.items())), 256, more, s>>>(a, kw);
  e = hipGetLastError();
  if (e != hipSuccess || !kw.nfirst) return e;
  const int64_t threads = (int64_t)a.B * a.Hkv * kw.nfirst * kw.rows * (2 * DP / 4);
  attn_first_kernel<E, DP><<<attn_grid((threads + 255) / 256), 256, 0, s>>>(a, kw);
  return hipGetLastError();
}

}  // namespace

size_t attn_first_bytes(const attn_desc* d) {
  const KeyWork w = key_work(d->Tq, d->Tk, d->window, d->sinks);
  return (size_t)d->B * d->Hkv * w.nfirst * (w.nchunk + 1) * w.rows * 2 * (d->D <= 64 ? 64 : 128) * sizeof(float);
}

hipError_t launch_attn_bwd(const attn_desc* d, const AttnPlan& p, AttnArgs& a, hipStream_t s) {
  const KeyWork w = key_work(d->Tq, d->Tk, d->window, d->sinks);
  if (d->dtype == LMHEAD_BF16) return p.DP == 64 ? bwd<bf16_tag, 64>(w, a, s) : bwd<bf16_tag, 128>(w, a, s);
  return p.DP == 64 ? bwd<f32_tag, 64>(w, a, s) : bwd<f32_tag, 128>(w, a, s);
}

}  // namespace lmhead
