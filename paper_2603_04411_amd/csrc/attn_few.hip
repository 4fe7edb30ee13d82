// Attention of a few rows (the queries of a step, times the heads of a key head: at most 32) over a long cache, in bf16, fp32 or 4 bits.
#include "attn_common.h"

namespace lmhead {

namespace {

constexpr int kFewWaves = 4;

// A tile of TK keys of one key head in registers, on its way: K as fragments (lane l holds keys 16 kb + l % 16), V as it lies in memory.
//
// kPast: keys and values that no cache will hold are asked for past them (decoding 64 x 8192, 1.3 GB: 252 us, so 225; 16 x 2048, 134 MB,
// called again and again: 29 us, so 33).
template <typename E, int DP, int TK, bool kPast>
struct Plain {
  using El = AttnElem<E>;
  using Frag = typename El::Frag;
  using Tile = AttnTile<E, DP, TK>;
  static constexpr int KS = DP / 32, KB = TK / 16, VL = Tile::BYTES / 1024;
  u32x4_t k[KB][KS][El::size / 2], v[VL];

  // First channel of this lane's eight of step ks.
  __device__ static inline int channel(int ks, int l) { return 32 * ks + 8 * (l >> 4); }

  __device__ inline void load(const AttnArgs& a, uint32_t, int b, int hk, int s, int n, int l) {
    const int rows = n < TK ? n : TK, width = a.D * El::size;
    const __amdgpu_buffer_rsrc_t kr = rsrc(a.k.p + b * a.k.seq + hk * a.k.head + s * a.k.slot, rows * (int)a.k.slot);
    const __amdgpu_buffer_rsrc_t vr = rsrc(a.v.p + b * a.v.seq + hk * a.v.head + s * a.v.slot, rows * (int)a.v.slot);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int c = 0; c < El::size / 2; ++c) {
        const int at = channel(ks, l) * El::size + 16 * c;
        const uint32_t off = at < width ? (uint32_t)(l & 15) * (uint32_t)a.k.slot + at : 0x80000000u;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) k[kb][ks][c] = fetch(kr, off, 16 * kb * (int)a.k.slot);
      }
    const int at = (l % Tile::CH) * 16;
    const uint32_t off = at < width ? (uint32_t)(l / Tile::CH) * (uint32_t)a.v.slot + at : 0x80000000u;
#pragma unroll
    for (int i = 0; i < VL; ++i) v[i] = fetch(vr, off, i * (64 / Tile::CH) * (int)a.v.slot);
  }
  __device__ inline Frag key(int kb, int ks) const {
    if constexpr (El::size == 2) return k[kb][ks][0];
    else return Frag{{__builtin_bit_cast(f32x4_t, k[kb][ks][0]), __builtin_bit_cast(f32x4_t, k[kb][ks][1])}};
  }
  __device__ inline void put_values(char* lds, int l) const {
#pragma unroll
    for (int i = 0; i < VL; ++i) *reinterpret_cast<u32x4_t*>(lds + Tile::at((i * 64 + l) / Tile::CH, l % Tile::CH)) = v[i];
  }
  __device__ static inline __amdgpu_buffer_rsrc_t rsrc(const char* p, int bytes) {
    const uint64_t x = reinterpret_cast<uint64_t>(p);
    const uint64_t first = (uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32 | (uint32_t)uniform((int)x);
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<char*>(first), 0, uniform(bytes), 0x00020000);
  }
  // `off` of the lane and `more` of the wavefront together are held against the buffer's length
  __device__ static inline u32x4_t fetch(__amdgpu_buffer_rsrc_t r, uint32_t off, int more) {
    return __builtin_amdgcn_raw_buffer_load_b128(r, off, more, kPast ? 2 : 0);
  }
};

// Eight values from a word of codes.
template <typename E>
__device__ inline typename AttnElem<E>::Frag decode8(uint32_t codes, float size) {
  if constexpr (AttnElem<E>::size == 2) {
    return u32x4_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, size, 0)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, size, 1)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, size, 2)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, size, 3))};
  } else {
    const auto x0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, size, 0), x1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, size, 1);
    const auto x2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, size, 2), x3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, size, 3);
    return typename AttnElem<E>::Frag{{f32x4_t{x0[0], x0[1], x1[0], x1[1]}, f32x4_t{x2[0], x2[1], x3[0], x3[1]}}};
  }
}

// The same in 4 bits.  A lane's channels of a key are DP / 4 consecutive ones (q is dealt out alike), so that its codes are one load and it
// needs no exchange; V is written to LDS in the storage type, which holds its values exactly.
template <typename E, int DP, int TK, bool kPast>
struct Coded {
  using El = AttnElem<E>;
  using Frag = typename El::Frag;
  using Tile = AttnTile<E, DP, TK>;
  static constexpr int KS = DP / 32, KB = TK / 16, VL = TK * DP / 2 / 1024;   // (of 16 bytes = a block)
  typedef __attribute__((ext_vector_type(KS))) uint32_t Codes;
  Codes k[KB];
  u32x4_t v[VL];
  uint32_t ks_[KB], vs[VL];

  __device__ static inline int channel(int ks, int l) { return (DP / 4) * (l >> 4) + 8 * ks; }

  __device__ inline void load(const AttnArgs& a, uint32_t bh, int, int, int s, int n, int l) {
    const int64_t row = (int64_t)bh * a.Tk + s;
    const int rows = n < TK ? n : TK, cb = a.D / 2, sb = a.D / 32;
    const __amdgpu_buffer_rsrc_t kr = P::rsrc((const char*)a.k_codes + row * cb, rows * cb), kq = P::rsrc((const char*)a.k_scales + row * sb, rows * sb);
    const __amdgpu_buffer_rsrc_t vr = P::rsrc((const char*)a.v_codes + row * cb, rows * cb), vq = P::rsrc((const char*)a.v_scales + row * sb, rows * sb);
    {
      const int r = l & 15, at = channel(0, l) / 2;
      const uint32_t off = at < cb ? r * cb + at : 0x80000000u, sc = at < cb ? r * sb + at / 16 : 0x80000000u;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        if constexpr (KS == 4) k[kb] = P::fetch(kr, off, 16 * kb * cb);
        else k[kb] = __builtin_amdgcn_raw_buffer_load_b64(kr, off, 16 * kb * cb, 0);
        ks_[kb] = __builtin_amdgcn_raw_buffer_load_b8(kq, sc, 16 * kb * sb, 0);
      }
    }
    const int r = l / (DP / 32), block = l % (DP / 32);
    const uint32_t off = block < sb ? r * cb + block * 16 : 0x80000000u, sc = block < sb ? r * sb + block : 0x80000000u;
#pragma unroll
    for (int i = 0; i < VL; ++i) {
      v[i] = P::fetch(vr, off, i * (2048 / DP) * cb);
      vs[i] = __builtin_amdgcn_raw_buffer_load_b8(vq, sc, i * (2048 / DP) * sb, 0);
    }
  }
  __device__ inline Frag key(int kb, int ks) const { return decode8<E>(k[kb][ks], __builtin_bit_cast(float, ks_[kb] << 23)); }
  __device__ inline void put_values(char* lds, int l) const {
#pragma unroll
    for (int i = 0; i < VL; ++i) {
      const int r = (i * 64 + l) / (DP / 32), block = l % (DP / 32);
      const float size = __builtin_bit_cast(float, vs[i] << 23);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const Frag f = decode8<E>(v[i][c], size);
        if constexpr (El::size == 2) {
          *reinterpret_cast<u32x4_t*>(lds + Tile::at(r, block * 4 + c)) = f;
        } else {
          *reinterpret_cast<f32x4_t*>(lds + Tile::at(r, block * 8 + 2 * c)) = f.x[0];
          *reinterpret_cast<f32x4_t*>(lds + Tile::at(r, block * 8 + 2 * c + 1)) = f.x[1];
        }
      }
    }
  }
  using P = Plain<E, DP, TK, kPast>;
};

template <typename E, int DP, int NN, int TK>
constexpr int few_lds() {      // of a wavefront: a tile of values, then its sums with their maxima and totals
  constexpr int tile = AttnTile<E, DP, TK>::BYTES, sums = NN * 16 * (DP + 4) * 4;
  return tile > sums ? tile : sums;
}

// A workgroup takes the rows of one key head and a part of the keys they see; its wavefronts take tiles in turn, each with sums of its own,
// and join them through LDS.  Nothing is shared in the loop, so there is no barrier in it: a wavefront asks for its next tile in registers
// before the softmax of this one.
//
// P goes into its product as two bf16 numbers (kFineP): one leaves out 1.3 times as far off as its own rounding does (2.2e-3 against 1.66e-3, relative
// to 64 bits), and beside the reading the second one's product costs nothing (64 x 8192: 229 us with and without).  Over 4 bits, where conversions count
// and the cache itself is off by far more, it is one: 1.96e-3, and 143 us instead of 147 of 64 sequences up to 16001.
//
// Bound by the reading of the cache.  Rows and keys are on 16x16 blocks: a group of four rows fills a quarter of one, which is cheaper than
// a product in vector instructions.  64 sequences of 2048 to 8192, 32 and 8 heads of 128: 225 us, 6.0 TB/s; in 4 bits, up to 16001: 129 us, and
// 32 rows over 131072 keys 45 us, where the exponentials and the conversion to bf16 weigh more than the 143 MB.
template <typename E, int DP, int NN, int TK, bool kCache, bool kPast>
__global__ __launch_bounds__(kFewWaves * 64, AttnElem<E>::size == 2 ? 2 : 1) void attn_few_kernel(AttnArgs a) {
  using El = AttnElem<E>;
  using Frag = typename El::Frag;
  using Load = typename std::conditional<kCache, Coded<E, DP, TK, kPast>, Plain<E, DP, TK, kPast>>::type;
  using Tile = AttnTile<E, DP, TK>;
  constexpr int KS = DP / 32, KB = TK / 16, DB = DP / 16, WLDS = few_lds<E, DP, NN, TK>();
  constexpr bool kFineP = El::size == 2 && !kCache;
  extern __shared__ char lds_all[];
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = l >> 4;
  char* const lds = lds_all + w * WLDS;
  report_lengths(a);
  Work work;
  if (!attn_work(a.B * a.Hkv, a.nsplit, work)) return;
  const int split = work.in;
  const uint32_t bh = work.bh;
  const int hk = uniform(bh % a.Hkv), b = uniform(bh / a.Hkv);
  const int lq = clamp_len(a.len_q, b, a.Tq), lk = clamp_len(a.len_k, b, a.Tk);
  const int R = a.Tq * a.G;

  Frag q[NN][KS];
  int p[NN];
#pragma unroll
  for (int nn = 0; nn < NN; ++nn) {
    const int r = nn * 16 + (l & 15), qi = r / (uint32_t)a.G, head = hk * a.G + r % (uint32_t)a.G;
    p[nn] = qi < lq ? lk - lq + qi : -1;
    const char* const src = a.q.p + b * a.q.seq + (int64_t)qi * a.q.slot + head * a.q.head;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const int d = Load::channel(ks, l);
      q[nn][ks] = p[nn] >= 0 && d < a.D ? El::load(src + d * El::size) : El::zero();
    }
  }
  const int pmin = lq ? max(0, lk - lq) : -1, pmax = lq ? lk - 1 : -1;
  KeyTiles kt = key_tiles<TK>(max(pmin, 0), pmax, a.window, a.sinks);
  if (pmax < 0) kt.n = 0;
  const int per = uniform((kt.n + a.nsplit - 1) / (uint32_t)a.nsplit), t1 = min(kt.n, (split + 1) * per);
  const bool blind = lk < lq || lq < a.Tq;      // some row sees nothing: no tile is seen whole

  f32x4_t o[NN][DB];
  float m[NN], sum[NN];
#pragma unroll
  for (int nn = 0; nn < NN; ++nn) {
    m[nn] = -INFINITY, sum[nn] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) o[nn][db] = f32x4_t{0, 0, 0, 0};
  }
  Load next;
  const uint32_t cbase = Tile::col_base16(l);
  auto fetch = [&](int i) {
    const int s = tile_start<TK>(kt, i);
    next.load(a, bh, b, hk, s, tile_end(kt, i) - s, l);
  };
  int t = split * per + w;
  if (t < t1) fetch(t);
  for (; t < t1; t += kFewWaves) {
    const int s0 = tile_start<TK>(kt, t), n = min(TK, tile_end(kt, t) - s0);
    next.put_values(lds, l);
    f32x4_t s[NN][KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int nn = 0; nn < NN; ++nn) s[nn][kb] = f32x4_t{0, 0, 0, 0};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const Frag kf = next.key(kb, ks);
#pragma unroll
        for (int nn = 0; nn < NN; ++nn) El::mma(s[nn][kb], kf, q[nn][ks]);
      }
    // (where logits are stored, behind their stores: a wait for loads then finds older stores only, not ones that were issued since)
    if (!a.logits && t + kFewWaves < t1) fetch(t + kFewWaves);
    const bool part = blind || n < TK || !all_seen(s0, n, pmin, pmax, a.window, a.sinks);
#pragma unroll
    for (int nn = 0; nn < NN; ++nn) {
      if (part) {
        const Seen sees(s0, n, p[nn], a.window, a.sinks, 4 * g);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[nn][kb][i] = sees(16 * kb + i) ? s[nn][kb][i] : -INFINITY;
      }
      if (a.logits) {      // [four keys][row][key]: sixteen bytes a lane, and what a tile leaves is one piece
        const int r = nn * 16 + (l & 15);
        if (r < R) {
          f32x4_t* const to = reinterpret_cast<f32x4_t*>(a.logits) + (((int64_t)bh * logit_groups(a.Tk) + (int64_t)t * (TK / 4) + g) * R + r);
#pragma unroll
          for (int kb = 0; kb < KB; ++kb) to[kb * 4 * R] = s[nn][kb] * a.scale2;
        }
        if (nn == NN - 1 && t + kFewWaves < t1) fetch(t + kFewWaves);
      }
      float top = s[nn][0][0];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[nn][kb][i]);
      top = max_quarters(top) * a.scale2;
      if (__any(top > m[nn] + kSlack)) {
        const float now = fmaxf(m[nn], top), keep = __builtin_amdgcn_exp2f(m[nn] - (now == -INFINITY ? 0.f : now));
        m[nn] = now;
        sum[nn] *= keep;
#pragma unroll
        for (int db = 0; db < DB; ++db) o[nn][db] *= keep;
      }
      const float base = m[nn] == -INFINITY ? 0.f : m[nn];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[nn][kb][i] = __builtin_amdgcn_exp2f(fmaf(s[nn][kb][i], a.scale2, -base));
      f32x4_t part = s[nn][0];
#pragma unroll
      for (int kb = 1; kb < KB; ++kb) part += s[nn][kb];
      sum[nn] += (part.x + part.y) + (part.z + part.w);
    }
#pragma unroll
    for (int kg = 0; kg < KB / 2; ++kg) {
      Frag pf[NN], low[NN];
#pragma unroll
      for (int nn = 0; nn < NN; ++nn) {
        const float x[8] = {s[nn][2 * kg][0], s[nn][2 * kg][1], s[nn][2 * kg][2], s[nn][2 * kg][3],
                            s[nn][2 * kg + 1][0], s[nn][2 * kg + 1][1], s[nn][2 * kg + 1][2], s[nn][2 * kg + 1][3]};
        if constexpr (kFineP) El::split(x, pf[nn], low[nn]);
        else pf[nn] = El::of(x);
      }
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const Frag vf = Tile::col_frag16(lds, cbase, db, kg);
#pragma unroll
        for (int nn = 0; nn < NN; ++nn) {
          El::mma(o[nn][db], vf, pf[nn]);
          if constexpr (kFineP) El::mma(o[nn][db], vf, low[nn]);
        }
      }
    }
  }

  // join: sums of a wavefront are rows of DP + 4 floats (a row further apart by four banks)
  __syncthreads();
  float* const mine = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int nn = 0; nn < NN; ++nn) {
    const float total = add_quarters(sum[nn]);
    float* const row = mine + (nn * 16 + (l & 15)) * (DP + 4);
#pragma unroll
    for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4_t*>(row + db * 16 + 4 * g) = o[nn][db];
    if (g == 0) {
      row[DP] = m[nn];
      row[DP + 1] = total;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < R * DP; i += kFewWaves * 64) {
    const int r = i / DP, d = i % DP;
    const float* const row = reinterpret_cast<const float*>(lds_all) + r * (DP + 4);
    constexpr int step = WLDS / 4;
    float top = -INFINITY;
#pragma unroll
    for (int x = 0; x < kFewWaves; ++x) top = fmaxf(top, row[x * step + DP]);
    const float base = top == -INFINITY ? 0.f : top;
    float total = 0.f, acc = 0.f;
#pragma unroll
    for (int x = 0; x < kFewWaves; ++x) {
      const float f = __builtin_amdgcn_exp2f(row[x * step + DP] - base);
      total += f * row[x * step + DP + 1];
      acc += f * row[x * step + d];
    }
    const int qi = r / (uint32_t)a.G, head = hk * a.G + r % (uint32_t)a.G;
    if (a.nsplit > 1 || a.logits) {
      float* const part = a.part + ((int64_t)(bh * a.nsplit + split) * R + r) * (DP + 4);
      part[d] = acc;
      if (d == 0) {
        part[DP] = top;
        part[DP + 1] = total;
      }
    }
    if (a.nsplit > 1) continue;
    if (d < a.D) {
      char* const out = a.o.p + b * a.o.seq + (int64_t)qi * a.o.slot + head * a.o.head;
      const float y = total == 0.f ? 0.f : acc / total;
      if constexpr (El::size == 2) reinterpret_cast<uint16_t*>(out)[d] = (uint16_t)pack_bf16(y, 0.f);
      else reinterpret_cast<float*>(out)[d] = y;
    }
    if (d == 0 && a.lse)
      a.lse[((int64_t)b * a.Hq + head) * a.Tq + qi] = lse_of(top, total);
  }
}

// What follows the parts.  Rows are joined by a workgroup each: 32 threads take a row's channels, four each (half of them where there are 64),
// and eight groups of them every eighth part.  The weight of the keys is added up from the logits that the parts left, by workgroups of
// kWeightKeys keys: no second reading of K, but a logit for a key and row written and read in fp32 (64 x 8192, four rows a key head: 50 us in
// the parts' kernel, whose reads they disturb, and 20 here; reading K again 130).
constexpr int kWeightKeys = 1024;
template <typename E, int DP, int TK>
__global__ __launch_bounds__(256) void attn_finish_kernel(AttnArgs a, int njoin, int nkey) {
  __shared__ float s_top[8], s_total[8];      // of a row that is joined: of its eight groups of parts; else: of the rows
  __shared__ f32x4_t s_sum[8][DP / 4];
  Work work;
  if (!attn_work(a.B * a.Hkv, njoin + nkey, work)) return;
  const uint32_t bh = work.bh;
  const int part_of = work.in, hk = uniform(bh % a.Hkv), b = uniform(bh / a.Hkv), R = a.Tq * a.G, ns = a.nsplit;
  const int lq = clamp_len(a.len_q, b, a.Tq), lk = clamp_len(a.len_k, b, a.Tk);
  const float* const part = a.part + (int64_t)bh * ns * R * (DP + 4);
  const int step = R * (DP + 4);
  const bool joins = part_of < njoin;
  // Four keys a thread: their logits are one load a row unless a range begins or ends among them, or keys and groups of logits are out of
  // step.  They are asked for before the parts are looked at.  Keys outside [0, e0) and [lo, e1) are seen by no row and have no logits.
  const int pmin = lq ? max(0, lk - lq) : 0, pmax = lq ? lk - 1 : -1, key0 = (part_of - njoin) * kWeightKeys + 4 * threadIdx.x;
  const KeyTiles kt = key_tiles<TK>(pmin, pmax, a.window, a.sinks);
  const f32x4_t* const logits = reinterpret_cast<const f32x4_t*>(a.logits) + (int64_t)bh * logit_groups(a.Tk) * R;
  auto place = [&](int key) { return key < kt.e0 ? key : kt.n0 * TK + key - kt.lo; };
  const bool all = !joins && key0 < lk && pmax >= 0 && (key0 + 3 < kt.e0 || key0 >= kt.lo) && (place(key0) & 3) == 0;
  f32x4_t z[kLogitRows];
#pragma unroll
  for (int r = 0; r < kLogitRows; ++r) z[r] = all && r < R ? logits[(int64_t)(place(key0) >> 2) * R + r] : f32x4_t{0, 0, 0, 0};
  if (joins) {
    const int r = part_of, c = threadIdx.x & 31, of = threadIdx.x >> 5;
    float top = -INFINITY, total = 0.f;
    f32x4_t acc = f32x4_t{0, 0, 0, 0};
    constexpr int U = 4;      // parts asked for at once
    for (int s0 = of; s0 < ns; s0 += 8 * U) {
      float m[U], l[U];
      f32x4_t x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int s = s0 + 8 * u;
        const float* const at = part + (int64_t)(s < ns ? s : s0) * step + (int64_t)r * (DP + 4);
        m[u] = s < ns ? at[DP] : -INFINITY;
        l[u] = at[DP + 1];
        x[u] = c < DP / 4 ? *reinterpret_cast<const f32x4_t*>(at + 4 * c) : f32x4_t{0, 0, 0, 0};
      }
      float now = top;
#pragma unroll
      for (int u = 0; u < U; ++u) now = fmaxf(now, m[u]);
      const float base = now == -INFINITY ? 0.f : now, keep = __builtin_amdgcn_exp2f(top - base);
      total *= keep;
      acc *= keep;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float f = __builtin_amdgcn_exp2f(m[u] - base);
        total = fmaf(f, l[u], total);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = fmaf(f, x[u][i], acc[i]);
      }
      top = now;
    }
    if (c < DP / 4) s_sum[of][c] = acc;
    if (c == 0) s_top[of] = top, s_total[of] = total;
    __syncthreads();
    float base = s_top[0];
#pragma unroll
    for (int x = 1; x < 8; ++x) base = fmaxf(base, s_top[x]);
    if (base == -INFINITY) base = 0.f;
    total = 0.f;
#pragma unroll
    for (int x = 0; x < 8; ++x) total = fmaf(__builtin_amdgcn_exp2f(s_top[x] - base), s_total[x], total);
    const int qi = r / (uint32_t)a.G, head = hk * a.G + r % (uint32_t)a.G;
    if (threadIdx.x < DP / 4 && 4 * (int)threadIdx.x < a.D) {
      f32x4_t y = f32x4_t{0, 0, 0, 0};
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const float f = __builtin_amdgcn_exp2f(s_top[x] - base);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = fmaf(f, s_sum[x][threadIdx.x][i], y[i]);
      }
      const float inv = total == 0.f ? 0.f : 1.f / total;
      if (total == 0.f) y = f32x4_t{0, 0, 0, 0};
      char* const out = a.o.p + b * a.o.seq + (int64_t)qi * a.o.slot + head * a.o.head;
      AttnElem<E>::store4(out + 4 * threadIdx.x * AttnElem<E>::size, y.x * inv, y.y * inv, y.z * inv, y.w * inv);
    }
    if (threadIdx.x == 0 && a.lse)
      a.lse[((int64_t)b * a.Hq + head) * a.Tq + qi] = lse_of(base, total);
    return;
  }
  // maximum and total of each row: a wavefront takes every fourth row, its lanes the parts
  {
    const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (int r = w; r < R; r += 4) {
      const float* const at = part + (int64_t)r * (DP + 4) + DP;
      float top = -INFINITY, total = 0.f;
      for (int s = l; s < ns; s += 64) top = fmaxf(top, at[(int64_t)s * step]);
#pragma unroll
      for (int x = 32; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
      const float base = top == -INFINITY ? 0.f : top;
      for (int s = l; s < ns; s += 64) total = fmaf(__builtin_amdgcn_exp2f(at[(int64_t)s * step] - base), at[(int64_t)s * step + 1], total);
#pragma unroll
      for (int x = 32; x; x >>= 1) total += __shfl_xor(total, x);
      if (l == 0) s_top[r] = base, s_total[r] = total;
    }
  }
  __syncthreads();
  if (threadIdx.x < R) s_total[threadIdx.x] = s_total[threadIdx.x] == 0.f ? 0.f : 1.f / s_total[threadIdx.x];
  __syncthreads();
  if (key0 >= lk) return;
  f32x4_t sum = f32x4_t{0, 0, 0, 0};
  // (a key that a row does not see has the logit -inf: it adds nothing, also where the row's sum is NaN, or 0 because it sees no key)
  if (all) {
#pragma unroll
    for (int r = 0; r < kLogitRows; ++r) {
      if (r >= R) break;
      const float top = s_top[r], inv = s_total[r];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float e = __builtin_amdgcn_exp2f(z[r][i] - top);
        sum[i] = e == 0.f ? sum[i] : fmaf(e, inv, sum[i]);
      }
    }
  } else if (pmax >= 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int key = key0 + i;
      if (key >= kt.e0 && key < kt.lo) continue;
      const float* const x = reinterpret_cast<const float*>(logits + (int64_t)(place(key) >> 2) * R) + (place(key) & 3);
      for (int r = 0; r < R; ++r) {
        const float e = __builtin_amdgcn_exp2f(x[r * 4] - s_top[r]);
        sum[i] = e == 0.f ? sum[i] : fmaf(e, s_total[r], sum[i]);
      }
    }
  }
  float* const to = a.weight + (int64_t)bh * a.Tk + key0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (key0 + i < lk) to[i] = a.decay == 0.f ? sum[i] : fmaf(a.decay, to[i], sum[i]);
}

template <typename E, int DP, int NN, int TK, bool kCache, bool kPast>
hipError_t few_with(const AttnArgs& a, hipStream_t s) {
  constexpr auto kernel = attn_few_kernel<E, DP, NN, TK, kCache, kPast>;
  constexpr int bytes = kFewWaves * few_lds<E, DP, NN, TK>();
  hipError_t e = allow_lds<kernel>(bytes);
  if (e != hipSuccess) return e;
  kernel<<<attn_grid(attn_wgs((int64_t)a.B * a.Hkv, a.nsplit)), kFewWaves * 64, bytes, s>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess || (a.nsplit == 1 && !a.logits)) return e;
  const int njoin = a.nsplit > 1 ? a.Tq * a.G : 0, nkey = a.logits ? (a.Tk + kWeightKeys - 1) / kWeightKeys : 0;
  attn_finish_kernel<E, DP, TK><<<attn_grid(attn_wgs((int64_t)a.B * a.Hkv, njoin + nkey)), 256, 0, s>>>(a, njoin, nkey);
  return hipGetLastError();
}

template <typename E, int DP, int NN, int TK, bool kCache>
hipError_t few(const AttnArgs& a, hipStream_t s) {
  return a.past ? few_with<E, DP, NN, TK, kCache, true>(a, s) : few_with<E, DP, NN, TK, kCache, false>(a, s);
}

template <typename E, int DP>
hipError_t few_rows(const AttnArgs& a, hipStream_t s) {
  const bool one = a.Tq * a.G <= 16;
  if (a.k_codes) return one ? few<E, DP, 1, 32, true>(a, s) : few<E, DP, 2, 32, true>(a, s);
  return one ? few<E, DP, 1, 32, false>(a, s) : few<E, DP, 2, 32, false>(a, s);
}

}  // namespace

hipError_t launch_attn_few(const attn_desc* d, const AttnPlan& p, const AttnArgs& a, hipStream_t s) {
  if (d->dtype == LMHEAD_BF16) return p.DP == 64 ? few_rows<bf16_tag, 64>(a, s) : few_rows<bf16_tag, 128>(a, s);
  return p.DP == 64 ? few_rows<f32_tag, 64>(a, s) : few_rows<f32_tag, 128>(a, s);
}

}  // namespace lmhead
