// Internal declarations of the attention operators: launchers, workspace layout, and the tiles and fragments that their kernels share.
#pragma once

#include "../../include/dynakv.h"
#include "common.h"
#include "gemm_core.h"

namespace lmhead {

struct AttnHeader {
  int32_t err;      // sticky error bits, where lmhead_check reads them
  int32_t nv;       // unused; lmhead_check copies it along
  int32_t pad[62];
};
static_assert(sizeof(AttnHeader) == 256, "header is one 256-byte line");

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f, kLn2Low = 0.6931471805599453 - (double)kLn2;
constexpr float kLog2eLow = 1.4426950408889634 - (double)kLog2e;

// One tensor as a kernel sees it: strides in bytes.
struct AttnTensor {
  char* p;
  int64_t seq, slot, head;
};

struct AttnArgs {
  int B, Tq, Tk, Hq, Hkv, G, D;
  int window, sinks;        // window: kNoWindow for none
  float scale, scale2;      // scale2 = scale * log2(e)
  AttnTensor q, k, v, o;
  const uint8_t *k_codes, *k_scales, *v_codes, *v_scales;   // the cache in 4 bits (k and v are not set then)
  const int32_t *len_q, *len_k;
  float* lse;
  float* weight;
  float decay;
  AttnHeader* hdr;
  int nblk, nsplit;         // blocks of rows, and parts of a block's keys
  bool past;                // few rows: read K and V past the caches
  bool past_out;            // more: write the output (the backward: dq) past them
  float* logits;            // of a few rows: [b][key head][key][row], for the weights
  float* part;              // [b][key head][split][row of the block-padded rows]{DP sums, maximum, sum}
  // weights of more rows than a few: see attn_weight_kernel
  int nsink, far, main;     // blocks with first tokens, parts of their queries behind the window, parts of a block's others
  float* sums;              // [b][key head][part][128], or null: one part, and the weights are written at once
  // backward
  AttnTensor g, dq, dk, dv;
  float* delta;             // [b][head][query]
  int64_t* before;          // [b][block of keys]: tiles of the items before
};

constexpr int kFewRows = 32;
// Groups of four keys whose logits a key head has room for: tiles of first tokens and of the window, rounded up.
__host__ __device__ inline int64_t logit_groups(int Tk) { return ((int64_t)Tk + 3) / 4 + 32; }
constexpr int kLogitRows = 8;      // up to so many rows their logits are kept for the weights; of more K is read again

// What a call needs in its workspace, and how its work is cut: the same for every call with this descriptor.
struct AttnPlan {
  int DP;            // width of a head in the kernels: 64 or 128
  int rows;          // rows (query, head of the key head) of a workgroup
  int nblk, nsplit;
  int nsink, far, main;                // how the weights of more rows are cut
  // offsets of the parts' sums, of the logits of a few rows, of the weights' sums, of lse where the caller has no use for it
  size_t part, logits, sums, lse, total;
};
AttnPlan attn_plan(const attn_desc* d);
int64_t attn_weight_parts(const attn_desc* d, const AttnPlan& p);      // of a key head, over all blocks

hipError_t launch_attn_few(const attn_desc* d, const AttnPlan& p, const AttnArgs& a, hipStream_t s);   // at most kFewRows rows
hipError_t launch_attn_fwd(const attn_desc* d, const AttnPlan& p, AttnArgs& a, hipStream_t s);
hipError_t launch_attn_weight(const attn_desc* d, const AttnPlan& p, AttnArgs& a, hipStream_t s);
size_t attn_before_bytes(const attn_desc* d);     // how dk and dv are cut: counts of tiles
size_t attn_parts_bytes(const attn_desc* d);      // and the sums of items that were cut
hipError_t launch_attn_bwd(const attn_desc* d, const AttnPlan& p, AttnArgs& a, hipStream_t s);
hipError_t launch_kv4_store(const attn_desc* d, const AttnArgs& a, uint8_t* const* cache, hipStream_t s);
hipError_t launch_evict(const evict_desc& d, const cache_plane* planes, int count, float* weight, const int32_t* len, int32_t* len_out,
                        int32_t* kept, char* ws, hipStream_t s);

// A launch has fewer than 2^32 threads along x: workgroups in rows of kAttnRow.
constexpr uint32_t kAttnRow = 1 << 21;
static inline dim3 attn_grid(int64_t wgs) {
  return dim3((unsigned)(wgs < kAttnRow ? wgs : kAttnRow), (unsigned)((wgs + kAttnRow - 1) / kAttnRow));
}

// A block of 128 keys of a key head, and the queries that see some of them in tiles of 32 of one head: those that the block reaches through its
// window and, for a block with first tokens, the ones behind.
struct KeyItem {
  int i0, main, far0, far;      // first query and tiles of a head through the window, and behind
  __host__ __device__ int tiles() const { return main + far; }
};
constexpr int kKeyBlock = 128, kQueryTile = 32;

__host__ __device__ inline KeyItem key_item(int s0, int lq, int lk, int window, int sinks) {
  KeyItem x{0, 0, 0, 0};
  if (s0 >= lk) return x;
  const int offset = lk - lq, last = (lk < s0 + kKeyBlock ? lk : s0 + kKeyBlock) - 1;
  x.i0 = s0 > offset ? s0 - offset : 0;
  const int64_t end = (int64_t)last + window - offset;
  const int i1 = end < lq ? (int)end : lq;
  if (i1 > x.i0) x.main = (i1 - x.i0 + kQueryTile - 1) / kQueryTile;
  x.far0 = i1 > x.i0 ? i1 : x.i0;
  if (s0 < sinks && lq > x.far0) x.far = (lq - x.far0 + kQueryTile - 1) / kQueryTile;
  return x;
}

// ---- device side --------------------------------------------------------------------------

__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
// A workgroup's place: which (sequence, key head), and which of the `inner` works on it.
struct Work {
  uint32_t bh, in;
};
// Workgroups go to the eight XCDs in turn.  The works of a key head read the same keys, so they go to one XCD's L2, and key heads go to
// the XCDs in turn, so that sequences of unequal lengths do not leave some XCDs idle (8 x 2048, lengths from 512: a range of consecutive
// work for each XCD 263 us).  Where their number is no multiple of eight each is dealt out to 2, 4 or 8 XCDs, its works in turn.
__host__ __device__ inline uint32_t attn_parts(uint32_t heads) { return heads % 8 == 0 ? 1 : heads % 4 == 0 ? 2 : heads % 2 == 0 ? 4 : 8; }
static inline int64_t attn_wgs(int64_t heads, int64_t inner) {
  const int64_t s = attn_parts((uint32_t)heads);
  return heads * s * ((inner + s - 1) / s);
}
// false: a workgroup without work.
__device__ inline bool attn_work(uint32_t heads, uint32_t inner, Work& x) {
  const uint32_t w = blockIdx.y * kAttnRow + blockIdx.x, s = attn_parts(heads), per = (inner + s - 1) / s;
  const uint32_t k = w / 8, unit = (uint32_t)uniform(k / per) * 8 + w % 8, bh = unit / s;
  x.bh = bh;
  x.in = (uint32_t)uniform(k % per) * s + unit % s;
  return bh < heads && x.in < inner;
}

__device__ inline int clamp_len(const int32_t* len, int b, int T) {
  if (!len) return T;
  const int n = uniform(len[b]);
  return n < 0 ? 0 : n > T ? T : n;
}

// The first workgroup reports the lengths that are out of range.
__device__ inline void report_lengths(const AttnArgs& a) {
  if (blockIdx.x | blockIdx.y) return;
  int bad = 0;
  for (int b = threadIdx.x; b < a.B; b += blockDim.x) {
    if (a.len_q) bad |= (uint32_t)a.len_q[b] > (uint32_t)a.Tq;
    if (a.len_k) bad |= (uint32_t)a.len_k[b] > (uint32_t)a.Tk;
  }
  bad = __syncthreads_or(bad);
  if (threadIdx.x == 0) a.hdr->err = bad ? kErrLen : 0;
}

__device__ inline uint32_t pack_bf16(float lo, float hi) {
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
  const bf16x2_t r = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, r);
}

// Fragments of the 32x32 MFMA blocks.  Sixteen values of K make a step: lane l holds row (or column) l % 32 and, with h = l / 32,
// eight of them.  In which order the sixteen are dealt out is immaterial as long as both operands agree:
//  - contiguous K (a tile's rows, or registers filled from memory): 8 h .. 8 h + 7;
//  - K along the rows of a tile, and accumulators that become an operand: 4 h .. 4 h + 3, then 8 + 4 h .. 8 + 4 h + 3, which is
//    where an accumulator block has its rows, so that the exponentials never leave their lane.
template <typename E>
struct AttnElem;
template <>
struct AttnElem<bf16_tag> {
  static constexpr int size = 2;
  using Frag = u32x4_t;
  __device__ static inline Frag zero() { return u32x4_t{0, 0, 0, 0}; }
  __device__ static inline void mma(f32x16_t& c, const Frag& a, const Frag& b) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
  }
  __device__ static inline void mma(f32x4_t& c, const Frag& a, const Frag& b) {
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
  }
  __device__ static inline Frag of(const float* x) {
    return u32x4_t{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
  }
  // x = high + low to sixteen bits
  __device__ static inline void split(const float* x, Frag& high, Frag& low) {
    high = of(x);
    float r[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = x[j] - value(high, j);
    low = of(r);
  }
  __device__ static inline Frag load(const char* p) { return *reinterpret_cast<const u32x4_t*>(p); }
  __device__ static inline float value(const Frag& f, int j) {
    const uint32_t w = f[j >> 1];
    return __builtin_bit_cast(float, j & 1 ? w & 0xffff0000u : w << 16);
  }
  __device__ static inline void store4(char* p, float a, float b, float c, float d) {
    *reinterpret_cast<u32x2_t*>(p) = u32x2_t{pack_bf16(a, b), pack_bf16(c, d)};
  }
};
template <>
struct AttnElem<f32_tag> {
  static constexpr int size = 4;
  struct Frag {
    f32x4_t x[2];
  };
  __device__ static inline Frag zero() { return Frag{{f32x4_t{0, 0, 0, 0}, f32x4_t{0, 0, 0, 0}}}; }
  __device__ static inline void mma(f32x16_t& c, const Frag& a, const Frag& b) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x[i].x, b.x[i].x, c, 0, 0, 0);
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x[i].y, b.x[i].y, c, 0, 0, 0);
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x[i].z, b.x[i].z, c, 0, 0, 0);
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x[i].w, b.x[i].w, c, 0, 0, 0);
    }
  }
  __device__ static inline void mma(f32x4_t& c, const Frag& a, const Frag& b) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x[i].x, b.x[i].x, c, 0, 0, 0);
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x[i].y, b.x[i].y, c, 0, 0, 0);
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x[i].z, b.x[i].z, c, 0, 0, 0);
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x[i].w, b.x[i].w, c, 0, 0, 0);
    }
  }
  __device__ static inline Frag of(const float* x) { return Frag{{f32x4_t{x[0], x[1], x[2], x[3]}, f32x4_t{x[4], x[5], x[6], x[7]}}}; }
  __device__ static inline Frag load(const char* p) {
    return Frag{{reinterpret_cast<const f32x4_t*>(p)[0], reinterpret_cast<const f32x4_t*>(p)[1]}};
  }
  __device__ static inline float value(const Frag& f, int j) { return f.x[j >> 2][j & 3]; }
  __device__ static inline void store4(char* p, float a, float b, float c, float d) {
    *reinterpret_cast<f32x4_t*>(p) = f32x4_t{a, b, c, d};
  }
};

// A transposing read.  With nothing known of its memory the compiler has it wait for all loads into LDS on their way, the next tile's too;
// `restrict` is what it needs to know (kernels wait for a tile themselves).
__device__ __attribute__((always_inline)) inline u32x2_t read_across(const char* __restrict p) {
  typedef __attribute__((address_space(3))) i16x4_t* tptr_t;
  return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tptr_t)p));
}

// ROWS rows of DP values in LDS.  A row is CH chunks of 16 bytes; chunk c of row r sits at position c ^ swz(r) of its row.  A read along rows
// takes a chunk of eight consecutive rows at a time, which then lie in different 16-byte banks (of 128 bytes, and sixteen rows in those of 256);
// a transposing read takes 64 bytes of four rows (32 of eight where blocks are sixteen wide), which cover 256 bytes.  (With pairs of chunks
// spread instead, the transposing reads met twice on every bank: a third of the forward's LDS cycles.)
template <typename E, int DP, int ROWS>
struct AttnTile {
  using El = AttnElem<E>;
  using Frag = typename El::Frag;
  static constexpr int CH = DP * El::size / 16;
  static constexpr int ROW = CH * 16;
  static constexpr int BYTES = ROWS * ROW;
  static constexpr int KS = DP / 16;      // steps along a row
  static_assert(64 % CH == 0 && BYTES % 1024 == 0, "a load instruction fills whole rows");

  __device__ static inline int swz(int r) {
    const int r0 = r & 1, r1 = (r >> 1) & 1, r2 = (r >> 2) & 1, r3 = (r >> 3) & 1;
    return CH == 8 ? r1 << 2 | r2 << 1 | (r0 ^ r3) : (r1 ^ r3) << 3 | r0 << 2 | r2 << 1 | r1;
  }
  __device__ static inline int at(int r, int c) { return r * ROW + ((c ^ swz(r)) << 4); }

  // Rows straight from memory by NW wavefronts (wavefront w, lane l): `p` is row 0, `valid` rows exist; the others, and columns from
  // `width` bytes on, become zeros: the offsets of theirs lie outside the buffer, and such a load touches no memory.
  template <int NW>
  __device__ static inline void load(char* lds, const char* p, uint32_t stride, int valid, int width, int w, int l) {
    constexpr int PER = BYTES / 1024 / NW;
    static_assert(PER * 1024 * NW == BYTES, "loads divide evenly");
    const int rows = valid < 0 ? 0 : valid < ROWS ? valid : ROWS;
    const uint64_t base = reinterpret_cast<uint64_t>(p);
    const uint64_t first = (uint64_t)(uint32_t)uniform((int)(base >> 32)) << 32 | (uint32_t)uniform((int)base);
    const __amdgpu_buffer_rsrc_t rsrc =
        __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<char*>(first), 0, uniform((int)(rows * stride)), 0x00020000);
    typedef __attribute__((address_space(3))) void* lptr_t;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int r = (w * PER + i) * (64 / CH) + l / CH, c = (l % CH) ^ swz(r);
      const uint32_t off = c * 16 < width ? (uint32_t)r * stride + c * 16 : 0x80000000u;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lptr_t)(lds + (w * PER + i) * 1024), 16, off, 0, 0, 0);
    }
  }
  // A lane's reads are a base of its own, with the step or the column block put in by xor or as a constant: chunk numbers and swizzles
  // meet bit by bit, and a row begins at a multiple of its length.
  //
  // Step `ks` of rows 32 rb + l % 32.
  __device__ static inline uint32_t row_base(int l) {
    const int r = l & 31, h = l >> 5;
    return r * ROW + (((El::size == 2 ? h : 2 * h) ^ swz(r)) << 4);
  }
  __device__ static inline Frag row_frag(const char* lds, uint32_t base, int rb, int ks) {
    if constexpr (El::size == 2) {
      return *reinterpret_cast<const u32x4_t*>(lds + (base ^ (ks << 5)) + rb * 32 * ROW);
    } else {
      return Frag{{*reinterpret_cast<const f32x4_t*>(lds + (base ^ (ks << 6)) + rb * 32 * ROW),
                   *reinterpret_cast<const f32x4_t*>(lds + (base ^ (ks << 6) ^ 16) + rb * 32 * ROW)}};
    }
  }
  __device__ static inline void put_row(char* lds, uint32_t base, int ks, const Frag& f) {
    if constexpr (El::size == 2) {
      *reinterpret_cast<u32x4_t*>(lds + (base ^ (ks << 5))) = f;
    } else {
      *reinterpret_cast<f32x4_t*>(lds + (base ^ (ks << 6))) = f.x[0];
      *reinterpret_cast<f32x4_t*>(lds + (base ^ (ks << 6) ^ 16)) = f.x[1];
    }
  }
  // Columns 32 db + l % 32 of rows 16 s .. 16 s + 15 (dealt out as accumulators are).
  __device__ static inline uint32_t col_base(int l) {
    const int h = l >> 5, t = l & 15;
    if constexpr (El::size == 2) return (4 * h + (t >> 2)) * ROW + (((((l >> 4) & 1) * 2 + ((t & 3) >> 1)) ^ swz(4 * h + (t >> 2))) << 4) + 8 * (t & 1);
    else return 4 * h * ROW + ((((l & 31) >> 2) ^ swz(4 * h)) << 4) + 4 * (l & 3);
  }
  __device__ static inline Frag col_frag(const char* lds, uint32_t base, int db, int s) {
    if constexpr (El::size == 2) {
      u32x4_t f;
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const uint32_t at = (base ^ (CH == 8 ? db << 6 | p << 4 : (db ^ p << 1) << 6)) + (16 * s + 8 * p) * ROW;
        const u32x2_t v = read_across(lds + at);
        f[2 * p] = v.x;
        f[2 * p + 1] = v.y;
      }
      return f;
    } else {
      Frag f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int row = 8 * (j >> 2) + (j & 3);
        const uint32_t at = (base ^ (swz(row) & 7) << 4) + ((db ^ swz(row) >> 3) << 7) + (16 * s + row) * ROW;
        f.x[j >> 2][j & 3] = *reinterpret_cast<const float*>(lds + at);
      }
      return f;
    }
  }
  // The same for 16x16 blocks (steps of 32): columns 16 db + l % 16 of rows 32 s .. 32 s + 31, of which lane group g = l / 16 holds
  // 4 g .. 4 g + 3 and 16 + 4 g .. 16 + 4 g + 3, as two accumulator blocks do.
  __device__ static inline uint32_t col_base16(int l) {
    const int g = l >> 4, t = l & 15;
    if constexpr (El::size == 2) return (4 * g + (t >> 2)) * ROW + ((((t & 3) >> 1) ^ swz(4 * g + (t >> 2))) << 4) + 8 * (t & 1);
    else return 4 * g * ROW + (((t >> 2) ^ swz(4 * g)) << 4) + 4 * (t & 3);
  }
  __device__ static inline Frag col_frag16(const char* lds, uint32_t base, int db, int s) {
    if constexpr (El::size == 2) {
      u32x4_t f;
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const uint32_t at = (base ^ (db << 5)) + (32 * s + 16 * p) * ROW;
        const u32x2_t v = read_across(lds + at);
        f[2 * p] = v.x;
        f[2 * p + 1] = v.y;
      }
      return f;
    } else {
      Frag f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t at = (base ^ (swz(j & 3) ^ db << 2) << 4) + (32 * s + 16 * (j >> 2) + (j & 3)) * ROW;
        f.x[j >> 2][j & 3] = *reinterpret_cast<const float*>(lds + at);
      }
      return f;
    }
  }
};

// The exponentials are taken against a maximum that is only moved once a logit passes it by so many powers of two: the sums then
// need no scaling in most tiles, and nothing comes near fp32's range.
constexpr float kSlack = 8.f;

// log sum exp from a maximum in powers of two and the sum of 2^(logit - maximum): rounded once, but for the sum's logarithm.
__device__ inline float lse_of(float m, float sum) {
  return sum == 0.f ? -INFINITY : fmaf(m, kLn2, fmaf(m, kLn2Low, logf(sum)));
}
// lse in powers of two, which fp32 holds to half a unit only: P is 2^(logit - a - b).  (b only matters where P is not rounded to bf16.)
struct Ends {
  float a, b;
  __device__ inline explicit Ends(float lse) {
    a = lse == -INFINITY ? INFINITY : lse * kLog2e;
    b = lse == -INFINITY || lse == INFINITY ? 0.f : fmaf(lse, kLog2e, -a) + lse * kLog2eLow;
  }
};

// Row of accumulator element i of a 32x32 block.
__device__ inline int acc_row(int i, int l) { return 8 * (i >> 2) + 4 * (l >> 5) + (i & 3); }

// Rows that lie in accumulators across (lane l has columns 32 db + acc_row(i, l) of row l % 32) go to memory by way of 32 rows of LDS that are
// this wavefront's: as they lie a store would write sixteen bytes here and there.  `to(row)`: where a row goes, or null.  `past`: past the caches,
// where they would not hold the result (the forward of 8 x 2048, 134 MB: 158 us as they lie, 153 by rows, 151 past the caches).
template <typename E, int DP, typename To>
__device__ inline void store_rows(char* lds, const f32x16_t (&x)[DP / 32], float factor, int D, bool past, int l, const To& to) {
  using El = AttnElem<E>;
  using Tile = AttnTile<E, DP, 32>;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int db = 0; db < DP / 32; ++db)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const int at = (db * 32 + acc_row(i, l)) * El::size;
      El::store4(lds + Tile::at(l & 31, at / 16) + at % 16, x[db][i] * factor, x[db][i + 1] * factor, x[db][i + 2] * factor, x[db][i + 3] * factor);
    }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const int c = l % Tile::CH;
#pragma unroll
  for (int it = 0; it < 32 * Tile::CH / 64; ++it) {
    const int row = it * (64 / Tile::CH) + l / Tile::CH;
    const u32x4_t v = *reinterpret_cast<const u32x4_t*>(lds + Tile::at(row, c));
    char* const p = to(row);
    if (!p || c * 16 >= D * El::size) continue;
    if (past) __builtin_nontemporal_store(v, reinterpret_cast<u32x4_t*>(p + c * 16));
    else *reinterpret_cast<u32x4_t*>(p + c * 16) = v;
  }
}

// A value and that of the lane 32 (16) further, each in both of them: what is symmetric in the two needs no more.
struct Pair {
  float a, b;
};
__device__ inline Pair halves(float x) {
  const u32x2_t r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  const uint32_t a = r.x, b = r.y;      // (bit casts of a vector's elements are avoided)
  return Pair{__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}
__device__ inline Pair quarters(float x) {
  const u32x2_t r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  const uint32_t a = r.x, b = r.y;      // (bit casts of a vector's elements are avoided)
  return Pair{__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}
__device__ inline float max_halves(float x) { const Pair p = halves(x); return fmaxf(p.a, p.b); }
__device__ inline float add_halves(float x) { const Pair p = halves(x); return p.a + p.b; }
__device__ inline float max_quarters(float x) { const Pair p = quarters(x); return max_halves(fmaxf(p.a, p.b)); }
__device__ inline float add_quarters(float x) { const Pair p = quarters(x); return add_halves(p.a + p.b); }

// The keys that a block of queries at positions [pmin, pmax] sees: [0, e0) and [lo, e1), in tiles of BK.
struct KeyTiles {
  int e0, lo, e1, n0, n;
};
template <int BK>
__device__ inline KeyTiles key_tiles(int pmin, int pmax, int window, int sinks) {
  KeyTiles t;
  t.lo = pmin - window + 1 > 0 ? pmin - window + 1 : 0;
  t.e0 = sinks < t.lo ? sinks : 0;
  if (sinks >= t.lo) t.lo = 0;
  t.e1 = pmax + 1;
  t.n0 = (t.e0 + BK - 1) / BK;
  t.n = t.n0 + (t.e1 > t.lo ? (int)(((int64_t)t.e1 - t.lo + BK - 1) / BK) : 0);
  return t;
}
template <int BK>
__device__ inline int tile_start(const KeyTiles& t, int i) { return i < t.n0 ? i * BK : t.lo + (i - t.n0) * BK; }
__device__ inline int tile_end(const KeyTiles& t, int i) { return i < t.n0 ? t.e0 : t.e1; }

// (query, key) pairs: whether all, or none, of keys [s, s + n) are seen from positions [pmin, pmax].
__device__ inline bool all_seen(int s, int n, int pmin, int pmax, int window, int sinks) {
  return (s + n - 1 <= pmin) & ((s > pmax - window) | (s + n <= sinks));
}
__device__ inline bool none_seen(int s, int n, int pmin, int pmax, int window, int sinks) {
  return (s > pmax) | ((s + n - 1 <= pmin - window) & (s >= sinks));
}
// `span` is the window, or more than any position where there is none.
__device__ inline bool seen(int key, int p, int span, int sinks) {
  return (key <= p) & ((key > p - span) | (key < sinks));
}
// The same for the keys s + c, c < n, of a tile from position p, less `lane` (what of c depends on the lane): comparisons with constants.
struct Seen {
  int last, before, first;
  __device__ inline Seen(int s, int n, int p, int span, int sinks, int lane)
      : last(min(n - 1, p - s) - lane), before(p - span - s - lane), first(sinks - s - lane) {}
  __device__ inline bool operator()(int c) const { return (c <= last) & ((c > before) | (c < first)); }
};
constexpr int kNoWindow = 1 << 30;    // Tk is at most this

}  // namespace lmhead
