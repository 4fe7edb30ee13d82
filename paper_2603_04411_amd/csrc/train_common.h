// Internal declarations of the operators around the head in a training step: preference loss, embedding lookup and its gradient,
// gradient norm and clipping.
#pragma once

#include "common.h"

namespace lmhead {

// A launch has fewer than 2^32 threads along x: workgroups in rows of kGridRow (the last row may be longer than what there is to do).
constexpr uint32_t kGridRow = 1 << 21;
static inline dim3 grid_of(int64_t wgs) {
  return dim3((unsigned)(wgs < kGridRow ? wgs : kGridRow), (unsigned)((wgs + kGridRow - 1) / kGridRow));
}
__device__ inline uint32_t grid_wg() { return blockIdx.y * kGridRow + blockIdx.x; }

// ---- preference loss (lmhead_pref.hip) --------------------------------------------------

// Up to so many responses and slots the loss is one workgroup: 8 x 32 8 us, 18 x 100 10 (in two launches 12), 32 x 64 14 (12).
constexpr int kPrefFewResponses = 24;
constexpr int kPrefFewSlots = 8192;
// Of more responses than kPrefTickets those of up to kPrefShort slots are a wavefront each (512 x 256: 12 us, a workgroup each 16;
// 8192 x 100: 26 and 124); up to kPrefTickets workgroups count themselves, and the last one adds up (a launch more costs what some 150
// counts on one word do).
constexpr int kPrefShort = 1024;
constexpr int kPrefTickets = 160;
// From more blocks of a response on they are added up once, by a launch of its own: 2 x 2 responses of 16 blocks 12.4 us, so 13.7;
// of 32 14.0 and 13.7; 4 x 4 of 128 53 and 25.
constexpr int kPrefBlocks = 16;
constexpr int kPrefCounted = 1024;      // up to so many responses each workgroup counts all pairs itself

struct PrefLayout {
  int64_t R, nb;         // responses, blocks of kLossSlotsPerBlock slots in one
  size_t done, sums, totals, rank, part, total;
};
static inline PrefLayout pref_layout(int64_t P, int64_t G, int32_t T) {
  PrefLayout L{};
  L.R = P * G;
  L.nb = loss_blocks(T);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += round_up(bytes, 256);
    return o;
  };
  L.done = take(256);
  L.sums = take((size_t)(L.R * L.nb) * 2 * sizeof(double));
  L.totals = take((size_t)L.R * 2 * sizeof(double));
  L.rank = take((size_t)L.R * 2 * sizeof(int32_t));
  L.part = take((size_t)L.R * 5 * sizeof(double));
  L.total = off;
  return L;
}
hipError_t launch_preference(const lmhead_preference& q, const float* lp, const float* lr, const float* reward, const int32_t* len,
                             int P, int G, int T, float* loss, float* g, float* ratio, float* stats, char* ws, hipStream_t s);

// ---- embedding (lmhead_embed.hip) -------------------------------------------------------

constexpr int kSortTile = 1024;      // slots per workgroup of a sorting pass
constexpr int kSortBits = 9;         // digits have at most so many bits
constexpr int kScanTiles = 64;       // up to so many tiles each adds up the counts of all of them itself
constexpr int kLongIdBytes = 16;
constexpr int kMergeTiles = 16;      // up to so many tiles are sorted by themselves and merged by ranks (64 KB of LDS)
constexpr int64_t kMergeCells = 64 << 20;   // unless more elements than these are to be zeroed
// Up to so many slots, and so many (slot, slot, 512 columns), the gradient is one launch without a sort.  Added to 152064 ids, one launch /
// sorted, us: 1024 x 1024 11 / 23   1024 x 4096 17 / 27   2048 x 1024 20 / 24   2048 x 4096 43 / 28   3000 x 1024 40 / 22.
constexpr int kFewSlots = 2048;
constexpr int64_t kFewWork = 12 << 20;
constexpr int kReportSlots = 4096;   // up to so many slots one workgroup of the lookup reports the errors of all

struct EmbedHeader {
  int32_t err;      // sticky error bits (kErrLen, kErrTok), where lmhead_check reads them
  int32_t nv;       // unused; lmhead_check copies it along
  int32_t nlong;    // ids whose rows span three chunks or more
  int32_t pad[61];
};
static_assert(sizeof(EmbedHeader) == 256, "header is one 256-byte line");

struct EmbedLayout {
  int64_t N;
  int bits, passes, digit;   // bits of a key (ids and V, the key of a slot that does not count), sorting passes, bits of a pass
  int64_t tiles, chunks;
  int C;                     // sorted slots per chunk of the sums
  int64_t ld_part;           // row pitch of the partial sums: a line more than d, or rows a power of two apart meet on one memory channel
  size_t hdr, key[2], slot[2], hist, list, part, total;
};
static inline EmbedLayout embed_layout(const lmhead_embed_desc* d) {
  EmbedLayout L{};
  L.N = (int64_t)d->R * d->T;
  L.bits = 1;
  while (((int64_t)d->V >> L.bits) != 0) ++L.bits;
  L.passes = (L.bits + kSortBits - 1) / kSortBits;
  L.digit = (L.bits + L.passes - 1) / L.passes;
  L.tiles = (L.N + kSortTile - 1) / kSortTile;
  // long chunks leave fewer partial sums; short ones keep 8192 wavefronts busy (eight per SIMD) where slots are few
  const int64_t cols = (d->d + 511) / 512;
  L.C = 64;
  while (L.C > 8 && L.N * cols < (int64_t)L.C * 8192) L.C /= 2;
  L.chunks = (L.N + L.C - 1) / L.C;
  // room for the chunks of any smaller batch: short ones are at most 16384 / cols
  int64_t room = (L.N + 7) / 8;
  if (room > 16384 / cols + 1) room = 16384 / cols + 1;
  if (room < L.chunks) room = L.chunks;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += round_up(bytes, 256);
    return o;
  };
  L.hdr = take(sizeof(EmbedHeader));
  for (int i = 0; i < 2; ++i) L.key[i] = take((size_t)L.N * 4);
  for (int i = 0; i < 2; ++i) L.slot[i] = take((size_t)L.N * 4);
  L.hist = take(((size_t)L.tiles << L.digit) * 4 + ((size_t)4 << L.digit));   // [digit][tile], then the totals
  L.list = take((size_t)room * kLongIdBytes);
  L.ld_part = d->d + 32;
  L.part = take((size_t)room * 2 * L.ld_part * 4);              // [chunk]{of an id that began earlier, of one that goes on}[d]
  L.total = off;
  return L;
}
hipError_t launch_embed_fwd(const lmhead_embed_desc& d, const void* W, const int32_t* tok, const int32_t* len, float scale, void* X,
                            EmbedHeader* hdr, hipStream_t s);
hipError_t launch_embed_bwd(const lmhead_embed_desc& d, const void* gX, const int32_t* tok, const int32_t* len, float scale, float* dW,
                            char* ws, hipStream_t s);

// ---- gradient norm and clipping (lmhead_grad.hip) -----------------------------------------

constexpr int kGradTensors = 96;     // tensors whose table one launch carries in its arguments
constexpr int kGradCount = 65536;    // tensors of one call
constexpr int kGradChunk = 8192;     // elements
constexpr int kClipParts = 4;        // workgroups of the scaling pass per chunk
constexpr int64_t kGradMost = 1ll << 37;   // elements of a tensor
constexpr int64_t kGradChunks = 1ll << 28; // chunks of a call
constexpr int kGradSpread = 2048;    // from twice so many chunks on a workgroup of the first pass takes several,
constexpr int kGradEach = 16;        // up to so many,
constexpr int kGradParts = 16384;    // and more where the partial sums would be more than these
constexpr int kGradShared = 512;     // up to so many partial sums every workgroup of the second pass adds up itself
constexpr int kFewChunk = 2048;      // elements of a chunk where the call is one workgroup:
constexpr int kGradFew = 48;         // up to so many of those
constexpr int kGradEntryBytes = 32;
static inline size_t grad_table_bytes() { return round_up((size_t)kGradCount * kGradEntryBytes, 256); }
static inline size_t grad_ws_bytes() { return grad_table_bytes() + (size_t)kGradParts * (sizeof(double) + sizeof(int32_t)); }
hipError_t launch_grads(const lmhead_tensor* g, const lmhead_tensor* out, int count, bool clip, float max_norm, float eps, float* norm,
                        char* ws, hipStream_t s);

}  // namespace lmhead
