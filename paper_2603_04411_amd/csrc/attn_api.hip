// extern "C" entry points of the attention operators.  As in lmhead_api.hip every argument error is returned before anything is
// enqueued.
#include <math.h>

#include <algorithm>
#include <initializer_list>

#include "attn_common.h"
#include "attn_regions.h"

namespace lmhead {

namespace {

// The queries of a block of keys are cut for about 4096 workgroups in all, into parts of eight tiles at least; those behind the window of a
// block with first tokens into parts of about the same length.
void weight_parts(const attn_desc* d, AttnPlan& p) {
  const int64_t G = d->Hq / d->Hkv, heads = (int64_t)d->B * d->Hkv, nkey = (d->Tk + kKeyBlock - 1) / kKeyBlock;
  const int64_t all = ((int64_t)d->Tq + kQueryTile - 1) / kQueryTile * G;
  const int64_t most = d->window ? std::min(all, (((int64_t)d->window + kKeyBlock - 1) / kQueryTile + 2) * G) : all;
  p.main = (int)std::max<int64_t>(1, std::min(4096 / (heads * nkey), most / 8));
  p.nsink = d->window && d->window < d->Tk ? (std::min(d->sinks, d->Tk) + kKeyBlock - 1) / kKeyBlock : 0;
  if (p.nsink == 0) return;
  const int64_t each = (most + p.main - 1) / p.main;
  p.far = (int)std::max<int64_t>(1, std::min((all + each - 1) / each, 16384 / (heads * p.nsink)));
}

}  // namespace

int64_t attn_weight_parts(const attn_desc* d, const AttnPlan& p) {
  return (int64_t)p.nsink * p.far + (int64_t)(d->Tk + kKeyBlock - 1) / kKeyBlock * p.main;
}

AttnPlan attn_plan(const attn_desc* d) {
  AttnPlan p{};
  p.DP = d->D <= 64 ? 64 : 128;
  const int64_t G = d->Hq / d->Hkv, R = d->Tq * G, heads = (int64_t)d->B * d->Hkv;
  const bool few = R <= kFewRows;
  p.rows = few ? (int)R : 128;
  p.nblk = (int)((R + p.rows - 1) / p.rows);
  const int64_t wgs = heads * p.nblk;
  const int64_t span = d->window ? std::min<int64_t>(d->Tk, (int64_t)d->window + d->sinks + p.rows / G + 1) : d->Tk;
  if (few) {
    // A workgroup's part: 1024 keys (its wavefronts' eight tiles each hide the start), less where that leaves compute units idle, down to
    // two tiles a wavefront; not more parts than the joining workgroups want to add up.
    const int64_t tiles = (span + 31) / 32;
    const int64_t want = std::max(tiles / 32, std::min(tiles / 8, 512 / heads));
    p.nsplit = (int)std::max<int64_t>(1, std::min<int64_t>({want, 4096 / heads, 256}));
  } else {
    p.nsplit = (int)std::max<int64_t>(1, std::min<int64_t>({512 / wgs, (span + 63) / 64, 256}));
  }
  size_t off = sizeof(AttnHeader);
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += round_up(bytes, 256);
    return o;
  };
  p.part = take(few || p.nsplit > 1 ? (size_t)wgs * p.nsplit * p.rows * (p.DP + 4) * sizeof(float) : 0);
  p.logits = take(R <= kLogitRows ? (size_t)heads * logit_groups(d->Tk) * R * 4 * sizeof(float) : 0);
  if (d->Tq >= kQueryTile) weight_parts(d, p);
  p.sums = take(d->Tq >= kQueryTile && R > kLogitRows && p.main + p.nsink > 1 ? (size_t)heads * attn_weight_parts(d, p) * kKeyBlock * sizeof(float) : 0);
  p.lse = take((size_t)d->B * d->Hq * d->Tq * sizeof(float));
  p.total = off;
  return p;
}

}  // namespace lmhead

using namespace lmhead;

namespace {

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

constexpr int64_t kMostStride = 1ll << 40;

bool strides(const attn_layout& x) {
  for (int64_t v : {x.seq, x.slot, x.head})
    if (v < 0 || v > kMostStride) return false;
  return true;
}

// Whether no two rows of `width` elements (n sequences, t slots, h heads) lie upon each other.
bool apart(const attn_layout& x, int64_t n, int64_t t, int64_t h, int64_t width) {
  struct Dim {
    int64_t stride, size;
  } d[3] = {{x.seq, n}, {x.slot, t}, {x.head, h}};
  std::sort(d, d + 3, [](const Dim& a, const Dim& b) { return a.stride < b.stride; });
  int64_t extent = width;      // of what the dimensions so far span
  for (const Dim& k : d) {
    if (k.size == 1) continue;
    if (k.stride < extent) return false;
    extent += spanned(k.stride, k.size);
  }
  return true;
}

// A layout that a tensor which is read can have: its slots lie apart, at most what a tile's 32-bit offsets reach.
int check_layout(const attn_layout& x, int64_t D, int esz) {
  if (!strides(x) || x.slot < D || x.slot * esz >= (1 << 24)) return LMHEAD_E_SHAPE;
  for (int64_t v : {x.seq, x.slot, x.head})
    if (v * esz % 16 != 0) return LMHEAD_E_ALIGN;
  return LMHEAD_OK;
}

int validate(const attn_desc* d) {
  if (!d) return LMHEAD_E_NULL;
  if (d->B <= 0 || d->B > 65535 || d->Tq <= 0 || d->Tk <= 0 || d->Hq <= 0 || d->Hkv <= 0 || d->Hq > 1024) return LMHEAD_E_SHAPE;
  if (d->Hq % d->Hkv != 0 || d->D <= 0 || d->D > 128 || d->D % 8 != 0) return LMHEAD_E_SHAPE;
  if (d->Tq > kNoWindow / 1024 || d->Tk > kNoWindow - 4096) return LMHEAD_E_SHAPE;
  if (d->window < 0 || d->sinks < 0 || !isfinite(d->scale * kLog2e) || d->scale <= 0.f) return LMHEAD_E_SHAPE;
  if (d->dtype != LMHEAD_F32 && d->dtype != LMHEAD_BF16) return LMHEAD_E_DTYPE;
  if (d->flags != 0) return LMHEAD_E_DTYPE;
  if (d->reserved != 0) return LMHEAD_E_SHAPE;
  const int esz = d->dtype == LMHEAD_BF16 ? 2 : 4;
  // work items are counted in 32 bits
  const int64_t rows = (int64_t)d->Tq * (d->Hq / d->Hkv), blocks = std::max((rows + 31) / 32, ((int64_t)d->Tk + 127) / 128);
  if ((int64_t)d->B * d->Hkv > ((int64_t)INT32_MAX - 8) / blocks) return LMHEAD_E_SHAPE;
  for (const attn_layout* x : {&d->q, &d->k, &d->v, &d->o}) {
    const int rc = check_layout(*x, d->D, esz);
    if (rc != LMHEAD_OK) return rc;
  }
  return apart(d->o, d->B, d->Tq, d->Hq, d->D) ? LMHEAD_OK : LMHEAD_E_SHAPE;
}

AttnTensor tensor(const void* p, const attn_layout& x, int esz) {
  return AttnTensor{static_cast<char*>(const_cast<void*>(p)), x.seq * esz, x.slot * esz, x.head * esz};
}

AttnArgs arguments(const attn_desc* d, const AttnPlan& p, const int32_t* len_q, const int32_t* len_k, void* ws) {
  AttnArgs a{};
  a.B = d->B, a.Tq = d->Tq, a.Tk = d->Tk, a.Hq = d->Hq, a.Hkv = d->Hkv, a.G = d->Hq / d->Hkv, a.D = d->D;
  a.window = d->window && d->window < kNoWindow ? d->window : kNoWindow;
  a.sinks = std::min(d->sinks, d->Tk);
  a.scale = d->scale;
  a.scale2 = d->scale * kLog2e;
  a.len_q = len_q, a.len_k = len_k;
  a.hdr = static_cast<AttnHeader*>(ws);
  a.nblk = p.nblk, a.nsplit = p.nsplit;
  // against what the eight L2s hold
  a.past_out = (int64_t)d->B * d->Tq * d->Hq * d->D * (d->dtype == LMHEAD_BF16 ? 2 : 4) > (32ll << 20);
  a.part = reinterpret_cast<float*>(static_cast<char*>(ws) + p.part);
  return a;
}

size_t lse_bytes(const attn_desc* d) { return round_up((size_t)d->B * d->Hq * d->Tq * sizeof(float), 256); }

int run_fwd(const attn_desc* d, const AttnPlan& p, AttnArgs& a, void* ws, float* lse, float* weight, float decay, hipStream_t s) {
  char* const base = static_cast<char*>(ws);
  a.weight = weight;
  a.decay = decay;
  const int64_t rows = (int64_t)d->Tq * a.G;
  // what the call reads of the cache, against what the last-level cache holds
  const int64_t span = d->window ? std::min<int64_t>(d->Tk, (int64_t)d->window + d->sinks + d->Tq) : d->Tk;
  const int64_t row = a.k_codes ? d->D / 2 + d->D / 32 : (int64_t)d->D * (d->dtype == LMHEAD_BF16 ? 2 : 4);
  a.past = 2 * (int64_t)d->B * d->Hkv * span * row > (256ll << 20);
  if (weight && rows <= kLogitRows) {
    a.lse = lse;
    a.logits = reinterpret_cast<float*>(base + p.logits);
    LM_TRY(launch_attn_few(d, p, a, s));
    return LMHEAD_OK;
  }
  // the weights need lse: where the caller does not want it, it stays in the workspace
  a.nsink = p.nsink, a.far = p.far, a.main = p.main;
  a.sums = p.main + p.nsink > 1 ? reinterpret_cast<float*>(base + p.sums) : nullptr;
  a.lse = lse || !weight ? lse : reinterpret_cast<float*>(base + p.lse);
  LM_TRY(rows <= kFewRows ? launch_attn_few(d, p, a, s) : launch_attn_fwd(d, p, a, s));
  if (weight) LM_TRY(launch_attn_weight(d, p, a, s));
  return LMHEAD_OK;
}

// Whether no output shares memory with another output or an input.
bool different(std::initializer_list<Region> outputs, std::initializer_list<Region> inputs) {
  for (auto o = outputs.begin(); o != outputs.end(); ++o) {
    for (auto x = outputs.begin(); x != o; ++x)
      if (share(*x, *o)) return false;
    for (const Region& x : inputs)
      if (share(x, *o)) return false;
  }
  return true;
}

// The tensors of a descriptor.
struct Regions {
  const attn_desc* d;
  int esz;
  explicit Regions(const attn_desc* desc) : d(desc), esz(desc->dtype == LMHEAD_BF16 ? 2 : 4) {}
  Region q(const void* p, const attn_layout& x) const { return Region(p, x, d->B, d->Tq, d->Hq, (int64_t)d->D * esz, esz); }
  Region k(const void* p, const attn_layout& x) const { return Region(p, x, d->B, d->Tk, d->Hkv, (int64_t)d->D * esz, esz); }
  Region added(const void* p, const attn_layout& x) const { return Region(p, x, d->B, d->Tq, d->Hkv, (int64_t)d->D * esz, esz); }
  Region len(const int32_t* p) const { return Region(p, (int64_t)d->B * 4); }
  Region lse(const float* p) const { return Region(p, (int64_t)d->B * d->Hq * d->Tq * 4); }
  Region weight(const float* p) const { return Region(p, rows() * 4); }
  Region codes(const uint8_t* p) const { return Region(p, rows() * (d->D / 2)); }
  Region scales(const uint8_t* p) const { return Region(p, rows() * (d->D / 32)); }
  int64_t rows() const { return (int64_t)d->B * d->Hkv * d->Tk; }
};

int check_weight(const float* weight, float decay) {
  return weight && !(decay >= 0.f && isfinite(decay)) ? LMHEAD_E_SHAPE : LMHEAD_OK;
}

int validate_evict(const evict_desc* d) {
  if (!d) return LMHEAD_E_NULL;
  if (d->B <= 0 || d->B > 65535 || d->T <= 0 || d->T > kNoWindow - 4096 || d->Hkv <= 0 || d->Hkv > 1024) return LMHEAD_E_SHAPE;
  if (d->keep <= 0 || d->keep > d->T || d->sinks < 0 || d->recent < 0 || d->sinks > d->keep || d->recent > d->keep - d->sinks) return LMHEAD_E_SHAPE;
  if (d->flags != 0) return LMHEAD_E_DTYPE;
  return d->reserved == 0 ? LMHEAD_OK : LMHEAD_E_SHAPE;
}

}  // namespace

extern "C" {

int attn_validate_desc(const attn_desc* desc) { return validate(desc); }

size_t attn_workspace_bytes(const attn_desc* desc) {
  if (validate(desc) != LMHEAD_OK) return 0;
  return attn_plan(desc).total;
}

int attn_fwd(const attn_desc* desc, const void* q, const void* k, const void* v, const int32_t* len_q, const int32_t* len_k, void* out,
             float* lse, float* weight, float decay, void* ws, size_t ws_bytes, void* stream) {
  int rc = validate(desc);
  if (rc != LMHEAD_OK) return rc;
  if (!q || !k || !v || !out || !ws) return LMHEAD_E_NULL;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) || !aligned(ws, 256)) return LMHEAD_E_ALIGN;
  rc = check_weight(weight, decay);
  if (rc != LMHEAD_OK) return rc;
  const AttnPlan p = attn_plan(desc);
  if (ws_bytes < p.total) return LMHEAD_E_WORKSPACE;
  const Regions x(desc);
  if (!different({x.q(out, desc->o), x.lse(lse), x.weight(weight), Region(ws, p.total)},
                 {x.q(q, desc->q), x.k(k, desc->k), x.k(v, desc->v), x.len(len_q), x.len(len_k)}))
    return LMHEAD_E_SHAPE;
  const int esz = desc->dtype == LMHEAD_BF16 ? 2 : 4;
  AttnArgs a = arguments(desc, p, len_q, len_k, ws);
  a.q = tensor(q, desc->q, esz), a.k = tensor(k, desc->k, esz), a.v = tensor(v, desc->v, esz), a.o = tensor(out, desc->o, esz);
  return run_fwd(desc, p, a, ws, lse, weight, decay, static_cast<hipStream_t>(stream));
}

size_t attn_bwd_workspace_bytes(const attn_desc* desc) {
  if (validate(desc) != LMHEAD_OK) return 0;
  return sizeof(AttnHeader) + lse_bytes(desc) + attn_before_bytes(desc) + attn_parts_bytes(desc);
}

int attn_bwd(const attn_desc* desc, const void* q, const void* k, const void* v, const int32_t* len_q, const int32_t* len_k,
             const void* out, const float* lse, const void* g_out, void* dq, void* dk, void* dv, void* ws, size_t ws_bytes,
             void* stream) {
  const int rc = validate(desc);
  if (rc != LMHEAD_OK) return rc;
  const int esz = desc->dtype == LMHEAD_BF16 ? 2 : 4;
  // gradients are written: theirs must not lie upon each other
  if (!apart(desc->q, desc->B, desc->Tq, desc->Hq, desc->D) || !apart(desc->k, desc->B, desc->Tk, desc->Hkv, desc->D) ||
      !apart(desc->v, desc->B, desc->Tk, desc->Hkv, desc->D))
    return LMHEAD_E_SHAPE;
  if (!q || !k || !v || !out || !lse || !g_out || !dq || !dk || !dv || !ws) return LMHEAD_E_NULL;
  for (const void* x : {q, k, v, out, g_out, static_cast<const void*>(dq), static_cast<const void*>(dk), static_cast<const void*>(dv)})
    if (!aligned(x, 16)) return LMHEAD_E_ALIGN;
  if (!aligned(ws, 256)) return LMHEAD_E_ALIGN;
  const size_t need = attn_bwd_workspace_bytes(desc);
  if (ws_bytes < need) return LMHEAD_E_WORKSPACE;
  const Regions x(desc);
  if (!different({x.q(dq, desc->q), x.k(dk, desc->k), x.k(dv, desc->v), Region(ws, need)},
                 {x.q(q, desc->q), x.k(k, desc->k), x.k(v, desc->v), x.q(out, desc->o), x.lse(lse), x.q(g_out, desc->o), x.len(len_q), x.len(len_k)}))
    return LMHEAD_E_SHAPE;
  const AttnPlan p = attn_plan(desc);
  AttnArgs a = arguments(desc, p, len_q, len_k, ws);
  a.q = tensor(q, desc->q, esz), a.k = tensor(k, desc->k, esz), a.v = tensor(v, desc->v, esz), a.o = tensor(out, desc->o, esz);
  a.g = tensor(g_out, desc->o, esz);
  a.dq = tensor(dq, desc->q, esz), a.dk = tensor(dk, desc->k, esz), a.dv = tensor(dv, desc->v, esz);
  a.lse = const_cast<float*>(lse);
  a.delta = reinterpret_cast<float*>(static_cast<char*>(ws) + sizeof(AttnHeader));
  a.before = reinterpret_cast<int64_t*>(static_cast<char*>(ws) + sizeof(AttnHeader) + lse_bytes(desc));
  a.part = reinterpret_cast<float*>(static_cast<char*>(ws) + sizeof(AttnHeader) + lse_bytes(desc) + attn_before_bytes(desc));
  LM_TRY(launch_attn_bwd(desc, p, a, static_cast<hipStream_t>(stream)));
  return LMHEAD_OK;
}

int kv4_store(const attn_desc* desc, const void* k, const void* v, const int32_t* len_q, const int32_t* len_k, uint8_t* k_codes,
              uint8_t* k_scales, uint8_t* v_codes, uint8_t* v_scales, void* ws, size_t ws_bytes, void* stream) {
  const int rc = validate(desc);
  if (rc != LMHEAD_OK) return rc;
  if (desc->D % 32 != 0) return LMHEAD_E_SHAPE;
  if (!k || !v || !k_codes || !k_scales || !v_codes || !v_scales || !ws) return LMHEAD_E_NULL;
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(k_codes, 16) || !aligned(v_codes, 16) || !aligned(k_scales, 4) ||
      !aligned(v_scales, 4) || !aligned(ws, 256))
    return LMHEAD_E_ALIGN;
  if (ws_bytes < sizeof(AttnHeader)) return LMHEAD_E_WORKSPACE;
  const Regions x(desc);
  if (!different({x.codes(k_codes), x.scales(k_scales), x.codes(v_codes), x.scales(v_scales), Region(ws, sizeof(AttnHeader))},
                 {x.added(k, desc->k), x.added(v, desc->v), x.len(len_q), x.len(len_k)}))
    return LMHEAD_E_SHAPE;
  const int esz = desc->dtype == LMHEAD_BF16 ? 2 : 4;
  AttnArgs a = arguments(desc, attn_plan(desc), len_q, len_k, ws);
  a.k = tensor(k, desc->k, esz), a.v = tensor(v, desc->v, esz);
  uint8_t* const cache[4] = {k_codes, k_scales, v_codes, v_scales};
  LM_TRY(launch_kv4_store(desc, a, cache, static_cast<hipStream_t>(stream)));
  return LMHEAD_OK;
}

int kv4_attn(const attn_desc* desc, const void* q, const uint8_t* k_codes, const uint8_t* k_scales, const uint8_t* v_codes,
             const uint8_t* v_scales, const int32_t* len_q, const int32_t* len_k, void* out, float* lse, float* weight, float decay,
             void* ws, size_t ws_bytes, void* stream) {
  int rc = validate(desc);
  if (rc != LMHEAD_OK) return rc;
  if (desc->D % 32 != 0) return LMHEAD_E_SHAPE;
  if (!q || !k_codes || !k_scales || !v_codes || !v_scales || !out || !ws) return LMHEAD_E_NULL;
  if (!aligned(q, 16) || !aligned(k_codes, 16) || !aligned(v_codes, 16) || !aligned(k_scales, 4) || !aligned(v_scales, 4) ||
      !aligned(out, 16) || !aligned(ws, 256))
    return LMHEAD_E_ALIGN;
  rc = check_weight(weight, decay);
  if (rc != LMHEAD_OK) return rc;
  const AttnPlan p = attn_plan(desc);
  if (ws_bytes < p.total) return LMHEAD_E_WORKSPACE;
  const Regions x(desc);
  if (!different({x.q(out, desc->o), x.lse(lse), x.weight(weight), Region(ws, p.total)},
                 {x.q(q, desc->q), x.codes(k_codes), x.scales(k_scales), x.codes(v_codes), x.scales(v_scales), x.len(len_q), x.len(len_k)}))
    return LMHEAD_E_SHAPE;
  const int esz = desc->dtype == LMHEAD_BF16 ? 2 : 4;
  AttnArgs a = arguments(desc, p, len_q, len_k, ws);
  a.q = tensor(q, desc->q, esz), a.o = tensor(out, desc->o, esz);
  a.k_codes = k_codes, a.k_scales = k_scales, a.v_codes = v_codes, a.v_scales = v_scales;
  return run_fwd(desc, p, a, ws, lse, weight, decay, static_cast<hipStream_t>(stream));
}

int evict_validate_desc(const evict_desc* desc) { return validate_evict(desc); }

size_t evict_workspace_bytes(const evict_desc* desc) { return validate_evict(desc) == LMHEAD_OK ? sizeof(AttnHeader) : 0; }

int cache_evict(const evict_desc* desc, const cache_plane* planes, int32_t count, float* weight, const int32_t* len, int32_t* len_out,
                int32_t* kept, void* ws, size_t ws_bytes, void* stream) {
  const int rc = validate_evict(desc);
  if (rc != LMHEAD_OK) return rc;
  if (!planes || !weight || !len_out || !kept || !ws) return LMHEAD_E_NULL;
  if (count < 1 || count > EVICT_PLANES) return LMHEAD_E_SHAPE;
  const int64_t heads = (int64_t)desc->B * desc->Hkv;
  const Region w(weight, heads * desc->T * 4), in(len, (int64_t)desc->B * 4), out(len_out, (int64_t)desc->B * 4), slots(kept, heads * desc->keep * 4);
  const Region scratch(ws, sizeof(AttnHeader));
  if (!different({w, out, slots, scratch}, {in})) return LMHEAD_E_SHAPE;
  Region moved[EVICT_PLANES];
  for (int i = 0; i < count; ++i) {
    const cache_plane& p = planes[i];
    if (!p.data) return LMHEAD_E_NULL;
    if (p.bytes < 4 || p.bytes > 4096) return LMHEAD_E_SHAPE;
    for (int64_t v : {p.seq, p.slot, p.head, p.bytes})
      if (v % 4 != 0) return LMHEAD_E_ALIGN;
    if (!aligned(p.data, 4)) return LMHEAD_E_ALIGN;
    const attn_layout x{p.seq, p.slot, p.head};
    if (!strides(x) || !apart(x, desc->B, desc->T, desc->Hkv, p.bytes)) return LMHEAD_E_SHAPE;
    moved[i] = Region(p.data, x, desc->B, desc->T, desc->Hkv, p.bytes, 1);
    for (int j = 0; j < i; ++j)
      if (share(moved[j], moved[i])) return LMHEAD_E_SHAPE;
    if (!different({moved[i]}, {w, in, out, slots, scratch})) return LMHEAD_E_SHAPE;
  }
  if (!aligned(ws, 256)) return LMHEAD_E_ALIGN;
  if (ws_bytes < sizeof(AttnHeader)) return LMHEAD_E_WORKSPACE;
  LM_TRY(launch_evict(*desc, planes, count, weight, len, len_out, kept, static_cast<char*>(ws), static_cast<hipStream_t>(stream)));
  return LMHEAD_OK;
}

}  // extern "C"
