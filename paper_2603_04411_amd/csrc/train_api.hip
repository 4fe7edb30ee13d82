// extern "C" entry points of the operators around the head in a training step.  As in lmhead_api.hip every argument error is
// returned before anything is enqueued.
#include <math.h>

#include <algorithm>
#include <new>

#include "train_common.h"

using namespace lmhead;

namespace {

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int element_bytes(int dtype) { return dtype == LMHEAD_BF16 ? 2 : 4; }

bool known(int dtype) { return dtype == LMHEAD_F32 || dtype == LMHEAD_BF16; }

int validate_embed(const lmhead_embed_desc* d) {
  if (!d) return LMHEAD_E_NULL;
  if (d->R <= 0 || d->T <= 0 || d->d <= 0 || d->V <= 0 || d->reserved != 0) return LMHEAD_E_SHAPE;
  if (!known(d->dtype) || !known(d->rows) || (d->flags & ~(uint32_t)LMHEAD_FLAG_ACCUM_DW)) return LMHEAD_E_DTYPE;
  if (d->d % 8 != 0 || d->d > 65536 || d->ldW < d->d || d->ldX < d->d) return LMHEAD_E_SHAPE;
  if ((int64_t)d->R * d->T > (int64_t)INT32_MAX - (1 << 20) + 1 || d->V > INT32_MAX - (1 << 20)) return LMHEAD_E_SHAPE;
  constexpr int64_t kMost = 1ll << 40;   // sizes that no memory holds are a mistake
  if (d->ldW > kMost || d->ldX > kMost || (int64_t)d->R * d->T > kMost / d->d || d->V > kMost / d->d) return LMHEAD_E_SHAPE;
  if (d->ldW * element_bytes(d->dtype) % 16 != 0 || d->ldX * element_bytes(d->rows) % 16 != 0) return LMHEAD_E_ALIGN;
  return LMHEAD_OK;
}

int validate_preference(const lmhead_preference* q) {
  if (!q) return LMHEAD_E_NULL;
  if (q->loss < LMHEAD_PREF_LOGISTIC || q->loss > LMHEAD_PREF_SQUARED || q->pairs < LMHEAD_PAIRS_ALL || q->pairs > LMHEAD_PAIRS_EXTREMES)
    return LMHEAD_E_SHAPE;
  if ((q->mean & ~1) || (q->weights & ~1) || q->reserved != 0) return LMHEAD_E_SHAPE;
  if (!isfinite(q->beta) || q->beta <= 0.f || !isfinite(q->margin) || !isfinite(q->margin_scale)) return LMHEAD_E_SHAPE;
  if (!(q->smoothing >= 0.f && q->smoothing <= 1.f) || (q->smoothing != 0.f && q->loss != LMHEAD_PREF_LOGISTIC)) return LMHEAD_E_SHAPE;
  if (!isfinite(q->nll_coef) || q->nll_coef < 0.f) return LMHEAD_E_SHAPE;
  return LMHEAD_OK;
}

int validate_tensors(const lmhead_tensor* t, int32_t count) {
  int64_t chunks = 0;
  for (int i = 0; i < count; ++i) {
    if (t[i].n < 0 || t[i].n > kGradMost || t[i].reserved != 0) return LMHEAD_E_SHAPE;
    if (!known(t[i].dtype)) return LMHEAD_E_DTYPE;
    if (t[i].n > 0 && !t[i].data) return LMHEAD_E_NULL;
    if (!aligned(t[i].data, element_bytes(t[i].dtype))) return LMHEAD_E_ALIGN;
    chunks += (t[i].n + kGradChunk - 1) / kGradChunk;
  }
  return chunks <= kGradChunks ? LMHEAD_OK : LMHEAD_E_SHAPE;
}

struct Span {
  uintptr_t lo, hi;
  bool written;
};

// Whether `norm` (of `norms` elements) and the workspace share no memory with a tensor, nor with each other.
bool scratch_apart(const lmhead_tensor* g, const lmhead_tensor* out, int32_t count, const float* norm, int norms, const void* ws) {
  const uintptr_t n0 = reinterpret_cast<uintptr_t>(norm), n1 = n0 + norms * sizeof(float);
  const uintptr_t w0 = reinterpret_cast<uintptr_t>(ws), w1 = w0 + grad_ws_bytes();
  auto clear = [&](const lmhead_tensor& t) {
    const uintptr_t lo = reinterpret_cast<uintptr_t>(t.data), hi = lo + (uintptr_t)t.n * element_bytes(t.dtype);
    return t.n == 0 || ((hi <= n0 || n1 <= lo) && (hi <= w0 || w1 <= lo));
  };
  for (int i = 0; i < count; ++i)
    if (!clear(g[i]) || (out && !clear(out[i]))) return false;
  return n1 <= w0 || w1 <= n0;
}

// Whether some output shares memory with another output, or with an input that is not itself.
int outputs_apart(const lmhead_tensor* g, const lmhead_tensor* out, int32_t count) {
  constexpr int kOnStack = 256;
  Span few[kOnStack];
  const size_t most = (size_t)count * (out ? 2 : 1);
  Span* const heap = most > kOnStack ? new (std::nothrow) Span[most] : nullptr;
  Span* const all = most > kOnStack ? heap : few;
  if (!all) return LMHEAD_E_WORKSPACE;
  size_t k = 0;
  auto put = [&](const lmhead_tensor& t, bool written) {
    if (t.n == 0) return;
    const uintptr_t lo = reinterpret_cast<uintptr_t>(t.data);
    all[k++] = Span{lo, lo + (uintptr_t)t.n * element_bytes(t.dtype), written};
  };
  for (int i = 0; i < count; ++i) {
    const bool itself = !out || (out[i].data == g[i].data && out[i].dtype == g[i].dtype);
    put(out ? out[i] : g[i], true);
    if (!itself) put(g[i], false);
  }
  std::sort(all, all + k, [](const Span& a, const Span& b) { return a.lo < b.lo; });
  uintptr_t read_to = 0, written_to = 0;
  int rc = LMHEAD_OK;
  for (size_t i = 0; i < k && rc == LMHEAD_OK; ++i) {
    if (all[i].lo < written_to || (all[i].written && all[i].lo < read_to)) rc = LMHEAD_E_SHAPE;
    uintptr_t& to = all[i].written ? written_to : read_to;
    to = std::max(to, all[i].hi);
  }
  delete[] heap;
  return rc;
}

}  // namespace

extern "C" {

size_t preference_workspace_bytes(int32_t P, int32_t G, int32_t T) {
  if (lmhead_loss_workspace_bytes(P, G, T) == 0) return 0;
  return pref_layout(P, G, T).total;
}

int preference_loss(const lmhead_preference* params, const float* logp, const float* logp_ref, const float* reward, const int32_t* len,
                    int32_t P, int32_t G, int32_t T, float* loss, float* g_logp, float* ratio, float* stats, void* ws, size_t ws_bytes,
                    void* stream) {
  const int rc = validate_preference(params);
  if (rc != LMHEAD_OK) return rc;
  const size_t need = preference_workspace_bytes(P, G, T);
  if (need == 0) return LMHEAD_E_SHAPE;
  if (!logp || !reward || !len || !loss || !ws) return LMHEAD_E_NULL;
  if (!aligned(ws, 256)) return LMHEAD_E_ALIGN;
  if (ws_bytes < need) return LMHEAD_E_WORKSPACE;
  LM_TRY(launch_preference(*params, logp, logp_ref, reward, len, P, G, T, loss, g_logp, ratio, stats, static_cast<char*>(ws),
                           static_cast<hipStream_t>(stream)));
  return LMHEAD_OK;
}

int embed_validate_desc(const lmhead_embed_desc* desc) { return validate_embed(desc); }

size_t embed_workspace_bytes(const lmhead_embed_desc* desc) {
  return validate_embed(desc) == LMHEAD_OK ? embed_layout(desc).total : 0;
}

int embed_fwd(const lmhead_embed_desc* desc, const void* W, const int32_t* tok, const int32_t* len, float scale, void* X, void* ws,
              size_t ws_bytes, void* stream) {
  const int rc = validate_embed(desc);
  if (rc != LMHEAD_OK) return rc;
  if (!W || !tok || !X || !ws) return LMHEAD_E_NULL;
  if (!aligned(W, 16) || !aligned(X, 16) || !aligned(ws, 256)) return LMHEAD_E_ALIGN;
  if (ws_bytes < sizeof(EmbedHeader)) return LMHEAD_E_WORKSPACE;
  LM_TRY(launch_embed_fwd(*desc, W, tok, len, scale, X, static_cast<EmbedHeader*>(ws), static_cast<hipStream_t>(stream)));
  return LMHEAD_OK;
}

int embed_bwd(const lmhead_embed_desc* desc, const void* gX, const int32_t* tok, const int32_t* len, float scale, float* dW, void* ws,
              size_t ws_bytes, void* stream) {
  const int rc = validate_embed(desc);
  if (rc != LMHEAD_OK) return rc;
  if (!gX || !tok || !dW || !ws) return LMHEAD_E_NULL;
  if (!aligned(gX, 16) || !aligned(dW, 16) || !aligned(ws, 256)) return LMHEAD_E_ALIGN;
  if (ws_bytes < embed_layout(desc).total) return LMHEAD_E_WORKSPACE;
  LM_TRY(launch_embed_bwd(*desc, gX, tok, len, scale, dW, static_cast<char*>(ws), static_cast<hipStream_t>(stream)));
  return LMHEAD_OK;
}

size_t grad_workspace_bytes(void) { return grad_ws_bytes(); }

int grad_norm(const lmhead_tensor* g, int32_t count, float* norm, void* ws, size_t ws_bytes, void* stream) {
  if (!g || !norm || !ws) return LMHEAD_E_NULL;
  if (count < 1 || count > kGradCount) return LMHEAD_E_SHAPE;
  const int rc = validate_tensors(g, count);
  if (rc != LMHEAD_OK) return rc;
  if (!aligned(ws, 256)) return LMHEAD_E_ALIGN;
  if (ws_bytes < grad_ws_bytes()) return LMHEAD_E_WORKSPACE;
  if (!scratch_apart(g, nullptr, count, norm, 1, ws)) return LMHEAD_E_SHAPE;
  LM_TRY(launch_grads(g, nullptr, count, false, 0.f, 0.f, norm, static_cast<char*>(ws), static_cast<hipStream_t>(stream)));
  return LMHEAD_OK;
}

int grad_clip(const lmhead_tensor* g, const lmhead_tensor* out, int32_t count, float max_norm, float eps, float* norm, void* ws,
              size_t ws_bytes, void* stream) {
  if (!g || !norm || !ws) return LMHEAD_E_NULL;
  if (count < 1 || count > kGradCount) return LMHEAD_E_SHAPE;
  if (!(max_norm >= 0.f) || !(eps >= 0.f) || !isfinite(eps)) return LMHEAD_E_SHAPE;
  int rc = validate_tensors(g, count);
  if (rc == LMHEAD_OK && out) rc = validate_tensors(out, count);
  if (rc != LMHEAD_OK) return rc;
  for (int i = 0; out && i < count; ++i)
    if (out[i].n != g[i].n) return LMHEAD_E_SHAPE;
  if (!aligned(ws, 256)) return LMHEAD_E_ALIGN;
  if (ws_bytes < grad_ws_bytes()) return LMHEAD_E_WORKSPACE;
  if (!scratch_apart(g, out, count, norm, 2, ws)) return LMHEAD_E_SHAPE;
  rc = outputs_apart(g, out, count);
  if (rc != LMHEAD_OK) return rc;
  LM_TRY(launch_grads(g, out, count, true, max_norm, eps, norm, static_cast<char*>(ws), static_cast<hipStream_t>(stream)));
  return LMHEAD_OK;
}

}  // extern "C"
