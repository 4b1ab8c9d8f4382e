// C ABI of the KVpop future-attention target library: argument validation, error
// reporting and dispatch to the gfx950 kernels. The semantics of every entry point
// are specified in include/kvpop.h and include/kvpop_cache.h.
#include "kvpop.h"
#include "kvpop_cache.h"

#include <hip/hip_runtime_api.h>

#include <cmath>
#include <cstdlib>
#include <cstdint>
#include <initializer_list>
#include <string>

#include "kvpop_internal.h"

namespace {

thread_local std::string g_err_text;

struct Sizes {
  int64_t q_elems, k_elems, row_elems;  // Q, K and [B, Hq, T] element counts
};

bool mul_ok(int64_t a, int64_t b, int64_t* r) {
  if (a != 0 && b > INT64_MAX / a) return false;
  *r = a * b;
  return true;
}

int check_dims(const kvpop_dims* d, Sizes* sz) {
  if (!d) return KVPOP_EINVAL;
  if (d->batch < 1 || d->n_q_heads < 1 || d->n_kv_heads < 1 || d->seq_len < 1 || d->head_dim < 1)
    return KVPOP_EINVAL;
  if (d->n_q_heads % d->n_kv_heads != 0) return KVPOP_EINVAL;
  if (!std::isfinite(d->scale) || !(d->scale > 0.f)) return KVPOP_EINVAL;
  if (d->head_dim != 64 && d->head_dim != 128) return KVPOP_EUNSUPPORTED;
  if (d->seq_len > KVPOP_MAX_SEQ_LEN) return KVPOP_EUNSUPPORTED;
  int64_t bh, bkh, t;
  if (!mul_ok(d->batch, d->n_q_heads, &bh) || !mul_ok(bh, d->seq_len, &sz->row_elems) ||
      !mul_ok(sz->row_elems, d->head_dim, &sz->q_elems) || !mul_ok(d->batch, d->n_kv_heads, &bkh) ||
      !mul_ok(bkh, d->seq_len, &t) || !mul_ok(t, d->head_dim, &sz->k_elems) ||
      sz->q_elems > INT64_MAX / 4)
    return KVPOP_EINVAL;
  // Grid sizes stay below 2^31 workgroups: at most B * Hq * ceil(T / 32) of them.
  if (sz->row_elems / 32 + bh > INT32_MAX) return KVPOP_EUNSUPPORTED;
  return KVPOP_OK;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

bool overlap(const void* a, int64_t abytes, const void* b, int64_t bbytes) {
  if (!a || !b) return false;
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
  return a0 < b0 + (uintptr_t)bbytes && b0 < a0 + (uintptr_t)abytes;
}

int check_band(int32_t window, int32_t horizon) {
  if (window < 0) return KVPOP_EINVAL;
  if (horizon >= 0 && horizon < window) return KVPOP_EINVAL;
  return KVPOP_OK;
}

int hip_status(int e) {
  if (e == 0) return KVPOP_OK;
  g_err_text = std::string("HIP error: ") + hipGetErrorString(static_cast<hipError_t>(e));
  return KVPOP_EHIP;
}

// Test hook for the KVPOP_EHIP path: with the environment variable
// KVPOP_TEST_FORCE_EHIP set to a nonzero hipError_t code, every entry point fails
// after validation as if its first launch had returned that code, and launches
// nothing. Unset (the normal case) it costs one getenv per call.
int forced_hip_error() {
  const char* e = std::getenv("KVPOP_TEST_FORCE_EHIP");
  return e ? std::atoi(e) : 0;
}

// Runs the launches of one entry point (a callable returning 0 or the hipError_t
// of the launch that failed) and maps the result to a status.
template <class F>
int launch(F&& f) {
  const int forced = forced_hip_error();
  if (forced != 0) return hip_status(forced);
  return hip_status(f());
}

kvpop::Launch make_launch(const kvpop_dims* d, const void* q, const void* k, const float* bias, void* stream) {
  kvpop::Launch L{};
  L.q = static_cast<const uint16_t*>(q);
  L.k = static_cast<const uint16_t*>(k);
  L.bias = bias;
  L.B = d->batch;
  L.Hq = d->n_q_heads;
  L.Hkv = d->n_kv_heads;
  L.T = d->seq_len;
  L.D = d->head_dim;
  L.scale = d->scale;
  L.stream = stream;
  return L;
}

// Validation shared by every entry point for the inputs q, k, key_bias.
int check_inputs(const kvpop_dims* d, const void* q, const void* k, const float* bias, Sizes* sz) {
  int st = check_dims(d, sz);
  if (st != KVPOP_OK) return st;
  if (!q || !k) return KVPOP_EINVAL;
  if (!aligned16(q) || !aligned16(k) || (bias && !aligned16(bias))) return KVPOP_EUNSUPPORTED;
  return KVPOP_OK;
}

// An output of `bytes` bytes must not overlap q, k, bias or `other`.
int check_output(const void* out, int64_t bytes, const Sizes& sz, const kvpop_dims* d, const void* q,
                 const void* k, const float* bias, const void* other, int64_t other_bytes) {
  if (!out) return KVPOP_EINVAL;
  if (!aligned16(out)) return KVPOP_EUNSUPPORTED;
  if (overlap(out, bytes, q, sz.q_elems * 2) || overlap(out, bytes, k, sz.k_elems * 2) ||
      overlap(out, bytes, bias, (int64_t)d->seq_len * 4) || overlap(out, bytes, other, other_bytes))
    return KVPOP_EINVAL;
  return KVPOP_OK;
}

// Validation shared by kvpop_running_topk and kvpop_running_topk_noalloc. The
// workspace (need bytes) is checked only when it is caller memory (ws != NULL).
int check_topk(const kvpop_topk_dims* d, const float* scores, const float* log_gamma, int32_t sinks, int32_t window,
               int32_t topk, int32_t* rank, int32_t* cutoff, int32_t* label, int32_t* boundary, int32_t* evict,
               const void* ws, size_t need) {
  if (!scores || !rank || !cutoff) return KVPOP_EINVAL;
  const void* ptrs[] = {scores, log_gamma, rank, cutoff, label, boundary, evict, ws};
  for (const void* p : ptrs)
    if (p && !aligned16(p)) return KVPOP_EUNSUPPORTED;
  const int64_t n = (int64_t)d->batch * d->n_heads * d->seq_len;
  if (n / d->seq_len / d->n_heads != d->batch || n * 4 > INT64_MAX / 2) return KVPOP_EINVAL;
  const int64_t b = n * 4;
  // Outputs must not overlap each other, the inputs or the workspace.
  const void* outs[] = {rank, cutoff, label, boundary, evict};
  for (int i = 0; i < 5; ++i) {
    if (!outs[i]) continue;
    if (overlap(outs[i], b, scores, b) || overlap(outs[i], b, log_gamma, (int64_t)d->n_heads * 4) ||
        overlap(outs[i], b, ws, (int64_t)need))
      return KVPOP_EINVAL;
    for (int j = i + 1; j < 5; ++j)
      if (overlap(outs[i], b, outs[j], b)) return KVPOP_EINVAL;
  }
  if (overlap(ws, (int64_t)need, scores, b) || overlap(ws, (int64_t)need, log_gamma, (int64_t)d->n_heads * 4))
    return KVPOP_EINVAL;
  return KVPOP_OK;
}

kvpop::TopkLaunch make_topk(const kvpop_topk_dims* d, const float* scores, const float* log_gamma, int32_t sinks,
                            int32_t window, int32_t topk, int32_t* rank, int32_t* cutoff, int32_t* label,
                            int32_t* boundary, int32_t* evict, void* workspace, void* stream) {
  kvpop::TopkLaunch L{};
  L.scores = scores;
  L.log_gamma = log_gamma;
  L.B = d->batch;
  L.H = d->n_heads;
  L.T = d->seq_len;
  L.sinks = sinks;
  L.window = window;
  L.topk = topk;
  L.rank = rank;
  L.cutoff = cutoff;
  L.label = label;
  L.boundary = boundary;
  L.evict = evict;
  L.workspace = workspace;
  L.stream = stream;
  return L;
}

// ---------------------------------------------------------------------------
// The compact cache (kvpop_cache.h)
// ---------------------------------------------------------------------------

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

int64_t pool_bytes(const kvpop_cache* c) { return (int64_t)c->n_pages * c->page_size * c->head_dim; }
int64_t cache_lists(const kvpop_cache* c) { return (int64_t)c->batch * c->n_kv_heads; }

// The sizes of a cache (its pointers are not looked at).
int check_cache_dims(const kvpop_cache* c) {
  if (!c) return KVPOP_EINVAL;
  if (c->batch < 1 || c->n_kv_heads < 1 || c->head_dim < 1 || c->page_size < 1 || c->n_pages < 1 || c->max_pages < 1)
    return KVPOP_EINVAL;
  if (c->head_dim != 64 && c->head_dim != 128) return KVPOP_EUNSUPPORTED;
  if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128) return KVPOP_EUNSUPPORTED;
  if (c->format != KVPOP_CACHE_INT8 && c->format != KVPOP_CACHE_E4M3) return KVPOP_EUNSUPPORTED;
  if ((int64_t)c->max_pages * c->page_size > KVPOP_MAX_SEQ_LEN) return KVPOP_EUNSUPPORTED;
  if (cache_lists(c) > INT32_MAX) return KVPOP_EUNSUPPORTED;
  return KVPOP_OK;
}

int check_cache(const kvpop_cache* c) {
  const int st = check_cache_dims(c);
  if (st != KVPOP_OK) return st;
  if (!c->k_pages || !c->v_pages || !c->k_exp || !c->v_exp || !c->page_table) return KVPOP_EINVAL;
  if (!aligned16(c->k_pages) || !aligned16(c->v_pages) || !aligned4(c->page_table)) return KVPOP_EUNSUPPORTED;
  return KVPOP_OK;
}

// A strided bf16 array [B, heads, tokens, D] and the bytes from its first element to its last.
int check_rows(const kvpop_rows& r, int64_t B, int64_t heads, int64_t tokens, int64_t D, int64_t* bytes) {
  if (!r.ptr || r.stride_b < 0 || r.stride_h < 0 || r.stride_t < 0) return KVPOP_EINVAL;
  int64_t x, y, z;
  if (!mul_ok(B - 1, r.stride_b, &x) || !mul_ok(heads - 1, r.stride_h, &y) || !mul_ok(tokens - 1, r.stride_t, &z) ||
      x > INT64_MAX / 16 || y > INT64_MAX / 16 || z > INT64_MAX / 16)
    return KVPOP_EINVAL;
  if (!aligned16(r.ptr) || r.stride_b % 8 != 0 || r.stride_h % 8 != 0 || r.stride_t % 8 != 0)
    return KVPOP_EUNSUPPORTED;
  *bytes = 2 * (x + y + z + D);
  return KVPOP_OK;
}

struct Span {
  const void* p;
  int64_t bytes;
};

// No two of `outs` overlap, and none overlaps one of `ins`; absent arrays are NULL.
template <size_t N, size_t M>
bool disjoint(const Span (&outs)[N], const Span (&ins)[M]) {
  for (size_t i = 0; i < N; ++i) {
    for (size_t j = 0; j < M; ++j)
      if (overlap(outs[i].p, outs[i].bytes, ins[j].p, ins[j].bytes)) return false;
    for (size_t j = i + 1; j < N; ++j)
      if (overlap(outs[i].p, outs[i].bytes, outs[j].p, outs[j].bytes)) return false;
  }
  return true;
}

kvpop::CacheView make_view(const kvpop_cache* c) {
  return {static_cast<uint8_t*>(c->k_pages), static_cast<uint8_t*>(c->v_pages), c->k_exp, c->v_exp, c->page_table,
          c->batch, c->n_kv_heads, c->head_dim, c->page_size, c->n_pages, c->max_pages, c->format};
}

kvpop::Rows make_rows(const kvpop_rows& r) {
  return {static_cast<const uint16_t*>(r.ptr), r.stride_b, r.stride_h, r.stride_t};
}

// Sizes of an attention call; fills what its plan depends on.
int check_cache_attn_dims(const kvpop_cache* c, int32_t Hq, int32_t N, kvpop::CacheAttnLaunch* L) {
  const int st = check_cache_dims(c);
  if (st != KVPOP_OK) return st;
  if (Hq < 1 || N < 1 || Hq % c->n_kv_heads != 0) return KVPOP_EINVAL;
  const int64_t G = Hq / c->n_kv_heads;
  int64_t rows, elems;
  if (!mul_ok((int64_t)c->batch * Hq, N, &rows) || !mul_ok(rows, c->head_dim, &elems) || elems > INT64_MAX / 512)
    return KVPOP_EINVAL;
  if (G > 1024 || N > KVPOP_MAX_SEQ_LEN || G * N > INT32_MAX / 2) return KVPOP_EUNSUPPORTED;
  *L = kvpop::CacheAttnLaunch{};
  L->c = make_view(c);
  L->Hq = Hq;
  L->N = N;
  if (kvpop::cache_attn_threads(*L) > UINT32_MAX) return KVPOP_EUNSUPPORTED;
  return KVPOP_OK;
}

int check_retain(const kvpop_retain* s) {
  if (!s || s->batch < 1 || s->n_heads < 1 || s->slots < 1 || !s->pos || !s->prio || !s->held) return KVPOP_EINVAL;
  if ((int64_t)s->batch * s->n_heads > INT32_MAX || s->slots > KVPOP_MAX_SEQ_LEN) return KVPOP_EUNSUPPORTED;
  if (!aligned4(s->pos) || !aligned4(s->prio) || !aligned4(s->held)) return KVPOP_EUNSUPPORTED;
  return KVPOP_OK;
}

kvpop::RetainLaunch make_retain(const kvpop_retain* s, const float* scores, const float* log_gamma, void* stream) {
  kvpop::RetainLaunch L{};
  L.B = s->batch;
  L.H = s->n_heads;
  L.S = s->slots;
  L.pos = s->pos;
  L.prio = s->prio;
  L.held = s->held;
  L.scores = scores;
  L.log_gamma = log_gamma;
  L.stream = stream;
  return L;
}

}  // namespace

extern "C" {

int kvpop_abi_version(void) { return KVPOP_ABI_VERSION; }

const char* kvpop_strerror(int status) {
  switch (status) {
    case KVPOP_OK:
      return "success";
    case KVPOP_EINVAL:
      return "invalid argument (null pointer, bad dimension, Hq % Hkv != 0, bad scale, bad window/horizon, "
             "or overlapping buffers)";
    case KVPOP_EUNSUPPORTED:
      return "unsupported configuration (head_dim not 64/128, pointer not 16-byte aligned, or size limit)";
    case KVPOP_EHIP:
      return g_err_text.empty() ? "HIP runtime error" : g_err_text.c_str();
    case KVPOP_ETOOBIG:
      return "problem too large for the no-allocation entry point (its workspace exceeds "
             "KVPOP_NOALLOC_SCRATCH_BYTES)";
    default:
      return "unknown status code";
  }
}

int kvpop_row_lse(const kvpop_dims* dims, const void* q, const void* k, const float* key_bias, float* lse,
                  void* stream) {
  Sizes sz;
  int st = check_inputs(dims, q, k, key_bias, &sz);
  if (st != KVPOP_OK) return st;
  st = check_output(lse, sz.row_elems * 4, sz, dims, q, k, key_bias, nullptr, 0);
  if (st != KVPOP_OK) return st;
  kvpop::Launch L = make_launch(dims, q, k, key_bias, stream);
  L.out = lse;
  return launch([&] { return kvpop::launch_row_lse(L); });
}

int kvpop_future_attn_from_lse(const kvpop_dims* dims, const void* q, const void* k, const float* key_bias,
                               const float* lse, int32_t window, int32_t horizon, float* out, void* stream) {
  Sizes sz;
  int st = check_inputs(dims, q, k, key_bias, &sz);
  if (st != KVPOP_OK) return st;
  if (!lse) return KVPOP_EINVAL;
  if (!aligned16(lse)) return KVPOP_EUNSUPPORTED;
  st = check_band(window, horizon);
  if (st != KVPOP_OK) return st;
  st = check_output(out, sz.row_elems * 4, sz, dims, q, k, key_bias, lse, sz.row_elems * 4);
  if (st != KVPOP_OK) return st;
  kvpop::Launch L = make_launch(dims, q, k, key_bias, stream);
  L.lse = lse;
  L.out = out;
  L.window = window;
  L.horizon = horizon;
  return launch([&] { return kvpop::launch_future_mass(L); });
}

int kvpop_future_attn_bands(const kvpop_dims* dims, const void* q, const void* k, const float* key_bias,
                            const float* lse, int32_t n_bands, const int32_t* windows, const int32_t* horizons,
                            float* const* outs, void* stream) {
  Sizes sz;
  int st = check_inputs(dims, q, k, key_bias, &sz);
  if (st != KVPOP_OK) return st;
  if (!lse) return KVPOP_EINVAL;
  if (!aligned16(lse)) return KVPOP_EUNSUPPORTED;
  if (n_bands < 1 || n_bands > 2 || !windows || !horizons || !outs) return KVPOP_EINVAL;
  for (int i = 0; i < n_bands; ++i) {
    st = check_band(windows[i], horizons[i]);
    if (st != KVPOP_OK) return st;
    st = check_output(outs[i], sz.row_elems * 4, sz, dims, q, k, key_bias, lse, sz.row_elems * 4);
    if (st != KVPOP_OK) return st;
  }
  if (n_bands == 2 && overlap(outs[0], sz.row_elems * 4, outs[1], sz.row_elems * 4)) return KVPOP_EINVAL;
  kvpop::Launch L = make_launch(dims, q, k, key_bias, stream);
  L.lse = lse;
  L.out = outs[0];
  L.window = windows[0];
  L.horizon = horizons[0];
  if (n_bands == 2) {
    L.out1 = outs[1];
    L.window1 = windows[1];
    L.horizon1 = horizons[1];
  }
  return launch([&] { return kvpop::launch_future_mass(L); });
}

int kvpop_future_attn_scores(const kvpop_dims* dims, const void* q, const void* k, const float* key_bias,
                             const float* lse, int32_t window, int32_t horizon, int32_t agg, float eps,
                             int32_t normalize, float* out, float* scores, void* stream) {
  Sizes sz;
  int st = check_inputs(dims, q, k, key_bias, &sz);
  if (st != KVPOP_OK) return st;
  if (!lse) return KVPOP_EINVAL;
  if (!aligned16(lse)) return KVPOP_EUNSUPPORTED;
  st = check_band(window, horizon);
  if (st != KVPOP_OK) return st;
  if ((agg != KVPOP_AGG_MAX && agg != KVPOP_AGG_MEAN) || (normalize != 0 && normalize != 1) || !std::isfinite(eps) ||
      eps < 0.f)
    return KVPOP_EINVAL;
  const int64_t score_bytes = (int64_t)dims->batch * dims->n_kv_heads * dims->seq_len * 4;
  st = check_output(scores, score_bytes, sz, dims, q, k, key_bias, lse, sz.row_elems * 4);
  if (st != KVPOP_OK) return st;
  if (out) {
    st = check_output(out, sz.row_elems * 4, sz, dims, q, k, key_bias, lse, sz.row_elems * 4);
    if (st != KVPOP_OK) return st;
    if (overlap(out, sz.row_elems * 4, scores, score_bytes)) return KVPOP_EINVAL;
  }
  kvpop::Launch L = make_launch(dims, q, k, key_bias, stream);
  L.lse = lse;
  L.out = out;
  L.window = window;
  L.horizon = horizon;
  L.scores = scores;
  L.agg = agg;
  L.eps = eps;
  L.normalize = normalize;
  return launch([&] { return kvpop::launch_future_mass(L); });
}

int kvpop_internal_scores_spread(const kvpop_dims* dims, int32_t window, int32_t horizon) {
  Sizes sz;
  if (check_dims(dims, &sz) != KVPOP_OK || check_band(window, horizon) != KVPOP_OK) return 0;
  kvpop::Launch L = make_launch(dims, nullptr, nullptr, nullptr, nullptr);
  L.window = window;
  L.horizon = horizon;
  return kvpop::scores_spread(L) ? 1 : 0;
}

size_t kvpop_running_topk_workspace_size(const kvpop_topk_dims* d) {
  if (!d || d->batch < 1 || d->n_heads < 1 || d->seq_len < 1 || d->seq_len > KVPOP_MAX_SEQ_LEN) return 0;
  const size_t seqs = (size_t)d->batch * (size_t)d->n_heads;
  const size_t words = kvpop::topk_workspace_words_per_seq(d->seq_len);
  if (seqs > SIZE_MAX / 4 / words) return 0;
  return seqs * words * 4;
}

int kvpop_running_topk(const kvpop_topk_dims* d, const float* scores, const float* log_gamma, int32_t sinks,
                       int32_t window, int32_t topk, int32_t* rank, int32_t* cutoff, int32_t* label,
                       int32_t* boundary, int32_t* evict, void* workspace, size_t workspace_bytes, void* stream) {
  if (!d || d->batch < 1 || d->n_heads < 1 || d->seq_len < 1) return KVPOP_EINVAL;
  if (d->seq_len > KVPOP_MAX_SEQ_LEN) return KVPOP_EUNSUPPORTED;
  if (sinks < 0 || window < 0 || topk < 1) return KVPOP_EINVAL;
  if (!scores || !rank || !cutoff || !workspace) return KVPOP_EINVAL;
  const size_t need = kvpop_running_topk_workspace_size(d);
  if (need == 0 || workspace_bytes < need) return KVPOP_EINVAL;
  const int st = check_topk(d, scores, log_gamma, sinks, window, topk, rank, cutoff, label, boundary, evict,
                            workspace, need);
  if (st != KVPOP_OK) return st;
  kvpop::TopkLaunch L = make_topk(d, scores, log_gamma, sinks, window, topk, rank, cutoff, label, boundary, evict,
                                  workspace, stream);
  return launch([&] { return kvpop::launch_running_topk(L); });
}

int kvpop_running_topk_noalloc(const kvpop_topk_dims* d, const float* scores, const float* log_gamma, int32_t sinks,
                               int32_t window, int32_t topk, int32_t* rank, int32_t* cutoff, int32_t* label,
                               int32_t* boundary, int32_t* evict, void* stream) {
  if (!d || d->batch < 1 || d->n_heads < 1 || d->seq_len < 1) return KVPOP_EINVAL;
  if (d->seq_len > KVPOP_MAX_SEQ_LEN) return KVPOP_EUNSUPPORTED;
  if (sinks < 0 || window < 0 || topk < 1) return KVPOP_EINVAL;
  const size_t need = kvpop_running_topk_workspace_size(d);
  if (need == 0) return KVPOP_EINVAL;
  if (need > (size_t)KVPOP_NOALLOC_SCRATCH_BYTES) return KVPOP_ETOOBIG;
  const int st = check_topk(d, scores, log_gamma, sinks, window, topk, rank, cutoff, label, boundary, evict,
                            nullptr, 0);
  if (st != KVPOP_OK) return st;
  return launch([&] {
    void* ws = nullptr;
    const int e = kvpop::noalloc_scratch(stream, &ws);
    if (e != 0) return e;
    kvpop::TopkLaunch L = make_topk(d, scores, log_gamma, sinks, window, topk, rank, cutoff, label, boundary,
                                    evict, ws, stream);
    return kvpop::launch_running_topk(L);
  });
}

int kvpop_sparse_attn_fwd(const kvpop_dims* dims, const void* q, const void* k, const void* v,
                          const float* key_bias, const int32_t* evict, void* o, float* lse, void* stream) {
  Sizes sz;
  int st = check_inputs(dims, q, k, key_bias, &sz);
  if (st != KVPOP_OK) return st;
  const int G = dims->n_q_heads / dims->n_kv_heads;
  if ((G & (G - 1)) != 0) return KVPOP_EUNSUPPORTED;
  if ((int64_t)dims->seq_len * dims->head_dim * 2 > INT32_MAX) return KVPOP_EUNSUPPORTED;
  if (!v || !evict) return KVPOP_EINVAL;
  if (!aligned16(v) || !aligned16(evict)) return KVPOP_EUNSUPPORTED;
  const int64_t ev_bytes = (int64_t)dims->batch * dims->n_kv_heads * dims->seq_len * 4;
  // o must not overlap q, k, key_bias, lse, v or evict; lse likewise.
  st = check_output(o, sz.q_elems * 2, sz, dims, q, k, key_bias, lse, sz.row_elems * 4);
  if (st != KVPOP_OK) return st;
  st = check_output(lse, sz.row_elems * 4, sz, dims, q, k, key_bias, o, sz.q_elems * 2);
  if (st != KVPOP_OK) return st;
  if (overlap(o, sz.q_elems * 2, v, sz.k_elems * 2) || overlap(o, sz.q_elems * 2, evict, ev_bytes) ||
      overlap(lse, sz.row_elems * 4, v, sz.k_elems * 2) || overlap(lse, sz.row_elems * 4, evict, ev_bytes))
    return KVPOP_EINVAL;
  kvpop::SparseLaunch L{};
  L.q = static_cast<const uint16_t*>(q);
  L.k = static_cast<const uint16_t*>(k);
  L.v = static_cast<const uint16_t*>(v);
  L.bias = key_bias;
  L.evict = evict;
  L.o = static_cast<uint16_t*>(o);
  L.lse = lse;
  L.B = dims->batch;
  L.Hq = dims->n_q_heads;
  L.Hkv = dims->n_kv_heads;
  L.T = dims->seq_len;
  L.D = dims->head_dim;
  L.scale = dims->scale;
  L.stream = stream;
  return launch([&] { return kvpop::launch_sparse_attn_fwd(L); });
}

int kvpop_future_attn_target(const kvpop_dims* dims, const void* q, const void* k, const float* key_bias,
                             int32_t window, int32_t horizon, float* lse_ws, float* out, void* stream) {
  Sizes sz;
  int st = check_inputs(dims, q, k, key_bias, &sz);
  if (st != KVPOP_OK) return st;
  st = check_band(window, horizon);
  if (st != KVPOP_OK) return st;
  st = check_output(lse_ws, sz.row_elems * 4, sz, dims, q, k, key_bias, out, sz.row_elems * 4);
  if (st != KVPOP_OK) return st;
  st = check_output(out, sz.row_elems * 4, sz, dims, q, k, key_bias, lse_ws, sz.row_elems * 4);
  if (st != KVPOP_OK) return st;
  kvpop::Launch L = make_launch(dims, q, k, key_bias, stream);
  return launch([&] {
    L.out = lse_ws;
    const int e = kvpop::launch_row_lse(L);
    if (e != 0) return e;
    L.lse = lse_ws;
    L.out = out;
    L.window = window;
    L.horizon = horizon;
    return kvpop::launch_future_mass(L);
  });
}

int kvpop_cache_append(const kvpop_cache* cache, const kvpop_append* a, void* stream) {
  int st = check_cache(cache);
  if (st != KVPOP_OK) return st;
  if (!a || a->n_tokens < 1 || a->n_entries < 1 || !a->held || (!a->src && a->n_entries != a->n_tokens))
    return KVPOP_EINVAL;
  const int64_t B = cache->batch, H = cache->n_kv_heads, D = cache->head_dim, lists = B * H, N = a->n_tokens;
  if (a->rot_dim < 0 || a->rot_dim > D || (a->adjacent != 0 && a->adjacent != 1) || a->n_q_heads < 0)
    return KVPOP_EINVAL;
  if (a->rot_dim % 16 != 0) return KVPOP_EUNSUPPORTED;
  if (a->rot_dim > 0 && (!a->cos || !a->sin || a->n_positions < 1)) return KVPOP_EINVAL;
  if (a->n_tokens > KVPOP_MAX_SEQ_LEN || a->n_entries > KVPOP_MAX_SEQ_LEN) return KVPOP_EUNSUPPORTED;
  int64_t kb = 0, vb = 0, qb = 0, qo = 0;
  if ((st = check_rows(a->k, B, H, N, D, &kb)) != KVPOP_OK) return st;
  if ((st = check_rows(a->v, B, H, N, D, &vb)) != KVPOP_OK) return st;
  if (a->q.ptr) {
    if (a->n_q_heads < 1 || !a->q_out) return KVPOP_EINVAL;
    int64_t rows;
    if (!mul_ok(B * a->n_q_heads, N, &rows) || rows > INT64_MAX / 512) return KVPOP_EINVAL;
    if ((st = check_rows(a->q, B, a->n_q_heads, N, D, &qb)) != KVPOP_OK) return st;
    if (!aligned16(a->q_out)) return KVPOP_EUNSUPPORTED;
    qo = rows * D * 2;
  }
  for (const void* p : {(const void*)a->held, (const void*)a->count, (const void*)a->start, (const void*)a->src,
                        (const void*)a->pos0})
    if (!aligned4(p)) return KVPOP_EUNSUPPORTED;
  if (a->rot_dim > 0 && (!aligned16(a->cos) || !aligned16(a->sin))) return KVPOP_EUNSUPPORTED;
  const int64_t table = a->rot_dim > 0 ? (int64_t)a->n_positions * (a->rot_dim / 2) * 4 : 0;
  const Span outs[] = {{cache->k_pages, pool_bytes(cache)}, {cache->v_pages, pool_bytes(cache)},
                       {cache->k_exp, cache->n_pages},      {cache->v_exp, cache->n_pages},
                       {a->q.ptr ? a->q_out : nullptr, qo}};
  const Span ins[] = {{a->k.ptr, kb},          {a->v.ptr, vb},          {a->q.ptr, qb},
                      {a->held, lists * 4},    {a->count, lists * 4},   {a->start, lists * 4},
                      {a->src, lists * a->n_entries * 4}, {a->pos0, B * 4},
                      {table ? a->cos : nullptr, table}, {table ? a->sin : nullptr, table},
                      {cache->page_table, lists * cache->max_pages * 4}};
  if (!disjoint(outs, ins)) return KVPOP_EINVAL;
  kvpop::AppendLaunch L{};
  L.c = make_view(cache);
  L.k = make_rows(a->k);
  L.v = make_rows(a->v);
  if (a->q.ptr) {
    L.q = make_rows(a->q);
    L.q_out = static_cast<uint16_t*>(a->q_out);
    L.Hq = a->n_q_heads;
  }
  L.held = a->held;
  L.count = a->count;
  L.start = a->start;
  L.src = a->src;
  L.pos0 = a->pos0;
  L.cos = a->cos;
  L.sin = a->sin;
  L.N = a->n_tokens;
  L.M = a->n_entries;
  L.n_positions = a->n_positions;
  L.rot = a->rot_dim;
  L.adjacent = a->adjacent;
  L.stream = stream;
  if (kvpop::cache_append_threads(L) > UINT32_MAX) return KVPOP_EUNSUPPORTED;
  return launch([&] { return kvpop::launch_cache_append(L); });
}

size_t kvpop_cache_attn_workspace_size(const kvpop_cache* cache, int32_t n_q_heads, int32_t n_tokens) {
  kvpop::CacheAttnLaunch L;
  if (check_cache_attn_dims(cache, n_q_heads, n_tokens, &L) != KVPOP_OK) return 0;
  return (size_t)kvpop::cache_attn_workspace_floats(L) * 4;
}

int kvpop_cache_attn(const kvpop_cache* cache, int32_t n_q_heads, int32_t n_tokens, float scale, const kvpop_rows* q,
                     const int32_t* held, const int32_t* q_lens, void* o, float* lse, void* workspace,
                     size_t workspace_bytes, void* stream) {
  kvpop::CacheAttnLaunch L;
  int st = check_cache_attn_dims(cache, n_q_heads, n_tokens, &L);
  if (st != KVPOP_OK) return st;
  if ((st = check_cache(cache)) != KVPOP_OK) return st;
  if (!q || !held || !o || !lse || !std::isfinite(scale) || !(scale > 0.f)) return KVPOP_EINVAL;
  int64_t qb;
  if ((st = check_rows(*q, cache->batch, n_q_heads, n_tokens, cache->head_dim, &qb)) != KVPOP_OK) return st;
  if (!aligned16(o) || !aligned4(lse) || !aligned4(held) || !aligned4(q_lens)) return KVPOP_EUNSUPPORTED;
  const int64_t need = kvpop::cache_attn_workspace_floats(L) * 4;
  if (need > 0) {
    if (!workspace || workspace_bytes < (size_t)need) return KVPOP_EINVAL;
    if (!aligned16(workspace)) return KVPOP_EUNSUPPORTED;
  }
  const int64_t rows = (int64_t)cache->batch * n_q_heads * n_tokens, lists = cache_lists(cache);
  const Span outs[] = {{o, rows * cache->head_dim * 2}, {lse, rows * 4}, {need ? workspace : nullptr, need}};
  const Span ins[] = {{q->ptr, qb}, {held, lists * 4}, {q_lens, (int64_t)cache->batch * 4},
                      {cache->k_pages, pool_bytes(cache)}, {cache->v_pages, pool_bytes(cache)},
                      {cache->k_exp, cache->n_pages}, {cache->v_exp, cache->n_pages},
                      {cache->page_table, lists * cache->max_pages * 4}};
  if (!disjoint(outs, ins)) return KVPOP_EINVAL;
  L.q = make_rows(*q);
  L.held = held;
  L.q_lens = q_lens;
  L.o = static_cast<uint16_t*>(o);
  L.lse = lse;
  L.workspace = static_cast<float*>(workspace);
  L.scale = scale;
  L.stream = stream;
  return launch([&] { return kvpop::launch_cache_attn(L); });
}

int kvpop_retain_prompt(const kvpop_retain* s, int32_t seq_len, const int32_t* evict, const float* scores,
                        const float* log_gamma, const int32_t* lens, void* stream) {
  int st = check_retain(s);
  if (st != KVPOP_OK) return st;
  if (seq_len < 1 || !evict || !scores) return KVPOP_EINVAL;
  if (seq_len > KVPOP_MAX_SEQ_LEN) return KVPOP_EUNSUPPORTED;
  if (!aligned4(evict) || !aligned4(scores) || !aligned4(log_gamma) || !aligned4(lens)) return KVPOP_EUNSUPPORTED;
  const int64_t lists = (int64_t)s->batch * s->n_heads;
  const Span outs[] = {{s->pos, lists * s->slots * 4}, {s->prio, lists * s->slots * 4}, {s->held, lists * 4}};
  const Span ins[] = {{evict, lists * seq_len * 4}, {scores, lists * seq_len * 4}, {log_gamma, (int64_t)s->n_heads * 4},
                      {lens, (int64_t)s->batch * 4}};
  if (!disjoint(outs, ins)) return KVPOP_EINVAL;
  kvpop::RetainLaunch L = make_retain(s, scores, log_gamma, stream);
  L.evict = evict;
  L.lens = lens;
  L.T = seq_len;
  if (kvpop::retain_prompt_threads(L) > UINT32_MAX) return KVPOP_EUNSUPPORTED;
  return launch([&] { return kvpop::launch_retain_prompt(L); });
}

int kvpop_retain_step(const kvpop_retain* s, const float* scores, const float* log_gamma, const int32_t* q_pos,
                      int32_t sinks, int32_t window, int32_t topk, int32_t* slot, void* stream) {
  int st = check_retain(s);
  if (st != KVPOP_OK) return st;
  if (!scores || !q_pos || !slot || sinks < 0 || window < 0 || topk < 1) return KVPOP_EINVAL;
  if ((int64_t)sinks + window + topk > s->slots) return KVPOP_EINVAL;
  if (!aligned4(scores) || !aligned4(log_gamma) || !aligned4(q_pos) || !aligned4(slot)) return KVPOP_EUNSUPPORTED;
  const int64_t lists = (int64_t)s->batch * s->n_heads;
  const Span outs[] = {{s->pos, lists * s->slots * 4}, {s->prio, lists * s->slots * 4}, {s->held, lists * 4},
                       {slot, lists * 4}};
  const Span ins[] = {{scores, lists * 4}, {log_gamma, (int64_t)s->n_heads * 4}, {q_pos, (int64_t)s->batch * 4}};
  if (!disjoint(outs, ins)) return KVPOP_EINVAL;
  kvpop::RetainLaunch L = make_retain(s, scores, log_gamma, stream);
  L.q_pos = q_pos;
  L.sinks = sinks;
  L.window = window;
  L.topk = topk;
  L.slot = slot;
  if (kvpop::retain_step_threads(L) > UINT32_MAX) return KVPOP_EUNSUPPORTED;
  return launch([&] { return kvpop::launch_retain_step(L); });
}

}  // extern "C"
