// Host side of the paged 4-bit cache and of the rotary tables: argument checking and the scheduling of the kernels.  No device allocation happens here.
#include <cmath>
#include <new>

#include "host_checks.h"
#include "paged.cuh"

using namespace mixkvq;

struct mixkvq_paged {
  mixkvq_paged_config cfg;
  char* mem;
  uint64_t page_bytes, layer_bytes, bytes;
  uint32_t tile_bytes, piece_bytes;
  int g, lg_page, n_sms;
  uint64_t launches;
  int last_form;                             // mixkvq_paged_last_attention
  uint32_t test_extra_tx, test_wait_polls;   // mixkvq_paged_test_arm_copy_timeout
};

namespace {

constexpr uint64_t kHeaderBytes = 256;       // the status word lies at offset 0

int check_config(const mixkvq_paged_config* c) {
  if (!c || c->n_layers < 1 || c->n_q_heads < 1 || c->n_kv_heads < 1 || c->n_pages < 1 || c->reserved != 0 || c->n_q_heads % c->n_kv_heads != 0)
    return MIXKVQ_E_INVALID_ARG;
  if (c->head_dim != kD || c->n_q_heads / c->n_kv_heads > 8) return MIXKVQ_E_UNSUPPORTED;
  if (c->group_size != 32 && c->group_size != 64 && c->group_size != 128) return MIXKVQ_E_UNSUPPORTED;
  if (c->page_tokens < 16 || c->page_tokens > 256 || (c->page_tokens & (c->page_tokens - 1))) return MIXKVQ_E_UNSUPPORTED;
  // (sizes fit 64 bits with room to spare)
  if ((double)c->n_layers * c->n_pages * c->n_kv_heads * c->page_tokens / kPagedTile * paged_tile_bytes(c->group_size) > 0x1p60) return MIXKVQ_E_UNSUPPORTED;
  return MIXKVQ_OK;
}

void plan(const mixkvq_paged_config* c, mixkvq_paged* h) {
  h->cfg = *c;
  h->g = c->n_q_heads / c->n_kv_heads;
  h->lg_page = 4;
  while (1 << h->lg_page < c->page_tokens) ++h->lg_page;
  h->tile_bytes = paged_tile_bytes(c->group_size);
  h->piece_bytes = h->tile_bytes * (uint32_t)(c->page_tokens / kPagedTile);
  h->page_bytes = (uint64_t)h->piece_bytes * c->n_kv_heads;
  h->layer_bytes = h->page_bytes * c->n_pages;
  h->bytes = kHeaderBytes + h->layer_bytes * c->n_layers;
}

// The sequences of a call.
int check_sequences(const mixkvq_paged* h, int layer, const mixkvq_paged_sequences* s, PagedView* v) {
  if (!h || !s || layer < 0 || layer >= h->cfg.n_layers || s->batch < 1 || s->n_tokens < 1 || s->max_pages < 1 || s->pages_stride < s->max_pages || !s->pages_dev ||
      !s->lens_dev)
    return MIXKVQ_E_INVALID_ARG;
  if (!aligned(s->pages_dev, 4) || !aligned(s->lens_dev, 4) || !aligned(s->counts_dev, 4)) return MIXKVQ_E_ALIGNMENT;
  if ((long long)s->max_pages * h->cfg.page_tokens > MIXKVQ_PAGED_MAX_TOKENS || (long long)s->batch * s->n_tokens > 0x7FFFFFFFll / 16 ||
      s->batch > MIXKVQ_PAGED_MAX_BATCH)
    return MIXKVQ_E_UNSUPPORTED;
  *v = PagedView{};
  v->pool = h->mem + kHeaderBytes + h->layer_bytes * (uint64_t)layer;
  v->status = reinterpret_cast<uint32_t*>(h->mem);
  v->pages = s->pages_dev;
  v->lens = s->lens_dev;
  v->counts = s->counts_dev;
  v->page_bytes = h->page_bytes;
  v->piece_bytes = h->piece_bytes;
  v->tile_bytes = h->tile_bytes;
  v->B = s->batch; v->n = s->n_tokens; v->Hq = h->cfg.n_q_heads; v->Hkv = h->cfg.n_kv_heads; v->g = h->g; v->G = h->cfg.group_size;
  v->n_pages = h->cfg.n_pages; v->lg_page = h->lg_page; v->max_pages = s->max_pages; v->pages_stride = s->pages_stride;
  return MIXKVQ_OK;
}
// What no output of a call may lie over, beside its own inputs.
void add_sequences(const mixkvq_paged* h, const mixkvq_paged_sequences* s, Ranges* r) {
  r->read(h->mem, h->bytes);
  r->read(s->pages_dev, 4 * ((size_t)(s->batch - 1) * s->pages_stride + s->max_pages));
  r->read(s->lens_dev, 4 * (size_t)s->batch);
  r->read(s->counts_dev, 4 * (size_t)s->batch);
}

int plan_append(const mixkvq_paged* h, int layer, const mixkvq_paged_sequences* s, const void* k_dev, const void* v_dev, const void* q_dev, const int64_t* strides_host,
                const mixkvq_rotation* rotation, void* q_out_dev, PagedAppend* a, Ranges* ranges) {
  *a = PagedAppend{};
  const int rc = check_sequences(h, layer, s, &a->view);
  if (rc != MIXKVQ_OK) return rc;
  if (!k_dev || !v_dev || (q_dev == nullptr) != (q_out_dev == nullptr)) return MIXKVQ_E_INVALID_ARG;
  const int B = s->batch, n = s->n_tokens;
  Ranges& r = *ranges;
  const void* in[3] = {q_dev, k_dev, v_dev};
  RopeTensor* t[3] = {&a->tq, &a->tk, &a->tv};
  for (int i = 0; i < 3; ++i) {
    const int H = i == 0 ? h->cfg.n_q_heads : h->cfg.n_kv_heads;
    *t[i] = strides_host ? RopeTensor{strides_host[3 * i], strides_host[3 * i + 1], strides_host[3 * i + 2]} : head_major(H, n);
    const int bad = check_strided(in[i], *t[i], B, H, n, &r, i == 0 && same_rows(in[0], *t[0], q_out_dev, B, H, n));
    if (bad != MIXKVQ_OK) return bad;
  }
  if (q_out_dev != nullptr) {
    if (!aligned16(q_out_dev)) return MIXKVQ_E_ALIGNMENT;
    r.write(q_out_dev, (size_t)B * h->cfg.n_q_heads * n * kD * 2);
  }
  if (rotation != nullptr) {
    const int bad = check_rotation(rotation, B, n, true, &a->turn, &r);
    if (bad != MIXKVQ_OK) return bad;
  }
  // the pool is written: the inputs do not lie in it either
  add_sequences(h, s, &r);
  if (r.clash() || r.touches(h->mem, h->bytes)) return MIXKVQ_E_INVALID_ARG;
  a->k = k_dev; a->v = v_dev; a->q = q_dev; a->q_out = q_out_dev;
  return MIXKVQ_OK;
}

// ranges: empty, or those of the append that the call begins with, which writes q_dev
int plan_attention(const mixkvq_paged* h, int layer, const mixkvq_paged_sequences* s, const void* q_dev, const void* out_dev, int out_type, float softmax_scale,
                   const void* workspace_dev, size_t workspace_bytes, PagedAttention* a, Ranges* ranges) {
  *a = PagedAttention{};
  const int rc = check_sequences(h, layer, s, &a->view);
  if (rc != MIXKVQ_OK) return rc;
  if (!q_dev || !out_dev || !workspace_dev || (out_type != MIXKVQ_OUT_FLOAT && out_type != MIXKVQ_OUT_BF16) || !(softmax_scale > 0.f) || !std::isfinite(softmax_scale))
    return MIXKVQ_E_INVALID_ARG;
  if (!aligned16(q_dev) || !aligned16(out_dev) || !aligned16(workspace_dev)) return MIXKVQ_E_ALIGNMENT;
  if ((long long)s->batch * s->n_tokens * h->cfg.n_q_heads > 0x7FFFFFFFll || (long long)s->n_tokens * h->g >= 1 << 28) return MIXKVQ_E_UNSUPPORTED;      // (thread blocks of a grid)
  const size_t need = paged_workspace_need(h->cfg.n_kv_heads, h->g, s->batch, s->n_tokens, (long long)s->max_pages * h->cfg.page_tokens);
  if (workspace_bytes < need) return MIXKVQ_E_BUFFER_TOO_SMALL;
  const size_t rows = (size_t)s->batch * h->cfg.n_q_heads * s->n_tokens * kD;
  Ranges& r = *ranges;
  const bool alone = r.n == 0;
  r.write(out_dev, rows * (out_type == MIXKVQ_OUT_BF16 ? 2 : 4));
  r.write(workspace_dev, need);
  if (alone) {
    r.read(q_dev, 2 * rows);
    add_sequences(h, s, &r);
  }
  if (r.clash()) return MIXKVQ_E_INVALID_ARG;
  a->q = q_dev;
  a->out = const_cast<void*>(out_dev);
  a->out_bf16 = out_type == MIXKVQ_OUT_BF16;
  a->scale_log2e = softmax_scale * 1.4426950408889634f;
  a->parts = static_cast<float*>(const_cast<void*>(workspace_dev));
  a->max_polls = h->test_wait_polls;
  a->test_extra = h->test_extra_tx;
  return MIXKVQ_OK;
}

int run_append(mixkvq_paged* h, const PagedAppend& a, cudaStream_t st) {
  if (launch_paged_append(a, h->n_sms, st) != cudaSuccess) return MIXKVQ_E_CUDA;
  h->launches += 1;
  return MIXKVQ_OK;
}
int run_attention(mixkvq_paged* h, const PagedAttention& a, cudaStream_t st) {
  int launches = 0;
  const cudaError_t e = launch_paged_attention(a, h->n_sms, st, &launches, &h->last_form);
  h->launches += launches;
  return e == cudaSuccess ? MIXKVQ_OK : MIXKVQ_E_CUDA;
}

}  // namespace

extern "C" {

int mixkvq_rope_tables(const mixkvq_rope_scaling* sc, int64_t start, int n_positions, float* cos_dev, float* sin_dev, void* stream) {
  if (!sc || !cos_dev || !sin_dev || n_positions < 1 || start < 0 || start > (1ll << 40) || sc->reserved != 0) return MIXKVQ_E_INVALID_ARG;
  if (sc->rotary_dim < 16 || sc->rotary_dim > kD || sc->rotary_dim % 16) return MIXKVQ_E_UNSUPPORTED;
  const int d = sc->rotary_dim;
  if (!(sc->base > 1.) || !std::isfinite(sc->base) || !(sc->factor > 0.) || !std::isfinite(sc->factor) || !(sc->attention_factor >= 0.) ||
      !std::isfinite(sc->attention_factor))
    return MIXKVQ_E_INVALID_ARG;
  const bool ranges = sc->kind == MIXKVQ_ROPE_BANDS || sc->kind == MIXKVQ_ROPE_YARN;
  if (sc->kind < MIXKVQ_ROPE_PLAIN || sc->kind > MIXKVQ_ROPE_YARN) return MIXKVQ_E_INVALID_ARG;
  if (ranges && (!(sc->original > 0.) || !std::isfinite(sc->original) || !(sc->low > 0.) || !(sc->high > sc->low) || !std::isfinite(sc->high)))
    return MIXKVQ_E_INVALID_ARG;
  if (!aligned16(cos_dev) || !aligned16(sin_dev)) return MIXKVQ_E_ALIGNMENT;
  Ranges r;
  r.write(cos_dev, 2 * (size_t)n_positions * d);
  r.write(sin_dev, 2 * (size_t)n_positions * d);
  if (r.clash()) return MIXKVQ_E_INVALID_ARG;
  RopeTables a{};
  const double pi = 3.14159265358979323846;
  double base = sc->base, m = 1.;
  if (sc->kind == MIXKVQ_ROPE_NTK) base *= std::pow(sc->factor, (double)d / (d - 2));
  double ramp_lo = 0., ramp_hi = 0.;
  if (sc->kind == MIXKVQ_ROPE_YARN) {
    auto dim = [&](double turns) { return d * std::log(sc->original / (turns * 2. * pi)) / (2. * std::log(base)); };
    ramp_lo = std::fmax(std::floor(dim(sc->high)), 0.);
    ramp_hi = std::fmin(std::ceil(dim(sc->low)), d - 1.);
    if (sc->factor > 1.) m = 0.1 * std::log(sc->factor) + 1.;
  }
  for (int i = 0; i < d / 2; ++i) {
    double f = std::pow(base, -2. * i / d), keep = 1.;           // keep: how much of the frequency is left unscaled
    if (sc->kind == MIXKVQ_ROPE_LINEAR) keep = 0.;
    if (sc->kind == MIXKVQ_ROPE_BANDS) keep = std::fmin(std::fmax((sc->original * f / (2. * pi) - sc->low) / (sc->high - sc->low), 0.), 1.);
    if (sc->kind == MIXKVQ_ROPE_YARN) keep = 1. - std::fmin(std::fmax((i - ramp_lo) / std::fmax(ramp_hi - ramp_lo, 1e-3), 0.), 1.);
    f = f * keep + f / sc->factor * (1. - keep);
    a.turns[i] = f / pi;
  }
  a.factor = sc->attention_factor > 0. ? sc->attention_factor : m;
  a.cos_t = cos_dev;
  a.sin_t = sin_dev;
  a.start = start;
  a.n = n_positions;
  a.half = d / 2;
  int dev = 0, n_sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n_sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return MIXKVQ_E_CUDA;
  return launch_rope_tables(a, n_sms, static_cast<cudaStream_t>(stream)) == cudaSuccess ? MIXKVQ_OK : MIXKVQ_E_CUDA;
}

int mixkvq_paged_bytes(const mixkvq_paged_config* cfg, size_t* pool_bytes) {
  const int rc = check_config(cfg);
  if (rc != MIXKVQ_OK) return rc;
  mixkvq_paged h{};
  plan(cfg, &h);
  if (pool_bytes) *pool_bytes = (size_t)h.bytes;
  return MIXKVQ_OK;
}

size_t mixkvq_paged_workspace_bytes(const mixkvq_paged_config* cfg, int batch, int n_tokens, int max_pages) {
  if (check_config(cfg) != MIXKVQ_OK || batch < 1 || n_tokens < 1 || max_pages < 1 || (long long)max_pages * cfg->page_tokens > MIXKVQ_PAGED_MAX_TOKENS) return 0;
  return paged_workspace_bytes(cfg->n_kv_heads, cfg->n_q_heads / cfg->n_kv_heads, batch, n_tokens, (long long)max_pages * cfg->page_tokens);
}

int mixkvq_paged_init(const mixkvq_paged_config* cfg, void* pool_dev, size_t bytes, void* stream, mixkvq_paged** out) {
  const int rc = check_config(cfg);
  if (rc != MIXKVQ_OK) return rc;
  if (!pool_dev || !out) return MIXKVQ_E_INVALID_ARG;
  if (!aligned(pool_dev, 256)) return MIXKVQ_E_ALIGNMENT;
  mixkvq_paged* h = new (std::nothrow) mixkvq_paged();
  if (!h) return MIXKVQ_E_INVALID_ARG;
  plan(cfg, h);
  h->mem = static_cast<char*>(pool_dev);
  int dev = 0, code = MIXKVQ_OK;
  if (bytes < h->bytes) code = MIXKVQ_E_BUFFER_TOO_SMALL;
  else if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&h->n_sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
           cudaMemsetAsync(h->mem, 0, kHeaderBytes, static_cast<cudaStream_t>(stream)) != cudaSuccess || paged_attention_setup() != cudaSuccess)
    code = MIXKVQ_E_CUDA;
  if (code != MIXKVQ_OK) {
    delete h;
    return code;
  }
  *out = h;
  return MIXKVQ_OK;
}

int mixkvq_paged_destroy(mixkvq_paged* cache) {
  delete cache;
  return MIXKVQ_OK;
}

int mixkvq_paged_append(mixkvq_paged* cache, int layer, const mixkvq_paged_sequences* seqs, const void* k_dev, const void* v_dev, const void* q_dev,
                        const int64_t* strides_host, const mixkvq_rotation* rotation, void* q_out_dev, void* stream) {
  PagedAppend a;
  Ranges r;
  const int rc = plan_append(cache, layer, seqs, k_dev, v_dev, q_dev, strides_host, rotation, q_out_dev, &a, &r);
  return rc != MIXKVQ_OK ? rc : run_append(cache, a, static_cast<cudaStream_t>(stream));
}

int mixkvq_paged_read(mixkvq_paged* cache, int layer, const mixkvq_paged_sequences* seqs, void* k_out_dev, void* v_out_dev, void* stream) {
  PagedRead a{};
  const int rc = check_sequences(cache, layer, seqs, &a.view);
  if (rc != MIXKVQ_OK) return rc;
  if (!k_out_dev || !v_out_dev) return MIXKVQ_E_INVALID_ARG;
  if (!aligned16(k_out_dev) || !aligned16(v_out_dev)) return MIXKVQ_E_ALIGNMENT;
  const size_t bytes = (size_t)seqs->batch * cache->cfg.n_kv_heads * seqs->n_tokens * kD * 2;
  Ranges r;
  r.write(k_out_dev, bytes);
  r.write(v_out_dev, bytes);
  add_sequences(cache, seqs, &r);
  if (r.clash()) return MIXKVQ_E_INVALID_ARG;
  a.k = k_out_dev;
  a.v = v_out_dev;
  if (launch_paged_read(a, cache->n_sms, static_cast<cudaStream_t>(stream)) != cudaSuccess) return MIXKVQ_E_CUDA;
  cache->launches += 1;
  return MIXKVQ_OK;
}

int mixkvq_paged_attention(mixkvq_paged* cache, int layer, const mixkvq_paged_sequences* seqs, const void* q_dev, void* out_dev, int out_type, float softmax_scale,
                           void* workspace_dev, size_t workspace_bytes, void* stream) {
  PagedAttention a;
  Ranges r;
  const int rc = plan_attention(cache, layer, seqs, q_dev, out_dev, out_type, softmax_scale, workspace_dev, workspace_bytes, &a, &r);
  return rc != MIXKVQ_OK ? rc : run_attention(cache, a, static_cast<cudaStream_t>(stream));
}

int mixkvq_paged_step(mixkvq_paged* cache, int layer, const mixkvq_paged_sequences* seqs, const void* k_dev, const void* v_dev, const void* q_dev,
                      const int64_t* strides_host, const mixkvq_rotation* rotation, void* q_out_dev, void* out_dev, int out_type, float softmax_scale,
                      void* workspace_dev, size_t workspace_bytes, void* stream) {
  PagedAppend a;
  PagedAttention b;
  if (!q_dev) return MIXKVQ_E_INVALID_ARG;
  Ranges r;
  int rc = plan_append(cache, layer, seqs, k_dev, v_dev, q_dev, strides_host, rotation, q_out_dev, &a, &r);
  if (rc != MIXKVQ_OK) return rc;
  rc = plan_attention(cache, layer, seqs, q_out_dev, out_dev, out_type, softmax_scale, workspace_dev, workspace_bytes, &b, &r);
  if (rc != MIXKVQ_OK) return rc;
  b.view.add_counts = 1;
  rc = run_append(cache, a, static_cast<cudaStream_t>(stream));
  return rc != MIXKVQ_OK ? rc : run_attention(cache, b, static_cast<cudaStream_t>(stream));
}

int mixkvq_paged_test_arm_copy_timeout(mixkvq_paged* cache, uint32_t extra_bytes, uint32_t max_polls) {
  if (!cache || (extra_bytes & 15u)) return MIXKVQ_E_INVALID_ARG;
  cache->test_extra_tx = extra_bytes;
  cache->test_wait_polls = max_polls;
  return MIXKVQ_OK;
}

int mixkvq_paged_query_status(mixkvq_paged* cache, int* device_status, void* stream) {
  if (!cache || !device_status) return MIXKVQ_E_INVALID_ARG;
  uint32_t w = 0;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (cudaMemcpyAsync(&w, cache->mem, sizeof(w), cudaMemcpyDeviceToHost, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess) return MIXKVQ_E_CUDA;
  *device_status = (int)w;
  return MIXKVQ_OK;
}

int mixkvq_paged_clear_status(mixkvq_paged* cache, void* stream) {
  if (!cache) return MIXKVQ_E_INVALID_ARG;
  return cudaMemsetAsync(cache->mem, 0, kHeaderBytes, static_cast<cudaStream_t>(stream)) == cudaSuccess ? MIXKVQ_OK : MIXKVQ_E_CUDA;
}

int mixkvq_paged_last_attention(const mixkvq_paged* cache) { return cache ? cache->last_form : 0; }

uint64_t mixkvq_paged_launch_count(const mixkvq_paged* cache) { return cache ? cache->launches : 0; }

}  // extern "C"
