// C ABI of the VarRate hot path (declared in include/varrate.h): argument validation, workspace
// carving and kernel launches. No device memory is allocated here.
#include <algorithm>
#include <atomic>
#include <initializer_list>

#include <float.h>
#include <math.h>
#include <stdint.h>

#include "common.cuh"
#include "kernels.h"
#include "paged.h"
#include "paged8.h"

using vr::Shape;

namespace {

constexpr int32_t kVersion = 1 * 10000 + 0 * 100 + 0;

bool valid_dtype(int32_t d) { return d == VARRATE_F32 || d == VARRATE_BF16; }

varrate_status check(const varrate_config* c) {
  if (c == nullptr) return VARRATE_ERR_ARG;
  if (c->n_layers < 1 || c->n_kv_heads < 1 || c->group < 1 || c->batch < 1 || c->window < 1 ||
      c->n_ctx < 1 || c->r_min < 1 || !valid_dtype(c->dtype) ||
      (c->mode != VARRATE_SALIENCE && c->mode != VARRATE_UNIFORM))
    return VARRATE_ERR_ARG;
  if (!(c->budget_frac > 0.0) || !(c->budget_frac <= 1.0)) return VARRATE_ERR_ARG;
  if (c->window > c->n_ctx || c->n_ctx >= (int64_t(1) << 31)) return VARRATE_ERR_ARG;
  if (c->pool_len < 1 || c->pool_len > 31 || (c->pool_len % 2) == 0) return VARRATE_ERR_ARG;
  if (c->head_dim != vr::kHeadDim) return VARRATE_ERR_UNSUPPORTED;
  if (c->r_min > c->head_dim) return VARRATE_ERR_ARG;
  if (c->group > 8 || (int64_t)c->group * c->window > 256) return VARRATE_ERR_UNSUPPORTED;
  if (c->dtype == VARRATE_BF16 &&
      (int64_t)c->batch * c->n_layers * c->n_kv_heads * c->n_ctx > (int64_t)INT32_MAX)
    return VARRATE_ERR_UNSUPPORTED;
  return VARRATE_OK;
}

int64_t coded_budget(const varrate_config* c) {
  return (int64_t)floor(c->budget_frac * (double)(c->n_ctx * (int64_t)c->head_dim)) -
         (int64_t)c->window * c->head_dim;
}

int64_t cap_elems(const varrate_config* c) {
  const int64_t n_coded = c->n_ctx - c->window;
  int64_t coded = coded_budget(c);
  if ((int64_t)c->r_min * n_coded > coded) coded = (int64_t)c->r_min * n_coded;
  if (coded < 0) coded = 0;
  int64_t pads = 0;
  for (int r = c->r_min; r <= c->head_dim; ++r) pads += 7 * r;
  const int64_t cap = coded + (int64_t)c->window * c->head_dim + pads;
  return (cap + 7) & ~int64_t(7);
}

Shape make_shape(const varrate_config* c, int64_t cap) {
  Shape s;
  s.B = c->batch; s.L = c->n_layers; s.G = c->n_kv_heads; s.grp = c->group;
  s.H = c->n_kv_heads * c->group; s.d = c->head_dim; s.w = c->window; s.pool = c->pool_len;
  s.r_min = c->r_min; s.r_max = c->head_dim; s.dtype = c->dtype; s.mode = c->mode;
  s.N = c->n_ctx; s.n_coded = c->n_ctx - c->window; s.Bc = coded_budget(c); s.cap = cap;
  return s;
}

// SM count of each device, cached per process (a property of the device: every thread that fills
// an entry writes the same value).
int num_sms() {
  static std::atomic<int> cached[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
  int n = cached[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) n = 148;
    cached[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}


size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

size_t ws_bytes(const varrate_config* c, int32_t which) {
  const Shape s = make_shape(c, cap_elems(c));
  const int sms = num_sms();
  switch (which) {
    case VARRATE_CALL_SALIENCE: return vr::salience_ws_bytes(s, sms);
    case VARRATE_CALL_PACK: return 0;
    case VARRATE_CALL_ENCODE:
      return vr::salience_ws_bytes(s, sms) + align256((size_t)s.B * s.L * s.n_coded * sizeof(float)) +
             align256((size_t)s.B * s.L * sizeof(int64_t));
    case VARRATE_CALL_DECODE: return vr::decode_ws_bytes(s, sms);
    case VARRATE_CALL_DECODE_WINDOW: return vr::decode_window_ws_bytes(s, sms);
    case VARRATE_CALL_DECODE_Q: return vr::decode_ws_bytes(s, sms);
    default: return 0;
  }
}

varrate_status launched() {
  return cudaGetLastError() == cudaSuccess ? VARRATE_OK : VARRATE_ERR_CUDA;
}

// Every device pointer must be 16-byte aligned: the kernels move data with 16-byte vector loads,
// 1-D bulk copies and TMA tiles, which fault on misaligned addresses. NULL passes.
bool aligned16(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if ((reinterpret_cast<uintptr_t>(p) & 15u) != 0) return false;
  return true;
}

int64_t qcap_bytes(const varrate_config* c, int bits) {
  const int64_t n_coded = c->n_ctx - c->window;
  int64_t sum = coded_budget(c);
  if ((int64_t)c->r_min * n_coded > sum) sum = (int64_t)c->r_min * n_coded;
  if (sum < 0) sum = 0;
  sum += (int64_t)c->window * c->head_dim;
  int64_t rsum = 0;
  for (int r = c->r_min; r <= c->head_dim; ++r) rsum += r;
  const int64_t full = vr::qrow_bytes(128, bits);
  const int64_t cap = (full * (sum + 7 * rsum) + 127) / 128 + 19 * rsum;
  return (cap + 15) & ~int64_t(15);
}

bool qpacked_ok(const varrate_config* c, const varrate_qpacked* p) {
  return p && p->data && p->qbase && p->bucket_count && (p->bits == 4 || p->bits == 8) &&
         p->qcap_bytes >= qcap_bytes(c, p->bits) && (p->qcap_bytes % 16) == 0 &&
         aligned16({p->data, p->qbase, p->bucket_count});
}

bool packed_ok(const varrate_config* c, const varrate_packed* p) {
  return p && p->coef && p->bucket_count && p->bucket_base && p->perm && p->pos && p->ranks &&
         p->cap_elems >= cap_elems(c) && (p->cap_elems % 8) == 0 &&
         aligned16({p->coef, p->bucket_count, p->bucket_base, p->perm, p->pos, p->ranks});
}

}  // namespace

extern "C" {

int32_t varrate_version(void) { return kVersion; }

const char* varrate_status_string(int32_t st) {
  switch (st) {
    case VARRATE_OK: return "ok";
    case VARRATE_FLOOR_BINDS: return "budget below the rank floor: every coded token at r_min";
    case VARRATE_ERR_ARG: return "invalid argument";
    case VARRATE_ERR_WORKSPACE: return "workspace too small";
    case VARRATE_ERR_CUDA: return "CUDA launch or runtime error";
    case VARRATE_ERR_TIMEOUT: return "bounded device wait timed out";
    case VARRATE_ERR_UNSUPPORTED: return "unsupported shape";
    case VARRATE_ERR_CORRUPT: return "rank or layout table out of range, or decode workspace left inconsistent";
    default: return "unknown status";
  }
}

varrate_status varrate_check_config(const varrate_config* cfg) { return check(cfg); }

int64_t varrate_coded_budget(const varrate_config* cfg) {
  return check(cfg) == VARRATE_OK ? coded_budget(cfg) : INT64_MIN;
}

int64_t varrate_packed_cap_elems(const varrate_config* cfg) {
  return check(cfg) == VARRATE_OK ? cap_elems(cfg) : -1;
}

size_t varrate_workspace_bytes(const varrate_config* cfg, int32_t which_call) {
  return check(cfg) == VARRATE_OK ? ws_bytes(cfg, which_call) : 0;
}

varrate_status varrate_salience(const varrate_config* cfg, const void* q_win, const void* k,
                                float* sal_out, void* ws, size_t ws_bytes_, void* stream) {
  varrate_status st = check(cfg);
  if (st != VARRATE_OK) return st;
  const bool empty = cfg->n_ctx == cfg->window;   // no coded token: nothing to score
  if (!empty && (!q_win || !k || !sal_out)) return VARRATE_ERR_ARG;
  if (cfg->mode == VARRATE_UNIFORM) return VARRATE_ERR_ARG;
  if (!aligned16({q_win, k, sal_out, ws})) return VARRATE_ERR_ARG;
  const size_t need = ws_bytes(cfg, VARRATE_CALL_SALIENCE);
  if (ws_bytes_ < need || (need > 0 && ws == nullptr)) return VARRATE_ERR_WORKSPACE;
  const Shape s = make_shape(cfg, cap_elems(cfg));
  if (vr::launch_salience(s, q_win, k, sal_out, ws, nullptr, num_sms(), (cudaStream_t)stream) < 0)
    return VARRATE_ERR_CUDA;
  return launched();
}

varrate_status varrate_allocate(const varrate_config* cfg, const float* sal, uint8_t* ranks,
                                int64_t* realized_sum, int32_t* dev_status, void* stream) {
  varrate_status st = check(cfg);
  if (st != VARRATE_OK) return st;
  if (!ranks || (cfg->mode == VARRATE_SALIENCE && !sal && cfg->n_ctx > cfg->window))
    return VARRATE_ERR_ARG;
  if (!aligned16({sal, ranks, realized_sum, dev_status})) return VARRATE_ERR_ARG;
  const Shape s = make_shape(cfg, cap_elems(cfg));
  if (vr::launch_allocate(s, sal, ranks, realized_sum, dev_status, num_sms(), (cudaStream_t)stream) < 0)
    return VARRATE_ERR_CUDA;
  return launched();
}

varrate_status varrate_pack(const varrate_config* cfg, const void* k, const void* v,
                            const void* basis_k, const void* basis_v, varrate_packed* out,
                            int32_t* dev_status, void* ws, size_t ws_bytes_, void* stream) {
  (void)ws; (void)ws_bytes_;
  varrate_status st = check(cfg);
  if (st != VARRATE_OK) return st;
  if (!k || !v || !basis_k || !basis_v || !packed_ok(cfg, out)) return VARRATE_ERR_ARG;
  if (!aligned16({k, v, basis_k, basis_v, dev_status})) return VARRATE_ERR_ARG;
  const Shape s = make_shape(cfg, out->cap_elems);
  if (!vr::pack_ready(s, k, v)) return VARRATE_ERR_CUDA;   // before anything is enqueued
  if (vr::launch_pack(s, k, v, basis_k, basis_v, *out, dev_status, num_sms(), (cudaStream_t)stream) < 0)
    return VARRATE_ERR_CUDA;
  return launched();
}

varrate_status varrate_encode(const varrate_config* cfg, const void* q_win, const void* k,
                              const void* v, const void* basis_k, const void* basis_v,
                              float* sal_out, varrate_packed* out, int64_t* realized_sum,
                              int32_t* dev_status, void* ws, size_t ws_bytes_, void* stream) {
  varrate_status st = check(cfg);
  if (st != VARRATE_OK) return st;
  if (!k || !v || !basis_k || !basis_v || !packed_ok(cfg, out)) return VARRATE_ERR_ARG;
  if (cfg->mode == VARRATE_SALIENCE && !q_win && cfg->n_ctx > cfg->window) return VARRATE_ERR_ARG;
  if (!aligned16({q_win, k, v, basis_k, basis_v, sal_out, realized_sum, dev_status, ws}))
    return VARRATE_ERR_ARG;
  const size_t need = ws_bytes(cfg, VARRATE_CALL_ENCODE);
  if (ws_bytes_ < need || ws == nullptr) return VARRATE_ERR_WORKSPACE;
  const Shape s = make_shape(cfg, out->cap_elems);
  if (!vr::pack_ready(s, k, v)) return VARRATE_ERR_CUDA;   // before anything is enqueued
  const int sms = num_sms();
  cudaStream_t cs = (cudaStream_t)stream;
  char* w = static_cast<char*>(ws);
  const size_t sal_ws = vr::salience_ws_bytes(s, sms);
  float* sal = sal_out ? sal_out : reinterpret_cast<float*>(w + sal_ws);
  int64_t* realized = realized_sum
      ? realized_sum
      : reinterpret_cast<int64_t*>(w + sal_ws + align256((size_t)s.B * s.L * s.n_coded * sizeof(float)));
  if (cfg->mode == VARRATE_SALIENCE && vr::launch_salience(s, q_win, k, sal, w, dev_status, sms, cs) < 0)
    return VARRATE_ERR_CUDA;
  if (vr::launch_allocate(s, sal, out->ranks, realized, dev_status, sms, cs) < 0) return VARRATE_ERR_CUDA;
  if (vr::launch_pack(s, k, v, basis_k, basis_v, *out, dev_status, sms, cs) < 0) return VARRATE_ERR_CUDA;
  return launched();
}

varrate_status varrate_decode_attn(const varrate_config* cfg, const varrate_packed* cache,
                                   const void* basis_k, const void* basis_v, const void* q,
                                   int32_t layer, const void* tail_k, const void* tail_v,
                                   int32_t n_tail, void* out, int32_t* dev_status, void* ws,
                                   size_t ws_bytes_, void* stream) {
  varrate_status st = check(cfg);
  if (st != VARRATE_OK) return st;
  if (!packed_ok(cfg, cache) || !basis_k || !basis_v || !q || !out) return VARRATE_ERR_ARG;
  if (layer < 0 || layer >= cfg->n_layers || n_tail < 0) return VARRATE_ERR_ARG;
  if (n_tail > 4096) return VARRATE_ERR_UNSUPPORTED;
  if (n_tail > 0 && (!tail_k || !tail_v)) return VARRATE_ERR_ARG;
  if (!aligned16({basis_k, basis_v, q, tail_k, tail_v, out, dev_status, ws})) return VARRATE_ERR_ARG;
  const size_t need = ws_bytes(cfg, VARRATE_CALL_DECODE);
  if (ws_bytes_ < need || ws == nullptr) return VARRATE_ERR_WORKSPACE;
  const Shape s = make_shape(cfg, cache->cap_elems);
  if (vr::launch_decode(s, *cache, basis_k, basis_v, q, layer, tail_k, tail_v, n_tail, out, dev_status,
                        ws, num_sms(), (cudaStream_t)stream) < 0)
    return VARRATE_ERR_CUDA;
  return launched();
}

varrate_status varrate_decode_window(const varrate_config* cfg, const varrate_packed* cache,
                                     const void* basis_k, const void* basis_v, const void* q,
                                     int32_t n_q, int32_t layer, const void* tail_k,
                                     const void* tail_v, int32_t n_tail, void* out,
                                     int32_t* dev_status, void* ws, size_t ws_bytes_, void* stream) {
  varrate_status st = check(cfg);
  if (st != VARRATE_OK) return st;
  if (cfg->dtype != VARRATE_BF16) return VARRATE_ERR_UNSUPPORTED;
  if (!packed_ok(cfg, cache) || !basis_k || !basis_v || !q || !out || !tail_k || !tail_v)
    return VARRATE_ERR_ARG;
  if (layer < 0 || layer >= cfg->n_layers || n_q < 1 || n_tail < n_q) return VARRATE_ERR_ARG;
  if (n_tail > 4096) return VARRATE_ERR_UNSUPPORTED;
  if (!aligned16({basis_k, basis_v, q, tail_k, tail_v, out, dev_status, ws})) return VARRATE_ERR_ARG;
  const Shape s = make_shape(cfg, cache->cap_elems);
  if (!vr::decode_window_supported(s, n_q, n_tail, num_sms())) return VARRATE_ERR_UNSUPPORTED;
  const size_t need = ws_bytes(cfg, VARRATE_CALL_DECODE_WINDOW);
  if (ws_bytes_ < need || ws == nullptr) return VARRATE_ERR_WORKSPACE;
  if (vr::launch_decode_window(s, *cache, basis_k, basis_v, q, n_q, layer, tail_k, tail_v, n_tail, out,
                               dev_status, ws, num_sms(), (cudaStream_t)stream) < 0)
    return VARRATE_ERR_CUDA;
  return launched();
}

int64_t varrate_qpacked_cap_bytes(const varrate_config* cfg, int32_t bits) {
  if (check(cfg) != VARRATE_OK || (bits != 4 && bits != 8)) return -1;
  return qcap_bytes(cfg, bits);
}

varrate_status varrate_quantize(const varrate_config* cfg, const varrate_packed* in,
                                varrate_qpacked* out, int32_t* dev_status, void* stream) {
  varrate_status st = check(cfg);
  if (st != VARRATE_OK) return st;
  if (cfg->dtype != VARRATE_BF16) return VARRATE_ERR_UNSUPPORTED;
  if (!packed_ok(cfg, in) || !qpacked_ok(cfg, out) || out->bucket_count != in->bucket_count)
    return VARRATE_ERR_ARG;
  if (!aligned16({dev_status})) return VARRATE_ERR_ARG;
  const Shape s = make_shape(cfg, in->cap_elems);
  if ((int64_t)s.B * s.L > 65535) return VARRATE_ERR_UNSUPPORTED;   // grid.y of the quantize kernel
  vr::launch_quantize(s, *in, *out, dev_status, num_sms(), (cudaStream_t)stream);
  return launched();
}

varrate_status varrate_decode_attn_q(const varrate_config* cfg, const varrate_qpacked* cache,
                                     const void* basis_k, const void* basis_v, const void* q,
                                     int32_t layer, const void* tail_k, const void* tail_v,
                                     int32_t n_tail, void* out, int32_t* dev_status, void* ws,
                                     size_t ws_bytes_, void* stream) {
  varrate_status st = check(cfg);
  if (st != VARRATE_OK) return st;
  if (cfg->dtype != VARRATE_BF16) return VARRATE_ERR_UNSUPPORTED;
  if (!qpacked_ok(cfg, cache) || !basis_k || !basis_v || !q || !out) return VARRATE_ERR_ARG;
  if (layer < 0 || layer >= cfg->n_layers || n_tail < 0) return VARRATE_ERR_ARG;
  if (n_tail > 4096) return VARRATE_ERR_UNSUPPORTED;
  if (n_tail > 0 && (!tail_k || !tail_v)) return VARRATE_ERR_ARG;
  if (!aligned16({basis_k, basis_v, q, tail_k, tail_v, out, dev_status, ws})) return VARRATE_ERR_ARG;
  const size_t need = ws_bytes(cfg, VARRATE_CALL_DECODE);
  if (ws_bytes_ < need || ws == nullptr) return VARRATE_ERR_WORKSPACE;
  const Shape s = make_shape(cfg, cap_elems(cfg));
  const int sms = num_sms();
  if (vr::decode_q_supported(s, cache->bits, cache->qcap_bytes, n_tail, sms) && aligned16({cache->data})) {
    char* w = static_cast<char*>(ws);
    if (vr::launch_decode_q_fused(s, *cache, basis_k, basis_v, q, layer, tail_k, tail_v, n_tail, out, dev_status,
                                  w, reinterpret_cast<float*>(w + vr::kDecodeCounterBytes), sms,
                                  (cudaStream_t)stream) < 0)
      return VARRATE_ERR_CUDA;
    return launched();
  }
  vr::launch_decode_q(s, *cache, basis_k, basis_v, q, layer, tail_k, tail_v, n_tail, out, ws, sms,
                      (cudaStream_t)stream);
  return launched();
}

size_t varrate_anchor_search_ws_bytes(const varrate_config* cfg, int32_t stride) {
  if (check(cfg) != VARRATE_OK || stride < 1 || stride > cfg->n_ctx) return 0;
  return vr::anchor_search_ws_bytes(make_shape(cfg, cap_elems(cfg)), stride);
}

varrate_status varrate_anchor_search(const varrate_config* cfg, const void* k, const void* v,
                                     int32_t stride, int32_t c, int32_t* idx_out, float* dist_out,
                                     int32_t* dev_status, void* ws, size_t ws_bytes_, void* stream) {
  varrate_status st = check(cfg);
  if (st != VARRATE_OK) return st;
  if (cfg->dtype != VARRATE_BF16) return VARRATE_ERR_UNSUPPORTED;
  if (!k || !v || !idx_out || stride < 1 || stride > cfg->n_ctx || c < 1) return VARRATE_ERR_ARG;
  if (!aligned16({k, v, idx_out, dist_out, dev_status, ws})) return VARRATE_ERR_ARG;
  const Shape s = make_shape(cfg, cap_elems(cfg));
  if (!vr::anchor_search_supported(s, stride, c)) return VARRATE_ERR_UNSUPPORTED;
  const size_t need = vr::anchor_search_ws_bytes(s, stride);
  if (ws_bytes_ < need || ws == nullptr) return VARRATE_ERR_WORKSPACE;
  if (vr::launch_anchor_search(s, k, v, stride, c, idx_out, dist_out, dev_status, ws,
                               (cudaStream_t)stream) < 0)
    return VARRATE_ERR_CUDA;
  return launched();
}

varrate_status varrate_anchor_residual(const varrate_config* cfg, const void* k, const void* v,
                                       int32_t stride, int32_t c, const int32_t* idx, void* e_out,
                                       int32_t* dev_status, void* stream) {
  varrate_status st = check(cfg);
  if (st != VARRATE_OK) return st;
  if (cfg->dtype != VARRATE_BF16) return VARRATE_ERR_UNSUPPORTED;
  if (!k || !v || !idx || !e_out || stride < 1 || stride > cfg->n_ctx || c < 1) return VARRATE_ERR_ARG;
  if (!aligned16({k, v, idx, e_out, dev_status})) return VARRATE_ERR_ARG;
  const Shape s = make_shape(cfg, cap_elems(cfg));
  if (!vr::anchor_residual_supported(s, stride, c)) return VARRATE_ERR_UNSUPPORTED;
  if (vr::launch_anchor_residual(s, k, v, stride, c, idx, e_out, dev_status, num_sms(), (cudaStream_t)stream) < 0)
    return VARRATE_ERR_CUDA;
  return launched();
}

static varrate_status paged_check(const varrate_pages* pages, const varrate_seqs* seqs) {
  if (pages == nullptr || seqs == nullptr) return VARRATE_ERR_ARG;
  if (!valid_dtype(pages->dtype) || pages->n_layers < 1 || pages->n_pages < 1 || pages->n_kv_heads < 1 ||
      pages->page_size < 1 || seqs->n_seqs < 0 || seqs->max_pages < 1 || seqs->n_rows < 0)
    return VARRATE_ERR_ARG;
  if (pages->head_dim != vr::kHeadDim) return VARRATE_ERR_UNSUPPORTED;
  const int32_t ps = pages->page_size;
  if (ps < 16 || ps > 256 || (ps & (ps - 1)) != 0 || pages->n_kv_heads > 4096) return VARRATE_ERR_UNSUPPORTED;
  if ((double)pages->n_pages * 2.0 * pages->n_kv_heads * ps > (double)INT32_MAX) return VARRATE_ERR_UNSUPPORTED;
  return VARRATE_OK;
}

static vr::Paged make_paged(const varrate_pages* pages, const varrate_seqs* seqs) {
  vr::Paged p;
  p.pool = static_cast<unsigned char*>(pages->pool);
  p.layer_rows = (int64_t)pages->n_pages * 2 * pages->n_kv_heads * pages->page_size;
  p.n_pages = pages->n_pages; p.G = pages->n_kv_heads; p.dtype = pages->dtype;
  p.page_log2 = 0;
  while ((1 << p.page_log2) < pages->page_size) ++p.page_log2;
  p.row_start = seqs->row_start; p.kv_len = seqs->kv_len; p.table = seqs->page_table;
  p.S = seqs->n_seqs; p.max_pages = seqs->max_pages; p.T = seqs->n_rows;
  return p;
}

// A batch's device pointers (looked at only where there are sequences).
static varrate_status paged_pointers(const varrate_pages* pages, const varrate_seqs* seqs, bool rows) {
  if (!pages->pool || !seqs->kv_len || !seqs->page_table || (rows && !seqs->row_start)) return VARRATE_ERR_ARG;
  return aligned16({pages->pool, seqs->kv_len, seqs->page_table, seqs->row_start}) ? VARRATE_OK : VARRATE_ERR_ARG;
}

varrate_status varrate_paged_append(const varrate_pages* pages, const varrate_seqs* seqs, int32_t layer,
                                    int32_t group, const void* q, int64_t q_stride, const void* k,
                                    int64_t k_stride, const void* v, int64_t v_stride, const void* q_norm,
                                    const void* k_norm, double eps, const double* freq, int32_t rot_dim,
                                    void* q_out, int32_t* dev_status, void* stream) {
  varrate_status st = paged_check(pages, seqs);
  if (st != VARRATE_OK) return st;
  if (layer < 0 || layer >= pages->n_layers || group < 1 || !(eps >= 0.0) || !isfinite((float)eps)) return VARRATE_ERR_ARG;
  if (group > 8) return VARRATE_ERR_UNSUPPORTED;
  if (rot_dim < 0 || rot_dim > vr::kHeadDim || (rot_dim % 16) != 0) return VARRATE_ERR_ARG;
  if (seqs->n_seqs == 0 || seqs->n_rows == 0) return VARRATE_OK;
  if ((st = paged_pointers(pages, seqs, true)) != VARRATE_OK) return st;
  if (!k || !v || (q && !q_out) || (rot_dim > 0 && !freq)) return VARRATE_ERR_ARG;
  if (!aligned16({q, k, v, q_norm, k_norm, freq, q_out, dev_status})) return VARRATE_ERR_ARG;
  const float eps32 = eps > 0.0 ? fmaxf((float)eps, FLT_TRUE_MIN) : 0.f;   // never rounded to 0: a head of zeros is no 0 / 0 then
  const int64_t vec = pages->dtype == VARRATE_F32 ? 4 : 8, kd = (int64_t)pages->n_kv_heads * vr::kHeadDim;
  if (k_stride < kd || k_stride % vec != 0 || v_stride < kd || v_stride % vec != 0) return VARRATE_ERR_ARG;
  if (q && (q_stride < kd * group || q_stride % vec != 0 || (q == q_out && q_stride != kd * group))) return VARRATE_ERR_ARG;
  if (vr::launch_paged_append(make_paged(pages, seqs), layer, group, q, q_stride, k, k_stride, v, v_stride, q_norm,
                              k_norm, eps32, freq, rot_dim, q_out, dev_status, num_sms(), (cudaStream_t)stream) < 0)
    return VARRATE_ERR_CUDA;
  return launched();
}

size_t varrate_paged_attn_ws_bytes(const varrate_pages* pages, const varrate_seqs* seqs, int32_t group) {
  if (paged_check(pages, seqs) != VARRATE_OK || group < 1 || group > 8) return 0;
  return vr::paged_attn_ws_bytes(make_paged(pages, seqs), group, num_sms());
}

varrate_status varrate_paged_attn(const varrate_pages* pages, const varrate_seqs* seqs, int32_t layer, int32_t group,
                                  const void* q, void* out, int32_t* dev_status, void* ws, size_t ws_bytes_,
                                  void* stream) {
  varrate_status st = paged_check(pages, seqs);
  if (st != VARRATE_OK) return st;
  if (layer < 0 || layer >= pages->n_layers || group < 1) return VARRATE_ERR_ARG;
  if (group > 8) return VARRATE_ERR_UNSUPPORTED;
  if (seqs->n_seqs == 0 || seqs->n_rows == 0) return VARRATE_OK;
  if ((st = paged_pointers(pages, seqs, true)) != VARRATE_OK) return st;
  if (!q || !out || q == out || !aligned16({q, out, dev_status, ws})) return VARRATE_ERR_ARG;
  const vr::Paged p = make_paged(pages, seqs);
  const int sms = num_sms();
  if (ws_bytes_ < vr::paged_attn_ws_bytes(p, group, sms) || ws == nullptr) return VARRATE_ERR_WORKSPACE;
  if (vr::launch_paged_attn(p, layer, group, q, out, dev_status, ws, sms, (cudaStream_t)stream) < 0) return VARRATE_ERR_CUDA;
  return launched();
}

varrate_status varrate_paged_gather(const varrate_pages* pages, const varrate_seqs* seqs, int32_t layer,
                                    int32_t n_layers, const int32_t* first, int32_t n, void* k_out, void* v_out,
                                    int32_t* dev_status, void* stream) {
  varrate_status st = paged_check(pages, seqs);
  if (st != VARRATE_OK) return st;
  if (layer < 0 || n_layers < 1 || n_layers > pages->n_layers - layer || n < 0) return VARRATE_ERR_ARG;
  if (seqs->n_seqs == 0 || n == 0 || (!k_out && !v_out)) return VARRATE_OK;
  if ((st = paged_pointers(pages, seqs, false)) != VARRATE_OK) return st;
  if (!aligned16({first, k_out, v_out, dev_status})) return VARRATE_ERR_ARG;
  if (vr::launch_paged_gather(make_paged(pages, seqs), layer, n_layers, first, n, k_out, v_out, dev_status, num_sms(),
                              (cudaStream_t)stream) < 0)
    return VARRATE_ERR_CUDA;
  return launched();
}

// The 8-bit pages' sizes as those of bf16 pages, for the checks and the kernels that both share.
static varrate_pages as_pages(const varrate_pages8* pages) {
  varrate_pages p = {};
  p.pool = pages->codes; p.n_layers = pages->n_layers; p.n_pages = pages->n_pages; p.n_kv_heads = pages->n_kv_heads;
  p.page_size = pages->page_size; p.head_dim = pages->head_dim; p.dtype = VARRATE_BF16;
  return p;
}

static varrate_status paged8_check(const varrate_pages8* pages, const varrate_seqs* seqs) {
  if (pages == nullptr) return VARRATE_ERR_ARG;
  const varrate_pages p = as_pages(pages);
  return paged_check(&p, seqs);
}

static varrate_status paged8_pointers(const varrate_pages8* pages, const varrate_seqs* seqs, bool rows) {
  const varrate_pages p = as_pages(pages);
  if (!pages->scale || !aligned16({pages->scale, pages->mass})) return VARRATE_ERR_ARG;
  return paged_pointers(&p, seqs, rows);
}

static vr::Paged8 make_paged8(const varrate_pages8* pages, const varrate_seqs* seqs) {
  const varrate_pages p = as_pages(pages);
  vr::Paged8 c;
  c.p = make_paged(&p, seqs);
  c.scale = static_cast<unsigned char*>(pages->scale);
  c.mass = pages->mass;
  return c;
}

varrate_status varrate_paged8_append(const varrate_pages8* pages, const varrate_seqs* seqs, int32_t layer, int32_t group,
                                     const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                                     int64_t v_stride, const void* q_norm, const void* k_norm, double eps,
                                     const double* freq, int32_t rot_dim, const int32_t* gone, void* q_out,
                                     int32_t* dev_status, void* stream) {
  varrate_status st = paged8_check(pages, seqs);
  if (st != VARRATE_OK) return st;
  if (layer < 0 || layer >= pages->n_layers || group < 1 || !(eps >= 0.0) || !isfinite((float)eps)) return VARRATE_ERR_ARG;
  if (group > 8) return VARRATE_ERR_UNSUPPORTED;
  if (rot_dim < 0 || rot_dim > vr::kHeadDim || (rot_dim % 16) != 0) return VARRATE_ERR_ARG;
  if (seqs->n_seqs == 0 || seqs->n_rows == 0) return VARRATE_OK;
  if ((st = paged8_pointers(pages, seqs, true)) != VARRATE_OK) return st;
  if (!k || !v || (q && !q_out) || (rot_dim > 0 && !freq)) return VARRATE_ERR_ARG;
  if (!aligned16({q, k, v, q_norm, k_norm, freq, gone, q_out, dev_status})) return VARRATE_ERR_ARG;
  const float eps32 = eps > 0.0 ? fmaxf((float)eps, FLT_TRUE_MIN) : 0.f;   // never rounded to 0: a head of zeros is no 0 / 0 then
  const int64_t kd = (int64_t)pages->n_kv_heads * vr::kHeadDim;
  if (k_stride < kd || k_stride % 8 != 0 || v_stride < kd || v_stride % 8 != 0) return VARRATE_ERR_ARG;
  if (q && (q_stride < kd * group || q_stride % 8 != 0 || (q == q_out && q_stride != kd * group))) return VARRATE_ERR_ARG;
  if (vr::launch_paged8_append(make_paged8(pages, seqs), layer, group, q, q_stride, k, k_stride, v, v_stride, q_norm, k_norm,
                               eps32, freq, rot_dim, gone, q_out, dev_status, num_sms(), (cudaStream_t)stream) < 0)
    return VARRATE_ERR_CUDA;
  return launched();
}

size_t varrate_paged8_attn_ws_bytes(const varrate_pages8* pages, const varrate_seqs* seqs, int32_t group) {
  if (paged8_check(pages, seqs) != VARRATE_OK || group < 1 || group > 8) return 0;
  return vr::paged8_attn_ws_bytes(make_paged8(pages, seqs), group, num_sms());
}

varrate_status varrate_paged8_attn(const varrate_pages8* pages, const varrate_seqs* seqs, int32_t layer, int32_t group,
                                   const void* q, void* out, float* lse, int32_t* dev_status, void* ws, size_t ws_bytes_,
                                   void* stream) {
  varrate_status st = paged8_check(pages, seqs);
  if (st != VARRATE_OK) return st;
  if (layer < 0 || layer >= pages->n_layers || group < 1) return VARRATE_ERR_ARG;
  if (group > 8) return VARRATE_ERR_UNSUPPORTED;
  if (seqs->n_seqs == 0 || seqs->n_rows == 0) return VARRATE_OK;
  if ((st = paged8_pointers(pages, seqs, true)) != VARRATE_OK) return st;
  if (!q || !out || q == out || !aligned16({q, out, lse, dev_status, ws})) return VARRATE_ERR_ARG;
  const vr::Paged8 c = make_paged8(pages, seqs);
  const int sms = num_sms();
  if (ws_bytes_ < vr::paged8_attn_ws_bytes(c, group, sms) || ws == nullptr) return VARRATE_ERR_WORKSPACE;
  if (vr::launch_paged8_attn(c, layer, group, q, out, lse, dev_status, ws, sms, (cudaStream_t)stream) < 0)
    return VARRATE_ERR_CUDA;
  return launched();
}

varrate_status varrate_paged8_mass(const varrate_pages8* pages, const varrate_seqs* seqs, int32_t layer, int32_t group,
                                   const void* q, const float* lse, int32_t* dev_status, void* stream) {
  varrate_status st = paged8_check(pages, seqs);
  if (st != VARRATE_OK) return st;
  if (layer < 0 || layer >= pages->n_layers || group < 1) return VARRATE_ERR_ARG;
  if (group > 8) return VARRATE_ERR_UNSUPPORTED;
  if (seqs->n_seqs == 0 || seqs->n_rows == 0) return VARRATE_OK;
  if ((st = paged8_pointers(pages, seqs, true)) != VARRATE_OK) return st;
  if (!pages->mass || !q || !lse || !aligned16({q, lse, dev_status})) return VARRATE_ERR_ARG;
  if (vr::launch_paged8_mass(make_paged8(pages, seqs), layer, group, q, lse, dev_status, num_sms(), (cudaStream_t)stream) < 0)
    return VARRATE_ERR_CUDA;
  return launched();
}

varrate_status varrate_paged8_evict(const varrate_pages8* pages, const varrate_seqs* seqs, int32_t layer, int32_t n_layers,
                                    int32_t budget, int32_t n_first, int32_t n_last, int32_t* kept, int32_t* new_len,
                                    int32_t* gone, int32_t* dev_status, void* stream) {
  varrate_status st = paged8_check(pages, seqs);
  if (st != VARRATE_OK) return st;
  if (layer < 0 || n_layers < 1 || n_layers > pages->n_layers - layer) return VARRATE_ERR_ARG;
  if (budget < 1 || n_first < 0 || n_last < 0 || n_first > budget - n_last) return VARRATE_ERR_ARG;
  if (seqs->n_seqs == 0) return VARRATE_OK;
  if ((st = paged8_pointers(pages, seqs, false)) != VARRATE_OK) return st;
  if (!pages->mass || !kept || !new_len || new_len == seqs->kv_len || gone == new_len || !aligned16({kept, new_len, gone, dev_status}))
    return VARRATE_ERR_ARG;
  if ((double)seqs->n_seqs * n_layers * pages->n_kv_heads > (double)(1 << 26)) return VARRATE_ERR_UNSUPPORTED;   // clusters of the grid
  if (vr::launch_paged8_evict(make_paged8(pages, seqs), layer, n_layers, budget, n_first, n_last, kept, new_len, gone,
                              dev_status, num_sms(), (cudaStream_t)stream) < 0)
    return VARRATE_ERR_CUDA;
  return launched();
}

}  // extern "C"
