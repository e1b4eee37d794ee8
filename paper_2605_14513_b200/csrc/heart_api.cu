// C ABI of the HEART hot path: argument validation, workspace carving and kernel sequencing.
// No device memory is allocated here and nothing synchronises except heart_get_status.
#include <math.h>

#include <initializer_list>
#include <mutex>
#include <stdio.h>
#include <string.h>

#include "common.cuh"
#include "cross.cuh"

using namespace heart;

namespace {

thread_local char g_errbuf[256] = "";
thread_local int g_launches = 0;

int cuda_fail(cudaError_t e, const char *where) {
  snprintf(g_errbuf, sizeof g_errbuf, "CUDA error in %s: %s", where, cudaGetErrorString(e));
  return HEART_ERR_CUDA;
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace

// Validates the shape part of a config and derives the geometry. Returns HEART_OK or an error.
int heart::make_geom(const heart_config *c, Geom *g) {
  if (c == nullptr) return HEART_ERR_INVALID;
  if (c->B <= 0 || c->H <= 0 || c->N <= 0) return HEART_ERR_INVALID;
  if (c->D != kD) return HEART_ERR_UNSUPPORTED;
  if (c->block != 64 && c->block != 128) return HEART_ERR_UNSUPPORTED;
  g->B = c->B;
  g->H = c->H;
  g->R = c->B * c->H;
  g->N = c->N;
  g->block = c->block;
  g->nb = (c->N + c->block - 1) / c->block;
  if (g->nb > HEART_MAX_BLOCKS) return HEART_ERR_UNSUPPORTED;
  g->W = (g->nb + 31) / 32;
  if (c->stride_b == 0 && c->stride_h == 0 && c->stride_n == 0) {
    g->sn = kD;
    g->sh = (long long)c->N * kD;
    g->sb = g->sh * c->H;
  } else {
    g->sb = c->stride_b;
    g->sh = c->stride_h;
    g->sn = c->stride_n;
    if (g->sn < kD || g->sh <= 0 || g->sb <= 0) return HEART_ERR_INVALID;
    if ((g->sn % 8) || (g->sh % 8) || (g->sb % 8)) return HEART_ERR_INVALID;
  }
  g->idx_stride = c->idx_stride;
  if (g->idx_stride < g->nb) return HEART_ERR_INVALID;
  g->scale = (c->scale > 0.0) ? c->scale : 1.0 / sqrt((double)kD);
  g->gate_lo = c->gate_lo;
  g->gate_hi = c->gate_hi;
  if (isnan(g->gate_lo) || isnan(g->gate_hi)) return HEART_ERR_INVALID;
  g->flags = c->flags;
  set_chunks(*g);
  return HEART_OK;
}

// The same for a heart_cache_config.
int heart::make_cache_geom(const heart_cache_config *c, CacheGeom *g) {
  if (c == nullptr) return HEART_ERR_INVALID;
  if (c->S <= 0 || c->T <= 0 || c->Hq <= 0 || c->Hkv <= 0 || c->n_pages <= 0 || c->table_stride <= 0) return HEART_ERR_INVALID;
#ifdef HEART_TEST_HOOKS
  g->test_skip = c->flags == 0x80000000u;
  const uint32_t flags = c->flags & 0x7fffffffu;
#else
  g->test_skip = 0;
  const uint32_t flags = c->flags;
#endif
  if (c->max_new < 0 || c->causal < 0 || c->window < 0 || c->sink < 0 || flags != 0) return HEART_ERR_INVALID;
  if (c->kind != HEART_CACHE_BF16 && c->kind != HEART_CACHE_E4M3) return HEART_ERR_INVALID;
  if (c->Hq % c->Hkv != 0) return HEART_ERR_INVALID;
  if (c->D != kD || c->Hq / c->Hkv > 128) return HEART_ERR_UNSUPPORTED;
  if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return HEART_ERR_UNSUPPORTED;
  constexpr long long kMost = (1LL << 31) - 256;  // rows, tokens and slots are counted in 32 bits
  if ((long long)c->table_stride * c->page >= kMost || (long long)c->T * c->Hq >= kMost || c->S >= (1 << 30)) return HEART_ERR_UNSUPPORTED;
  g->S = c->S;
  g->T = c->T;
  g->Hq = c->Hq;
  g->Hkv = c->Hkv;
  g->G = c->Hq / c->Hkv;
  g->page = c->page;
  g->n_pages = c->n_pages;
  g->table_stride = c->table_stride;
  g->e4m3 = c->kind == HEART_CACHE_E4M3;
  g->max_new = c->max_new == 0 || c->max_new > c->T ? c->T : c->max_new;
  g->causal = c->causal;
  g->window = c->window;
  g->sink = c->sink;
  auto strides_ok = [](long long a, long long b, int multiple) {
    constexpr long long kMostStride = 1LL << 38;
    return a >= kD && b >= kD && a < kMostStride && b < kMostStride && a % multiple == 0 && b % multiple == 0;
  };
  const bool q_plain = c->q_stride_t == 0 && c->q_stride_h == 0, kv_plain = c->kv_stride_t == 0 && c->kv_stride_h == 0;
  const bool pool_plain = c->pool_stride_page == 0 && c->pool_stride_h == 0 && c->pool_stride_t == 0;
  g->qt = q_plain ? (long long)c->Hq * kD : c->q_stride_t;
  g->qh = q_plain ? kD : c->q_stride_h;
  g->kvt = kv_plain ? (long long)c->Hkv * kD : c->kv_stride_t;
  g->kvh = kv_plain ? kD : c->kv_stride_h;
  g->pt = pool_plain ? kD : c->pool_stride_t;
  g->ph = pool_plain ? (long long)c->page * kD : c->pool_stride_h;
  g->pp = pool_plain ? (long long)c->Hkv * c->page * kD : c->pool_stride_page;
  const int multiple = g->e4m3 ? 16 : 8;
  if (!strides_ok(g->qt, g->qh, 8) || !strides_ok(g->kvt, g->kvh, 8) || !strides_ok(g->pt, g->ph, multiple) || !strides_ok(g->pp, g->pp, multiple))
    return HEART_ERR_INVALID;
  if (!isfinite(c->scale)) return HEART_ERR_INVALID;
  g->scale = c->scale > 0.0 ? c->scale : 1.0 / sqrt((double)kD);
  if (g->scale < 1e-30 || g->scale > 1e30) return HEART_ERR_INVALID;  // (a normal fp32 number)
  return HEART_OK;
}

// The same for a heart_cross_config.
int heart::make_cross_geom(const heart_cross_config *c, CrossGeom *g) {
  if (c == nullptr) return HEART_ERR_INVALID;
  if (c->S <= 0 || c->T <= 0 || c->Tk <= 0 || c->Hq <= 0 || c->Hkv <= 0 || c->max_q < 0) return HEART_ERR_INVALID;
#ifdef HEART_TEST_HOOKS
  g->test_skip = c->flags == 0x80000000u;
  const uint32_t flags = c->flags & 0x7fffffffu;
#else
  g->test_skip = 0;
  const uint32_t flags = c->flags;
#endif
  if (flags != 0 || c->Hq % c->Hkv != 0) return HEART_ERR_INVALID;
  if (c->D != kD || c->Hq / c->Hkv > 128) return HEART_ERR_UNSUPPORTED;
  constexpr long long kMost = (1LL << 31) - 256;  // rows are counted in 32 bits
  if ((long long)c->T * c->Hq >= kMost || c->Tk >= kMost || c->S >= (1 << 30)) return HEART_ERR_UNSUPPORTED;
  g->S = c->S;
  g->T = c->T;
  g->Tk = c->Tk;
  g->Hq = c->Hq;
  g->Hkv = c->Hkv;
  g->G = c->Hq / c->Hkv;
  g->max_q = c->max_q == 0 || c->max_q > c->T ? c->T : c->max_q;
  auto strides_ok = [](long long a, long long b) {
    constexpr long long kMostStride = 1LL << 38;
    return a >= kD && b >= kD && a < kMostStride && b < kMostStride && a % 8 == 0 && b % 8 == 0;
  };
  const bool q_plain = c->q_stride_t == 0 && c->q_stride_h == 0, kv_plain = c->kv_stride_t == 0 && c->kv_stride_h == 0;
  g->qt = q_plain ? (long long)c->Hq * kD : c->q_stride_t;
  g->qh = q_plain ? kD : c->q_stride_h;
  g->kt = kv_plain ? (long long)c->Hkv * kD : c->kv_stride_t;
  g->kh = kv_plain ? kD : c->kv_stride_h;
  if (!strides_ok(g->qt, g->qh) || !strides_ok(g->kt, g->kh) || !strides_ok(g->G * g->qh, kD)) return HEART_ERR_INVALID;  // (from key head to key head)
  if (!isfinite(c->scale)) return HEART_ERR_INVALID;
  g->scale = c->scale > 0.0 ? c->scale : 1.0 / sqrt((double)kD);
  if (g->scale < 1e-30 || g->scale > 1e30) return HEART_ERR_INVALID;  // (a normal fp32 number)
  return HEART_OK;
}

namespace {

// What the three calls on a cache check alike, and the arrays as the kernels take them.
int cache_call(const heart_cache_config *cfg, const heart_cache *cache, const int32_t *page_table, const int32_t *row_start,
               const int32_t *kv_len, void *workspace, CacheGeom *g, CacheWorkspace *w, CacheIndex *ix) {
  const int rc = make_cache_geom(cfg, g);
  if (rc != HEART_OK) return rc;
  if (!cache || !cache->k || !cache->v || !page_table || !row_start || !kv_len || !workspace) return HEART_ERR_INVALID;
  if (!aligned16(cache->k) || !aligned16(cache->v) || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return HEART_ERR_INVALID;
  if (((reinterpret_cast<uintptr_t>(page_table) | reinterpret_cast<uintptr_t>(row_start) | reinterpret_cast<uintptr_t>(kv_len)) & 3u) != 0)
    return HEART_ERR_INVALID;
  if (g->e4m3 && (!cache->k_scale || !cache->v_scale || !aligned16(cache->k_scale) || !aligned16(cache->v_scale))) return HEART_ERR_INVALID;
  *w = carve_cache(*g, workspace);
  ix->table = page_table;
  ix->row_start = row_start;
  ix->kv_len = kv_len;
  ix->status = w->status;
  ix->S = g->S;
  ix->T = g->T;
  ix->page_log2 = g->page == 16 ? 4 : g->page == 32 ? 5 : g->page == 64 ? 6 : 7;
  ix->n_pages = g->n_pages;
  ix->table_stride = g->table_stride;
  ix->causal = g->causal;
  ix->window = g->window;
  ix->sink = g->sink;
  return HEART_OK;
}

// Arrays of 32-bit words that a call needs.
bool words_ok(std::initializer_list<const void *> words) {
  for (const void *p : words)
    if (!p || (reinterpret_cast<uintptr_t>(p) & 3u)) return false;
  return true;
}

bool state_ok(const heart_state *st) {
  return st && st->anchor_q && st->anchor_k && st->has_anchor && st->mask_bits && st->kv_idx && st->kv_cnt;
}

// The steps between the block sums and the attention: drift, decision, masks of the refreshed heads.
cudaError_t decide_for_step(const Geom &g, const Workspace &w, const void *Q, const void *K, const double *delta, const double *tau,
                            heart_state st, double *drift_out, uint8_t *refresh_out, cudaStream_t s) {
  if (rows_kernel_fits(g)) return launch_decide_and_predict(g, w, decide_args(g, w, delta, st, drift_out, refresh_out), tau, st, s, &g_launches);
  cudaError_t e = launch_decide(g, w, delta, st, drift_out, refresh_out, s, &g_launches);
  if (e != cudaSuccess) return e;
  if (g.flags & HEART_ESTIMATOR_ANTIDIAG) {
    e = launch_antidiag_scores(g, w, Q, K, w.refresh, s, &g_launches);
    if (e != cudaSuccess) return e;
    return launch_top_p(g, w, tau, w.refresh, st, s, &g_launches, 0);
  }
  return launch_predict_mask(g, w, tau, w.refresh, st, s, &g_launches);
}

__global__ void fill_dense_outputs_kernel(int R, double *drift_out, uint8_t *refresh_out, uint8_t *refresh_ws) {
  const int r = blockIdx.x * blockDim.x + threadIdx.x;
  if (r < R) {
    if (drift_out) drift_out[r] = __longlong_as_double(0x7ff0000000000000LL);
    if (refresh_out) refresh_out[r] = 0;
    refresh_ws[r] = 0;
  }
}

}  // namespace

extern "C" {

size_t heart_workspace_bytes(const heart_config *cfg) {
  Geom g;
  if (make_geom(cfg, &g) != HEART_OK) return 0;
  return carve(g, nullptr).bytes;
}

size_t heart_drift_workspace_bytes(const heart_config *cfg) {
  Geom g;
  if (make_geom(cfg, &g) != HEART_OK) return 0;
  return carve(g, nullptr).bytes_no_scores;
}

int heart_state_reset(const heart_config *cfg, heart_state *st, heart_stream_t stream) {
  Geom g;
  int rc = make_geom(cfg, &g);
  if (rc != HEART_OK) return rc;
  if (!state_ok(st)) return HEART_ERR_INVALID;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaMemsetAsync(st->has_anchor, 0, (size_t)g.R, s);
  if (e != cudaSuccess) return cuda_fail(e, "heart_state_reset");
  e = cudaMemsetAsync(st->kv_cnt, 0, sizeof(int32_t) * (size_t)g.R * g.nb, s);
  if (e != cudaSuccess) return cuda_fail(e, "heart_state_reset");
  return HEART_OK;
}

int heart_drift(const heart_config *cfg, const void *Q, const void *K, const double *delta,
                heart_state *st, double *drift_out, uint8_t *refresh_out, void *workspace,
                heart_stream_t stream) {
  Geom g;
  int rc = make_geom(cfg, &g);
  if (rc != HEART_OK) return rc;
  if (!Q || !K || !delta || !workspace || !state_ok(st)) return HEART_ERR_INVALID;
  if (!aligned16(Q) || !aligned16(K) || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return HEART_ERR_INVALID;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  Workspace w = carve(g, workspace);
  g_launches = 0;
  cudaError_t e = launch_block_sums(g, Q, K, w, s, &g_launches);
  if (e != cudaSuccess) return cuda_fail(e, "block_sums");
  e = launch_decide(g, w, delta, *st, drift_out, refresh_out, s, &g_launches);
  if (e != cudaSuccess) return cuda_fail(e, "decide");
  return HEART_OK;
}

int heart_predict_mask(const heart_config *cfg, const void *Q, const void *K, const double *tau,
                       const uint8_t *refresh, heart_state *st, void *workspace, heart_stream_t stream) {
  Geom g;
  int rc = make_geom(cfg, &g);
  if (rc != HEART_OK) return rc;
  if (!Q || !K || !tau || !workspace || !state_ok(st)) return HEART_ERR_INVALID;
  if (!aligned16(Q) || !aligned16(K) || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return HEART_ERR_INVALID;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  Workspace w = carve(g, workspace);
  g_launches = 0;
  cudaError_t e;
  unsigned long long expect_sig = 0;
  if (g.flags & HEART_ESTIMATOR_ANTIDIAG) {
    // this estimator works on the tokens themselves: no block means needed
    e = launch_antidiag_scores(g, w, Q, K, refresh, s, &g_launches);
    if (e != cudaSuccess) return cuda_fail(e, "antidiag_scores");
    e = launch_top_p(g, w, tau, refresh, *st, s, &g_launches, 0);
    if (e != cudaSuccess) return cuda_fail(e, "top_p");
    return HEART_OK;
  }
  if (g.flags & HEART_BLOCK_MEANS_VALID) {
    // the caller vouches that a heart_drift (or heart_predict_mask) on these very tensors left the block
    // means in this workspace: no second pass over Q and K; the kernels verify the workspace's signature
    expect_sig = block_means_signature(g, Q, K);
  } else {
    e = launch_block_sums(g, Q, K, w, s, &g_launches);
    if (e != cudaSuccess) return cuda_fail(e, "block_sums");
  }
  e = launch_predict_mask(g, w, tau, refresh, *st, s, &g_launches, expect_sig);
  if (e != cudaSuccess) return cuda_fail(e, "predict_mask");
  return HEART_OK;
}

int heart_block_sparse_attn(const heart_config *cfg, const void *Q, const void *K, const void *V,
                            const int32_t *kv_idx, const int32_t *kv_cnt, void *O, float *lse,
                            void *workspace, heart_stream_t stream) {
  Geom g;
  int rc = make_geom(cfg, &g);
  if (rc != HEART_OK) return rc;
  const bool dense = (g.flags & HEART_FORCE_DENSE) != 0;
  if (!Q || !K || !V || !O || !workspace) return HEART_ERR_INVALID;
  if (!dense && (!kv_idx || !kv_cnt)) return HEART_ERR_INVALID;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) ||
      (reinterpret_cast<uintptr_t>(workspace) & 255u))
    return HEART_ERR_INVALID;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  Workspace w = carve(g, workspace);
  g_launches = 0;
  cudaError_t e = launch_attention(g, w, Q, K, V, kv_idx, kv_cnt, dense, O, lse, s, &g_launches);
  if (e != cudaSuccess) return cuda_fail(e, "attention");
  return HEART_OK;
}

int heart_step(const heart_config *cfg, const void *Q, const void *K, const void *V,
               const double *delta, const double *tau, heart_state *st, void *O, float *lse,
               double *drift_out, uint8_t *refresh_out, void *workspace, heart_stream_t stream) {
  Geom g;
  int rc = make_geom(cfg, &g);
  if (rc != HEART_OK) return rc;
  if (!Q || !K || !V || !O || !delta || !tau || !workspace || !state_ok(st)) return HEART_ERR_INVALID;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) ||
      (reinterpret_cast<uintptr_t>(workspace) & 255u))
    return HEART_ERR_INVALID;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  Workspace w = carve(g, workspace);
  g_launches = 0;
  cudaError_t e;
  if (g.flags & HEART_FORCE_DENSE) {
    fill_dense_outputs_kernel<<<(g.R + 127) / 128, 128, 0, s>>>(g.R, drift_out, refresh_out, w.refresh);
    ++g_launches;
    if ((e = cudaGetLastError()) != cudaSuccess) return cuda_fail(e, "fill_dense_outputs");
    e = launch_attention(g, w, Q, K, V, nullptr, nullptr, true, O, lse, s, &g_launches);
    if (e != cudaSuccess) return cuda_fail(e, "attention");
    return HEART_OK;
  }
  e = launch_block_sums(g, Q, K, w, s, &g_launches);
  if (e != cudaSuccess) return cuda_fail(e, "block_sums");
  e = decide_for_step(g, w, Q, K, delta, tau, *st, drift_out, refresh_out, s);
  if (e != cudaSuccess) return cuda_fail(e, "decide, predict_mask");
  e = launch_attention(g, w, Q, K, V, st->kv_idx, st->kv_cnt, false, O, lse, s, &g_launches);
  if (e != cudaSuccess) return cuda_fail(e, "attention");
  return HEART_OK;
}

namespace {

// Streams and events of heart_step_host, created on first use on each device and kept.
constexpr int kHostGroups = 16;  // head groups the V copy, the attention and the O copy are pipelined over
struct HostPipe {
  bool ready = false;
  cudaStream_t s_in = nullptr, s_out = nullptr;
  cudaEvent_t ev_qk = nullptr, ev_join = nullptr, ev_v[kHostGroups] = {}, ev_o[kHostGroups] = {};
};
constexpr int kMaxPipeDevices = 64;
std::mutex g_pipe_mu;
HostPipe g_pipe[kMaxPipeDevices];

cudaError_t pipe_for_current_device(HostPipe **out) {
  int dev = -1;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= kMaxPipeDevices) return cudaErrorInvalidDevice;
  HostPipe &p = g_pipe[dev];
  if (!p.ready) {
    if ((e = cudaStreamCreateWithFlags(&p.s_in, cudaStreamNonBlocking)) != cudaSuccess) return e;
    if ((e = cudaStreamCreateWithFlags(&p.s_out, cudaStreamNonBlocking)) != cudaSuccess) return e;
    if ((e = cudaEventCreateWithFlags(&p.ev_qk, cudaEventDisableTiming)) != cudaSuccess) return e;
    if ((e = cudaEventCreateWithFlags(&p.ev_join, cudaEventDisableTiming)) != cudaSuccess) return e;
    for (int i = 0; i < kHostGroups; ++i) {
      if ((e = cudaEventCreateWithFlags(&p.ev_v[i], cudaEventDisableTiming)) != cudaSuccess) return e;
      if ((e = cudaEventCreateWithFlags(&p.ev_o[i], cudaEventDisableTiming)) != cudaSuccess) return e;
    }
    p.ready = true;
  }
  *out = &p;
  return cudaSuccess;
}

}  // namespace

// Pipeline: Q and K go up on `stream`, then drift and mask prediction run there while V goes up on
// an internal stream, one group of heads at a time; the attention of a head group starts when its V
// has landed and its O goes down on a second internal stream while the next group computes.  `stream`
// finally waits for the last download, so everything is ordered before later work on `stream`.
int heart_step_host(const heart_config *cfg, const void *Q_host, const void *K_host, const void *V_host,
                    const double *delta, const double *tau, heart_state *st, void *O_host,
                    double *drift_host, uint8_t *refresh_host, void *Q_dev, void *K_dev, void *V_dev,
                    void *O_dev, void *workspace, heart_stream_t stream) {
  Geom g;
  int rc = make_geom(cfg, &g);
  if (rc != HEART_OK) return rc;
  if (cfg->stride_b != 0 || cfg->stride_h != 0 || cfg->stride_n != 0) return HEART_ERR_INVALID;
  if (!Q_host || !K_host || !V_host || !O_host || !Q_dev || !K_dev || !V_dev || !O_dev || !delta || !tau ||
      !workspace || !state_ok(st))
    return HEART_ERR_INVALID;
  if (!aligned16(Q_dev) || !aligned16(K_dev) || !aligned16(V_dev) || !aligned16(O_dev) ||
      (reinterpret_cast<uintptr_t>(workspace) & 255u))
    return HEART_ERR_INVALID;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  Workspace w = carve(g, workspace);
  std::lock_guard<std::mutex> lock(g_pipe_mu);  // the events are shared by the calls on a device
  HostPipe *pp = nullptr;
  cudaError_t e = pipe_for_current_device(&pp);
  if (e != cudaSuccess) return cuda_fail(e, "heart_step_host (streams)");
  const size_t head_bytes = sizeof(uint16_t) * (size_t)g.N * kD;
  const size_t bytes = head_bytes * g.R;
  g_launches = 0;
  e = cudaMemcpyAsync(Q_dev, Q_host, bytes, cudaMemcpyHostToDevice, s);
  if (e == cudaSuccess) e = cudaMemcpyAsync(K_dev, K_host, bytes, cudaMemcpyHostToDevice, s);
  if (e == cudaSuccess) e = cudaEventRecord(pp->ev_qk, s);
  if (e == cudaSuccess) e = cudaStreamWaitEvent(pp->s_in, pp->ev_qk, 0);  // V queues behind Q and K
  if (e != cudaSuccess) return cuda_fail(e, "heart_step_host (host to device)");
  const bool dense = (g.flags & HEART_FORCE_DENSE) != 0;
  if (dense) {
    fill_dense_outputs_kernel<<<(g.R + 127) / 128, 128, 0, s>>>(g.R, w.drift, nullptr, w.refresh);
    ++g_launches;
    if ((e = cudaGetLastError()) != cudaSuccess) return cuda_fail(e, "fill_dense_outputs");
  } else {
    e = launch_block_sums(g, Q_dev, K_dev, w, s, &g_launches);
    if (e != cudaSuccess) return cuda_fail(e, "block_sums");
    e = decide_for_step(g, w, Q_dev, K_dev, delta, tau, *st, w.drift, nullptr, s);
    if (e != cudaSuccess) return cuda_fail(e, "decide, predict_mask");
  }
  const int groups = g.H < kHostGroups ? g.H : kHostGroups;
  for (int gi = 0; gi < groups; ++gi) {
    const int h0 = (int)((long long)g.H * gi / groups), h1 = (int)((long long)g.H * (gi + 1) / groups);
    for (int b = 0; b < g.B && e == cudaSuccess; ++b) {  // one copy per batch entry: its heads h0..h1 are contiguous
      const size_t off = ((size_t)b * g.H + h0) * head_bytes;
      e = cudaMemcpyAsync(static_cast<char *>(V_dev) + off, static_cast<const char *>(V_host) + off,
                          head_bytes * (h1 - h0), cudaMemcpyHostToDevice, pp->s_in);
    }
    if (e == cudaSuccess) e = cudaEventRecord(pp->ev_v[gi], pp->s_in);
    if (e == cudaSuccess) e = cudaStreamWaitEvent(s, pp->ev_v[gi], 0);
    if (e != cudaSuccess) return cuda_fail(e, "heart_step_host (host to device)");
    e = launch_attention(g, w, Q_dev, K_dev, V_dev, dense ? nullptr : st->kv_idx, dense ? nullptr : st->kv_cnt, dense,
                         O_dev, nullptr, s, &g_launches, h0, h1 - h0);
    if (e != cudaSuccess) return cuda_fail(e, "attention");
    e = cudaEventRecord(pp->ev_o[gi], s);
    if (e == cudaSuccess) e = cudaStreamWaitEvent(pp->s_out, pp->ev_o[gi], 0);
    for (int b = 0; b < g.B && e == cudaSuccess; ++b) {
      const size_t off = ((size_t)b * g.H + h0) * head_bytes;
      e = cudaMemcpyAsync(static_cast<char *>(O_host) + off, static_cast<const char *>(O_dev) + off,
                          head_bytes * (h1 - h0), cudaMemcpyDeviceToHost, pp->s_out);
    }
    if (e != cudaSuccess) return cuda_fail(e, "heart_step_host (device to host)");
  }
  // drift and refresh were final before the first attention launch: ev_o[0] on s_out covers them
  if (drift_host)
    e = cudaMemcpyAsync(drift_host, w.drift, sizeof(double) * (size_t)g.R, cudaMemcpyDeviceToHost, pp->s_out);
  if (e == cudaSuccess && refresh_host)
    e = cudaMemcpyAsync(refresh_host, w.refresh, (size_t)g.R, cudaMemcpyDeviceToHost, pp->s_out);
  if (e == cudaSuccess) e = cudaEventRecord(pp->ev_join, pp->s_out);
  if (e == cudaSuccess) e = cudaStreamWaitEvent(s, pp->ev_join, 0);
  if (e != cudaSuccess) return cuda_fail(e, "heart_step_host (device to host)");
  return HEART_OK;
}

int heart_full_token_drift(const heart_config *cfg, const void *Qa, const void *Ka, const void *Qb,
                           const void *Kb, double *drift_out, void *workspace, heart_stream_t stream) {
  Geom g;
  int rc = make_geom(cfg, &g);
  if (rc != HEART_OK) return rc;
  if (!Qa || !Ka || !Qb || !Kb || !drift_out || !workspace) return HEART_ERR_INVALID;
  if (!aligned16(Qa) || !aligned16(Ka) || !aligned16(Qb) || !aligned16(Kb) ||
      (reinterpret_cast<uintptr_t>(workspace) & 255u))
    return HEART_ERR_INVALID;
  Workspace w = carve(g, workspace);
  int rows = 0;
  const size_t need = (size_t)g.R * token_drift_chunks(g, &rows);  // partials live in the block-sum area
  if (need > 2 * (size_t)g.R * g.nb * kD) return HEART_ERR_INVALID;
  g_launches = 0;
  cudaError_t e = launch_token_drift(g, Qa, Ka, Qb, Kb, w, drift_out, static_cast<cudaStream_t>(stream), &g_launches);
  if (e != cudaSuccess) return cuda_fail(e, "token_drift");
  return HEART_OK;
}

int heart_mask_iou(const heart_config *cfg, const uint32_t *mask_a, const uint32_t *mask_b,
                   double *iou_out, int64_t *counts_out, heart_stream_t stream) {
  Geom g;
  int rc = make_geom(cfg, &g);
  if (rc != HEART_OK) return rc;
  if (!mask_a || !mask_b || !iou_out) return HEART_ERR_INVALID;
  g_launches = 0;
  cudaError_t e = launch_mask_iou(g, mask_a, mask_b, iou_out, reinterpret_cast<long long *>(counts_out),
                                  static_cast<cudaStream_t>(stream), &g_launches);
  if (e != cudaSuccess) return cuda_fail(e, "mask_iou");
  return HEART_OK;
}

size_t heart_cache_workspace_bytes(const heart_cache_config *cfg) {
  CacheGeom g;
  if (make_cache_geom(cfg, &g) != HEART_OK) return 0;
  return carve_cache(g, nullptr).bytes;
}

int heart_cache_write(const heart_cache_config *cfg, const void *K, const void *V, const heart_cache *cache,
                      const int32_t *page_table, const int32_t *row_start, const int32_t *kv_len, void *workspace,
                      heart_stream_t stream) {
  CacheGeom g;
  CacheWorkspace w;
  CacheIndex ix;
  const int rc = cache_call(cfg, cache, page_table, row_start, kv_len, workspace, &g, &w, &ix);
  if (rc != HEART_OK) return rc;
  if (!K || !V || !aligned16(K) || !aligned16(V)) return HEART_ERR_INVALID;
  g_launches = 0;
  cudaError_t e = launch_cache_write(g, ix, K, V, *cache, static_cast<cudaStream_t>(stream), &g_launches);
  if (e != cudaSuccess) return cuda_fail(e, "cache_write");
  return HEART_OK;
}

int heart_cache_read(const heart_cache_config *cfg, const heart_cache *cache, const int32_t *page_table,
                     const int32_t *row_start, const int32_t *kv_len, void *K_out, void *V_out, void *workspace,
                     heart_stream_t stream) {
  CacheGeom g;
  CacheWorkspace w;
  CacheIndex ix;
  const int rc = cache_call(cfg, cache, page_table, row_start, kv_len, workspace, &g, &w, &ix);
  if (rc != HEART_OK) return rc;
  if (!K_out || !V_out || !aligned16(K_out) || !aligned16(V_out)) return HEART_ERR_INVALID;
  g_launches = 0;
  cudaError_t e = launch_cache_read(g, ix, *cache, K_out, V_out, static_cast<cudaStream_t>(stream), &g_launches);
  if (e != cudaSuccess) return cuda_fail(e, "cache_read");
  return HEART_OK;
}

size_t heart_cross_workspace_bytes(const heart_cross_config *cfg) {
  CrossGeom g;
  if (make_cross_geom(cfg, &g) != HEART_OK) return 0;
  return carve_cross(nullptr).bytes;
}

int heart_cross_attn(const heart_cross_config *cfg, const void *Q, const void *K, const void *V, const int32_t *q_start, const int32_t *k_start,
                     const int32_t *k_len, void *O, float *lse, void *workspace, heart_stream_t stream) {
  CrossGeom g;
  const int rc = make_cross_geom(cfg, &g);
  if (rc != HEART_OK) return rc;
  if (!Q || !K || !V || !O || !aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O)) return HEART_ERR_INVALID;
  if (!words_ok({q_start, k_start, k_len}) || (reinterpret_cast<uintptr_t>(lse) & 3u)) return HEART_ERR_INVALID;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return HEART_ERR_INVALID;
  const CrossWorkspace w = carve_cross(workspace);
  CacheIndex ix = {};
  ix.table = k_start;
  ix.row_start = q_start;
  ix.kv_len = k_len;
  ix.status = w.status;
  ix.S = g.S;
  ix.T = g.T;
  ix.table_stride = g.Tk;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  g_launches = 0;
  const CrossKernel kernel = cross_kernel(g);
  const bool rows = kernel == CrossKernel::kRows8 || kernel == CrossKernel::kRows16;
  cudaError_t e = rows ? launch_cross_rows(g, ix, w, Q, K, V, O, lse, kernel == CrossKernel::kRows8, s, &g_launches)
                       : launch_cross_tiles(g, ix, w, Q, K, V, O, lse, kernel == CrossKernel::kPairs, s, &g_launches);
  if (e != cudaSuccess) return cuda_fail(e, "cross_attention");
  return HEART_OK;
}

int heart_cache_extend(const heart_cache_config *cfg, const int32_t *new_len, const int32_t *kv_len, const int32_t *free_pages,
                       const int32_t *free_count, int32_t *page_table, int32_t *row_start, int32_t *kv_len_out, int32_t *free_count_out,
                       int64_t *slots, void *workspace, heart_stream_t stream) {
  CacheGeom g;
  const int rc = make_cache_geom(cfg, &g);
  if (rc != HEART_OK) return rc;
  if (!words_ok({new_len, kv_len, free_pages, free_count, page_table, row_start, kv_len_out, free_count_out})) return HEART_ERR_INVALID;
  if ((reinterpret_cast<uintptr_t>(slots) & 7u) || !workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return HEART_ERR_INVALID;
  g_launches = 0;
  cudaError_t e = launch_cache_extend(g, carve_cache(g, workspace), new_len, kv_len, free_pages, free_count, page_table, row_start, kv_len_out,
                                      free_count_out, slots, static_cast<cudaStream_t>(stream), &g_launches);
  if (e != cudaSuccess) return cuda_fail(e, "cache_extend");
  return HEART_OK;
}

int heart_cache_release(const heart_cache_config *cfg, const uint8_t *ended, const int32_t *kv_len, int32_t *free_pages, const int32_t *free_count,
                        const int32_t *page_table, int32_t *kv_len_out, int32_t *free_count_out, void *workspace, heart_stream_t stream) {
  CacheGeom g;
  const int rc = make_cache_geom(cfg, &g);
  if (rc != HEART_OK) return rc;
  if (!ended || !words_ok({kv_len, free_pages, free_count, page_table, kv_len_out, free_count_out})) return HEART_ERR_INVALID;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return HEART_ERR_INVALID;
  g_launches = 0;
  cudaError_t e = launch_cache_release(g, carve_cache(g, workspace), ended, kv_len, free_pages, free_count, page_table, kv_len_out, free_count_out,
                                       static_cast<cudaStream_t>(stream), &g_launches);
  if (e != cudaSuccess) return cuda_fail(e, "cache_release");
  return HEART_OK;
}

int heart_cache_attn(const heart_cache_config *cfg, const void *Q, const heart_cache *cache, const int32_t *page_table,
                     const int32_t *row_start, const int32_t *kv_len, void *O, float *lse, void *workspace,
                     heart_stream_t stream) {
  CacheGeom g;
  CacheWorkspace w;
  CacheIndex ix;
  const int rc = cache_call(cfg, cache, page_table, row_start, kv_len, workspace, &g, &w, &ix);
  if (rc != HEART_OK) return rc;
  if (!Q || !O || !aligned16(Q) || !aligned16(O) || (reinterpret_cast<uintptr_t>(lse) & 3u)) return HEART_ERR_INVALID;
  g_launches = 0;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = (long long)g.max_new * g.G <= kRowsOfRowsKernel ? launch_cache_rows(g, ix, w, Q, *cache, O, lse, s, &g_launches)
                                                                  : launch_cache_tiles(g, ix, w, Q, *cache, O, lse, s, &g_launches);
  if (e != cudaSuccess) return cuda_fail(e, "cache_attention");
  return HEART_OK;
}

size_t heart_band_error_workspace_bytes(int32_t C, int32_t T, int32_t H, int32_t W) {
  if (C < 1 || T < 1 || H < 1 || W < 1 || (long long)C * T * H * W > (1LL << 31)) return 0;
  return band_error_workspace_bytes(C, T, H, W);
}

int heart_band_error(const float *y_sparse, const float *y_dense, int32_t C, int32_t T, int32_t H, int32_t W,
                     const double *weights, double eps, double *out, void *workspace, heart_stream_t stream) {
  if (heart_band_error_workspace_bytes(C, T, H, W) == 0) return HEART_ERR_INVALID;
  if (!y_sparse || !y_dense || !weights || !out || !workspace || !(eps >= 0.0)) return HEART_ERR_INVALID;
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return HEART_ERR_INVALID;
  g_launches = 0;
  cudaError_t e = launch_band_error(y_sparse, y_dense, C, T, H, W, weights, eps, out, workspace,
                                    static_cast<cudaStream_t>(stream), &g_launches);
  if (e != cudaSuccess) return cuda_fail(e, "band_error");
  return HEART_OK;
}

int heart_get_status(void *workspace, heart_stream_t stream, int32_t *code_out) {
  if (!workspace || !code_out) return HEART_ERR_INVALID;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int32_t words[2] = {0, 0};
  cudaError_t e = cudaMemcpyAsync(words, workspace, sizeof words, cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e != cudaSuccess) return cuda_fail(e, "heart_get_status");
  *code_out = words[0];
  if (words[0] != 0) {
    e = cudaMemsetAsync(workspace, 0, sizeof words, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    if (e != cudaSuccess) return cuda_fail(e, "heart_get_status");
  }
  return HEART_OK;
}

const char *heart_strerror(int code) {
  switch (code) {
    case HEART_OK: return "ok";
    case HEART_ERR_INVALID: return "invalid argument (null pointer, size, stride or alignment)";
    case HEART_ERR_UNSUPPORTED:
      return "unsupported shape (head_dim must be 128, block 64 or 128, at most 1024 blocks; caches: page 16, 32, 64 or 128; caches and cross "
             "attention: at most 128 query heads a key head, fewer than 2^31 rows and tokens)";
    case HEART_ERR_CUDA: return g_errbuf[0] ? g_errbuf : "CUDA error";
    case HEART_ERR_TOO_LARGE: return "shape needs more scratch than the built-in HEART_STATIC_SCRATCH_BYTES array holds";
    case HEART_ERR_INFEASIBLE: return "no assignment of one candidate per head meets the sparsity budget";
    case HEART_ERR_DEVICE_CHECK: return "device-side check failed (index-list entry out of range or a bounded wait ran out)";
    default: return "unknown code";
  }
}

int heart_last_launch_count(void) { return g_launches; }

#ifdef HEART_TEST_HOOKS
// Test-hook builds only: the kernel that a call takes (a CrossKernel), or -1.
int heart_test_cross_kernel(const heart_cross_config *cfg) {
  CrossGeom g;
  return make_cross_geom(cfg, &g) == HEART_OK ? static_cast<int>(cross_kernel(g)) : -1;
}
#endif

}  // extern "C"
