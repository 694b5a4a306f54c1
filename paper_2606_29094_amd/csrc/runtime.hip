// Host runtime behind include/dlm.h: argument validation, the per-step row
// plan, KV-slot bookkeeping, workspace layout and the kernel sequence of one
// denoising step. Device memory is always the caller's.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdint>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <mutex>
#include <new>
#include <string>
#include <utility>
#include <vector>

#include "../../include/dlm.h"
#include "common.h"
#include "kernels.h"
#include "mx_common.h"
#include "mx_kernels.h"

using namespace dlm;

namespace dlm {
thread_local LaunchTiming g_launch_timing;
}

namespace {

thread_local std::string g_err;

dlm_status fail(dlm_status s, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  g_err = buf;
  return s;
}

#define HIPCHECK(expr)                                                               \
  do {                                                                               \
    hipError_t e_ = (expr);                                                          \
    if (e_ != hipSuccess)                                                            \
      return fail(DLM_EHIP, "%s failed: %s", #expr, hipGetErrorString(e_));          \
  } while (0)

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

}  // namespace

// Scratch of dlm_denoise_step_noalloc: one copy per device, in the library's
// code object. Host code never uses this name as an address: the device
// address of each GPU's copy comes from hipGetSymbolAddress (scratch_address).
static __device__ __align__(256) char scratch[DLM_SCRATCH_BYTES];

namespace {

constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
void* g_scratch_ptr[kMaxDevices] = {};

// Device address of the current device's scratch, looked up once per device.
dlm_status scratch_address(void** out) {
  int dev = 0;
  HIPCHECK(hipGetDevice(&dev));
  if (dev < 0 || dev >= kMaxDevices)
    return fail(DLM_EUNSUPPORTED, "device %d outside [0, %d)", dev, kMaxDevices);
  std::lock_guard<std::mutex> lock(g_scratch_mu);
  if (!g_scratch_ptr[dev]) {
    void* p = nullptr;
    HIPCHECK(hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)));
    if (!p || reinterpret_cast<uintptr_t>(p) % 256 != 0)
      return fail(DLM_EHIP, "scratch of device %d is not 256-byte aligned", dev);
    g_scratch_ptr[dev] = p;
  }
  *out = g_scratch_ptr[dev];
  return DLM_OK;
}

}  // namespace

// Enqueue one kernel class (`expr`, a launch returning hipError_t); when the
// model's profiler times this launch, its kernel
// carries a pair of events in its own dispatch (DLM_LAUNCH), so the measured
// time is the kernel's and the stream gets no extra commands. (A class that
// enqueues no kernel this time returns the events unused.)
#define LAUNCH(model, stream, name, expr)                                           \
  do {                                                                            \
    Profiler& pf_ = (model)->prof;                                                \
    hipEvent_t a_ = nullptr, b_ = nullptr;                                        \
    if (pf_.wants(name)) {                                                        \
      a_ = pf_.take();                                                            \
      b_ = pf_.take();                                                            \
      if (a_ && b_) g_launch_timing = LaunchTiming{a_, b_};                       \
    }                                                                             \
    const hipError_t le_ = (expr);                                                \
    const bool used_ = a_ && b_ && !g_launch_timing.start && !g_launch_timing.stop; \
    g_launch_timing = LaunchTiming{};                                             \
    if (used_) {                                                                  \
      pf_.pending.push_back({pf_.kind_of(name), a_, b_});                         \
    } else {                                                                      \
      if (a_) pf_.pool.push_back(a_);                                             \
      if (b_) pf_.pool.push_back(b_);                                             \
    }                                                                             \
    if (le_ != hipSuccess)                                                        \
      return fail(DLM_EHIP, "%s failed: %s", #expr, hipGetErrorString(le_));      \
  } while (0)

// Per-kernel-class event timing (dlm_profile_*).
struct Profiler {
  bool on = false;
  std::string only;        // empty: every class
  int every = 1;           // time one launch in `every` of each class
  std::vector<long> seen;  // launches of each class since enable / sample (sampling phase)
  std::vector<int> since_read;   // launches of each class since the last read
  bool wants(const char* n) {
    if (!on || !(only.empty() || only == n)) return false;
    const int k = kind_of(n);
    if ((int)seen.size() <= k) seen.resize(k + 1, 0);
    if ((int)since_read.size() <= k) since_read.resize(k + 1, 0);
    since_read[k] += 1;
    return seen[k]++ % every == 0;
  }
  struct Rec { int kind; hipEvent_t a, b; };
  std::vector<Rec> pending;
  std::vector<hipEvent_t> pool;
  std::vector<std::string> names;
  int kind_of(const char* n) {
    for (size_t i = 0; i < names.size(); ++i)
      if (names[i] == n) return (int)i;
    names.emplace_back(n);
    return (int)names.size() - 1;
  }
  hipEvent_t take() {
    if (pool.empty()) {
      hipEvent_t e;
      if (hipEventCreate(&e) != hipSuccess) return nullptr;
      return e;
    }
    hipEvent_t e = pool.back();
    pool.pop_back();
    return e;
  }
  ~Profiler() {
    for (auto& r : pending) { (void)hipEventDestroy(r.a); (void)hipEventDestroy(r.b); }
    for (auto e : pool) (void)hipEventDestroy(e);
  }
};

struct dlm_model {
  Profiler prof;
  dlm_config cfg;
  const void* embed;
  const void* lm_head;
  const float* final_norm;
  std::vector<dlm_layer_weights> layers;
  std::vector<dlm_layer_mx> mx;   // packed projections (dlm_load_weights_mx), or empty
  int num_cu;
  size_t es;   // element size
};

struct SlotState {
  bool valid = false;
  int block_start = -1;
  int seq_len = -1;
};

struct dlm_cache {
  const dlm_model* model;
  int n_slots;
  int s_max;          // positions per slot (multiple of 64)
  char* base;
  size_t region;      // bytes of one layer's K (or V) region
  std::vector<SlotState> slots;
  bool mx = false;            // 4-bit slots: region is then the bytes of one layer's codes
  size_t scale_region = 0;    // and this the bytes of one layer's scales (keys or values)
  void* k_layer(int l) const { return base + (size_t)(2 * l) * region; }
  void* v_layer(int l) const { return base + (size_t)(2 * l + 1) * region; }
  MxKv mx_layer(int l) const {
    uint8_t* b = reinterpret_cast<uint8_t*>(base) + (size_t)(2 * l) * (region + scale_region);
    return {b, b + region, b + 2 * region, b + 2 * region + scale_region, s_max};
  }
};

namespace {

// Workspace layout of a step with n recomputed rows and n_req requests.
struct Layout {
  size_t h, a, qkv, cs, q, ao, part, act, lm_rows, lm_count, req_off, req_cnt, u, pm, ps, pi,
      conf, tok, mx, total;
  GemmPlan g_qkv, g_o, g_gu, g_down, g_lm, g_logits;
  MxPlan q_qkv, q_o, q_gu, q_down;   // of a model with packed projections
  int s_qkv, s_o, s_down, tiles, m_max;
};

MxView mx_view(const dlm_mx& w) {
  const int groups = ceil_div(w.k, kMxGroup);
  return {reinterpret_cast<uint8_t*>(w.codes), w.scales, w.n, groups, ceil_div(groups, 16) * 16};
}

GemmPlan projection_plan(int es, int rows, int N, int K, int num_cu) {
  return gemm_plan(es, rows, N, K, true, num_cu);
}
// the SwiGLU GEMM keeps 16x16 tiles: its 32x32 variants measured 5-6 % slower on
// every gate/up shape
GemmPlan gate_up_plan(int es, int rows, int F, int K, int num_cu) {
  return gemm_plan(es, rows, 2 * F, K, false, num_cu, false, true, false);
}

Layout layout(const dlm_model* m, int n, int n_req) {
  const dlm_config& c = m->cfg;
  Layout L{};
  const int qkv_dim = (c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim;
  const int qd = c.n_q_heads * c.head_dim;
  const int es_i = (int)m->es;
  if (m->mx.empty()) {
    L.g_qkv = projection_plan(es_i, n, qkv_dim, c.d_model, m->num_cu);
    L.g_o = projection_plan(es_i, n, c.d_model, qd, m->num_cu);
    L.g_gu = gate_up_plan(es_i, n, c.d_ffn, c.d_model, m->num_cu);
    L.g_down = projection_plan(es_i, n, c.d_model, c.d_ffn, m->num_cu);
    L.s_qkv = L.g_qkv.splits;
    L.s_o = L.g_o.splits;
    L.s_down = L.g_down.splits;
  } else {
    // (the rotation and the residual norms add K slices as they read them)
    L.q_qkv = mx_plan(es_i, n, qkv_dim, c.d_model, c.d_model, false, true, true, false, m->num_cu);
    L.q_o = mx_plan(es_i, n, c.d_model, qd, qd, false, true, true, false, m->num_cu);
    L.q_gu = mx_plan(es_i, n, 2 * c.d_ffn, c.d_model, c.d_model, true, true, true, true, m->num_cu);
    L.q_down = mx_plan(es_i, n, c.d_model, c.d_ffn, c.d_ffn, false, true, true, false, m->num_cu);
    auto slices = [](const MxPlan& p) { return p.gemm ? p.g.splits : p.tile.slices; };
    L.s_qkv = slices(L.q_qkv), L.s_o = slices(L.q_o), L.s_down = slices(L.q_down);
  }
  L.m_max = std::min(n, n_req * kMaxBlock);
  L.g_lm = lm_head_plan(es_i, L.m_max, c.vocab, c.d_model, m->num_cu);
  L.g_logits = L.g_lm;
  L.tiles = lm_head_tiles(L.g_lm, c.vocab);
  const size_t es = m->es;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    size_t o = off;
    off = align_up(off + bytes, 256);
    return o;
  };
  L.h = take((size_t)n * c.d_model * 4);
  L.a = take((size_t)n * c.d_model * es);
  L.qkv = take((size_t)L.s_qkv * n * qkv_dim * 4);
  L.cs = take((size_t)n * (c.head_dim / 2) * 8);
  L.q = take((size_t)n * qd * es);
  L.ao = take((size_t)n * qd * es);
  L.part = take((size_t)std::max(L.s_o, L.s_down) * n * c.d_model * 4);
  L.act = take((size_t)n * c.d_ffn * es);
  L.lm_rows = take((size_t)std::max(L.m_max, 1) * 4);
  L.lm_count = take(4);
  L.req_off = take((size_t)kMaxReq * 4);
  L.req_cnt = take((size_t)kMaxReq * 4);
  L.u = take((size_t)std::max(L.m_max, 1) * c.d_model * es);
  L.pm = take((size_t)L.tiles * std::max(L.m_max, 1) * 4);
  L.ps = take((size_t)L.tiles * std::max(L.m_max, 1) * 4);
  L.pi = take((size_t)L.tiles * std::max(L.m_max, 1) * 4);
  L.conf = take((size_t)std::max(L.m_max, 1) * 4);
  L.tok = take((size_t)std::max(L.m_max, 1) * 4);
  L.mx = take(std::max({L.q_qkv.scratch, L.q_o.scratch, L.q_gu.scratch, L.q_down.scratch}));
  L.total = off;
  return L;
}

dlm_status check_config(const dlm_config* c) {
  if (!c) return fail(DLM_EINVAL, "config is NULL");
  if (c->dtype != DLM_F32 && c->dtype != DLM_BF16)
    return fail(DLM_EINVAL, "dtype %d is not DLM_F32 or DLM_BF16", c->dtype);
  if (c->n_layers < 1 || c->d_model < 1 || c->n_q_heads < 1 || c->n_kv_heads < 1 ||
      c->head_dim < 1 || c->d_ffn < 1 || c->vocab < 2)
    return fail(DLM_EINVAL, "non-positive model dimension");
  if (c->head_dim != 64 && c->head_dim != 128)
    return fail(DLM_EUNSUPPORTED, "head_dim %d (supported: 64, 128)", c->head_dim);
  if (c->n_q_heads % c->n_kv_heads != 0)
    return fail(DLM_EINVAL, "n_q_heads %d is not a multiple of n_kv_heads %d", c->n_q_heads,
                c->n_kv_heads);
  if (c->d_model % 64 != 0)
    return fail(DLM_EUNSUPPORTED, "d_model %d is not a multiple of 64", c->d_model);
  if (c->d_ffn % 16 != 0)
    return fail(DLM_EUNSUPPORTED, "d_ffn %d is not a multiple of 16", c->d_ffn);
  if (c->mask_id < 0 || c->mask_id >= c->vocab)
    return fail(DLM_EINVAL, "mask_id %d outside [0, vocab)", c->mask_id);
  if (!(c->rms_eps >= 0.f) || !(c->rope_theta > 0.f) || !std::isfinite(c->inv_tau) ||
      !(c->inv_tau > 0.f))
    return fail(DLM_EINVAL, "rms_eps, rope_theta or inv_tau out of range");
  return DLM_OK;
}

// Row plan of one step; returns the error status (nothing enqueued yet).
dlm_status make_plan(const dlm_model* m, const dlm_cache* c, const dlm_batch* b,
                     const float* thr, bool force_refresh, StepPlan* p) {
  if (!b) return fail(DLM_EINVAL, "batch is NULL");
  if (b->n_req < 1 || b->n_req > kMaxReq)
    return fail(DLM_EINVAL, "n_req %d outside [1, %d]", b->n_req, kMaxReq);
  if (!b->reqs || !b->tokens || !b->mask) return fail(DLM_EINVAL, "batch pointer is NULL");
  if (b->mode < DLM_CACHE_NONE || b->mode > DLM_CACHE_DUAL)
    return fail(DLM_EINVAL, "cache mode %d", b->mode);
  std::vector<char> used(c->n_slots, 0);
  int row = 0, tile = 0, blk = 0;
  p->n_req = b->n_req;
  for (int r = 0; r < b->n_req; ++r) {
    const dlm_req& q = b->reqs[r];
    if (q.slot < 0 || q.slot >= c->n_slots)
      return fail(DLM_EINVAL, "request %d: slot %d outside [0, %d)", r, q.slot, c->n_slots);
    if (used[q.slot]) return fail(DLM_EINVAL, "request %d: slot %d used twice", r, q.slot);
    used[q.slot] = 1;
    if (q.seq_len < 1 || q.seq_len > c->s_max)
      return fail(DLM_ESIZE, "request %d: seq_len %d outside [1, %d]", r, q.seq_len, c->s_max);
    if (q.prompt_len < 0 || q.prompt_len > q.block_start)
      return fail(DLM_EINVAL, "request %d: prompt_len %d vs block_start %d", r, q.prompt_len,
                  q.block_start);
    if (q.block_len < 1 || q.block_len > kMaxBlock || q.block_start + q.block_len > q.seq_len)
      return fail(DLM_EINVAL, "request %d: block [%d, %d) invalid for seq_len %d", r,
                  q.block_start, q.block_start + q.block_len, q.seq_len);
    if (q.tok_offset < 0) return fail(DLM_EINVAL, "request %d: negative tok_offset", r);
    if (q.flags & ~DLM_REQ_REFRESH) return fail(DLM_EINVAL, "request %d: unknown flags", r);
    float g = 0.f;
    if (thr) {
      g = thr[r];
      if (!(g >= 0.f && g <= 1.f))
        return fail(DLM_EINVAL, "request %d: threshold outside [0, 1]", r);
    }
    const bool refresh = force_refresh || b->mode == DLM_CACHE_NONE || (q.flags & DLM_REQ_REFRESH);
    int r0, r1;
    if (refresh) {
      r0 = 0; r1 = q.seq_len;
    } else {
      const SlotState& s = c->slots[q.slot];
      if (!s.valid || s.block_start != q.block_start || s.seq_len != q.seq_len)
        return fail(DLM_ESTATE,
                    "request %d: cache step on slot %d whose cache is not current (refreshed at "
                    "block %d, seq_len %d; step at block %d, seq_len %d)",
                    r, q.slot, s.valid ? s.block_start : -1, s.valid ? s.seq_len : -1,
                    q.block_start, q.seq_len);
      r0 = q.block_start;
      r1 = b->mode == DLM_CACHE_DUAL ? q.block_start + q.block_len : q.seq_len;
    }
    ReqPlan& rp = p->r[r];
    rp.row0 = row;
    rp.nrows = r1 - r0;
    rp.pos0 = r0;
    rp.seq_len = q.seq_len;
    rp.prompt_len = q.prompt_len;
    rp.slot = q.slot;
    rp.tok_off = q.tok_offset;
    rp.blk_s = q.block_start;
    rp.blk_len = q.block_len;
    rp.tile0 = tile;
    rp.blk0 = blk;
    rp.gamma = g;
    row += rp.nrows;
    tile += ceil_div(rp.nrows, kQTile);
    blk += q.block_len;
  }
  // the requests' packed token ranges must be disjoint (each step updates its
  // request's tokens and mask in place)
  std::vector<std::pair<long, long>> ranges(b->n_req);
  for (int r = 0; r < b->n_req; ++r)
    ranges[r] = {(long)b->reqs[r].tok_offset, (long)b->reqs[r].tok_offset + b->reqs[r].seq_len};
  std::sort(ranges.begin(), ranges.end());
  for (int r = 1; r < b->n_req; ++r)
    if (ranges[r].first < ranges[r - 1].second)
      return fail(DLM_EINVAL, "token ranges [%ld, %ld) and [%ld, %ld) overlap", ranges[r - 1].first,
                  ranges[r - 1].second, ranges[r].first, ranges[r].second);
  if (ranges.back().second > INT32_MAX)
    return fail(DLM_EINVAL, "token range end %ld exceeds the int32 index range", ranges.back().second);
  p->n_rows = row;
  p->n_tiles = tile;
  p->n_blk = blk;
  (void)m;
  return DLM_OK;
}

dlm_status check_ws(const dlm_model* m, const StepPlan& p, void* ws, size_t ws_bytes,
                    Layout* L) {
  *L = layout(m, p.n_rows, p.n_req);
  if (!ws) return fail(DLM_EINVAL, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(ws) % 256 != 0)
    return fail(DLM_EINVAL, "workspace is not 256-byte aligned");
  if (ws_bytes < L->total)
    return fail(DLM_ESIZE, "workspace of %zu bytes; this step needs %zu (%d rows)", ws_bytes,
                L->total, p.n_rows);
  return DLM_OK;
}

enum class Tail { Unmask, Logits, None };

// Device-to-device copy of a recorded intermediate (dlm_debug_trace); a NULL
// destination records nothing.
#define TRACE_COPY(dst, src, bytes)                                                    \
  do {                                                                                 \
    if (dst) HIPCHECK(hipMemcpyAsync((dst), (src), (bytes), hipMemcpyDeviceToDevice, st)); \
  } while (0)

template <typename T>
dlm_status run_forward(dlm_model* m, dlm_cache* c, const dlm_batch* b, const StepPlan& p,
                       const Layout& L, char* ws, const dlm_trace* tr, hipStream_t st) {
  const dlm_config& cf = m->cfg;
  const int d = cf.d_model, hq = cf.n_q_heads, hkv = cf.n_kv_heads, dh = cf.head_dim;
  const int qkv_dim = (hq + 2 * hkv) * dh, qd = hq * dh, n = p.n_rows;
  float* h = reinterpret_cast<float*>(ws + L.h);
  T* a = reinterpret_cast<T*>(ws + L.a);
  float* qkv = reinterpret_cast<float*>(ws + L.qkv);
  float2* cs = reinterpret_cast<float2*>(ws + L.cs);
  T* q = reinterpret_cast<T*>(ws + L.q);
  T* ao = reinterpret_cast<T*>(ws + L.ao);
  float* part = reinterpret_cast<float*>(ws + L.part);
  T* act = reinterpret_cast<T*>(ws + L.act);
  // part and act (consecutive) hold nothing while attention runs: its key splits' partials go there
  const AttnPlan ap = attention_plan(p, hq, hkv, dh, sizeof(T), L.lm_rows - L.part, m->num_cu);
  const MxAttnPlan mx_ap =
      c->mx ? mx_attention_plan(p, hq, hkv, dh, sizeof(T), L.lm_rows - L.part, m->num_cu) : MxAttnPlan{};
  const bool w4 = !m->mx.empty();
  void* const mxs = ws + L.mx;

  LAUNCH(m, st, "embed_norm", embed_norm_rows<T>(p, reinterpret_cast<const T*>(m->embed), d, cf.vocab,
                         cf.mask_id, b->tokens, b->mask, m->layers[0].attn_norm, cf.rms_eps, dh,
                         cf.rope_theta, h, a, cs, st));
  const size_t es = sizeof(T);
  for (int l = 0; l < cf.n_layers; ++l) {
    const dlm_layer_weights& w = m->layers[l];
    const dlm_layer_mx* w4l = w4 ? &m->mx[l] : nullptr;
    const MxKv kv4 = c->mx ? c->mx_layer(l) : MxKv{};
    T* kc = c->mx ? nullptr : reinterpret_cast<T*>(c->k_layer(l));
    T* vc = c->mx ? nullptr : reinterpret_cast<T*>(c->v_layer(l));
    const dlm_trace* t = tr && tr->layer == l ? tr : nullptr;
    if (t) {
      TRACE_COPY(t->h_in, h, (size_t)n * d * 4);
      TRACE_COPY(t->a_attn, a, (size_t)n * d * es);
    }
    if (w4)
      LAUNCH(m, st, "gemm_qkv", mx_matmul<T>(L.q_qkv, a, d, n, mx_view(w4l->w_qkv), d, DLM_MX_STORE, qkv,
                                             qkv_dim, mxs, st));
    else
      LAUNCH(m, st, "gemm_qkv", gemm_store_f32<T>(L.g_qkv, a, d, reinterpret_cast<const T*>(w.w_qkv), d, n,
                                                      qkv_dim, d, qkv, qkv_dim, st));
    if (t) TRACE_COPY(t->qkv, qkv, (size_t)L.s_qkv * n * qkv_dim * 4);
    if (c->mx)
      LAUNCH(m, st, "rope_kv_write", mx_kv_append<T>(p, qkv, L.s_qkv, (long)n * qkv_dim, cs, hq, hkv, dh,
                                                     q, kv4, st));
    else
      LAUNCH(m, st, "rope_kv_write", qkv_rope_scatter<T>(p, qkv, L.s_qkv, (long)n * qkv_dim, cs, hq, hkv, dh, q, kc, vc,
                                 c->s_max, st));
    if (t) TRACE_COPY(t->q, q, (size_t)n * qd * es);
    if (c->mx) {
      LAUNCH(m, st, "attention", mx_attention<T>(p, q, kv4, hq, hkv, dh, ao, mx_ap, part, st));
    } else {
      LAUNCH(m, st, "attention", attention<T>(p, q, kc, vc, c->s_max, hq, hkv, dh, ao, ap, part, st));
      if constexpr (sizeof(T) == 2)
        if (ap.splits > 1)
          LAUNCH(m, st, "attention_merge", attention_merge(p, hq, dh, ap.splits, part, ao, st));
    }
    if (t) TRACE_COPY(t->attn_out, ao, (size_t)n * qd * es);
    // O projection; its residual update is fused into the FFN norm when K is split
    if (L.s_o == 1) {
      if (w4)
        LAUNCH(m, st, "gemm_o", mx_matmul<T>(L.q_o, ao, qd, n, mx_view(w4l->w_o), qd, DLM_MX_ADD, h, d,
                                             mxs, st));
      else
        LAUNCH(m, st, "gemm_o", gemm_add_f32<T>(L.g_o, ao, qd, reinterpret_cast<const T*>(w.w_o), qd, n, d,
                                                  qd, h, d, st));
      LAUNCH(m, st, "rmsnorm", rmsnorm_rows<T>(h, w.ffn_norm, n, d, cf.rms_eps, a, st));
    } else {
      if (w4)
        LAUNCH(m, st, "gemm_o", mx_matmul<T>(L.q_o, ao, qd, n, mx_view(w4l->w_o), qd, DLM_MX_STORE, part, d,
                                             mxs, st));
      else
        LAUNCH(m, st, "gemm_o", gemm_store_f32<T>(L.g_o, ao, qd, reinterpret_cast<const T*>(w.w_o), qd, n, d,
                                                    qd, part, d, st));
      LAUNCH(m, st, "residual_rmsnorm", add_rmsnorm_rows<T>(h, part, L.s_o, (long)n * d, w.ffn_norm, n, d,
                                                                cf.rms_eps, a, st));
    }
    if (t) {
      TRACE_COPY(t->h_mid, h, (size_t)n * d * 4);
      TRACE_COPY(t->a_ffn, a, (size_t)n * d * es);
    }
    if (w4)
      LAUNCH(m, st, "gemm_gate_up_swiglu", mx_matmul<T>(L.q_gu, a, d, n, mx_view(w4l->w_gate_up), d,
                                                        DLM_MX_SWIGLU, act, cf.d_ffn, mxs, st));
    else
      LAUNCH(m, st, "gemm_gate_up_swiglu", gemm_swiglu<T>(L.g_gu, a, d, reinterpret_cast<const T*>(w.w_gate_up), d, n, cf.d_ffn, d, act,
                            cf.d_ffn, st));
    if (t) TRACE_COPY(t->act, act, (size_t)n * cf.d_ffn * es);
    // down projection; its residual update is fused into the next layer's norm
    const float* next_norm = l + 1 < cf.n_layers ? m->layers[l + 1].attn_norm : nullptr;
    T* next_a = l + 1 < cf.n_layers ? a : nullptr;
    if (L.s_down == 1) {
      if (w4)
        LAUNCH(m, st, "gemm_down", mx_matmul<T>(L.q_down, act, cf.d_ffn, n, mx_view(w4l->w_down), cf.d_ffn,
                                                DLM_MX_ADD, h, d, mxs, st));
      else
        LAUNCH(m, st, "gemm_down", gemm_add_f32<T>(L.g_down, act, cf.d_ffn, reinterpret_cast<const T*>(w.w_down), cf.d_ffn, n, d,
                               cf.d_ffn, h, d, st));
      if (next_a) LAUNCH(m, st, "rmsnorm", rmsnorm_rows<T>(h, next_norm, n, d, cf.rms_eps, a, st));
    } else {
      if (w4)
        LAUNCH(m, st, "gemm_down", mx_matmul<T>(L.q_down, act, cf.d_ffn, n, mx_view(w4l->w_down), cf.d_ffn,
                                                DLM_MX_STORE, part, d, mxs, st));
      else
        LAUNCH(m, st, "gemm_down", gemm_store_f32<T>(L.g_down, act, cf.d_ffn, reinterpret_cast<const T*>(w.w_down),
                                                       cf.d_ffn, n, d, cf.d_ffn, part, d, st));
      LAUNCH(m, st, "residual_rmsnorm", add_rmsnorm_rows<T>(h, part, L.s_down, (long)n * d, next_norm, n, d,
                                                                cf.rms_eps, next_a, st));
    }
    if (t) TRACE_COPY(t->h_out, h, (size_t)n * d * 4);
  }
  return DLM_OK;
}

template <typename T>
dlm_status run_step(dlm_model* m, dlm_cache* c, const dlm_batch* b, const StepPlan& p,
                    const Layout& L, char* ws, Tail tail, const dlm_step_out* out,
                    float* logits, const dlm_trace* tr, hipStream_t st) {
  dlm_status s = run_forward<T>(m, c, b, p, L, ws, tr, st);
  if (s != DLM_OK || tail == Tail::None) return s;
  const dlm_config& cf = m->cfg;
  const int d = cf.d_model;
  float* h = reinterpret_cast<float*>(ws + L.h);
  int* lm_rows = reinterpret_cast<int*>(ws + L.lm_rows);
  int* lm_count = reinterpret_cast<int*>(ws + L.lm_count);
  int* req_off = reinterpret_cast<int*>(ws + L.req_off);
  int* req_cnt = reinterpret_cast<int*>(ws + L.req_cnt);
  T* u = reinterpret_cast<T*>(ws + L.u);
  const int m_max = p.n_blk;
  LAUNCH(m, st, "lm_select", lm_select_rows(p, b->mask, tail == Tail::Logits ? 1 : 0, lm_rows, lm_count, req_off,
                          req_cnt, st));
  LAUNCH(m, st, "final_norm", final_norm_gather<T>(h, m->final_norm, lm_rows, lm_count, m_max, d, cf.rms_eps, u, st));
  if (tr && tail == Tail::Logits) TRACE_COPY(tr->u, u, (size_t)m_max * d * sizeof(T));
  if (tail == Tail::Logits) {
    LAUNCH(m, st, "gemm_logits", gemm_scaled_f32<T>(L.g_logits, u, d, reinterpret_cast<const T*>(m->lm_head), d, m_max, cf.vocab,
                                d, cf.inv_tau, logits, cf.vocab, st));
    return DLM_OK;
  }
  float* pm = reinterpret_cast<float*>(ws + L.pm);
  float* ps = reinterpret_cast<float*>(ws + L.ps);
  int* pi = reinterpret_cast<int*>(ws + L.pi);
  float* conf = reinterpret_cast<float*>(ws + L.conf);
  int* tok = reinterpret_cast<int*>(ws + L.tok);
  LAUNCH(m, st, "lm_head", gemm_lm_head<T>(L.g_lm, u, d, reinterpret_cast<const T*>(m->lm_head), m_max, cf.vocab, d,
                           cf.inv_tau, pm, ps, pi, L.m_max, lm_count, st));
  LAUNCH(m, st, "lm_combine", lm_combine(pm, ps, pi, L.tiles, L.m_max, lm_count, m_max, conf, tok, st));
  LAUNCH(m, st, "unmask", unmask_select(p, conf, tok, req_off, b->tokens, b->mask, out->n_unmasked, out->pos,
                         out->tok, out->conf, out->block_conf, out->block_tok, b->tok_conf,
                         out->stats, st));
  return DLM_OK;
}

void mark_refreshed(dlm_cache* c, const dlm_batch* b, bool force_refresh) {
  for (int r = 0; r < b->n_req; ++r) {
    const dlm_req& q = b->reqs[r];
    if (force_refresh || b->mode == DLM_CACHE_NONE || (q.flags & DLM_REQ_REFRESH)) {
      SlotState& s = c->slots[q.slot];
      s.valid = true;
      s.block_start = q.block_start;
      s.seq_len = q.seq_len;
    }
  }
}

dlm_status dispatch(dlm_model* m, dlm_cache* c, const dlm_batch* b, const StepPlan& p,
                    const Layout& L, void* ws, Tail tail, const dlm_step_out* out,
                    float* logits, void* stream, const dlm_trace* tr = nullptr) {
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  char* w = reinterpret_cast<char*>(ws);
  if (m->cfg.dtype == DLM_BF16) return run_step<bf16>(m, c, b, p, L, w, tail, out, logits, tr, st);
  return run_step<float>(m, c, b, p, L, w, tail, out, logits, tr, st);
}

int device_cus() {
  int dev = 0, cu = 0;
  const bool ok = hipGetDevice(&dev) == hipSuccess &&
                  hipDeviceGetAttribute(&cu, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess &&
                  cu > 0;
  (void)hipGetLastError();
  return ok ? cu : 256;
}

// ---- 4-bit operands ----
bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// A packed matrix of the given shape (n, k < 0: any), with buffers the kernels can read.
dlm_status check_mx(const dlm_mx* w, int n, int k, const char* what) {
  if (!w || !w->codes || !w->scales) return fail(DLM_EINVAL, "%s: packed matrix pointer is NULL", what);
  if (w->n < 1 || w->k < 1) return fail(DLM_EINVAL, "%s: packed matrix of %d x %d", what, w->n, w->k);
  if ((n >= 0 && w->n != n) || (k >= 0 && w->k != k))
    return fail(DLM_EINVAL, "%s: packed matrix is %d x %d, expected %d x %d", what, w->n, w->k, n, k);
  // (the kernels count k in int, whole groups with a chunk to spare)
  if (w->n > INT32_MAX - 1024 || w->k > INT32_MAX - 1024)
    return fail(DLM_EUNSUPPORTED, "%s: packed matrix of %d x %d", what, w->n, w->k);
  if (!aligned16(w->codes) || !aligned16(w->scales))
    return fail(DLM_EINVAL, "%s: packed matrix is not 16-byte aligned", what);
  return DLM_OK;
}

dlm_status check_dtype(int32_t dtype) {
  if (dtype != DLM_F32 && dtype != DLM_BF16)
    return fail(DLM_EINVAL, "dtype %d is not DLM_F32 or DLM_BF16", dtype);
  return DLM_OK;
}

// Row plan of an operator call on a 4-bit cache: `rows` lists the requests. writes: the
// rows' own positions are written, so each must exist and no slot may come twice.
dlm_status make_kv_plan(const dlm_cache* c, int32_t layer, int32_t n_req, const dlm_kv_rows* rows,
                        bool positions, bool writes, StepPlan* p) {
  if (!c) return fail(DLM_EINVAL, "cache is NULL");
  if (!c->mx) return fail(DLM_EUNSUPPORTED, "the cache is not a 4-bit one (dlm_kv_cache_alloc_mx)");
  if (layer < 0 || layer >= c->model->cfg.n_layers)
    return fail(DLM_EINVAL, "layer %d outside [0, %d)", layer, c->model->cfg.n_layers);
  if (n_req < 1 || n_req > kMaxReq) return fail(DLM_EINVAL, "n_req %d outside [1, %d]", n_req, kMaxReq);
  if (!rows) return fail(DLM_EINVAL, "rows is NULL");
  memset(p, 0, sizeof *p);
  p->n_req = n_req;
  long total = 0;
  for (int r = 0; r < n_req; ++r) {
    const dlm_kv_rows& q = rows[r];
    if (q.slot < 0 || q.slot >= c->n_slots)
      return fail(DLM_EINVAL, "request %d: slot %d outside [0, %d)", r, q.slot, c->n_slots);
    if (q.seq_len < 0 || q.seq_len > c->s_max)
      return fail(DLM_ESIZE, "request %d: seq_len %d outside [0, %d]", r, q.seq_len, c->s_max);
    if (q.n_rows < 0) return fail(DLM_EINVAL, "request %d: n_rows %d < 0", r, q.n_rows);
    if (positions && (q.pos0 < 0 || (long)q.pos0 + q.n_rows > q.seq_len))
      return fail(DLM_EINVAL, "request %d: positions [%d, %ld) outside [0, %d)", r, q.pos0,
                  (long)q.pos0 + q.n_rows, q.seq_len);
    for (int s = 0; writes && s < r; ++s)
      if (rows[s].slot == q.slot) return fail(DLM_EINVAL, "request %d: slot %d used twice", r, q.slot);
    ReqPlan& rp = p->r[r];
    rp.row0 = (int)total;
    rp.nrows = q.n_rows;
    rp.pos0 = positions ? q.pos0 : 0;
    rp.seq_len = q.seq_len;
    rp.slot = q.slot;
    total += q.n_rows;
    if (total > DLM_MAX_REQ * DLM_MAX_SEQ)
      return fail(DLM_ESIZE, "more than %d rows", DLM_MAX_REQ * DLM_MAX_SEQ);
  }
  p->n_rows = (int)total;
  return DLM_OK;
}

dlm_status check_handles(dlm_model* m, dlm_cache* c) {
  if (!m) return fail(DLM_EINVAL, "model is NULL");
  if (!c) return fail(DLM_EINVAL, "cache is NULL");
  if (c->model != m) return fail(DLM_EINVAL, "cache was allocated for another model");
  return DLM_OK;
}

}  // namespace

extern "C" {

const char* dlm_last_error(void) { return g_err.c_str(); }

dlm_status dlm_load_weights(const dlm_config* cfg, const dlm_weights* w, dlm_model** out) {
  g_err.clear();
  if (!out) return fail(DLM_EINVAL, "out is NULL");
  *out = nullptr;
  dlm_status s = check_config(cfg);
  if (s != DLM_OK) return s;
  if (!w || !w->embed || !w->lm_head || !w->final_norm || !w->layers)
    return fail(DLM_EINVAL, "weights pointer is NULL");
  for (int l = 0; l < cfg->n_layers; ++l) {
    const dlm_layer_weights& lw = w->layers[l];
    if (!lw.attn_norm || !lw.w_qkv || !lw.w_o || !lw.ffn_norm || !lw.w_gate_up || !lw.w_down)
      return fail(DLM_EINVAL, "layer %d: weight pointer is NULL", l);
  }
  dlm_model* m = new dlm_model();
  m->cfg = *cfg;
  m->embed = w->embed;
  m->lm_head = w->lm_head;
  m->final_norm = w->final_norm;
  m->layers.assign(w->layers, w->layers + cfg->n_layers);
  m->es = cfg->dtype == DLM_BF16 ? 2 : 4;
  m->num_cu = device_cus();
  *out = m;
  return DLM_OK;
}

dlm_status dlm_load_weights_mx(const dlm_config* cfg, const dlm_weights_mx* w, dlm_model** out) {
  g_err.clear();
  if (!out) return fail(DLM_EINVAL, "out is NULL");
  *out = nullptr;
  dlm_status s = check_config(cfg);
  if (s != DLM_OK) return s;
  if (!w || !w->embed || !w->lm_head || !w->final_norm || !w->layers)
    return fail(DLM_EINVAL, "weights pointer is NULL");
  const int qd = cfg->n_q_heads * cfg->head_dim, qkv_dim = qd + 2 * cfg->n_kv_heads * cfg->head_dim;
  for (int l = 0; l < cfg->n_layers; ++l) {
    const dlm_layer_mx& lw = w->layers[l];
    char what[48];
    if (!lw.attn_norm || !lw.ffn_norm) return fail(DLM_EINVAL, "layer %d: weight pointer is NULL", l);
    const struct { const dlm_mx* w; int n, k; const char* name; } parts[4] = {
        {&lw.w_qkv, qkv_dim, cfg->d_model, "w_qkv"},
        {&lw.w_o, cfg->d_model, qd, "w_o"},
        {&lw.w_gate_up, 2 * cfg->d_ffn, cfg->d_model, "w_gate_up"},
        {&lw.w_down, cfg->d_model, cfg->d_ffn, "w_down"}};
    for (const auto& q : parts) {
      snprintf(what, sizeof what, "layer %d: %s", l, q.name);
      if ((s = check_mx(q.w, q.n, q.k, what)) != DLM_OK) return s;
    }
  }
  dlm_model* m = nullptr;
  try {
    m = new dlm_model();
    m->mx.assign(w->layers, w->layers + cfg->n_layers);
    for (const dlm_layer_mx& lw : m->mx)
      m->layers.push_back({lw.attn_norm, nullptr, nullptr, lw.ffn_norm, nullptr, nullptr});
  } catch (const std::bad_alloc&) {
    delete m;
    return fail(DLM_ESIZE, "out of host memory for %d layers", cfg->n_layers);
  }
  m->cfg = *cfg;
  m->embed = w->embed;
  m->lm_head = w->lm_head;
  m->final_norm = w->final_norm;
  m->es = cfg->dtype == DLM_BF16 ? 2 : 4;
  m->num_cu = device_cus();
  *out = m;
  return DLM_OK;
}

void dlm_model_destroy(dlm_model* m) { delete m; }

dlm_status dlm_profile_enable(dlm_model* m, int32_t on, const char* only_class) {
  g_err.clear();
  if (!m) return fail(DLM_EINVAL, "model is NULL");
  m->prof.on = on != 0;
  m->prof.only = only_class ? only_class : "";
  m->prof.seen.clear();
  return DLM_OK;
}

dlm_status dlm_profile_sample(dlm_model* m, int32_t every) {
  g_err.clear();
  if (!m) return fail(DLM_EINVAL, "model is NULL");
  if (every < 1) return fail(DLM_EINVAL, "every %d < 1", every);
  m->prof.every = every;
  m->prof.seen.clear();
  return DLM_OK;
}

dlm_status dlm_profile_read(dlm_model* m, dlm_profile_entry* out, int32_t cap, int32_t* n_out) {
  g_err.clear();
  if (!m || !n_out || cap < 0 || (cap > 0 && !out)) return fail(DLM_EINVAL, "NULL argument or cap < 0");
  Profiler& pf = m->prof;
  std::vector<int> calls(pf.names.size(), 0);
  std::vector<double> ms(pf.names.size(), 0.0);
  dlm_status st = DLM_OK;
  for (auto& r : pf.pending) {
    float t = 0.f;
    hipError_t e = hipEventSynchronize(r.b);
    if (e == hipSuccess) e = hipEventElapsedTime(&t, r.a, r.b);
    if (e != hipSuccess && st == DLM_OK)
      st = fail(DLM_EHIP, "profile event: %s", hipGetErrorString(e));
    calls[r.kind] += 1;
    ms[r.kind] += t;
    pf.pool.push_back(r.a);
    pf.pool.push_back(r.b);
  }
  pf.pending.clear();
  int n = 0;
  for (size_t k = 0; k < pf.names.size(); ++k) {
    const int launches = k < pf.since_read.size() ? pf.since_read[k] : 0;
    if (calls[k] == 0 && launches == 0) continue;
    if (n < cap) {
      snprintf(out[n].name, sizeof out[n].name, "%s", pf.names[k].c_str());
      out[n].calls = calls[k];
      out[n].total_ms = ms[k];
      out[n].launches = launches;
    }
    ++n;
  }
  pf.since_read.assign(pf.since_read.size(), 0);
  *n_out = n < cap ? n : cap;
  return st;
}

dlm_status dlm_workspace_bytes(const dlm_model* m, int32_t max_rows, int32_t max_reqs,
                               size_t* out_bytes) {
  g_err.clear();
  if (!m || !out_bytes) return fail(DLM_EINVAL, "NULL argument");
  if (max_rows < 1 || max_reqs < 1 || max_reqs > kMaxReq)
    return fail(DLM_EINVAL, "max_rows %d / max_reqs %d out of range", max_rows, max_reqs);
  // the planner's split-K factors (and with them the slice buffers) depend on
  // the row count and are not monotonic in it: take the largest layout over
  // every row count up to max_rows
  size_t best = 0;
  for (int n = 1; n <= max_rows; ++n) best = std::max(best, layout(m, n, max_reqs).total);
  *out_bytes = best;
  return DLM_OK;
}

static dlm_status kv_cache_alloc(const dlm_model* m, bool mx, int32_t n_slots, int32_t max_seq_len,
                                 void* dev_buf, size_t buf_bytes, size_t* required_bytes,
                                 dlm_cache** out) {
  g_err.clear();
  if (!m) return fail(DLM_EINVAL, "model is NULL");
  if (n_slots < 1) return fail(DLM_EINVAL, "n_slots %d < 1", n_slots);
  if (max_seq_len < 1 || max_seq_len > DLM_MAX_SEQ)
    return fail(DLM_ESIZE, "max_seq_len %d outside [1, %d]", max_seq_len, DLM_MAX_SEQ);
  const dlm_config& c = m->cfg;
  const int s_max = (int)align_up(max_seq_len, 64);
  const size_t vecs = (size_t)n_slots * c.n_kv_heads * s_max;
  const size_t region = mx ? vecs * (c.head_dim / 2) : vecs * c.head_dim * m->es;
  const size_t scale_region = mx ? align_up(vecs * (c.head_dim / kMxGroup), 256) : 0;
  const size_t need = (region + scale_region) * 2 * c.n_layers;
  if (required_bytes) *required_bytes = need;
  if (!dev_buf) {
    if (out) *out = nullptr;
    return DLM_OK;
  }
  if (!out) return fail(DLM_EINVAL, "out is NULL");
  *out = nullptr;
  if (buf_bytes < need) return fail(DLM_ESIZE, "cache buffer %zu bytes < %zu", buf_bytes, need);
  if (reinterpret_cast<uintptr_t>(dev_buf) % 256 != 0)
    return fail(DLM_EINVAL, "cache buffer is not 256-byte aligned");
  dlm_cache* k = nullptr;
  try {
    k = new dlm_cache();
    k->slots.assign(n_slots, SlotState{});
  } catch (const std::bad_alloc&) {
    delete k;
    return fail(DLM_ESIZE, "out of host memory for %d slots", n_slots);
  }
  k->model = m;
  k->n_slots = n_slots;
  k->s_max = s_max;
  k->base = reinterpret_cast<char*>(dev_buf);
  k->region = region;
  k->mx = mx;
  k->scale_region = scale_region;
  *out = k;
  return DLM_OK;
}

dlm_status dlm_kv_cache_alloc(const dlm_model* m, int32_t n_slots, int32_t max_seq_len,
                              void* dev_buf, size_t buf_bytes, size_t* required_bytes,
                              dlm_cache** out) {
  return kv_cache_alloc(m, false, n_slots, max_seq_len, dev_buf, buf_bytes, required_bytes, out);
}

dlm_status dlm_kv_cache_alloc_mx(const dlm_model* m, int32_t n_slots, int32_t max_seq_len,
                                 void* dev_buf, size_t buf_bytes, size_t* required_bytes,
                                 dlm_cache** out) {
  return kv_cache_alloc(m, true, n_slots, max_seq_len, dev_buf, buf_bytes, required_bytes, out);
}

void dlm_cache_destroy(dlm_cache* c) { delete c; }

dlm_status dlm_cache_invalidate(dlm_cache* c, int32_t slot) {
  g_err.clear();
  if (!c) return fail(DLM_EINVAL, "cache is NULL");
  if (slot < 0 || slot >= c->n_slots) return fail(DLM_EINVAL, "slot %d out of range", slot);
  c->slots[slot] = SlotState{};
  return DLM_OK;
}

dlm_status dlm_denoise_step(dlm_model* m, dlm_cache* c, const dlm_batch* b,
                            const float* thresholds, const dlm_step_out* out, void* workspace,
                            size_t ws_bytes, void* stream) {
  g_err.clear();
  dlm_status s = check_handles(m, c);
  if (s != DLM_OK) return s;
  if (!thresholds) return fail(DLM_EINVAL, "thresholds is NULL");
  if (!out || !out->n_unmasked || !out->pos || !out->tok || !out->conf)
    return fail(DLM_EINVAL, "step output pointer is NULL");
  if (out->stats && (!b || !b->tok_conf))
    return fail(DLM_EINVAL, "confidence statistics need batch.tok_conf");
  StepPlan p;
  s = make_plan(m, c, b, thresholds, false, &p);
  if (s != DLM_OK) return s;
  Layout L;
  s = check_ws(m, p, workspace, ws_bytes, &L);
  if (s != DLM_OK) return s;
  s = dispatch(m, c, b, p, L, workspace, Tail::Unmask, out, nullptr, stream);
  if (s == DLM_OK) mark_refreshed(c, b, false);
  return s;
}

dlm_status dlm_denoise_step_noalloc(dlm_model* m, dlm_cache* c, const dlm_batch* b,
                                    const float* thresholds, const dlm_step_out* out,
                                    void* stream) {
  g_err.clear();
  dlm_status s = check_handles(m, c);
  if (s != DLM_OK) return s;
  if (!thresholds) return fail(DLM_EINVAL, "thresholds is NULL");
  if (!out || !out->n_unmasked || !out->pos || !out->tok || !out->conf)
    return fail(DLM_EINVAL, "step output pointer is NULL");
  if (out->stats && (!b || !b->tok_conf))
    return fail(DLM_EINVAL, "confidence statistics need batch.tok_conf");
  StepPlan p;
  s = make_plan(m, c, b, thresholds, false, &p);
  if (s != DLM_OK) return s;
  const size_t need = layout(m, p.n_rows, p.n_req).total;
  if (need > (size_t)DLM_SCRATCH_BYTES)
    return fail(DLM_ESIZE, "this step needs %zu bytes of scratch (%d rows); the fixed scratch "
                "holds %zu", need, p.n_rows, (size_t)DLM_SCRATCH_BYTES);
  void* ws = nullptr;
  s = scratch_address(&ws);
  if (s != DLM_OK) return s;
  Layout L;
  s = check_ws(m, p, ws, (size_t)DLM_SCRATCH_BYTES, &L);
  if (s != DLM_OK) return s;
  // no kernel timing here (its events would be created on first use)
  const bool prof_on = m->prof.on;
  m->prof.on = false;
  s = dispatch(m, c, b, p, L, ws, Tail::Unmask, out, nullptr, stream);
  m->prof.on = prof_on;
  if (s == DLM_OK) mark_refreshed(c, b, false);
  return s;
}

dlm_status dlm_cache_refresh(dlm_model* m, dlm_cache* c, const dlm_batch* b, void* workspace,
                             size_t ws_bytes, void* stream) {
  g_err.clear();
  dlm_status s = check_handles(m, c);
  if (s != DLM_OK) return s;
  StepPlan p;
  s = make_plan(m, c, b, nullptr, true, &p);
  if (s != DLM_OK) return s;
  Layout L;
  s = check_ws(m, p, workspace, ws_bytes, &L);
  if (s != DLM_OK) return s;
  s = dispatch(m, c, b, p, L, workspace, Tail::None, nullptr, nullptr, stream);
  if (s == DLM_OK) mark_refreshed(c, b, true);
  return s;
}

dlm_status dlm_debug_logits(dlm_model* m, dlm_cache* c, const dlm_batch* b, float* logits_out,
                            void* workspace, size_t ws_bytes, void* stream) {
  g_err.clear();
  dlm_status s = check_handles(m, c);
  if (s != DLM_OK) return s;
  if (!logits_out) return fail(DLM_EINVAL, "logits_out is NULL");
  StepPlan p;
  s = make_plan(m, c, b, nullptr, false, &p);
  if (s != DLM_OK) return s;
  Layout L;
  s = check_ws(m, p, workspace, ws_bytes, &L);
  if (s != DLM_OK) return s;
  s = dispatch(m, c, b, p, L, workspace, Tail::Logits, nullptr, logits_out, stream);
  if (s == DLM_OK) mark_refreshed(c, b, false);
  return s;
}

dlm_status dlm_debug_trace(dlm_model* m, dlm_cache* c, const dlm_batch* b, dlm_trace* tr,
                           void* workspace, size_t ws_bytes, void* stream) {
  g_err.clear();
  dlm_status s = check_handles(m, c);
  if (s != DLM_OK) return s;
  if (!tr) return fail(DLM_EINVAL, "trace is NULL");
  if (tr->layer < 0 || tr->layer >= m->cfg.n_layers)
    return fail(DLM_EINVAL, "trace layer %d outside [0, %d)", tr->layer, m->cfg.n_layers);
  if (tr->u && !tr->logits) return fail(DLM_EINVAL, "trace.u needs trace.logits");
  StepPlan p;
  s = make_plan(m, c, b, nullptr, false, &p);
  if (s != DLM_OK) return s;
  Layout L;
  s = check_ws(m, p, workspace, ws_bytes, &L);
  if (s != DLM_OK) return s;
  if (tr->qkv && tr->qkv_cap < L.s_qkv)
    return fail(DLM_ESIZE, "trace.qkv holds %d K-split slices; this step writes %d", tr->qkv_cap,
                L.s_qkv);
  tr->qkv_splits = L.s_qkv;
  s = dispatch(m, c, b, p, L, workspace, tr->logits ? Tail::Logits : Tail::None, nullptr,
               tr->logits, stream, tr);
  if (s == DLM_OK) mark_refreshed(c, b, false);
  return s;
}

dlm_status dlm_head_confidence(dlm_model* m, const void* u_rows, int32_t m_rows, float* conf,
                               int32_t* tok, void* workspace, size_t ws_bytes, void* stream) {
  g_err.clear();
  if (!m) return fail(DLM_EINVAL, "model is NULL");
  if (!u_rows || !conf || !tok) return fail(DLM_EINVAL, "NULL buffer");
  if (m_rows < 1) return fail(DLM_EINVAL, "m_rows %d < 1", m_rows);
  if (!workspace) return fail(DLM_EINVAL, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(workspace) % 256 != 0)
    return fail(DLM_EINVAL, "workspace is not 256-byte aligned");
  const GemmPlan gp = lm_head_plan((int)m->es, m_rows, m->cfg.vocab, m->cfg.d_model, m->num_cu);
  const int tiles = lm_head_tiles(gp, m->cfg.vocab);
  const size_t stat = align_up((size_t)tiles * m_rows * 4, 256);
  const size_t need = 3 * stat + 256;
  if (ws_bytes < need) return fail(DLM_ESIZE, "workspace of %zu bytes; needs %zu", ws_bytes, need);
  char* w = reinterpret_cast<char*>(workspace);
  float* pm = reinterpret_cast<float*>(w);
  float* ps = reinterpret_cast<float*>(w + stat);
  int* pi = reinterpret_cast<int*>(w + 2 * stat);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const dlm_config& cf = m->cfg;
  if (cf.dtype == DLM_BF16) {
    HIPCHECK(gemm_lm_head<bf16>(gp, reinterpret_cast<const bf16*>(u_rows), cf.d_model,
                                reinterpret_cast<const bf16*>(m->lm_head), m_rows, cf.vocab,
                                cf.d_model, cf.inv_tau, pm, ps, pi, m_rows, nullptr, st));
  } else {
    HIPCHECK(gemm_lm_head<float>(gp, reinterpret_cast<const float*>(u_rows), cf.d_model,
                                 reinterpret_cast<const float*>(m->lm_head), m_rows, cf.vocab,
                                 cf.d_model, cf.inv_tau, pm, ps, pi, m_rows, nullptr, st));
  }
  HIPCHECK(lm_combine(pm, ps, pi, tiles, m_rows, nullptr, m_rows, conf, tok, st));
  return DLM_OK;
}

dlm_status dlm_debug_gemm_plan(int32_t elem_bytes, int32_t M, int32_t N, int32_t K, int32_t kind,
                               int32_t num_cu, int32_t out[4]) {
  g_err.clear();
  if (!out) return fail(DLM_EINVAL, "out is NULL");
  if ((elem_bytes != 2 && elem_bytes != 4) || M < 1 || N < 1 || K < 1 || num_cu < 1 || kind < 0 ||
      kind > 2 || (kind == 1 && N % 2 != 0))
    return fail(DLM_EINVAL, "elem_bytes %d, M %d N %d K %d, kind %d, %d CUs", elem_bytes, M, N, K,
                kind, num_cu);
  const GemmPlan p = kind == 0   ? projection_plan(elem_bytes, M, N, K, num_cu)
                     : kind == 1 ? gate_up_plan(elem_bytes, M, N / 2, K, num_cu)
                                 : lm_head_plan(elem_bytes, M, N, K, num_cu);
  out[0] = p.cfg;
  out[1] = p.splits;
  out[2] = p.sub;
  out[3] = p.n_tail;
  return DLM_OK;
}

dlm_status dlm_debug_attention_plan(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                    int32_t n_req, const int32_t* rows, const int32_t* seq_len,
                                    size_t scratch_bytes, int32_t num_cu, int32_t* kernel,
                                    int32_t* splits) {
  g_err.clear();
  if (!rows || !seq_len) return fail(DLM_EINVAL, "NULL array");
  if (n_req < 1 || n_req > kMaxReq) return fail(DLM_EINVAL, "n_req %d outside [1, %d]", n_req, kMaxReq);
  if (n_q_heads < 1 || n_kv_heads < 1 || n_q_heads % n_kv_heads != 0 || num_cu < 1 ||
      (head_dim != 64 && head_dim != 128))
    return fail(DLM_EINVAL, "heads %d / %d of %d on %d CUs", n_q_heads, n_kv_heads, head_dim, num_cu);
  StepPlan p{};
  p.n_req = n_req;
  for (int r = 0; r < n_req; ++r) {
    if (rows[r] < 1 || seq_len[r] < 1)
      return fail(DLM_EINVAL, "request %d: %d rows over %d keys", r, rows[r], seq_len[r]);
    p.r[r].row0 = p.n_rows;
    p.r[r].nrows = rows[r];
    p.r[r].seq_len = seq_len[r];
    p.n_rows += rows[r];
  }
  const AttnPlan ap = attention_plan(p, n_q_heads, n_kv_heads, head_dim, 2, scratch_bytes, num_cu);
  if (kernel) *kernel = ap.kernel;
  if (splits) *splits = ap.splits;
  return DLM_OK;
}

dlm_status dlm_debug_gemm_info(int32_t cfg, int32_t* bm, int32_t* bn, int32_t* subs) {
  g_err.clear();
  int tm = 0, tn = 0, th = 0;
  if (!gemm_dl_tile(cfg, &tm, &tn, &th)) return fail(DLM_EINVAL, "no GEMM configuration %d", cfg);
  if (bm) *bm = tm;
  if (bn) *bn = tn;
  if (subs) *subs = gemm_dl_subs(cfg) | (gemm_dl_odd(cfg) ? 8 : 0);
  return DLM_OK;
}

dlm_status dlm_debug_gemm(int32_t cfg, int32_t epilogue, int32_t sub, int32_t n_tail,
                          int32_t group_m, int32_t splits, const void* a, const void* b, void* c,
                          int32_t M, int32_t N, int32_t K, void* stream) {
  g_err.clear();
  if (!a || !b || !c) return fail(DLM_EINVAL, "NULL buffer");
  if (M < 1 || N < 1 || K < 1 || K % 64 != 0)
    return fail(DLM_EINVAL, "sizes M %d N %d K %d (K a positive multiple of 64)", M, N, K);
  if (epilogue < 0 || epilogue > 2) return fail(DLM_EINVAL, "epilogue %d", epilogue);
  if (epilogue == 1 && N % 2 != 0) return fail(DLM_EINVAL, "odd N %d for the SwiGLU epilogue", N);
  if (group_m < 0 || n_tail < 0) return fail(DLM_EINVAL, "negative group_m or n_tail");
  if (splits < 1 || (splits > 1 && epilogue != 0) || (K / 64) % splits != 0)
    return fail(DLM_EINVAL, "splits %d (K slices of the plain store only, dividing the %d k-tiles)",
                splits, K / 64);
  int tm = 0, tn = 0, th = 0;
  if (!gemm_dl_tile(cfg, &tm, &tn, &th)) return fail(DLM_EINVAL, "no GEMM configuration %d", cfg);
  // the gate/up interleave pairs columns in groups of the MFMA tile width
  const int pair = gemm_dl_mfma(cfg) == 32 ? 32 : 16;
  if (epilogue == 1 && (N / 2) % pair != 0)
    return fail(DLM_EINVAL, "SwiGLU width %d is not a multiple of %d", N / 2, pair);
  if (epilogue == 1 && gemm_dl_odd(cfg))
    return fail(DLM_EINVAL, "configuration %d has no SwiGLU epilogue (odd fragment count)", cfg);
  if (sub != 0 && ((sub != 2 && sub != 4) || !(gemm_dl_subs(cfg) & sub)))
    return fail(DLM_EINVAL, "configuration %d has no %d-way sub-tiles", cfg, sub);
  if (sub != 0 && (long)n_tail > (long)ceil_div(M, tm) * ceil_div(N, tn) * splits)
    return fail(DLM_EINVAL, "n_tail %d beyond the tile count", n_tail);
  const hipError_t e = gemm_debug_launch(cfg, epilogue, sub, n_tail, group_m, splits,
                                         reinterpret_cast<const bf16*>(a),
                                         reinterpret_cast<const bf16*>(b), c, M, N, K,
                                         reinterpret_cast<hipStream_t>(stream));
  if (e == hipErrorInvalidValue)
    return fail(DLM_EINVAL, "GEMM configuration %d rejects this launch", cfg);
  if (e != hipSuccess) return fail(DLM_EHIP, "GEMM launch: %s", hipGetErrorString(e));
  return DLM_OK;
}

// ---- operators on 4-bit operands ----

dlm_status dlm_mx_bytes(int32_t n, int32_t k, size_t* codes_bytes, size_t* scales_bytes) {
  g_err.clear();
  if (n < 1 || k < 1) return fail(DLM_EINVAL, "packed matrix of %d x %d", n, k);
  const size_t groups = ((size_t)k + kMxGroup - 1) / kMxGroup;
  if (codes_bytes) *codes_bytes = (size_t)n * groups * 16;
  if (scales_bytes) *scales_bytes = (size_t)n * align_up(groups, 16);
  return DLM_OK;
}

dlm_status dlm_mx_pack(int32_t dtype, const void* w, int64_t ldw, const dlm_mx* out, void* stream) {
  g_err.clear();
  dlm_status s = check_dtype(dtype);
  if (s != DLM_OK || (s = check_mx(out, -1, -1, "out")) != DLM_OK) return s;
  if (!w) return fail(DLM_EINVAL, "w is NULL");
  if (ldw < out->k) return fail(DLM_EINVAL, "row stride %lld < %d", (long long)ldw, out->k);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (dtype == DLM_BF16)
    HIPCHECK(mx_pack<bf16>(reinterpret_cast<const bf16*>(w), ldw, out->k, mx_view(*out), st));
  else
    HIPCHECK(mx_pack<float>(reinterpret_cast<const float*>(w), ldw, out->k, mx_view(*out), st));
  return DLM_OK;
}

dlm_status dlm_mx_unpack(const dlm_mx* w, int32_t dtype, void* out, int64_t ldo, void* stream) {
  g_err.clear();
  dlm_status s = check_dtype(dtype);
  if (s != DLM_OK || (s = check_mx(w, -1, -1, "w")) != DLM_OK) return s;
  if (!out) return fail(DLM_EINVAL, "out is NULL");
  if (ldo < w->k) return fail(DLM_EINVAL, "row stride %lld < %d", (long long)ldo, w->k);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (dtype == DLM_BF16)
    HIPCHECK(mx_unpack<bf16>(mx_view(*w), w->k, reinterpret_cast<bf16*>(out), ldo, st));
  else
    HIPCHECK(mx_unpack<float>(mx_view(*w), w->k, reinterpret_cast<float*>(out), ldo, st));
  return DLM_OK;
}

static dlm_status check_linear(int32_t dtype, int32_t m_rows, const dlm_mx* w, int32_t epilogue) {
  dlm_status s = check_dtype(dtype);
  if (s != DLM_OK || (s = check_mx(w, -1, -1, "w")) != DLM_OK) return s;
  if (m_rows < 0 || m_rows > DLM_MAX_REQ * DLM_MAX_SEQ)
    return fail(DLM_EINVAL, "m_rows %d outside [0, %d]", m_rows, DLM_MAX_REQ * DLM_MAX_SEQ);
  if (epilogue < DLM_MX_STORE || epilogue > DLM_MX_SWIGLU) return fail(DLM_EINVAL, "epilogue %d", epilogue);
  if (epilogue == DLM_MX_SWIGLU && w->n % 2 != 0)
    return fail(DLM_EINVAL, "odd number of rows %d for the SwiGLU epilogue", w->n);
  return DLM_OK;
}

dlm_status dlm_mx_linear_workspace(int32_t dtype, int32_t m_rows, const dlm_mx* w, int32_t epilogue,
                                   size_t* out_bytes) {
  g_err.clear();
  dlm_status s = check_linear(dtype, m_rows, w, epilogue);
  if (s != DLM_OK) return s;
  if (!out_bytes) return fail(DLM_EINVAL, "out_bytes is NULL");
  // whatever the addresses and the row strides of x and y turn out to be
  size_t need = 0;
  for (int al = 0; al < 4; ++al)
    need = std::max(need, mx_plan(dtype == DLM_BF16 ? 2 : 4, m_rows, w->n, w->k, w->k,
                                  epilogue == DLM_MX_SWIGLU, al & 1, al & 2, true, device_cus()).scratch);
  *out_bytes = need;
  return DLM_OK;
}

dlm_status dlm_mx_linear(int32_t dtype, const void* x, int64_t ldx, int32_t m_rows, const dlm_mx* w,
                         int32_t epilogue, void* y, int64_t ldy, void* workspace, size_t ws_bytes,
                         void* stream) {
  g_err.clear();
  dlm_status s = check_linear(dtype, m_rows, w, epilogue);
  if (s != DLM_OK) return s;
  if (m_rows == 0) return DLM_OK;
  if (!x || !y) return fail(DLM_EINVAL, "NULL buffer");
  const bool swiglu = epilogue == DLM_MX_SWIGLU;
  if (ldx < w->k || ldy < (swiglu ? w->n / 2 : w->n))
    return fail(DLM_EINVAL, "row strides %lld, %lld too small for %d inputs and %d outputs",
                (long long)ldx, (long long)ldy, w->k, swiglu ? w->n / 2 : w->n);
  const int es = dtype == DLM_BF16 ? 2 : 4;
  const bool x_al = aligned16(x) && ldx * es % 16 == 0 && w->k * (long)es % 16 == 0 && ldx <= kMxTileK;
  const bool y_al = aligned16(y) && ldy % 8 == 0 && ldy < INT32_MAX;
  const MxPlan plan = mx_plan(es, m_rows, w->n, w->k, (long)ldx, swiglu, x_al, y_al, true, device_cus());
  if (plan.scratch) {
    if (!workspace) return fail(DLM_EINVAL, "workspace is NULL");
    if (reinterpret_cast<uintptr_t>(workspace) % 256 != 0)
      return fail(DLM_EINVAL, "workspace is not 256-byte aligned");
    if (ws_bytes < plan.scratch)
      return fail(DLM_ESIZE, "workspace of %zu bytes; needs %zu", ws_bytes, plan.scratch);
  }
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (dtype == DLM_BF16)
    HIPCHECK(mx_matmul<bf16>(plan, reinterpret_cast<const bf16*>(x), ldx, m_rows, mx_view(*w), w->k,
                             epilogue, y, ldy, workspace, st));
  else
    HIPCHECK(mx_matmul<float>(plan, reinterpret_cast<const float*>(x), ldx, m_rows, mx_view(*w), w->k,
                              epilogue, y, ldy, workspace, st));
  return DLM_OK;
}

dlm_status dlm_debug_mx_linear_plan(int32_t dtype, int32_t m_rows, int32_t n, int32_t k, int64_t ldx,
                                    int32_t epilogue, int32_t aligned, int32_t join, int32_t num_cu,
                                    int32_t out[3]) {
  g_err.clear();
  uint8_t unused[16] __attribute__((aligned(16)));   // (buffers for the check; not looked at)
  const dlm_mx w{unused, unused, n, k};
  dlm_status s = check_linear(dtype, m_rows, &w, epilogue);
  if (s != DLM_OK) return s;
  if (!out) return fail(DLM_EINVAL, "out is NULL");
  if (m_rows < 1 || ldx < k || num_cu < 1 || (!join && epilogue != DLM_MX_STORE))
    return fail(DLM_EINVAL, "%d rows, row stride %lld, %d CUs, join %d", m_rows, (long long)ldx, num_cu, join);
  const MxPlan p = mx_plan(dtype == DLM_BF16 ? 2 : 4, m_rows, n, k, (long)ldx, epilogue == DLM_MX_SWIGLU,
                           aligned & 1, aligned & 2, join != 0, num_cu);
  out[0] = p.gemm ? 4 : p.tile.kind;
  out[1] = p.gemm ? p.g.splits : p.tile.slices;
  out[2] = p.staged;
  return DLM_OK;
}

dlm_status dlm_debug_mx_attention_plan(int32_t dtype, int32_t n_q_heads, int32_t n_kv_heads,
                                       int32_t head_dim, int32_t n_req, const int32_t* rows,
                                       const int32_t* seq_len, size_t scratch_bytes, int32_t num_cu,
                                       int32_t* kernel, int32_t* splits) {
  g_err.clear();
  dlm_status s = check_dtype(dtype);
  if (s != DLM_OK) return s;
  if (!rows || !seq_len || !kernel || !splits) return fail(DLM_EINVAL, "NULL array or output");
  if (n_req < 1 || n_req > kMaxReq) return fail(DLM_EINVAL, "n_req %d outside [1, %d]", n_req, kMaxReq);
  if (n_q_heads < 1 || n_kv_heads < 1 || n_q_heads % n_kv_heads != 0 || num_cu < 1 ||
      (head_dim != 64 && head_dim != 128))
    return fail(DLM_EINVAL, "heads %d / %d of %d on %d CUs", n_q_heads, n_kv_heads, head_dim, num_cu);
  StepPlan p{};
  p.n_req = n_req;
  for (int r = 0; r < n_req; ++r) {
    if (rows[r] < 0 || rows[r] > DLM_MAX_SEQ || seq_len[r] < 0 || seq_len[r] > DLM_MAX_SEQ)
      return fail(DLM_EINVAL, "request %d: %d rows over %d keys", r, rows[r], seq_len[r]);
    p.r[r].row0 = p.n_rows;
    p.r[r].nrows = rows[r];
    p.r[r].seq_len = seq_len[r];
    p.n_rows += rows[r];
  }
  const MxAttnPlan ap = mx_attention_plan(p, n_q_heads, n_kv_heads, head_dim, dtype == DLM_BF16 ? 2 : 4,
                                          scratch_bytes, num_cu);
  *kernel = ap.kind;
  *splits = ap.splits;
  return DLM_OK;
}

dlm_status dlm_mx_kv_append(dlm_cache* c, int32_t layer, int32_t n_req, const dlm_kv_rows* rows,
                            const float* qkv, int32_t splits, const float* rot, void* q_out,
                            void* stream) {
  g_err.clear();
  StepPlan p;
  dlm_status s = make_kv_plan(c, layer, n_req, rows, true, true, &p);
  if (s != DLM_OK) return s;
  if (splits < 1) return fail(DLM_EINVAL, "splits %d < 1", splits);
  if (p.n_rows == 0) return DLM_OK;
  if (!qkv || !rot || !q_out) return fail(DLM_EINVAL, "NULL buffer");
  if (!aligned16(qkv) || !aligned16(rot) || !aligned16(q_out))
    return fail(DLM_EINVAL, "a buffer is not 16-byte aligned");
  const dlm_config& cf = c->model->cfg;
  const long stride = (long)p.n_rows * (cf.n_q_heads + 2 * cf.n_kv_heads) * cf.head_dim;
  const float2* cs = reinterpret_cast<const float2*>(rot);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (cf.dtype == DLM_BF16)
    HIPCHECK(mx_kv_append<bf16>(p, qkv, splits, stride, cs, cf.n_q_heads, cf.n_kv_heads, cf.head_dim,
                                reinterpret_cast<bf16*>(q_out), c->mx_layer(layer), st));
  else
    HIPCHECK(mx_kv_append<float>(p, qkv, splits, stride, cs, cf.n_q_heads, cf.n_kv_heads, cf.head_dim,
                                 reinterpret_cast<float*>(q_out), c->mx_layer(layer), st));
  return DLM_OK;
}

dlm_status dlm_mx_kv_read(const dlm_cache* c, int32_t layer, int32_t n_req, const dlm_kv_rows* rows,
                          void* k_out, void* v_out, void* stream) {
  g_err.clear();
  StepPlan p;
  dlm_status s = make_kv_plan(c, layer, n_req, rows, true, false, &p);
  if (s != DLM_OK) return s;
  if (p.n_rows == 0) return DLM_OK;
  if (!k_out || !v_out) return fail(DLM_EINVAL, "NULL buffer");
  if (!aligned16(k_out) || !aligned16(v_out)) return fail(DLM_EINVAL, "a buffer is not 16-byte aligned");
  const dlm_config& cf = c->model->cfg;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (cf.dtype == DLM_BF16)
    HIPCHECK(mx_kv_read<bf16>(p, cf.n_kv_heads, cf.head_dim, c->mx_layer(layer),
                              reinterpret_cast<bf16*>(k_out), reinterpret_cast<bf16*>(v_out), st));
  else
    HIPCHECK(mx_kv_read<float>(p, cf.n_kv_heads, cf.head_dim, c->mx_layer(layer),
                               reinterpret_cast<float*>(k_out), reinterpret_cast<float*>(v_out), st));
  return DLM_OK;
}

dlm_status dlm_mx_kv_attention_workspace(const dlm_cache* c, int32_t n_req, const dlm_kv_rows* rows,
                                         size_t* out_bytes) {
  g_err.clear();
  StepPlan p;
  dlm_status s = make_kv_plan(c, 0, n_req, rows, false, false, &p);
  if (s != DLM_OK) return s;
  if (!out_bytes) return fail(DLM_EINVAL, "out_bytes is NULL");
  const dlm_model* m = c->model;
  const dlm_config& cf = m->cfg;
  *out_bytes = mx_attention_scratch(
      p.n_rows, cf.n_q_heads, cf.head_dim,
      mx_attention_plan(p, cf.n_q_heads, cf.n_kv_heads, cf.head_dim, m->es, SIZE_MAX, m->num_cu).splits);
  return DLM_OK;
}

dlm_status dlm_mx_kv_attention(const dlm_cache* c, int32_t layer, int32_t n_req,
                               const dlm_kv_rows* rows, const void* q, void* out, void* workspace,
                               size_t ws_bytes, void* stream) {
  g_err.clear();
  StepPlan p;
  dlm_status s = make_kv_plan(c, layer, n_req, rows, false, false, &p);
  if (s != DLM_OK) return s;
  if (p.n_rows == 0) return DLM_OK;
  if (!q || !out) return fail(DLM_EINVAL, "NULL buffer");
  if (!aligned16(q) || !aligned16(out)) return fail(DLM_EINVAL, "a buffer is not 16-byte aligned");
  const dlm_model* m = c->model;
  const dlm_config& cf = m->cfg;
  const MxAttnPlan plan =
      mx_attention_plan(p, cf.n_q_heads, cf.n_kv_heads, cf.head_dim, m->es, SIZE_MAX, m->num_cu);
  const size_t need = mx_attention_scratch(p.n_rows, cf.n_q_heads, cf.head_dim, plan.splits);
  if (need) {
    if (!workspace) return fail(DLM_EINVAL, "workspace is NULL");
    if (reinterpret_cast<uintptr_t>(workspace) % 256 != 0)
      return fail(DLM_EINVAL, "workspace is not 256-byte aligned");
    if (ws_bytes < need) return fail(DLM_ESIZE, "workspace of %zu bytes; needs %zu", ws_bytes, need);
  }
  float* scratch = reinterpret_cast<float*>(workspace);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (cf.dtype == DLM_BF16)
    HIPCHECK(mx_attention<bf16>(p, reinterpret_cast<const bf16*>(q), c->mx_layer(layer), cf.n_q_heads,
                                cf.n_kv_heads, cf.head_dim, reinterpret_cast<bf16*>(out), plan, scratch,
                                st));
  else
    HIPCHECK(mx_attention<float>(p, reinterpret_cast<const float*>(q), c->mx_layer(layer), cf.n_q_heads,
                                 cf.n_kv_heads, cf.head_dim, reinterpret_cast<float*>(out), plan, scratch,
                                 st));
  return DLM_OK;
}

}  // extern "C"
