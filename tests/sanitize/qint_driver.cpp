// Drives the host side of the calls on 8-bit integers (include/dlm.h) over random and
// edge-case arguments: sizes, workspaces and plans of products (those whose rows are taken in
// parts too), models with projections in 8 bits, and the refusals. No call here reaches a
// launch. Exit status 0 when every valid call returned DLM_OK and every other one an error.
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <random>
#include <vector>

#include "../../include/dlm.h"

// The library is compiled without its GPU code here; there is nothing to register.
extern "C" {
void** __hipRegisterFatBinary(const void*) {
  static void* none = nullptr;
  return &none;
}
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void*, char*, const char*, unsigned, void*, void*, void*, void*, int*) {}
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
}

static int failures = 0;
#define EXPECT(cond)                                          \
  do {                                                        \
    if (!(cond)) {                                            \
      std::fprintf(stderr, "line %d: %s\n", __LINE__, #cond); \
      ++failures;                                             \
    }                                                         \
  } while (0)

static void* at(uintptr_t a) { return reinterpret_cast<void*>(a); }
static dlm_qint matrix(int n, int k) {
  return dlm_qint{static_cast<int8_t*>(at(0x10000)), static_cast<float*>(at(0x20000)), n, k};
}

int main() {
  std::mt19937_64 rng(5);
  auto ri = [&](long a, long b) { return std::uniform_int_distribution<long>(a, b)(rng); };
  auto size = [&](int bits) { return (int32_t)(ri(0, 3) ? ri(1, 1L << ri(0, bits)) : 1L << ri(0, bits)); };
  const int max_rows = DLM_MAX_REQ * DLM_MAX_SEQ;

  // products: plans of any size, and a missing, short or unaligned workspace refused
  for (int trial = 0; trial < 60000; ++trial) {
    const int k = std::min<int>(size(17), DLM_QINT_MAX_K), epi = (int)ri(0, 2);
    const long row = (k + DLM_QINT_ROW - 1L) / DLM_QINT_ROW * DLM_QINT_ROW;
    int n = size(ri(0, 4) ? 16 : 25), m = ri(0, 3) ? size(13) : (int)ri(1, max_rows);
    if (epi == DLM_QINT_SWIGLU) n += n % 2;
    const dlm_qint w = matrix(n, k), x = matrix(m, k);
    const bool wide = (n + 31L) / 32 * 32 * row >= 1L << 33;
    size_t codes = 0, scales = 0, need = ~(size_t)0;
    EXPECT(dlm_qint_bytes(n, k, &codes, &scales) == DLM_OK && codes == (size_t)n * row && scales == 4 * (size_t)n);
    EXPECT(dlm_qint_linear_workspace(m, &w, epi, &need) == (wide ? DLM_EUNSUPPORTED : DLM_OK));
    int32_t p[4];
    const int cus = (int)(ri(0, 1) ? 256 : ri(1, 400));
    EXPECT(dlm_debug_qint_linear_plan(m, n, k, epi, cus, p) == (wide ? DLM_EUNSUPPORTED : DLM_OK));
    if (wide) continue;
    EXPECT(need != ~(size_t)0 && p[1] >= 1);
    if (m * row >= 1L << 33) EXPECT(need == 0 && p[1] == 1 && p[2] == 0);     // parts: whole tiles, no slices
    if (!need) continue;
    const int dtype = DLM_F32;
    void* y = at(0x2000);
    auto call = [&](void* ws, size_t bytes) {
      return dlm_qint_linear(&x, &w, epi, static_cast<float*>(y), n, dtype, y, n, ws, bytes, nullptr);
    };
    EXPECT(call(nullptr, SIZE_MAX) == DLM_EINVAL);
    EXPECT(call(at(0x110), SIZE_MAX) == DLM_EINVAL);
    EXPECT(call(at(0x100), need - 1) == DLM_ESIZE);
  }
  // refusals of the other calls
  for (int trial = 0; trial < 2000; ++trial) {
    dlm_qint q = matrix(size(20), std::min<int>(size(17), DLM_QINT_MAX_K));
    const int kind = (int)ri(0, 4);
    if (kind == 0) q.codes += ri(1, 15);
    if (kind == 1) q.scales = static_cast<float*>(at(0x20000 + ri(1, 3)));
    if (kind == 2) q.k = (int)(ri(0, 1) ? DLM_QINT_MAX_K + 1 : INT32_MAX);
    if (kind == 3) q.n = (int)(ri(0, 1) ? -1 : INT32_MIN);
    const long ld = kind == 4 ? q.k - 1L : INT32_MAX;
    const float* h = static_cast<float*>(at(0x30000));
    EXPECT(dlm_qint_pack(DLM_BF16, at(0x1000), ld, &q, nullptr) != DLM_OK);
    EXPECT(dlm_qint_unpack(&q, DLM_F32, at(0x1000), ld, nullptr) != DLM_OK);
    EXPECT(dlm_qint_norm(h, ld, nullptr, 0, DLM_F32, nullptr, 0, 0, 0, h, 1e-5f, &q, nullptr) != DLM_OK);
  }

  // models: workspaces, the attention's scratch, caches
  for (int trial = 0; trial < 60; ++trial) {
    const int dh = ri(0, 1) ? 64 : 128, hkv = (int)ri(1, 8), hq = hkv * (int)ri(1, 8), layers = (int)ri(1, 5);
    dlm_config cfg{};
    cfg.n_layers = layers, cfg.d_model = 64 * (int)ri(1, 40), cfg.n_q_heads = hq, cfg.n_kv_heads = hkv;
    cfg.head_dim = dh, cfg.d_ffn = 32 * (int)ri(1, 300), cfg.vocab = 64 * (int)ri(2, 200);
    cfg.mask_id = cfg.vocab - 1, cfg.rms_eps = 1e-5f, cfg.rope_theta = 10000.f, cfg.inv_tau = 1.f;
    cfg.dtype = ri(0, 1) ? DLM_BF16 : DLM_F32;
    const int qd = hq * dh, qkv = qd + 2 * hkv * dh;
    const float* norm = static_cast<float*>(at(0x30000));
    std::vector<dlm_layer_qint> ls(layers, dlm_layer_qint{norm, matrix(qkv, cfg.d_model), matrix(cfg.d_model, qd), norm,
                                                          matrix(2 * cfg.d_ffn, cfg.d_model),
                                                          matrix(cfg.d_model, cfg.d_ffn)});
    dlm_weights_qint w{at(0x40000), at(0x50000), norm, ls.data()};
    dlm_model* m = nullptr;
    const dlm_status s = dlm_load_weights_qint(&cfg, &w, &m);
    if (s != DLM_OK) {
      EXPECT(s == DLM_EUNSUPPORTED || s == DLM_EINVAL);
      std::fprintf(stderr, "note: configuration refused: %s\n", dlm_last_error());
      continue;
    }
    size_t ws = 0, less = 0, room = 0;
    EXPECT(dlm_workspace_bytes(m, 3000, 8, &ws) == DLM_OK && dlm_workspace_bytes(m, 700, 8, &less) == DLM_OK);
    EXPECT(less <= ws);
    for (int i = 0; i < 200; ++i) {
      const int rows = (int)ri(1, 700);
      EXPECT(dlm_debug_attention_scratch(m, rows, (int)ri(1, DLM_MAX_REQ), &room) == DLM_OK && room <= less);
    }
    ls.back().w_down.k += 1;
    dlm_model* other = nullptr;
    EXPECT(dlm_load_weights_qint(&cfg, &w, &other) == DLM_EINVAL && !other);
    size_t need = 0;
    EXPECT(dlm_kv_cache_alloc_mx(m, 3, (int)ri(1, 8192), nullptr, 0, &need, nullptr) == DLM_OK && need % 256 == 0);
    dlm_model_destroy(m);
  }
  std::printf("%d failures\n", failures);
  return failures ? 1 : 0;
}
