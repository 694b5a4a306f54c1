// Drives the host side of the 4-bit calls (include/dlm.h) over random and edge-case
// arguments: sizes, workspaces and plans of products and of attention, packed models and
// caches, and the refusals. No call here reaches a launch. Exit status 0 when every valid
// call returned DLM_OK and every other one an error.
#include <cstdint>
#include <cstdio>
#include <random>
#include <vector>

#include "../../include/dlm.h"

static int failures = 0;
#define EXPECT(cond)                                          \
  do {                                                        \
    if (!(cond)) {                                            \
      std::fprintf(stderr, "line %d: %s\n", __LINE__, #cond); \
      ++failures;                                             \
    }                                                         \
  } while (0)

static void* at(uintptr_t a) { return reinterpret_cast<void*>(a); }

int main() {
  std::mt19937_64 rng(3);
  auto ri = [&](long a, long b) { return std::uniform_int_distribution<long>(a, b)(rng); };
  auto size = [&](int bits) { return (int32_t)(ri(0, 3) ? ri(1, 1L << ri(0, bits)) : 1L << ri(0, bits)); };

  // products: every workspace has a size, and a NULL or a short one is refused
  for (int trial = 0; trial < 20000; ++trial) {
    dlm_mx w{at(0x10000), reinterpret_cast<uint8_t*>(at(0x20000)), size(trial % 50 ? 16 : 30),
             size(trial % 50 ? 16 : 30)};
    const int dtype = (int)ri(0, 1), epi = (int)ri(0, 2), m = (int)(ri(0, 9) ? size(13) : size(19));
    if (epi == DLM_MX_SWIGLU) w.n += w.n % 2;
    size_t codes = 0, scales = 0, need = ~(size_t)0;
    EXPECT(dlm_mx_bytes(w.n, w.k, &codes, &scales) == DLM_OK);
    EXPECT(codes >= (size_t)w.n * w.k / 2 && codes % 16 == 0 && scales % 16 == 0);
    EXPECT(dlm_mx_linear_workspace(dtype, m, &w, epi, &need) == DLM_OK && need != ~(size_t)0);
    EXPECT(dlm_mx_linear_workspace(dtype, 0, &w, epi, &need) == DLM_OK);
    EXPECT(dlm_mx_linear(dtype, at(0x1000), w.k, 0, &w, epi, at(0x2000), w.n, nullptr, 0, nullptr) == DLM_OK);
    EXPECT(dlm_mx_linear(dtype, at(0x1000), w.k - 1, m, &w, epi, at(0x2000), w.n, nullptr, 0, nullptr) != DLM_OK);
    EXPECT(dlm_mx_linear(DLM_F32, at(0x1000), w.k, m, &w, epi, at(0x2000), w.n, nullptr, 0, nullptr) ==
           DLM_EINVAL);   // (fp32 x always takes a workspace)
    EXPECT(dlm_mx_linear(DLM_F32, at(0x1000), w.k, m, &w, epi, at(0x2000), w.n, at(0x100), 255, nullptr) ==
           DLM_ESIZE);
    EXPECT(dlm_mx_linear(DLM_F32, at(0x1000), w.k, m, &w, epi, at(0x2000), w.n, at(0x110), SIZE_MAX, nullptr) ==
           DLM_EINVAL);
  }

  // packed models, their workspaces and caches, and the requests of the cache's calls
  for (int trial = 0; trial < 60; ++trial) {
    const int dh = ri(0, 1) ? 64 : 128, hkv = (int)ri(1, 8), hq = hkv * (int)ri(1, 8), layers = (int)ri(1, 5);
    dlm_config cfg{};
    cfg.n_layers = layers, cfg.d_model = 64 * (int)ri(1, 40), cfg.n_q_heads = hq, cfg.n_kv_heads = hkv;
    cfg.head_dim = dh, cfg.d_ffn = 32 * (int)ri(1, 300), cfg.vocab = 64 * (int)ri(2, 200);
    cfg.mask_id = cfg.vocab - 1, cfg.rms_eps = 1e-5f, cfg.rope_theta = 10000.f, cfg.inv_tau = 1.f;
    cfg.dtype = ri(0, 1) ? DLM_BF16 : DLM_F32;
    auto mx = [&](int n, int k) { return dlm_mx{at(0x10000), reinterpret_cast<uint8_t*>(at(0x20000)), n, k}; };
    const int qd = hq * dh, qkv = qd + 2 * hkv * dh;
    const float* norm = reinterpret_cast<const float*>(at(0x30000));
    std::vector<dlm_layer_mx> ls(layers, dlm_layer_mx{norm, mx(qkv, cfg.d_model), mx(cfg.d_model, qd), norm,
                                                      mx(2 * cfg.d_ffn, cfg.d_model), mx(cfg.d_model, cfg.d_ffn)});
    dlm_weights_mx w{at(0x40000), at(0x50000), norm, ls.data()};
    dlm_model* m = nullptr;
    const dlm_status s = dlm_load_weights_mx(&cfg, &w, &m);
    if (s != DLM_OK) {
      EXPECT(s == DLM_EUNSUPPORTED || s == DLM_EINVAL);
      std::fprintf(stderr, "note: configuration refused: %s\n", dlm_last_error());
      continue;
    }
    size_t ws = 0, less = 0;
    EXPECT(dlm_workspace_bytes(m, 3000, 8, &ws) == DLM_OK && dlm_workspace_bytes(m, 700, 8, &less) == DLM_OK);
    EXPECT(less <= ws);
    ls.back().w_down.k += 1;
    dlm_model* other = nullptr;
    EXPECT(dlm_load_weights_mx(&cfg, &w, &other) == DLM_EINVAL && !other);

    const int slots = (int)ri(1, 70), seq = (int)ri(1, 8192);
    size_t need = 0;
    EXPECT(dlm_kv_cache_alloc_mx(m, slots, seq, nullptr, 0, &need, nullptr) == DLM_OK && need % 256 == 0);
    dlm_cache* c = nullptr;
    EXPECT(dlm_kv_cache_alloc_mx(m, slots, seq, at(0x100000), need - 1, nullptr, &c) == DLM_ESIZE && !c);
    EXPECT(dlm_kv_cache_alloc_mx(m, slots, seq, at(0x100000), need, nullptr, &c) == DLM_OK && c);
    for (int i = 0; i < 300; ++i) {
      const int n_req = (int)ri(1, DLM_MAX_REQ);
      std::vector<dlm_kv_rows> rows(n_req);
      long total = 0;
      for (auto& r : rows) {
        r.seq_len = (int)ri(0, seq), r.slot = (int)ri(0, slots - 1), r.pos0 = 0;
        r.n_rows = ri(0, 2) ? (int)ri(0, 64) : (int)ri(0, 8192);
        total += r.n_rows;
      }
      size_t a = ~(size_t)0;
      EXPECT(dlm_mx_kv_attention_workspace(c, n_req, rows.data(), &a) == DLM_OK && a != ~(size_t)0);
      if (total && a)
        EXPECT(dlm_mx_kv_attention(c, 0, n_req, rows.data(), at(0x1000), at(0x2000), at(0x100), a - 1, nullptr) ==
               DLM_ESIZE);
      // one field of one request out of its range
      dlm_kv_rows& r = rows[ri(0, n_req - 1)];
      const int kind = (int)ri(0, 4);
      if (kind == 0) r.slot = ri(0, 1) ? -1 : slots;
      if (kind == 1) r.seq_len = ri(0, 1) ? -1 : INT32_MAX;
      if (kind == 2) r.n_rows = -1;
      if (kind == 3) r.n_rows = INT32_MAX;
      if (kind == 4) r.slot = INT32_MIN;
      EXPECT(dlm_mx_kv_attention_workspace(c, n_req, rows.data(), &a) != DLM_OK);
      EXPECT(dlm_mx_kv_attention(c, 0, n_req, rows.data(), at(0x1000), at(0x2000), at(0x100), SIZE_MAX, nullptr) !=
             DLM_OK);
      r.pos0 = INT32_MAX;
      EXPECT(dlm_mx_kv_read(c, 0, n_req, rows.data(), at(0x1000), at(0x2000), nullptr) != DLM_OK);
      EXPECT(dlm_mx_kv_append(c, 0, n_req, rows.data(), norm, 1, norm, at(0x2000), nullptr) != DLM_OK);
    }
    dlm_cache_destroy(c);
    dlm_model_destroy(m);
  }
  std::printf("%d failures\n", failures);
  return failures ? 1 : 0;
}
