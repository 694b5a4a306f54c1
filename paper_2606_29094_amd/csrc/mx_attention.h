// Attention over a cache in 4 bits (mx_common.h). Part of attention.hip.
#pragma once

#include <algorithm>

#include "kernels.h"
#include "mx_common.h"

namespace dlm {

namespace {

// --------------------------------------------------------------- attention --
// The query rows of a request that read one key/value head are numbered (row,
// query head), heads fastest: item t is row t / gh, head t % gh of the group.
struct MxAttn {
  MxKv kv;
  int hq, hkv, splits;
  float c;               // log2(e) / sqrt(dh)
  float* po;             // splits > 1: partial outputs [split][row][head][dh], unnormalised,
  float2* ml;            // and [split][row][head] (largest score, sum of weights)
};

typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kLdsPad = 32;   // bytes: rows of V start 8 banks apart

// eight keys (8 g .. 8 g + 7 of the 32 rows at `rows`) of V column d0 + lane % 16, from
// rows of `stride` bytes: two transposing reads, each of which hands a 16-lane
// group the columns of a [4 keys][16 columns] block
__device__ __forceinline__ bf16x8 v_columns(const char* rows, int stride, int d0, int lane) {
  typedef __attribute__((address_space(3))) s16x4* lds_t;
  const char* at = rows + (8 * (lane >> 4) + ((lane & 15) >> 2)) * stride + d0 * 2 + (lane & 3) * 8;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)at);
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(at + 4 * stride));
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  return __builtin_bit_cast(bf16x8, s16x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
}

// Waves that split the keys: one block = 16 QT items of one key/value head, wave w
// takes the 64-key tiles w, w + W, ... of the block's key range, each with its own
// online softmax, merged in LDS at the end. Scores as S^T = K Q^T (16x16x32 MFMA, keys
// as the A operand straight from the codes in registers: lane l holds group l / 16 of key
// l % 16, whose dword j is the A fragment of step j), so a lane owns one query and 16
// keys; the keys of a tile are dealt to the rows of S^T so that a lane's weights are
// the B operand of O^T = V^T P^T as they stand. V is unpacked into the wave's part of
// LDS key by key (its scales belong to keys) and read back transposed.
// NP bf16 terms for each query element and weight: 1 for bf16 queries (a weight is then
// off by at most 2^-9 of itself, the rounding the output gets too), 3 for fp32 ones.
template <typename T, int DH, int QT, int W>
__global__ __launch_bounds__(W * 64) void mx_attn_kernel(StepPlan p, const T* __restrict__ q,
                                                         MxAttn a, T* __restrict__ out) {
  constexpr int NP = sizeof(T) == 2 ? 1 : 3;
  constexpr int GROUPS = DH / kMxGroup;
  constexpr int KS = DH / 32;               // MFMA steps over dh
  constexpr int PER = DH / 4;               // elements of a key in a lane: 32 or 16
  constexpr int DT = DH / 16;
  constexpr int STRIDE = DH * 2 + kLdsPad;
  constexpr int VBYTES = 64 * STRIDE;
  static_assert(VBYTES >= QT * 16 * DH * 4, "the merge reuses the wave's part");
  __shared__ __attribute__((aligned(16))) char smem[W * VBYTES];
  __shared__ float2 stat[W][QT * 16];

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, g = lane >> 4;
  const int gh = a.hq / a.hkv;
  const int tile = blockIdx.x;
  const int r = plan_req_of_tile(p, tile);
  const ReqPlan& rq = p.r[r];
  const int item0 = (tile - rq.tile0) * 16 * QT, items = rq.nrows * gh;
  const int head = blockIdx.y;
  const int split = blockIdx.z;
  const int len = rq.seq_len;
  const int tiles = ceil_div(len, 64), per = ceil_div(tiles, a.splits);
  const int t0 = min(split * per, tiles), t1 = min(t0 + per, tiles);

  // queries: B fragment of step j is elements PER g + 8 j .. of the item's query
  bf16x8 qf[QT][KS][NP];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int it = min(item0 + 16 * t + col, items - 1);
    const T* src = q + ((long)(rq.row0 + it / gh) * a.hq + head * gh + it % gh) * DH + PER * g;
#pragma unroll
    for (int j = 0; j < KS; ++j) {
      if constexpr (NP == 1) {
        qf[t][j][0] = *reinterpret_cast<const bf16x8*>(src + 8 * j);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          bf16 hi, mid, lo;
          split3(to_f32(src[8 * j + e]), hi, mid, lo);
          qf[t][j][0][e] = hi;
          qf[t][j][1][e] = mid;
          qf[t][j][2][e] = lo;
        }
      }
    }
  }
  const long base = ((long)rq.slot * a.hkv + head) * a.kv.s_max;
  const uint8_t* kc = a.kv.kc + base * (DH / 2);
  const uint8_t* vc = a.kv.vc + base * (DH / 2);
  const uint8_t* ks = a.kv.ks + base * GROUPS;
  const uint8_t* vs = a.kv.vs + base * GROUPS;
  char* vrows = smem + wave * VBYTES;

  f32x4 o[DT][QT];
  float m[QT], l[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m[t] = -INFINITY;
    l[t] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  for (int kt = t0 + wave; kt < t1; kt += W) {
    const int k0 = kt * 64;
    // V: whole groups, key by key (a slot holds a multiple of 64 positions; those
    // behind the sequence become zeros, whatever they hold)
    constexpr int VN = 64 * GROUPS / 64;
#pragma unroll
    for (int u = 0; u < VN; ++u) {
      const int at = u * 64 + lane, key = at / GROUPS, gr = at % GROUPS;
      u32x4 c = reinterpret_cast<const u32x4*>(vc)[(long)k0 * GROUPS + at];
      uint32_t e = vs[(long)k0 * GROUPS + at];
      if (k0 + key >= len) c = u32x4{0u, 0u, 0u, 0u}, e = 127u;
      const float s = mx_scale(e);
#pragma unroll
      for (int w = 0; w < 4; ++w)
        *reinterpret_cast<bf16x8*>(vrows + key * STRIDE + gr * 64 + w * 16) = mx_bf16x8(c[w], s);
    }
    // S^T: row x of key tile n is key 32 (n / 2) + 8 (x / 4) + 4 (n % 2) + x % 4
    f32x4 s[4][QT];
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int key = k0 + 32 * (n >> 1) + 8 * (col >> 2) + 4 * (n & 1) + (col & 3);
      uint32_t c[PER / 8];
      if constexpr (PER == 32) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(kc + (long)key * 64 + g * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) c[j] = v[j];
      } else {
        const u32x2 v = *reinterpret_cast<const u32x2*>(kc + (long)key * 32 + g * 8);
        c[0] = v[0], c[1] = v[1];
      }
      const float sc = mx_scale(ks[(long)key * GROUPS + g * PER / kMxGroup]);
#pragma unroll
      for (int t = 0; t < QT; ++t) s[n][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < KS; ++j) {
        const bf16x8 kf = mx_bf16x8(c[j], sc);
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int w = NP - 1; w >= 0; --w) s[n][t] = mfma16_bf16(kf, qf[t][j][w], s[n][t]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (k0 + 32 * (n >> 1) + 8 * g + 4 * (n & 1) + i >= len)
#pragma unroll
          for (int t = 0; t < QT; ++t) s[n][t][i] = -INFINITY;
    }
    bf16x8 pf[QT][2][NP];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      float mx = m[t];
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[n][t][i]);
      mx = fmaxf(mx, __shfl_xor(mx, 16, kWave));
      mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
      const float ref = mx == -INFINITY ? 0.f : mx;   // (no key with a score yet)
      const float keep = exp2f((m[t] - ref) * a.c);
      m[t] = mx;
      l[t] *= keep;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d][t] *= keep;
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float w = exp2f((s[n][t][i] - ref) * a.c);
          l[t] += w;
          const int e = 4 * (n & 1) + i;
          if constexpr (NP == 1) {
            pf[t][n >> 1][0][e] = (bf16)w;
          } else {
            bf16 hi, mid, lo;
            split3(w, hi, mid, lo);
            pf[t][n >> 1][0][e] = hi;
            pf[t][n >> 1][1][e] = mid;
            pf[t][n >> 1][2][e] = lo;
          }
        }
    }
    // the wave's own stores to LDS, before it reads them
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const bf16x8 vf = v_columns(vrows + 32 * h * STRIDE, STRIDE, 16 * d, lane);
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int w = NP - 1; w >= 0; --w) o[d][t] = mfma16_bf16(vf, pf[t][h][w], o[d][t]);
      }
    // and its reads, before the next tile's stores
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }

  // merge the waves: item x of the block, [x][dh] fp32 in each wave's part
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    l[t] += __shfl_xor(l[t], 16, kWave);
    l[t] += __shfl_xor(l[t], 32, kWave);
    if (g == 0) stat[wave][16 * t + col] = make_float2(m[t], l[t]);
#pragma unroll
    for (int d = 0; d < DT; ++d)
      *reinterpret_cast<f32x4*>(vrows + ((16 * t + col) * DH + 16 * d + 4 * g) * 4) = o[d][t];
  }
  __syncthreads();
  constexpr int QUADS = DH / 4;
  for (int i = threadIdx.x; i < 16 * QT * QUADS; i += W * 64) {
    const int x = i / QUADS, d = i % QUADS * 4;
    if (item0 + x >= items) continue;
    float mx = stat[0][x].x;
#pragma unroll
    for (int w = 1; w < W; ++w) mx = fmaxf(mx, stat[w][x].x);
    const float ref = mx == -INFINITY ? 0.f : mx;
    float sum = 0.f;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = exp2f((stat[w][x].x - ref) * a.c);
      sum += stat[w][x].y * f;
      v += *reinterpret_cast<const f32x4*>(smem + w * VBYTES + (x * DH + d) * 4) * f;
    }
    const int it = item0 + x;
    const long at = (long)(rq.row0 + it / gh) * a.hq + head * gh + it % gh;
    if (a.splits > 1) {
      const long rows = (long)p.n_rows * a.hq;
      *reinterpret_cast<f32x4*>(a.po + (split * rows + at) * DH + d) = v;
      // a row over no keys: weight one on an output of zeros
      if (d == 0)
        a.ml[split * rows + at] = len == 0 && split == 0 ? make_float2(0.f, 1.f) : make_float2(mx, sum);
      continue;
    }
    const float inv = len > 0 ? 1.f / sum : 0.f;
    typedef T T4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<T4*>(out + at * DH + d) = T4{from_f32<T>(v[0] * inv), from_f32<T>(v[1] * inv),
                                                   from_f32<T>(v[2] * inv), from_f32<T>(v[3] * inv)};
  }
}

// The key splits of each (row, head), added in order. A split without keys has
// weight zero.
template <typename T, int DH>
__global__ __launch_bounds__(256) void mx_merge_kernel(MxAttn a, long items, T* __restrict__ out) {
  constexpr int QUADS = DH / 4;
  const long at = ((long)blockIdx.x * 256 + threadIdx.x) / QUADS;
  const int d = threadIdx.x % QUADS * 4;
  if (at >= items) return;
  float mx = -INFINITY;
  for (int s = 0; s < a.splits; ++s) mx = fmaxf(mx, a.ml[s * items + at].x);
  const float ref = mx == -INFINITY ? 0.f : mx;
  float sum = 0.f;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < a.splits; ++s) {
    const float2 ml = a.ml[s * items + at];
    const float f = exp2f((ml.x - ref) * a.c);
    sum += ml.y * f;
    v += *reinterpret_cast<const f32x4*>(a.po + (s * items + at) * DH + d) * f;
  }
  const float inv = 1.f / sum;
  typedef T T4 __attribute__((ext_vector_type(4)));
  *reinterpret_cast<T4*>(out + at * DH + d) = T4{from_f32<T>(v[0] * inv), from_f32<T>(v[1] * inv),
                                                 from_f32<T>(v[2] * inv), from_f32<T>(v[3] * inv)};
}

constexpr int kMxSplits = 16;

template <typename T, int DH>
hipError_t launch_attention(const StepPlan& p, const T* q, const MxAttn& a, T* out, hipStream_t st) {
  constexpr int QT = sizeof(T) == 2 ? 2 : 1, W = 4;
  const int gh = a.hq / a.hkv;
  const StepPlan t = plan_with_tiles(p, [&](int n) { return ceil_div(n * gh, 16 * QT); });
  if (t.n_tiles == 0) return hipSuccess;
  DLM_LAUNCH((mx_attn_kernel<T, DH, QT, W>), dim3(t.n_tiles, a.hkv, a.splits), dim3(W * 64), 0, st, t, q,
             a, out);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  const long items = (long)p.n_rows * a.hq;
  DLM_LAUNCH((mx_merge_kernel<T, DH>), dim3((unsigned)((items * (DH / 4) + 255) / 256)), dim3(256), 0,
             st, a, items, out);
  return hipGetLastError();
}

}  // namespace

size_t mx_attention_scratch(int rows, int hq, int dh, int splits) {
  if (splits <= 1) return 0;
  return (size_t)splits * rows * hq * (dh * sizeof(float) + sizeof(float2));
}

int mx_attention_splits(const StepPlan& p, int hq, int hkv, int dh, size_t elem,
                        size_t scratch_bytes, int num_cu) {
  const int gh = hq / hkv, rows = elem == 2 ? 32 : 16;
  long blocks = 0;
  int longest = 0;
  for (int r = 0; r < p.n_req; ++r) {
    blocks += (long)hkv * ceil_div(p.r[r].nrows * gh, rows);
    longest = std::max(longest, p.r[r].nrows ? p.r[r].seq_len : 0);
  }
  if (blocks == 0) return 1;
  const int tiles = ceil_div(longest, 64);
  int s = (int)std::min<long>(kMxSplits, num_cu / blocks);
  s = std::min(s, tiles / 8);
  while (s > 1 && mx_attention_scratch(p.n_rows, hq, dh, s) > scratch_bytes) --s;
  return std::max(s, 1);
}

template <typename T>
hipError_t mx_attention(const StepPlan& p, const T* q, const MxKv& kv, int hq, int hkv, int dh,
                        T* out, int splits, float* scratch, hipStream_t st) {
  if (hkv < 1 || hq % hkv != 0 || splits < 1 || splits > kMxSplits || (splits > 1 && !scratch))
    return hipErrorInvalidValue;
  if (p.n_rows == 0) return hipSuccess;
  MxAttn a{kv, hq, hkv, splits, 1.4426950408889634f / sqrtf((float)dh), scratch,
           reinterpret_cast<float2*>(scratch + (size_t)splits * p.n_rows * hq * dh)};
  if (dh == 128) return launch_attention<T, 128>(p, q, a, out, st);
  if (dh == 64) return launch_attention<T, 64>(p, q, a, out, st);
  return hipErrorInvalidValue;
}

#define INST(T)                                                                                  \
  template hipError_t mx_attention<T>(const StepPlan&, const T*, const MxKv&, int, int, int, T*, \
                                      int, float*, hipStream_t);
INST(bf16)
INST(float)
#undef INST

}  // namespace dlm
