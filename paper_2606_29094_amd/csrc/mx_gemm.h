// Products with 4-bit matrices (mx_common.h), y[m][n] = sum_k x[m][k] w[n][k]. Part of
// gemm.hip.
#pragma once

#include "../../include/dlm.h"
#include "kernels.h"
#include "mx_common.h"

namespace dlm {

namespace {

// --------------------------------------------------------------- products --
// x for the product kernel: NP planes of [rows, kp] bf16 (one for bf16 x, three for
// fp32 x: split3), kp = 32 groups, zero from k on.
template <typename T, int NP>
__global__ __launch_bounds__(256) void mx_stage_kernel(const T* __restrict__ x, long ldx, int k,
                                                       int kp, long plane, bf16* __restrict__ out,
                                                       long total) {
  const long at = (long)blockIdx.x * 256 + threadIdx.x;
  if (at >= total) return;
  const long row = at / kp;
  const int c = (int)(at - row * kp);
  const float v = c < k ? to_f32(x[row * ldx + c]) : 0.f;
  if constexpr (NP == 1) {
    out[at] = (bf16)v;
  } else {
    bf16 a, b, d;
    split3(v, a, b, d);
    out[at] = a;
    out[at + plane] = b;
    out[at + 2 * plane] = d;
  }
}

__device__ __forceinline__ float silu_mul(float g, float u) { return g / (1.f + __expf(-g)) * u; }

// One block: 16 MT rows x 16 NF columns, W waves that take the 128-wide k chunks
// in turn and add their partial sums in LDS, in wave order. In a chunk lane l reads
// the 32 codes of group l / 16 of weight row l % 16 as one 16-byte load; the MFMA
// j = 0..3 multiplies their dword j with the same eight elements of x (the order
// of k inside a chunk is the same on both sides). The weights are read once, by
// the one block row that needs them; x comes from the caches.
template <int MT, int NF, int W, int NP>
__global__ __launch_bounds__(W * 64) void mx_linear_kernel(MxLinear a) {
  __shared__ f32x4 part[W][MT * NF][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, g = lane >> 4;
  const int n0 = blockIdx.x * (a.swiglu ? NF * 8 : NF * 16), m0 = blockIdx.y * MT * 16;
  const int n_end = a.swiglu ? a.w.n / 2 : a.w.n;   // columns of the output

  const uint8_t* wc[NF];
  const uint8_t* ws[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) {
    int n;
    if (a.swiglu) {   // the first half of the fragments are gate rows, the second the up rows
      n = min(n0 + 16 * (f % (NF > 1 ? NF / 2 : 1)) + col, n_end - 1) + (2 * f >= NF ? n_end : 0);
    } else {
      n = min(n0 + 16 * f + col, n_end - 1);
    }
    wc[f] = a.w.codes + ((long)n * a.w.groups + g) * 16;
    ws[f] = a.w.scales + (long)n * a.w.scale_ld + g;
  }
  const bf16* xr[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t)
    xr[t] = a.x + (long)min(m0 + 16 * t + col, a.m - 1) * a.ldx + 32 * g;

  f32x4 acc[MT][NF];
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int f = 0; f < NF; ++f) acc[t][f] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int chunks = (a.w.groups + 3) / 4;
  for (int c = wave; c < chunks; c += W) {
    const bool ok = 4 * c + g < a.w.groups;
    u32x4 codes[NF];
    float s[NF];
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      codes[f] = ok ? *reinterpret_cast<const u32x4*>(wc[f] + (long)c * 64) : u32x4{0u, 0u, 0u, 0u};
      s[f] = mx_scale(ok ? ws[f][4 * c] : 127u);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      bf16x8 b[NF];
#pragma unroll
      for (int f = 0; f < NF; ++f) b[f] = mx_bf16x8(codes[f][j], s[f]);
      const bool in = 128 * c + 32 * g + 8 * j < a.k;
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          bf16x8 v = {};
          if (in) v = *reinterpret_cast<const bf16x8*>(xr[t] + p * a.plane + 128 * c + 8 * j);
#pragma unroll
          for (int f = 0; f < NF; ++f) acc[t][f] = mfma16_bf16(v, b[f], acc[t][f]);
        }
    }
  }
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int f = 0; f < NF; ++f) part[wave][t * NF + f][lane] = acc[t][f];
  __syncthreads();

  // fragment (or gate / up pair of fragments) i of the tile is wave i % W's
  auto sum = [&](int i) {
    f32x4 v = part[0][i][lane];
#pragma unroll
    for (int w = 1; w < W; ++w) v += part[w][i][lane];
    return v;
  };
  if (a.swiglu) {
    constexpr int H = NF > 1 ? NF / 2 : 1;
    for (int i = wave; i < MT * H; i += W) {
      const int t = i / H, f = i % H;
      const f32x4 gate = sum(t * NF + f), up = sum(t * NF + f + NF / 2);
      const int n = n0 + 16 * f + col;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int m = m0 + 16 * t + 4 * g + e;
        if (m >= a.m || n >= n_end) continue;
        const float v = silu_mul(gate[e], up[e]);
        if constexpr (NP == 1) reinterpret_cast<bf16*>(a.y)[(long)m * a.ldy + n] = (bf16)v;
        else reinterpret_cast<float*>(a.y)[(long)m * a.ldy + n] = v;
      }
    }
    return;
  }
  for (int i = wave; i < MT * NF; i += W) {
    const int t = i / NF, f = i % NF;
    const f32x4 v = sum(i);
    const int n = n0 + 16 * f + col;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int m = m0 + 16 * t + 4 * g + e;
      if (m >= a.m || n >= n_end) continue;
      float* o = reinterpret_cast<float*>(a.y) + (long)m * a.ldy + n;
      *o = a.add ? *o + v[e] : v[e];
    }
  }
}

template <int NP>
hipError_t launch_linear(const MxLinear& a, hipStream_t st) {
  const int n_out = a.swiglu ? a.w.n / 2 : a.w.n;
#define MX_LAUNCH(MT_, NF_, W_)                                                              \
  do {                                                                                       \
    const int bn_ = a.swiglu ? NF_ * 8 : NF_ * 16;                                           \
    DLM_LAUNCH((mx_linear_kernel<MT_, NF_, W_, NP>),                                         \
               dim3(ceil_div(n_out, bn_), ceil_div(a.m, MT_ * 16)), dim3(W_ * 64), 0, st, a); \
    return hipGetLastError();                                                                \
  } while (0)
  if (a.m <= 16) MX_LAUNCH(1, 2, 8);
  if (a.m <= 32) MX_LAUNCH(2, 2, 8);
  MX_LAUNCH(4, 2, 8);
#undef MX_LAUNCH
}

}  // namespace

namespace {
template <typename T>
bool direct_x(const T* x, long ldx, int k) {
  return sizeof(T) == 2 && k % 8 == 0 && ldx % 8 == 0 && reinterpret_cast<uintptr_t>(x) % 16 == 0;
}
}  // namespace

size_t mx_linear_scratch(int elem, int rows, int k, bool aligned) {
  if (elem == 2 && aligned) return 0;
  return (size_t)rows * ceil_div(k, kMxGroup) * kMxGroup * 2 * (elem == 2 ? 1 : 3);
}

template <typename T>
hipError_t mx_linear(const T* x, long ldx, int rows, const MxView& w, int k, bool swiglu, bool add,
                     void* y, long ldy, void* scratch, hipStream_t st) {
  if (rows <= 0 || w.n <= 0) return hipSuccess;
  MxLinear a{};
  a.w = w, a.m = rows, a.k = k, a.swiglu = swiglu, a.add = add, a.y = y, a.ldy = ldy;
  if constexpr (sizeof(T) == 2) {
    if (direct_x(x, ldx, k)) {
      a.x = x, a.ldx = ldx;
      return launch_linear<1>(a, st);
    }
  }
  constexpr int NP = sizeof(T) == 2 ? 1 : 3;
  const int kp = w.groups * kMxGroup;
  const long total = (long)rows * kp;
  bf16* xs = reinterpret_cast<bf16*>(scratch);
  DLM_LAUNCH((mx_stage_kernel<T, NP>), dim3((unsigned)((total + 255) / 256)), dim3(256), 0, st, x,
             ldx, k, kp, total, xs, total);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  a.x = xs, a.ldx = kp, a.plane = total, a.k = kp;
  return launch_linear<NP>(a, st);
}

// Above this many rows the matrix is unpacked once and goes through the GEMM kernels.
constexpr int kMxDirectRows = 256;

MxPlan mx_plan(int elem, int rows, int n, int k, bool swiglu, bool aligned, int num_cu) {
  MxPlan p;
  if (aligned && rows > kMxDirectRows && k % (16 / elem) == 0 && (!swiglu || n % 32 == 0)) {
    p.gemm = true;
    p.g = gemm_plan(elem, rows, n, k, false, num_cu, !swiglu, true, !swiglu);
    p.scratch = (size_t)n * k * elem;
  } else {
    p.scratch = mx_linear_scratch(elem, rows, k, aligned && k % 8 == 0);
  }
  return p;
}

template <typename T>
hipError_t mx_matmul(const MxPlan& plan, const T* x, long ldx, int rows, const MxView& w, int k,
                     int epilogue, void* y, long ldy, void* scratch, hipStream_t st) {
  const bool swiglu = epilogue == DLM_MX_SWIGLU, add = epilogue == DLM_MX_ADD;
  if (!plan.gemm) return mx_linear<T>(x, ldx, rows, w, k, swiglu, add, y, ldy, scratch, st);
  T* dense = reinterpret_cast<T*>(scratch);
  const hipError_t e = mx_unpack<T>(w, k, dense, k, st);
  if (e != hipSuccess) return e;
  if (swiglu)
    return gemm_swiglu<T>(plan.g, x, (int)ldx, dense, k, rows, w.n / 2, k, reinterpret_cast<T*>(y),
                          (int)ldy, st);
  float* c = reinterpret_cast<float*>(y);
  return add ? gemm_add_f32<T>(plan.g, x, (int)ldx, dense, k, rows, w.n, k, c, (int)ldy, st)
             : gemm_store_f32<T>(plan.g, x, (int)ldx, dense, k, rows, w.n, k, c, (int)ldy, st);
}

#define INST(T)                                                                                 \
  template hipError_t mx_linear<T>(const T*, long, int, const MxView&, int, bool, bool, void*,  \
                                   long, void*, hipStream_t);                                  \
  template hipError_t mx_matmul<T>(const MxPlan&, const T*, long, int, const MxView&, int, int, \
                                   void*, long, void*, hipStream_t);
INST(bf16)
INST(float)
#undef INST

}  // namespace dlm
