// Products of 8-bit integers (qint_kernels.h), p[m][n] = (sum_k x[m][k] w[n][k]) sx[m] sw[n] over
// the codes. The sums are whole numbers in 32 bits (2^14 * 131071 < 2^31): they are the same in any
// order, so a row's result depends neither on the rows beside it nor on how K is split.
#pragma once

#include <algorithm>

#include "../../include/dlm.h"
#include "qint_kernels.h"

namespace dlm {

namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

// 16x16x64 int8: lane l supplies A[row = l%16][k = 16*(l/16) .. +15] and B[col = l%16] of the same
// k; D[row = 4*(l/16) + i][col = l%16] = acc[i].
__device__ __forceinline__ i32x4 mfma16_i8(const u32x4& a, const u32x4& b, const i32x4& c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b),
                                               c, 0, 0, 0);
}

// acc sx sw in fp32, off by at most three roundings: the smaller scale first, so that nothing on
// the way overflows or falls below the normal numbers where the result does not (scales
// that packing writes are 2^-126 at least).
__device__ __forceinline__ float qint_value(int acc, float sx, float sw) {
  const bool less = sx < sw;
  return (float)acc * (less ? sx : sw) * (less ? sw : sx);
}
__device__ __forceinline__ float qint_silu_mul(float g, float u) { return g / (1.f + __expf(-g)) * u; }

__device__ __forceinline__ void qint_store(const QintOut& o, int m, int n, float v) {
  const long at = (long)m * o.ldy + n;
  if (o.wide) reinterpret_cast<float*>(o.y)[at] = v;
  else reinterpret_cast<bf16*>(o.y)[at] = (bf16)v;
}

// Few rows. One block: 16 of them and 16 NF columns (SwiGLU: 8 NF, as many gate fragments as up
// fragments), W waves that take chunks of 512 k in turn and add their sums in LDS. A lane's loads
// are 16 bytes of a row, 64 consecutive bytes over the four lanes that share it; a chunk's are all
// requested before the first is used. The weights are read once, by the one block row that needs
// them; x comes from the caches.
constexpr int kQintChunk = 512;

template <int NF, int W>
__global__ __launch_bounds__(W * 64) void qint_few_kernel(const int8_t* __restrict__ x,
                                                        const int8_t* __restrict__ w, int row_bytes,
                                                        QintOut o) {
  constexpr int U = kQintChunk / 64, H = NF > 1 ? NF / 2 : 1;
  __shared__ i32x4 part[W][NF][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, g = lane >> 4;
  const bool swiglu = o.mode == DLM_QINT_SWIGLU;
  const int n0 = blockIdx.x * (swiglu ? NF * 8 : NF * 16), m0 = blockIdx.y * 16;
  const int n_end = swiglu ? o.f : o.n;          // columns of the output
  // column of fragment f in this lane (of the output; the up fragments are f / 2 .. of it)
  auto out_col = [&](int f) { return n0 + 16 * (swiglu ? f % H : f) + col; };
  auto w_row = [&](int f) {
    return min(out_col(f), n_end - 1) + (swiglu && 2 * f >= NF ? o.f : 0);
  };
  const int8_t* wr[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) wr[f] = w + (long)w_row(f) * row_bytes + 16 * g;
  const int8_t* const xr = x + (long)min(m0 + col, o.m - 1) * row_bytes + 16 * g;

  i32x4 acc[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) acc[f] = i32x4{0, 0, 0, 0};
  for (int k0 = wave * kQintChunk; k0 < row_bytes; k0 += W * kQintChunk) {
    u32x4 b[U][NF], a[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool in = k0 + 64 * u < row_bytes;       // (uniform)
#pragma unroll
      for (int f = 0; f < NF; ++f)
        b[u][f] = in ? *reinterpret_cast<const u32x4*>(wr[f] + k0 + 64 * u) : u32x4{0u, 0u, 0u, 0u};
      a[u] = in ? *reinterpret_cast<const u32x4*>(xr + k0 + 64 * u) : u32x4{0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int f = 0; f < NF; ++f) acc[f] = mfma16_i8(a[u], b[u][f], acc[f]);
  }
#pragma unroll
  for (int f = 0; f < NF; ++f) part[wave][f][lane] = acc[f];
  __syncthreads();

  // wave f finishes fragment f (or pair of gate and up fragments)
  auto sum = [&](int f) {
    i32x4 v = part[0][f][lane];
#pragma unroll
    for (int i = 1; i < W; ++i) v += part[i][f][lane];
    return v;
  };
  if (wave >= (swiglu ? H : NF)) return;
  const int n = out_col(wave);
  if (n >= n_end) return;
  const i32x4 v = sum(wave);
  i32x4 up = {0, 0, 0, 0};
  if (swiglu) up = sum(wave + H);
  const float sw = o.sw[n], su = swiglu ? o.sw[o.f + n] : 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int m = m0 + 4 * g + e;
    if (m >= o.m) continue;
    const float sx = o.sx[m];
    float p = qint_value(v[e], sx, sw);
    if (swiglu) p = qint_silu_mul(p, qint_value(up[e], sx, su));
    if (o.mode == DLM_QINT_ADD) p += o.res[(long)m * o.ldr + n];
    qint_store(o, m, n, p);
  }
}

}  // namespace

QintPlan qint_plan(int rows, int n, int k, bool swiglu, int num_cu) {
  QintPlan p;
  p.nf = swiglu ? 2 : 1;
  return p;
}

hipError_t qint_matmul(const QintPlan& plan, const QintView& x, const QintView& w, QintOut o, void* scratch,
                     hipStream_t st) {
  if (x.n == 0) return hipSuccess;
  const int row_bytes = qint_row(w.k);
  o.m = x.n, o.n = w.n, o.f = w.n / 2, o.sx = x.scales, o.sw = w.scales;
  const bool swiglu = o.mode == DLM_QINT_SWIGLU;
  const dim3 grid(ceil_div(swiglu ? o.f : o.n, plan.nf * (swiglu ? 8 : 16)), ceil_div(o.m, 16));
  if (plan.nf == 2)
    DLM_LAUNCH((qint_few_kernel<2, 8>), grid, dim3(512), 0, st, x.codes, w.codes, row_bytes, o);
  else
    DLM_LAUNCH((qint_few_kernel<1, 8>), grid, dim3(512), 0, st, x.codes, w.codes, row_bytes, o);
  return hipGetLastError();
}

}  // namespace dlm
