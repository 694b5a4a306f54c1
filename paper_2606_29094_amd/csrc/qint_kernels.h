// Launch functions of the kernels on 8-bit integers (qint_gemm.h, qint_rowwise.h), internal to
// libdlm.so. An 8-bit matrix [n, k]: signed codes, rows of qint_row(k) bytes whose codes behind k
// are zero, and one fp32 scale for each row; a value is code * scale.
#pragma once

#include "common.h"
#include "mx_kernels.h"

namespace dlm {

constexpr int kQintRow = 128;            // bytes of a row are a multiple of this
__host__ __device__ constexpr int qint_row(int k) { return (k + kQintRow - 1) / kQintRow * kQintRow; }

struct QintView { int8_t* codes; float* scales; int n, k; };

template <typename T>
hipError_t qint_pack(const T* x, long ldx, const QintView& o, hipStream_t st);
template <typename T>
hipError_t qint_unpack(const QintView& x, T* out, long ldo, hipStream_t st);

// acc sx sw in fp32, off by at most three roundings: the token's scale first, except where that
// could leave fp32's range on the way (|acc| < 2^31) though the result does not. Scales that
// packing writes are 2^-126 at least, so nothing falls below the normal numbers on the way. FAST:
// the rows' scales are known to be kQintWide at most.
constexpr float kQintWide = 0x1p96f;
template <bool FAST = false>
__device__ __forceinline__ float qint_value(int acc, float sx, float sw) {
  if constexpr (FAST) return (float)acc * sx * sw;
  const bool wide = sx > kQintWide;
  return (float)acc * (wide ? sw : sx) * (wide ? sx : sw);
}
// (rounded by itself whatever the kernel: no fused multiply-add)
__device__ __forceinline__ float qint_add(float res, float p) {
#pragma clang fp contract(off)
  return res + p;
}

// Rows of fp32 [o.n, o.k]: h + slices 0, 1, .. (T, `splits` of them, stride elements apart, rows
// lda) goes to h_out (may be h or null), its norm times g in 8 bits to o. T = int32_t: the K slices
// that a product left unjoined, h + qint_value(their sum, sx, sw) (sx may be o's scales).
template <typename T>
struct QintNorm {
  const float* h;
  long ldh;
  float* h_out;
  long ldo;
  const T* add;
  int splits;
  long stride, lda;
  const float* g;
  float eps;
  const float* sx = nullptr;
  const float* sw = nullptr;
};
template <typename T>
hipError_t qint_norm(const QintNorm<T>& a, const QintView& o, hipStream_t st);

// What a product does with p[m][n] = sum_k x[m][k] w[n][k] (mode: dlm_qint_epilogue): y = p (fp32,
// or bf16 where wide is false), y = res + p (fp32), or silu(gate) * up; f = w's rows / 2 there.
struct QintOut {
  void* y;
  long ldy;
  const float* res;
  long ldr;
  const float* sx;
  const float* sw;
  int m, n, f;
  int mode;
  bool wide;
};
// A product's way: (gemm) the GEMM tiles, or blocks of 16 rows and columns straight from memory.
// slices > 1: as many K slices [slices, rows, n] go to scratch and are added by a second kernel, or,
// without join, left there.
struct QintPlan {
  bool gemm = false, join = true;
  GemmPlan g{};
  int slices = 1;
  size_t scratch = 0;
};
QintPlan qint_plan(int rows, int n, int k, bool swiglu, int num_cu);
hipError_t qint_matmul(const QintPlan& plan, const QintView& x, const QintView& w, QintOut o, void* scratch,
                     hipStream_t st);

}  // namespace dlm
