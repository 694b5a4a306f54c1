// 8-bit integers row by row (qint_kernels.h): packing, unpacking, and the norm that packs what it
// makes. Part of rowwise.hip.
#pragma once

#include <float.h>

#include <algorithm>
#include <type_traits>

#include "qint_kernels.h"

namespace dlm {

namespace {

// A row's largest magnitude A decides its scale, max(A / 127, 2^-126), and its codes, the
// integers nearest to x min(127 / A, 2^126) (ties to the even one). The floor keeps 127 / A
// finite and the scale a normal number for rows of zeros and of the smallest magnitudes.
//
// The codes are decided in 64 bits, x r with r = 127 / A rounded. That product is off by up to
// 2^-46, which alone would let the rounding of r decide exact middles (x = A / 2 is always one, 63.5:
// its code was 63 instead of 64 for 69 of the 128 bf16 mantissas of A). So it is rounded twice: to a
// whole number of 2^-42, which a middle meets exactly, then to an integer, ties to the even one, left
// in the low bits of the sum. Of 24-bit x and A any other quotient lies 2^-32 from a middle or more
// (254 x - (2 c + 1) A is a multiple of 2^-7 steps of A, 2 A less than 2^25 of them): the codes of
// packing are those of the exact quotient, for every row. (In 32 bits the product is off by up to
// 2^-17. The second addition costs no time: 4096 x 18944 bf16 packed and read back 90 us with
// one or two.)
constexpr double kQintRound = 6755399441055744.0;   // 1.5 * 2^52
constexpr double kQintGrid = 1536.0;                 // 1.5 * 2^10
constexpr double kQintMinScale = 0x1p-126;

__device__ __forceinline__ int qint_code(double x, double r) {
  return __double2loint(__builtin_fma(x, r, kQintGrid) + (kQintRound - kQintGrid));
}
__device__ __forceinline__ uint32_t qint_bytes4(int a, int b, int c, int d) {
  const uint32_t lo = __builtin_amdgcn_perm((uint32_t)b, (uint32_t)a, 0x0c0c0400u);
  const uint32_t hi = __builtin_amdgcn_perm((uint32_t)d, (uint32_t)c, 0x0c0c0400u);
  return lo | hi << 16;
}

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}
__device__ __forceinline__ double wave_max64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmax(v, __shfl_xor(v, o, kWave));
  return v;
}

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

// elements [at, at + V) of a row of k, zeros behind it. VEC: whole vectors of V elements.
template <int V, bool VEC, typename T>
__device__ __forceinline__ void load_row(const T* row, int at, int k, float (&v)[V]) {
  typedef T vt __attribute__((ext_vector_type(V)));
  if constexpr (VEC) {
    vt x = vt{};
    if (at < k) x = *reinterpret_cast<const vt*>(row + at);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = to_f32((T)x[i]);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = at + i < k ? to_f32(row[at + i]) : 0.f;
  }
}

// ------------------------------------------------------------ pack, unpack --
// One row a block, C vectors of 16 bytes a thread that stay in registers between the search
// for the largest magnitude and the rounding (LOOP: rows longer than that are read twice).
// Bound by memory.
template <typename T, bool VEC, int C, bool LOOP>
__global__ __launch_bounds__(1024) void qint_pack_kernel(const T* __restrict__ x, long ldx, QintView o) {
  constexpr int V = 16 / sizeof(T);
  __shared__ uint32_t red[16];
  const int row_bytes = qint_row(o.k), step = blockDim.x * V * C;
  for (long row = blockIdx.x; row < o.n; row += gridDim.x) {
    const T* const src = x + row * ldx;
    float v[C][V];
    uint32_t amax = 0;
    auto load = [&](int at0) {
#pragma unroll
      for (int c = 0; c < C; ++c) load_row<V, VEC>(src, at0 + (c * blockDim.x + threadIdx.x) * V, o.k, v[c]);
    };
    for (int at0 = 0; at0 < (LOOP ? row_bytes : 1); at0 += step) {
      load(at0);
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) amax = max(amax, __float_as_uint(v[c][i]) & 0x7fffffffu);
    }
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, s, kWave));
    if (blockDim.x > kWave) {
      if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = amax;
      __syncthreads();
      for (int w = 0; w < (int)blockDim.x / kWave; ++w) amax = max(amax, red[w]);
      __syncthreads();
    }
    const bool bad = amax >= 0x7f800000u;    // an infinity or a NaN
    const double a = (double)__uint_as_float(amax);
    const double r = fmin(127.0 / a, 1 / kQintMinScale);
    if (threadIdx.x == 0)
      o.scales[row] = bad ? __uint_as_float(0x7fc00000u) : (float)fmax(a / 127.0, kQintMinScale);
    int8_t* const codes = o.codes + row * row_bytes;
    for (int at0 = 0; at0 < (LOOP ? row_bytes : 1); at0 += step) {
      if (LOOP) load(at0);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int at = at0 + (c * blockDim.x + threadIdx.x) * V;
        if (at >= row_bytes) continue;
        uint32_t q[V / 4];
#pragma unroll
        for (int i = 0; i < V / 4; ++i)
          q[i] = bad ? 0u : qint_bytes4(qint_code(v[c][4 * i], r), qint_code(v[c][4 * i + 1], r),
                                      qint_code(v[c][4 * i + 2], r), qint_code(v[c][4 * i + 3], r));
        if constexpr (V == 8) *reinterpret_cast<u32x2*>(codes + at) = u32x2{q[0], q[1]};
        else *reinterpret_cast<uint32_t*>(codes + at) = q[0];
      }
    }
  }
}

// A thread makes 16 bytes of the wide matrix. Bound by memory.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void qint_unpack_kernel(QintView x, T* __restrict__ out, long ldo) {
  constexpr int V = 16 / sizeof(T), U = 4;
  typedef T vt __attribute__((ext_vector_type(V)));
  const int row_bytes = qint_row(x.k), at0 = (blockIdx.x * 256 * U + threadIdx.x) * V;
  for (long row = blockIdx.y; row < x.n; row += gridDim.y) {
    const float s = x.scales[row];
    u32x2 q[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = at0 + u * 256 * V;
      if (at >= x.k) continue;
      const int8_t* p = x.codes + row * row_bytes + at;
      if constexpr (V == 8) q[u] = *reinterpret_cast<const u32x2*>(p);
      else q[u][0] = *reinterpret_cast<const uint32_t*>(p);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = at0 + u * 256 * V;
      if (at >= x.k) continue;
      vt v;
#pragma unroll
      for (int i = 0; i < V; ++i)
        v[i] = from_f32<T>((float)(int8_t)(q[u][i / 4] >> (8 * (i % 4))) * s);
      T* p = out + row * ldo + at;
      if constexpr (VEC) {
        *reinterpret_cast<vt*>(p) = v;
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (at + i < x.k) p[i] = v[i];
      }
    }
  }
}

// -------------------------------------------------------------------- norm --
// One row a block, C float4 of it a thread, kept in registers (LOOP: rows longer than that go
// through memory twice). y = h' g inv with inv = 1 / sqrt(mean h'^2 + eps), all in 64 bits; inv
// is the same for the whole row, so the codes follow from t = h' g alone, which 64 bits hold
// exactly: x 127 / max|t|. The statistic and the largest |t| are found in one pass, and one
// exchange over the block serves both; only the scale needs inv. Bound by memory.
// S: slices whose loads are issued together (-1: a.splits of them, one at a time).
template <typename T, int S, bool VEC, int C, bool LOOP>
__global__ __launch_bounds__(1024) void qint_norm_kernel(QintNorm<T> a, QintView o) {
  __shared__ double red[2][16];
  const int row_bytes = qint_row(o.k), step = blockDim.x * 4 * C, k = o.k;
  for (long row = blockIdx.x; row < o.n; row += gridDim.x) {
    const float* const src = a.h + row * a.ldh;
    const T* const part = a.add + row * a.lda;
    float* const dst = a.h_out ? a.h_out + row * a.ldo : nullptr;
    float v[C][4];
    auto at_of = [&](int at0, int c) { return at0 + (c * (int)blockDim.x + (int)threadIdx.x) * 4; };
    auto load = [&](int at0) {
#pragma unroll
      for (int c = 0; c < C; ++c) load_row<4, VEC>(src, at_of(at0, c), k, v[c]);
      if constexpr (std::is_same<T, int32_t>::value) {
        i32x4 sum[C];
        float w[C][4];
#pragma unroll
        for (int c = 0; c < C; ++c) sum[c] = i32x4{0, 0, 0, 0}, load_row<4, VEC>(a.sw, at_of(at0, c), k, w[c]);
#pragma unroll 2
        for (int s = 0; s < a.splits; ++s)
#pragma unroll
          for (int c = 0; c < C; ++c) {
            const int at = at_of(at0, c);
            const int32_t* const p = part + s * a.stride + at;
            if constexpr (VEC) {
              if (at < k) sum[c] += *reinterpret_cast<const i32x4*>(p);
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (at + i < k) sum[c][i] += p[i];
            }
          }
        const float x = a.sx[row];
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) v[c][i] = qint_add(v[c][i], qint_value(sum[c][i], x, w[c][i]));
      } else if constexpr (S > 0) {
        float p[S][C][4];
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
          for (int c = 0; c < C; ++c) load_row<4, VEC>(part + s * a.stride, at_of(at0, c), k, p[s][c]);
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
          for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[c][i] += p[s][c][i];
      } else if constexpr (S < 0) {
        for (int s = 0; s < a.splits; ++s) {
          float p[C][4];
#pragma unroll
          for (int c = 0; c < C; ++c) load_row<4, VEC>(part + s * a.stride, at_of(at0, c), k, p[c]);
#pragma unroll
          for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[c][i] += p[c][i];
        }
      }
    };
    auto gain = [&](int at0, float (&g)[C][4]) {
#pragma unroll
      for (int c = 0; c < C; ++c) load_row<4, VEC>(a.g, at_of(at0, c), k, g[c]);
    };
    float g[C][4];
    double ss = 0, tmax = 0;
    bool bad = false;
    for (int at0 = 0; at0 < (LOOP ? row_bytes : 1); at0 += step) {
      load(at0);
      gain(at0, g);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int at = at_of(at0, c);
        if (dst) {
          if constexpr (VEC) {
            if (at < k) *reinterpret_cast<f32x4*>(dst + at) = f32x4{v[c][0], v[c][1], v[c][2], v[c][3]};
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (at + i < k) dst[at + i] = v[c][i];
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const double x = v[c][i], t = fabs(x * (double)g[c][i]);
          ss = __builtin_fma(x, x, ss);
          tmax = fmax(tmax, t);
          bad |= !(t <= DBL_MAX);      // (fmax drops a NaN)
        }
      }
    }
    if (bad) tmax = INFINITY;
    ss = wave_sum64(ss);
    tmax = wave_max64(tmax);
    const int waves = blockDim.x / kWave;
    if (waves > 1) {
      const int w = threadIdx.x / kWave;
      if (threadIdx.x % kWave == 0) red[0][w] = ss, red[1][w] = tmax;
      __syncthreads();
      ss = red[0][0], tmax = red[1][0];
      for (int i = 1; i < waves; ++i) ss += red[0][i], tmax = fmax(tmax, red[1][i]);
      __syncthreads();
    }
    const double inv = 1.0 / sqrt(ss / k + (double)a.eps);
    const float scale = (float)fmax(tmax * inv / 127.0, kQintMinScale);
    bad = !(scale <= FLT_MAX) || !(ss <= DBL_MAX);
    const double r = fmin(127.0 / tmax, inv / kQintMinScale);
    // (a.sx may be these scales: every lane has read its row's by the exchange above)
    if (threadIdx.x == 0) o.scales[row] = bad ? __uint_as_float(0x7fc00000u) : scale;
    int8_t* const codes = o.codes + row * row_bytes;
    for (int at0 = 0; at0 < (LOOP ? row_bytes : 1); at0 += step) {
      if constexpr (LOOP) {
        if (dst) {     // (the thread's own stores; h itself may be what they replaced)
#pragma unroll
          for (int c = 0; c < C; ++c) load_row<4, VEC>((const float*)dst, at_of(at0, c), k, v[c]);
        } else {
          load(at0);
        }
        gain(at0, g);
      }
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int at = at_of(at0, c);
        if (at >= row_bytes) continue;
        int q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = qint_code((double)v[c][i] * (double)g[c][i], r);
        *reinterpret_cast<uint32_t*>(codes + at) = bad ? 0u : qint_bytes4(q[0], q[1], q[2], q[3]);
      }
    }
  }
}

constexpr int kQintBlocks = 1 << 20;     // rows beyond go round

// Threads of a block whose C vectors each cover `vecs` (1024: not all of them).
int qint_threads(int vecs, int c) {
  return std::min(1024, ceil_div(ceil_div(vecs, c), kWave) * kWave);
}

// whether rows, ld elements apart, start at multiples of a vector of v elements, and end there
template <typename T>
bool vector_rows(const T* p, long ld, int k, int v) {
  return reinterpret_cast<uintptr_t>(p) % (v * sizeof(T)) == 0 && ld % v == 0 && k % v == 0;
}

}  // namespace

template <typename T>
hipError_t qint_pack(const T* x, long ldx, const QintView& o, hipStream_t st) {
  if (o.n == 0) return hipSuccess;
  constexpr int V = 16 / sizeof(T);
  const int vecs = qint_row(o.k) / V, blocks = std::min(o.n, kQintBlocks);
  const bool vec = vector_rows(x, ldx, o.k, V);
#define PACK(VEC_, C_, LOOP_)                                                                     \
  DLM_LAUNCH((qint_pack_kernel<T, VEC_, C_, LOOP_>), dim3(blocks), dim3(qint_threads(vecs, C_)), 0, st, \
             x, ldx, o)
  if (vecs > 4096) { if (vec) PACK(true, 4, true); else PACK(false, 4, true); }
  else if (vecs > 64) { if (vec) PACK(true, 4, false); else PACK(false, 4, false); }
  else { if (vec) PACK(true, 1, false); else PACK(false, 1, false); }
#undef PACK
  return hipGetLastError();
}

template <typename T>
hipError_t qint_unpack(const QintView& x, T* out, long ldo, hipStream_t st) {
  if (x.n == 0) return hipSuccess;
  constexpr int V = 16 / sizeof(T);
  const dim3 grid(ceil_div(x.k, 1024 * V), std::min(x.n, 65535));
  if (vector_rows(out, ldo, x.k, V))
    DLM_LAUNCH((qint_unpack_kernel<T, true>), grid, dim3(256), 0, st, x, out, ldo);
  else
    DLM_LAUNCH((qint_unpack_kernel<T, false>), grid, dim3(256), 0, st, x, out, ldo);
  return hipGetLastError();
}

template <typename T>
hipError_t qint_norm(const QintNorm<T>& a, const QintView& o, hipStream_t st) {
  if (o.n == 0) return hipSuccess;
  const int quads = qint_row(o.k) / 4, blocks = std::min(o.n, kQintBlocks);
  const bool vec = vector_rows(a.h, a.ldh, o.k, 4) && vector_rows(a.g, 4, o.k, 4) &&
                   (!a.h_out || vector_rows(a.h_out, a.ldo, o.k, 4)) &&
                   (a.splits == 0 || (vector_rows(a.add, a.lda, o.k, 4) && a.stride % 4 == 0)) &&
                   (!a.sw || vector_rows(a.sw, 4, o.k, 4));
#define NORM(S_, VEC_, C_, LOOP_)                                                                  \
  DLM_LAUNCH((qint_norm_kernel<T, S_, VEC_, C_, LOOP_>), dim3(blocks), dim3(qint_threads(quads, C_)), 0, \
             st, a, o)
// Four vectors a thread; two where the slices' loads take as many registers again (4096 x 4096, two
// slices: 52 us against 59, one slice 40.9 against 40.4; one vector 77 and 72).
#define NORM_C(S_)                                                                                 \
  do {                                                                                             \
    if (quads > 4096) NORM(S_, true, 4, true);                                                     \
    else if (a.splits > 1 && quads <= 2048) NORM(S_, true, 2, false);                              \
    else NORM(S_, true, 4, false);                                                                 \
  } while (0)
  if (!vec) {
    if (quads > 4096) NORM(-1, false, 4, true);
    else NORM(-1, false, 4, false);
  } else if constexpr (std::is_same<T, int32_t>::value) {
    NORM_C(-1);
  } else {
    if (a.splits == 0) NORM_C(0);
    else if (a.splits == 1) NORM_C(1);
    else if (a.splits == 2) NORM_C(2);
    else NORM_C(-1);
  }
#undef NORM_C
#undef NORM
  return hipGetLastError();
}

#define INST(T)                                                                   \
  template hipError_t qint_pack<T>(const T*, long, const QintView&, hipStream_t);     \
  template hipError_t qint_unpack<T>(const QintView&, T*, long, hipStream_t);         \
  template hipError_t qint_norm<T>(const QintNorm<T>&, const QintView&, hipStream_t);
INST(bf16)
INST(float)
#undef INST
template hipError_t qint_norm<int32_t>(const QintNorm<int32_t>&, const QintView&, hipStream_t);

}  // namespace dlm
