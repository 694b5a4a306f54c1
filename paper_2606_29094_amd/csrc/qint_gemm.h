// Products of 8-bit integers (qint_kernels.h), p[m][n] = (sum_k x[m][k] w[n][k]) sx[m] sw[n] over
// the codes. The sums are whole numbers in 32 bits (2^14 * 131071 < 2^31): they are the same in any
// order, so a row's result depends neither on the rows beside it nor on how K is split. Part of
// gemm_dl.hip, whose tiles serve all but the fewest rows.
#pragma once

#include <algorithm>
#include <cmath>

#include "../../include/dlm.h"
#include "qint_kernels.h"

namespace dlm {

namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef f32x4 f32x4u __attribute__((aligned(4)));      // at a float's alignment

// 16x16x64 int8: lane l supplies A[row = l%16][k = 16*(l/16) .. +15] and B[col = l%16] of the same
// k; D[row = 4*(l/16) + i][col = l%16] = acc[i].
__device__ __forceinline__ i32x4 mfma16_i8(const u32x4& a, const u32x4& b, const i32x4& c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b),
                                               c, 0, 0, 0);
}

// (the reciprocal by the hardware's instruction, within 1 ulp)
__device__ __forceinline__ float qint_silu_mul(float g, float u) {
  return g * __builtin_amdgcn_rcpf(1.f + __expf(-g)) * u;
}

__device__ __forceinline__ void qint_store(const QintOut& o, int m, int n, float v) {
  const long at = (long)m * o.ldy + n;
  if (o.wide) reinterpret_cast<float*>(o.y)[at] = v;
  else reinterpret_cast<bf16*>(o.y)[at] = (bf16)v;
}

// Few rows. One block: 16 of them and 16 columns (SwiGLU: of the output, with their gate and up
// rows of w), kQintWaves waves that take chunks of 256 k of the block's K slice in turn and add their sums
// in LDS. A lane's loads are 16 bytes of a row, 64 consecutive bytes over the four lanes that
// share it; a chunk's are all requested before the first is used. No wave needs what another one
// loads, so nothing waits on a barrier until the end, and the weights are read once. Bound by
// memory (one row of 3584 x 18944 15.5 us, 4.4 TB/s). Chunks of 512 k take 17.4 us there, 16 waves
// 16.2; for more rows several row fragments a block lose to the tiles, which read x through
// LDS (64 rows of 3584 x 18944: 40 us, tiles 21).
constexpr int kQintWaves = 8, kQintChunk = 256, kQintWalk = kQintWaves * kQintChunk;

template <bool SWIGLU>
__global__ __launch_bounds__(kQintWaves * 64) void qint_few_kernel(const int8_t* __restrict__ x,
                                                                   const int8_t* __restrict__ w, int row_bytes,
                                                                   int per_slice, int32_t* __restrict__ slices,
                                                                   QintOut o) {
  constexpr int NF = SWIGLU ? 2 : 1, U = kQintChunk / 64;
  __shared__ i32x4 part[kQintWaves][NF][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int g = lane >> 4, m0 = blockIdx.y * 16;
  const int n = blockIdx.x * 16 + (lane & 15), n_end = SWIGLU ? o.f : o.n;     // column of the output
  const int8_t* wr[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) wr[f] = w + (long)(min(n, n_end - 1) + f * o.f) * row_bytes + 16 * g;
  const int8_t* const xr = x + (long)min(m0 + (lane & 15), o.m - 1) * row_bytes + 16 * g;

  i32x4 acc[NF] = {};
  const int k_end = min(row_bytes, ((int)blockIdx.z + 1) * per_slice);
  for (int k0 = blockIdx.z * per_slice + wave * kQintChunk; k0 < k_end; k0 += kQintWalk) {
    u32x4 b[U][NF], a[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool in = k0 + 64 * u < k_end;       // (uniform)
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

  // wave e finishes rows 4 g + e
  if (wave >= 4) return;
  const int m = m0 + 4 * g + wave;
  if (m >= o.m || n >= n_end) return;
  int sum[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) {
    sum[f] = part[0][f][lane][wave];
#pragma unroll
    for (int j = 1; j < kQintWaves; ++j) sum[f] += part[j][f][lane][wave];
  }
  if (slices) {
#pragma unroll
    for (int f = 0; f < NF; ++f) slices[((long)blockIdx.z * o.m + m) * o.n + n + f * o.f] = sum[f];
    return;
  }
  const float sx = o.sx[m];
  float p = qint_value(sum[0], sx, o.sw[n]);
  if constexpr (SWIGLU) p = qint_silu_mul(p, qint_value(sum[NF - 1], sx, o.sw[o.f + n]));
  if (o.mode == DLM_QINT_ADD) p = qint_add(o.res[(long)m * o.ldr + n], p);
  qint_store(o, m, n, p);
}

// ------------------------------------------------- the tiles of gemm_dl.hip --
struct MulI8 {
  typedef i32x4 Acc16;
  __device__ __forceinline__ static Acc16 mma16(const u32x4& a, const u32x4& b, const Acc16& c) {
    return mfma16_i8(a, b, c);
  }
};

// What the epilogues have in common with those of the dense GEMMs (gemm_common.h).
struct EpiQintBase {
  typedef MulI8 Mul;
  static constexpr bool kRotateK = false;
  static constexpr bool kMf32 = false;
  static constexpr bool kTailSplit = true;
  static constexpr bool kWaveLocal = false;
  static constexpr bool kHead = false;
  QintOut o;
  bool vec;         // rows of y (and of the residual) are whole vectors of four
  __host__ __device__ void set_mfma(int) {}
  __device__ bool skip_tile(int) const { return false; }

  // The block's scales, in LDS (free by now): tokens m0 .. of bm rows, channels row(n0) .. of bn
  // columns. (Loaded by every lane for itself, fragment by fragment, each waits for memory: 37888 x
  // 3584 SwiGLU at 4096 rows 547 us against 518.) Whether all of the tokens' are kQintWide at most.
  template <class Row>
  __device__ __forceinline__ bool scales(float* s, int m0, int bm, int n0, int bn, int n_end, const Row& row) const {
    for (int i = threadIdx.x; i < bm + bn; i += blockDim.x)
      s[i] = i < bm ? o.sx[min(m0 + i, o.m - 1)] : o.sw[row(min(n0 + i - bm, n_end - 1))];
    __syncthreads();
    bool wide = false;
    for (int i = threadIdx.x & 63; i < bm; i += 64) wide |= s[i] > kQintWide;
    return !__any(wide);
  }
  // A wave's accumulators go through LDS, kRows rows at a time, so that a lane finishes four adjacent
  // columns of a row and a row's stores are whole lines. Those rows are finished in rounds of PER
  // quads a lane, body(round, r0, place): place(t, r, q) gives the lane's t-th one, row r0 + r of
  // the wave's, quad q of QUADS, at buf + r kStride. Only the writes to LDS name accumulators, so
  // only they are unrolled over them.
  template <int FN> static constexpr int kStride = FN * 16 + 4;
  template <int FM> static constexpr int kRows = FM % 2 == 0 ? 32 : 16;
  template <int QUADS, int PER, int FM, int FN, class Body>
  __device__ __forceinline__ void by_rows(const i32x4 (&acc)[FM][FN], int32_t* buf, int lane, const Body& body) const {
    constexpr int G = kRows<FM> / 16, ROUNDS = kRows<FM> * QUADS / 64 / PER;
    static_assert(ROUNDS * PER * 64 == kRows<FM> * QUADS, "rounds");
#pragma unroll
    for (int f0 = 0; f0 < FM; f0 += G) {
#pragma unroll
      for (int f = 0; f < G; ++f)
#pragma unroll
        for (int fn = 0; fn < FN; ++fn)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            buf[(f * 16 + 4 * (lane >> 4) + i) * kStride<FN> + fn * 16 + (lane & 15)] = acc[f0 + f][fn][i];
      // (the wave's own LDS accesses, which complete in order)
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll 1
      for (int round = 0; round < ROUNDS; ++round)
        body(f0 / G * ROUNDS + round, f0 * 16, [&](int t, int& r, int& q) {
          const int at = (round * PER + t) * 64 + lane;
          r = at / QUADS, q = at % QUADS;
        });
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
  }
  // four adjacent outputs of row m from column n on
  __device__ __forceinline__ void put(const f32x4& y, int m, int n, int n_end) const {
    if (m >= o.m) return;
    if (vec) {
      if (n >= n_end) return;
      const long at = (long)m * o.ldy + n;
      if (o.wide) *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(o.y) + at) = y;
      else *reinterpret_cast<bf16x4*>(reinterpret_cast<bf16*>(o.y) + at) = bf16x4{(bf16)y[0], (bf16)y[1], (bf16)y[2], (bf16)y[3]};
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n + i < n_end) qint_store(o, m, n + i, y[i]);
    }
  }
};

// LDS of an epilogue: the scales of the block's rows and columns, then a buffer for each wave.
template <int FM, int FN>
__device__ __forceinline__ int32_t* qint_wave_buf(char* smem, int scales) {
  return reinterpret_cast<int32_t*>(smem) + scales +
         (threadIdx.x >> 6) * (EpiQintBase::kRows<FM> * EpiQintBase::kStride<FN>);
}

// y = p, or res + p (ADD).
template <bool ADD>
struct EpiQint : EpiQintBase {
  static constexpr bool kOddFragments = true;
  __device__ int b_row(int n) const { return n; }
  template <bool FAST, int FM, int FN>
  __device__ __forceinline__ void finish(const i32x4 (&acc)[FM][FN], int m0, int n0, const float* sx,
                                         const float* sw, int32_t* buf, int lane) const {
    constexpr int Q = FN * 4, LAST = FM * 16 * Q / 64 / FN - 1;      // quads of a row; the last round
    f32x4 res[FN], next[FN];
    // (Rounds go over the wave's rows in order. A place beyond the matrix reads the channels' scales,
    // which nobody writes, instead of a value that another wave may be storing where the residual is
    // in place: by a choice of the address, since branches here spill the accumulators, 4096 x
    // 4096 at 4096 rows 83 -> 182 us.)
    auto load = [&](f32x4 (&v)[FN], int round) {
#pragma unroll
      for (int t = 0; t < FN; ++t) {
        const int at = (round * FN + t) * 64 + lane, m = m0 + at / Q, n = n0 + at % Q * 4;
        const float* const r = o.res + (long)m * o.ldr + n;
        if (vec) {
          v[t] = *reinterpret_cast<const f32x4u*>(m < o.m && n < o.n ? r : o.sw);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) v[t][i] = *(m < o.m && n + i < o.n ? r + i : o.sw);
        }
      }
    };
    if constexpr (ADD) load(next, 0);
    by_rows<Q, FN>(acc, buf, lane, [&](int round, int r0, auto place) {
      if constexpr (ADD) {         // (the next rows' loads before these rows' stores)
#pragma unroll
        for (int t = 0; t < FN; ++t) res[t] = next[t];
        load(next, min(round + 1, LAST));
      }
#pragma unroll
      for (int t = 0; t < FN; ++t) {
        int r, q;
        place(t, r, q);
        const i32x4 v = *reinterpret_cast<const i32x4*>(buf + r * kStride<FN> + 4 * q);
        const f32x4 w = *reinterpret_cast<const f32x4*>(sw + 4 * q);
        const float x = sx[r0 + r];
        f32x4 y;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          y[i] = qint_value<FAST>(v[i], x, w[i]);
          if constexpr (ADD) y[i] = qint_add(res[t][i], y[i]);
        }
        put(y, m0 + r0 + r, n0 + 4 * q, o.n);
      }
    });
  }
  template <int FM, int FN>
  __device__ void operator()(i32x4 (&acc)[FM][FN], int m0, int n0, int lane, int wave_n, char* smem, int waves_n,
                             int bm, int block_m0, int, int) const {
    const int block_n0 = n0 - wave_n * FN * 16, bn = waves_n * FN * 16;
    float* const s = reinterpret_cast<float*>(smem);
    const bool fast = scales(s, block_m0, bm, block_n0, bn, o.n, [](int n) { return n; });
    int32_t* const buf = qint_wave_buf<FM, FN>(smem, bm + bn);
    if (fast) finish<true>(acc, m0, n0, s + (m0 - block_m0), s + bm + (n0 - block_n0), buf, lane);
    else finish<false>(acc, m0, n0, s + (m0 - block_m0), s + bm + (n0 - block_n0), buf, lane);
  }
};

// silu(gate) * up over columns that come as 16 of the gate, then the 16 of the up matrix (as in
// EpiSwiGLU): column n is output (n / 32) 16 + n % 16, the GEMM's N = 2 f rounded up to 32.
struct EpiQintSwiGLU : EpiQintBase {
  static constexpr bool kOddFragments = false;
  __device__ int b_row(int n) const {
    const int f = min(((n >> 5) << 4) + (n & 15), o.f - 1);
    return (n >> 4) & 1 ? o.f + f : f;
  }
  template <bool FAST, int FM, int FN>
  __device__ __forceinline__ void finish(const i32x4 (&acc)[FM][FN], int m0, int n0, const float* sx,
                                         const float* sw, int32_t* buf, int lane) const {
    by_rows<FN * 2, FN / 2>(acc, buf, lane, [&](int, int r0, auto place) {
#pragma unroll
      for (int t = 0; t < FN / 2; ++t) {
        int r, q;
        place(t, r, q);
        const int c = q / 4 * 32 + q % 4 * 4;            // the gate's column, the up one is 16 behind it
        const i32x4 g = *reinterpret_cast<const i32x4*>(buf + r * kStride<FN> + c);
        const i32x4 u = *reinterpret_cast<const i32x4*>(buf + r * kStride<FN> + c + 16);
        const f32x4 wg = *reinterpret_cast<const f32x4*>(sw + c), wu = *reinterpret_cast<const f32x4*>(sw + c + 16);
        const float x = sx[r0 + r];
        f32x4 y;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          y[i] = qint_silu_mul(qint_value<FAST>(g[i], x, wg[i]), qint_value<FAST>(u[i], x, wu[i]));
        put(y, m0 + r0 + r, (n0 >> 1) + q * 4, o.f);
      }
    });
  }
  template <int FM, int FN>
  __device__ void operator()(i32x4 (&acc)[FM][FN], int m0, int n0, int lane, int wave_n, char* smem, int waves_n,
                             int bm, int block_m0, int, int) const {
    static_assert(FN % 2 == 0, "gate/up pairs");
    const int block_n0 = n0 - wave_n * FN * 16, bn = waves_n * FN * 16;
    float* const s = reinterpret_cast<float*>(smem);
    const bool fast = scales(s, block_m0, bm, block_n0, bn, INT32_MAX, [&](int n) { return b_row(n); });
    int32_t* const buf = qint_wave_buf<FM, FN>(smem, bm + bn);
    if (fast) finish<true>(acc, m0, n0, s + (m0 - block_m0), s + bm + (n0 - block_n0), buf, lane);
    else finish<false>(acc, m0, n0, s + (m0 - block_m0), s + bm + (n0 - block_n0), buf, lane);
  }
};

// The whole numbers of each K slice, [slice][m][n], for qint_join_kernel.
struct EpiQintSlices : EpiQintBase {
  static constexpr bool kOddFragments = true;
  int32_t* slices;
  __device__ int b_row(int n) const { return n; }
  template <int FM, int FN>
  __device__ void operator()(i32x4 (&acc)[FM][FN], int m0, int n0, int lane, int, char*, int, int, int, int,
                             int split) const {
    int32_t* const s = slices + (long)split * o.m * o.n;
#pragma unroll
    for (int fm = 0; fm < FM; ++fm)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int m = m0 + fm * 16 + 4 * (lane >> 4) + i;
        if (m >= o.m) continue;
#pragma unroll
        for (int fn = 0; fn < FN; ++fn) {
          const int n = n0 + fn * 16 + (lane & 15);
          if (n < o.n) s[(long)m * o.n + n] = acc[fm][fn][i];
        }
      }
  }
};

// The K slices of a product, added, and its epilogue: V columns of a row a thread (four where rows
// are whole vectors of that: 1000 x 3584, four slices 24.3 -> 17.7 us). Everything it reads is
// requested before the first use.
template <int V>
__global__ __launch_bounds__(256) void qint_join_kernel(const int32_t* __restrict__ slices, int n_slices,
                                                        QintOut o) {
  typedef int32_t iv __attribute__((ext_vector_type(V)));
  typedef float fv __attribute__((ext_vector_type(V)));
  const bool swiglu = o.mode == DLM_QINT_SWIGLU;
  const int n_out = swiglu ? o.f : o.n, n = (blockIdx.x * 256 + threadIdx.x) * V;
  if (n >= n_out) return;
  float sw[V], su[V];
#pragma unroll
  for (int i = 0; i < V; ++i) sw[i] = o.sw[n + i], su[i] = swiglu ? o.sw[o.f + n + i] : 0.f;
  for (int m = blockIdx.y; m < o.m; m += gridDim.y) {
    const int32_t* const p = slices + (long)m * o.n + n;
    const long slice = (long)o.m * o.n;
    const float sx = o.sx[m];
    fv res = {};
    if (o.mode == DLM_QINT_ADD) res = *reinterpret_cast<const fv*>(o.res + (long)m * o.ldr + n);
    iv v = {}, up = {};
#pragma unroll 4
    for (int s = 0; s < n_slices; ++s) {
      v += *reinterpret_cast<const iv*>(p + s * slice);
      if (swiglu) up += *reinterpret_cast<const iv*>(p + s * slice + o.f);
    }
    fv y;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      y[i] = qint_value(v[i], sx, sw[i]);
      if (swiglu) y[i] = qint_silu_mul(y[i], qint_value(up[i], sx, su[i]));
      if (o.mode == DLM_QINT_ADD) y[i] = qint_add(res[i], y[i]);
    }
    const long at = (long)m * o.ldy + n;
    if (o.wide) {
      *reinterpret_cast<fv*>(reinterpret_cast<float*>(o.y) + at) = y;
    } else {
      typedef bf16 bv __attribute__((ext_vector_type(V)));
      bv b;
#pragma unroll
      for (int i = 0; i < V; ++i) b[i] = (bf16)y[i];
      *reinterpret_cast<bv*>(reinterpret_cast<bf16*>(o.y) + at) = b;
    }
  }
}

}  // namespace

// Way of a product. The GEMM tiles' times are those of bf16 operands of as many bytes (gemm_plan;
// the matrix cores take the same time over them), K slices by a join of their own. Up to 16 rows
// also blocks that read memory directly (qint_few_kernel), us on MI355X with the weights from HBM:
// 3.4 + the weights at 5.6 TB/s (less where CUs have unequal shares) + x, once for each column tile, at
// 11 TB/s out of the L2s, and for K slices 2 + 0.8 a MB of them. Direct / tiles: one row of 4096 x
// 4096 6.4 / 8.3, 3584 x 18944 15.5 / 18.1, 24576 x 4096 SwiGLU 21.6 / 21.3; 16 rows 8.0 / 8.9, 22.4 /
// 18.6, 26.0 / 21.6.
constexpr int kQintFewRows = 16, kQintSmallTile = 94;

// Rows that the tiles can address (32-bit offsets of 2-byte units); more are taken in turn, all by
// one plan: whole tiles over whole K, whose last round has no sub-tiles (their number is that of one
// launch's tiles; 65280 rows and more are many rounds).
static int qint_near_rows(int units) { return (int)std::min<long>(((1L << 32) / units - 1) & ~255L, 1 << 30); }

QintPlan qint_plan(int rows, int n, int k, bool swiglu, int num_cu) {
  QintPlan p;
  if (rows <= 0) return p;
  const int units = qint_row(k) / 2, cols = swiglu ? ceil_div(n, 32) * 32 : n;   // 2-byte units of a row
  const bool near = rows <= qint_near_rows(units), split = !swiglu && near;
  double us, best;
  p.gemm = true;
  p.g = gemm_plan(2, rows, cols, units, split, num_cu, false, near, !swiglu, kFewRows, false, split, &best);
  if (swiglu && (long)rows * cols < 64 * 64 * (long)num_cu) {     // (the smallest tiles leave CUs idle)
    const GemmPlan g = gemm_plan(2, rows, n, units, true, num_cu, false, true, true, kFewRows, false, true, &us);
    if (g.splits > 1 && us < best) best = us, p.g = g;
  }
  // Weights that fill half of the 256 MB last-level cache, or many rows: row tiles in groups of 8, so
  // that an XCD's blocks share weight columns as well as rows. Plain order / groups, us: 37888 x 3584
  // SwiGLU at 1500 rows 205 / 188, 4096 503 / 477, 10240 1243 / 1183; 4096 x 12288 at 10240 494 / 474;
  // 3584 x 18944 at 4096 237 / 236, 10240 648 / 639. Fewer rows of smaller ones: 24576 x 4096 at 4096
  // 340 / 342, 12288 x 4096 174 / 180, 4096 x 4096 at 1000 rows 23 / 27. One row tile has no rows to
  // share and keeps the plain order: 37888 x 3584 SwiGLU at 32 rows 26.8 / 27.0, 128 31.5 / 31.8, 256
  // 44.4 / 44.8 (28672 x 8192 at 32 rows 45.1 / 44.3, 192 63.0 / 63.6).
  int bm, bn, th;
  if (((double)n * units > 64e6 || rows >= 8192) && p.g.splits == 1 && gemm_dl_tile(p.g.cfg, &bm, &bn, &th) && rows > bm)
    p.g.group_m = 8;
  // Small products: tiles of 32 x 32 with eight stages, 3.45 + 0.1875 for each k-tile where every CU
  // has a block, 15 % more where it has two, beside the stream. The other tiles / these, us: 2048 x
  // 2048 at 64 rows 8.7 / 6.3, 3584 x 3584 10.9 / 8.8, 4608 x 3584 11.3 / 9.6, 4096 x 4096 at 128 rows
  // 12.7 / 10.8, 689 x 1031 6.7 / 5.4, 256 x 688 5.0 / 4.0; long walks and many tiles are the others':
  // 4096 x 12288 at 64 rows 17.4 / 22.4, 12288 x 4096 15.9 / 22.6, 4608 x 3584 at 128 rows 12.4 / 15.9. (The
  // models of both are off by up to a tenth, which the others keep.)
  if (!swiglu) {
    const long tiles = (long)ceil_div(rows, 32) * ceil_div(n, 32), full = tiles / (2 * num_cu), rem = tiles - full * 2 * num_cu;
    const double rounds = 1.15 * full + (rem > num_cu ? 1.15 : rem ? 1.0 : 0.0);
    const double walk = units / 64 * 0.1875 * rounds, stream = (double)n * units * 2e-6 / 7.1;
    const double t = 3.45 + (double)rows * n * 4e-6 / 6.46 + std::sqrt(walk * walk + stream * stream);
    if (t < 0.9 * best) best = t, p.g = GemmPlan{kQintSmallTile, 1, 0};
  }
  p.slices = p.g.splits;
  if (rows <= kQintFewRows) {
    const int blocks = ceil_div(swiglu ? n / 2 : n, 16), walks = ceil_div(units * 2, kQintWalk);
    const double mb = (double)n * units * 2e-6, x_mb = (double)rows * units * 2e-6 * blocks;
    for (int s = 1; s <= 16 && s <= walks; s *= 2) {
      if (ceil_div(walks, ceil_div(walks, s)) != s) continue;     // (none of them empty)
      const double shares = (double)blocks * s / num_cu;
      double t = 3.4 + mb * std::max(1.0, 0.875 * std::ceil(shares) / shares) / 5.6 + x_mb / 11;
      if (s > 1) t += 2 + 0.8 * s * rows * (double)n * 4e-6;
      if (t < best) best = t, p.gemm = false, p.slices = s;
    }
  }
  if (p.slices > 1) p.scratch = (size_t)p.slices * rows * n * sizeof(int32_t);
  return p;
}

hipError_t qint_matmul(const QintPlan& plan, const QintView& x, const QintView& w, QintOut o, void* scratch,
                       hipStream_t st) {
  if (x.n == 0) return hipSuccess;
  const int row_bytes = qint_row(w.k), near = qint_near_rows(row_bytes / 2);
  if (x.n > near) {
    const LaunchSpan span(true);
    for (int at = 0; at < x.n; at += near) {
      const QintView part{x.codes + (long)at * row_bytes, x.scales + at, std::min(near, x.n - at), x.k};
      QintOut op = o;
      op.y = reinterpret_cast<char*>(o.y) + (long)at * o.ldy * (o.wide ? 4 : 2);
      if (o.mode == DLM_QINT_ADD) op.res = o.res + (long)at * o.ldr;
      if (at + near >= x.n) span.last();
      const hipError_t e = qint_matmul(plan, part, w, op, scratch, st);
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  }
  o.m = x.n, o.n = w.n, o.f = w.n / 2, o.sx = x.scales, o.sw = w.scales;
  const bool swiglu = o.mode == DLM_QINT_SWIGLU;
  const int n_out = swiglu ? o.f : o.n, es = o.wide ? 4 : 2;
  // outputs (and what is read beside them) in vectors of four
  const bool vec = n_out % 4 == 0 && o.ldy % 4 == 0 && reinterpret_cast<uintptr_t>(o.y) % (4 * es) == 0 &&
                   (o.mode != DLM_QINT_ADD || (o.ldr % 4 == 0 && reinterpret_cast<uintptr_t>(o.res) % 16 == 0));
  auto join = [&](const int32_t* slices) {
    if (!plan.join) return hipSuccess;
    const int rows = std::min(o.m, 65535);
    if (vec)
      DLM_LAUNCH((qint_join_kernel<4>), dim3(ceil_div(n_out, 1024), rows), dim3(256), 0, st, slices, plan.slices, o);
    else
      DLM_LAUNCH((qint_join_kernel<1>), dim3(ceil_div(n_out, 256), rows), dim3(256), 0, st, slices, plan.slices, o);
    return hipGetLastError();
  };
  if (plan.gemm) {
    const bf16 *a = reinterpret_cast<const bf16*>(x.codes), *b = reinterpret_cast<const bf16*>(w.codes);
    const int units = row_bytes / 2;
    const GemmPlan& g = plan.g;
    if (plan.slices == 1) {
      auto launch = [&](auto e, int n) {
        e.o = o, e.vec = vec;
        return gemm_dl_launch<decltype(e)>(g.cfg, a, units, b, units, o.m, n, units, 1, g.group_m, g.sub,
                                           g.n_tail, e, st);
      };
      if (swiglu) return launch(EpiQintSwiGLU{}, ceil_div(o.n, 32) * 32);
      return o.mode == DLM_QINT_ADD ? launch(EpiQint<true>{}, o.n) : launch(EpiQint<false>{}, o.n);
    }
    const LaunchSpan span(plan.join);
    EpiQintSlices e{};
    e.o = o, e.slices = reinterpret_cast<int32_t*>(scratch);
    const hipError_t err = gemm_dl_launch<EpiQintSlices>(g.cfg, a, units, b, units, o.m, o.n, units, g.splits,
                                                         g.group_m, g.sub, g.n_tail, e, st);
    if (err != hipSuccess) return err;
    span.last();
    return join(e.slices);
  }
  const LaunchSpan span(plan.slices > 1 && plan.join);
  int32_t* const slices = plan.slices > 1 ? reinterpret_cast<int32_t*>(scratch) : nullptr;
  const int per_slice = ceil_div(ceil_div(row_bytes, kQintWalk), plan.slices) * kQintWalk;
  const dim3 grid(ceil_div(n_out, 16), ceil_div(o.m, 16), plan.slices);
  if (swiglu)
    DLM_LAUNCH((qint_few_kernel<true>), grid, dim3(kQintWaves * 64), 0, st, x.codes, w.codes, row_bytes, per_slice,
               slices, o);
  else
    DLM_LAUNCH((qint_few_kernel<false>), grid, dim3(kQintWaves * 64), 0, st, x.codes, w.codes, row_bytes, per_slice,
               slices, o);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess || !slices) return err;
  span.last();
  return join(slices);
}

}  // namespace dlm
