// Products with 4-bit matrices (mx_common.h), y[m][n] = sum_k x[m][k] w[n][k]. Part of
// gemm.hip.
#pragma once

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "../../include/dlm.h"
#include "mx_common.h"
#include "mx_kernels.h"

namespace dlm {

namespace {

// --------------------------------------------------------------- products --
// x for the product kernels: NP planes of [rows, kp] bf16 (one for bf16 x, three for
// fp32 x: split3), kp = 32 groups, zero from k on. A thread makes eight elements of a row.
template <typename T, int NP>
__global__ __launch_bounds__(256) void mx_stage_kernel(const T* __restrict__ x, long ldx, int rows,
                                                       int k, int kp, long plane,
                                                       bf16* __restrict__ out) {
  const long at = ((long)blockIdx.x * 256 + threadIdx.x) * 8;
  if (at >= kp) return;
  for (long row = blockIdx.y; row < rows; row += gridDim.y) {
    bf16x8 v[NP];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float e = at + i < k ? to_f32(x[row * ldx + at + i]) : 0.f;
      if constexpr (NP == 1) {
        v[0][i] = (bf16)e;
      } else {
        bf16 hi, mid, lo;
        split3(e, hi, mid, lo);
        v[0][i] = hi;
        v[1][i] = mid;
        v[2][i] = lo;
      }
    }
#pragma unroll
    for (int p = 0; p < NP; ++p) *reinterpret_cast<bf16x8*>(out + p * plane + row * kp + at) = v[p];
  }
}

// The first `keep` codes of a group, the others zero. (What is behind k may be anything: x is
// zero there, but a code that its scale makes infinite would still give NaN.)
__device__ __forceinline__ u32x4 keep_codes(u32x4 c, int keep) {
#pragma unroll
  for (int d = 0; d < 4; ++d) c[d] &= (uint32_t)((1ull << 4 * min(max(keep - 8 * d, 0), 8)) - 1);
  return c;
}

// Infinite weights meet the first term of an fp32 x alone, whose product is the right
// infinity; the others would be 0 * inf, or an infinity of the other sign. Whether a scale
// byte makes any code infinite, and eight weights with the infinite ones zero.
__device__ __forceinline__ bool mx_may_be_infinite(uint32_t e) { return e - 253u < 2u; }
__device__ __forceinline__ bf16x8 finite_or_zero(const bf16x8& w) {
  u32x4 v = __builtin_bit_cast(u32x4, w);
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    if ((v[d] & 0x7fffu) == 0x7f80u) v[d] &= 0xffff0000u;
    if ((v[d] & 0x7fff0000u) == 0x7f800000u) v[d] &= 0xffffu;
  }
  return __builtin_bit_cast(bf16x8, v);
}

// The same of a group's codes: 4 and 6 under byte 253, and 2 and 3 under 254.
__device__ __forceinline__ u32x4 finite_or_zero(u32x4 c, uint32_t e) {
#pragma unroll
  for (int d = 0; d < 4; ++d)
    c[d] &= ~(15u * (c[d] >> 2 & (e == 254u ? ~0u : c[d] >> 1) & 0x11111111u));
  return c;
}

__device__ __forceinline__ float silu_mul(float g, float u) { return g / (1.f + __expf(-g)) * u; }

// Few rows. One block: 16 of them and 16 NF columns, W waves that take the 512-wide k ranges
// ("walks") of the block's K slice in turn and add their partial sums in LDS, in
// wave order. In a chunk of 128 k lane l reads the 32 codes of group l / 16 of weight
// row l % 16 as one 16-byte load; four register swaps between the 16-lane groups turn
// that into the dword of group j that the MFMA j = 0..3 takes (whose lanes then read
// 64 consecutive bytes of each x row). A walk's codes and scales (one 16-byte load for
// its 16 groups) are all requested before the first is used. The weights are read once,
// by the one block row that needs them; x comes from the caches, once for every 16 NF
// columns. (One row: 4096 x 4096 4.9 us, 24576 x 4096 17.6, 3.0 TB/s.)
constexpr int kWalk = 512;

template <int NF, int W, int NP>
__global__ __launch_bounds__(W * 64) void mx_linear_kernel(MxLinear a) {
  __shared__ f32x4 part[W][NF][64];
  constexpr int XJ = NP > 1 ? 1 : 2;   // k steps whose x is requested together
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, g = lane >> 4;
  const int n0 = blockIdx.x * (a.swiglu ? NF * 8 : NF * 16), m0 = blockIdx.y * 16;
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
    ws[f] = a.w.scales + (long)n * a.w.scale_ld;
  }
  const bf16* const xr = a.x + (long)min(m0 + col, a.m - 1) * a.ldx + 8 * g;

  f32x4 acc[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) acc[f] = f32x4{0.f, 0.f, 0.f, 0.f};

  // one walk; TAIL: the last one, whose groups and elements may end inside it
  auto walk = [&](int s, auto tail) {
    constexpr bool TAIL = decltype(tail)::value;
    const int k0 = s * kWalk;
    u32x4 codes[4][NF], scales[NF];
#pragma unroll
    for (int f = 0; f < NF; ++f) {
#pragma unroll
      for (int c = 0; c < 4; ++c)
        codes[c][f] = !TAIL || 16 * s + 4 * c + g < a.w.groups
                          ? *reinterpret_cast<const u32x4*>(wc[f] + (long)s * 256 + c * 64)
                          : u32x4{0u, 0u, 0u, 0u};
      scales[f] = *reinterpret_cast<const u32x4*>(ws[f] + 16 * s);
    }
    bool infinite = false;   // (of any lane: a lane looks at its own groups)
    if constexpr (NP > 1) {
#pragma unroll
      for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int c = 0; c < 4; ++c) infinite |= mx_may_be_infinite((scales[f][c] >> (8 * g)) & 255u);
      infinite = __any(infinite);
    }
    bf16x8 xv[2][XJ][NP];
    auto xload = [&](int i) {   // x of steps XJ i .. of the walk
#pragma unroll
      for (int u = 0; u < XJ; ++u) {
        const int c = (XJ * i + u) / 4, j = (XJ * i + u) % 4;
        const bool in = !TAIL || k0 + 128 * c + 32 * j + 8 * g < a.k;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          bf16x8 v = {};
          if (in) v = *reinterpret_cast<const bf16x8*>(xr + p * a.plane + k0 + 128 * c + 32 * j);
          xv[i & 1][u][p] = v;
        }
      }
    };
    xload(0);
#pragma unroll
    for (int i = 0; i < 16 / XJ; ++i) {
      if (i + 1 < 16 / XJ) xload(i + 1);
      __builtin_amdgcn_sched_barrier(0);   // (or the loads are moved down to their uses)
#pragma unroll
      for (int u = 0; u < XJ; ++u) {
        const int c = (XJ * i + u) / 4, j = (XJ * i + u) % 4;
        if (j == 0) {
#pragma unroll
          for (int f = 0; f < NF; ++f) {
            if (TAIL && a.tail && 16 * s + 4 * c + g == a.w.groups - 1)
              codes[c][f] = keep_codes(codes[c][f], a.tail);
            codes[c][f] = transpose_groups(codes[c][f]);
          }
        }
        bf16x8 b[NF];
#pragma unroll
        for (int f = 0; f < NF; ++f) {
          uint32_t e = (scales[f][c] >> (8 * j)) & 255u;
          if (TAIL && 16 * s + 4 * c + j >= a.w.groups) e = 127u;
          b[f] = mx_bf16x8(codes[c][f][j], mx_scale(e));
        }
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          if (NP > 1 && p == 1 && infinite) {
#pragma unroll
            for (int f = 0; f < NF; ++f) b[f] = finite_or_zero(b[f]);
          }
#pragma unroll
          for (int f = 0; f < NF; ++f) acc[f] = mfma16_bf16(xv[i & 1][u][p], b[f], acc[f]);
        }
      }
    }
  };
  const int walks = ceil_div(a.w.groups, kWalk / kMxGroup);
  const int s_end = min(((int)blockIdx.z + 1) * a.per_slice, walks);
  // (x holds every k of the full ones, and their groups are whole)
  const int full = (a.k - (a.tail ? 1 : 0)) / kWalk;
  for (int s = blockIdx.z * a.per_slice + wave; s < s_end; s += W) {
    if (s < full) walk(s, std::false_type{});
    else walk(s, std::true_type{});
  }
#pragma unroll
  for (int f = 0; f < NF; ++f) part[wave][f][lane] = acc[f];
  __syncthreads();

  // wave f finishes fragment f (or gate / up pair of fragments)
  auto sum = [&](int i) {
    f32x4 v = part[0][i][lane];
#pragma unroll
    for (int w = 1; w < W; ++w) v += part[w][i][lane];
    return v;
  };
  const bool sliced = gridDim.z > 1;   // fp32 sums to the scratch, mx_join_kernel does the rest
  if (a.swiglu && !sliced) {
    constexpr int H = NF > 1 ? NF / 2 : 1;
    if (wave < H) {
      const int f = wave;
      const f32x4 gate = sum(f), up = sum(f + NF / 2);
      const int n = n0 + 16 * f + col;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int m = m0 + 4 * g + e;
        if (m >= a.m || n >= n_end) continue;
        const float v = silu_mul(gate[e], up[e]);
        if constexpr (NP == 1) reinterpret_cast<bf16*>(a.y)[(long)m * a.ldy + n] = (bf16)v;
        else reinterpret_cast<float*>(a.y)[(long)m * a.ldy + n] = v;
      }
    }
    return;
  }
  float* out = sliced ? a.slices + (long)blockIdx.z * a.m * a.w.n : reinterpret_cast<float*>(a.y);
  const long ldo = sliced ? a.w.n : a.ldy;
  if (wave < NF) {
    const int f = wave;
    const f32x4 v = sum(f);
    int n = n0 + 16 * f + col;
    bool ok = n < n_end;
    if (a.swiglu) {
      n = n0 + 16 * (f % (NF > 1 ? NF / 2 : 1)) + col;
      ok = n < n_end;
      n += 2 * f >= NF ? n_end : 0;
    }
    float* o = out + (long)(m0 + 4 * g) * ldo + n;
    f32x4 old = {0.f, 0.f, 0.f, 0.f};
    if (a.add && !sliced) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (ok && m0 + 4 * g + e < a.m) old[e] = o[e * ldo];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (ok && m0 + 4 * g + e < a.m) o[e * ldo] = old[e] + v[e];
  }
}

// More rows: WN waves compute 16 MT rows x 16 NF WN columns. x goes through LDS in chunks
// of 128 k by direct loads, NS stages of them, shared by the waves; each wave reads its
// own columns' codes from memory into registers NS - 1 chunks ahead, and their scales
// for four chunks (a walk) at a time one walk ahead, and unpacks them there (once for 16 MT
// rows), so the weights need no LDS. Bound by the chain of a chunk where a CU has one block
// of few rows, beyond by the matrix cores and by LDS, which each wave reads all rows from
// (37888 x 3584 SwiGLU, 1000 rows 248 us, 1.09 PFLOP/s).
// Row r of a stage is 256 bytes, its 16-byte slot s stored at s ^ (r & 15): the 16 rows
// that a fragment reads at one slot come from distinct banks.
// Blocks 8 apart in the launch run on one XCD: each XCD takes an eighth of the tiles, the row
// tiles of a column tile one after the other, so they read its codes through one L2. (An
// eighth of the column tiles to each left XCDs idle where there are few: 41 x 2608 at 3636
// rows, one column tile, 33 us against 10.)
__device__ const uint4 kZeros[1] = {};   // what x holds behind k

// TAIL: k is not a multiple of 32 (an instance of its own: the test of each chunk for the
// codes behind k costs 1 to 5 %, 256 rows of 4096 x 4096 18.9 us against 17.9). The second
// launch bound keeps four blocks of the smallest tile on a CU.
template <int WN, int MT, int NF, int NS, bool PLANES, bool TAIL>
__global__ __launch_bounds__(WN * 64, MT == 2 ? 4 : 1) void mx_tile_kernel(MxLinear a, int n_tiles, int m_tiles) {
  typedef typename std::conditional<PLANES, float, bf16>::type T;
  constexpr int BM = 16 * MT, STAGE = BM * 256;
  constexpr int XL = STAGE / 1024 / WN;    // direct loads of a wave for a stage
  constexpr int LOADS = XL + NF;           // memory operations of a wave for a chunk, without scales
  static_assert(STAGE % (1024 * WN) == 0 && 4 % NS == 0, "whole loads, whole walks");
  __shared__ __attribute__((aligned(16))) char smem[NS * STAGE];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, g = lane >> 4;
  const int per_xcd = ceil_div(n_tiles * m_tiles, kXcds);
  const int id = blockIdx.x % kXcds * per_xcd + blockIdx.x / kXcds;
  if (id >= n_tiles * m_tiles) return;
  const int n_tile = id / m_tiles, m0 = id % m_tiles * BM;
  const int n_end = a.swiglu ? a.w.n / 2 : a.w.n;
  constexpr int H = NF / 2;
  const int n0 = (n_tile * WN + wave) * (a.swiglu ? 16 * H : 16 * NF);   // the wave's first column

  // Addresses as a base of the wave, which scalar registers hold, and an offset of the
  // lane in 32 bits; with SwiGLU the second half of the fragments are the up rows.
  const int n_base = min(n0, n_end - 1);
  const uint8_t* const codes0 = a.w.codes + (long)n_base * a.w.groups * 16;
  const uint8_t* const scales0 = a.w.scales + (long)n_base * a.w.scale_ld;
  const long up_codes = a.swiglu ? (long)n_end * a.w.groups * 16 : 0;
  const long up_scales = a.swiglu ? (long)n_end * a.w.scale_ld : 0;
  uint32_t wc[NF], ws[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) {
    const int n = min(n0 + 16 * (a.swiglu ? f % H : f) + col, n_end - 1) - n_base;
    wc[f] = (uint32_t)(n * a.w.groups + g) * 16;
    ws[f] = (uint32_t)n * a.w.scale_ld;
  }
  const char* const x0 = reinterpret_cast<const char*>(a.x + (long)m0 * a.ldx);
  uint32_t xs[XL];         // this lane's slot in each of the wave's direct loads
#pragma unroll
  for (int u = 0; u < XL; ++u) {
    const int r = 4 * (u * WN + wave) + g;
    xs[u] = (uint32_t)min(r, a.m - 1 - m0) * (uint32_t)a.ldx * 2 + 16 * (col ^ (r & 15));
  }
  uint32_t slot[4];        // of the lane's fragments in a row of a stage
#pragma unroll
  for (int j = 0; j < 4; ++j) slot[j] = col * 256 + ((4 * j + g) ^ col) * 16;

  // The walks of this block's slice; the planes of fp32 x are so many products with the
  // same weights, one after the other.
  const int walks = ceil_div(a.w.groups, kWalk / kMxGroup);
  const int s0 = blockIdx.z * a.per_slice, s1 = min(s0 + a.per_slice, walks * a.planes);
  const int turns = s1 - s0;
  auto walk = [&](int i) { return min(s0 + i, s1 - 1); };   // (past the end: loaded, not used)

  f32x4 acc[MT][NF];
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int f = 0; f < NF; ++f) acc[t][f] = f32x4{0.f, 0.f, 0.f, 0.f};
  u32x4 codes[NS][NF], scales[2][NF];
  auto load = [&](int b, int i, int c4) {   // chunk c4 of turn i into stage b
    const int s = walk(i), c = 4 * (PLANES ? s % walks : s) + c4;
    char* dst = smem + b * STAGE + wave * 1024;
    const char* xc = x0 + (PLANES ? s / walks * a.plane * 2 : 0) + (long)c * 256;
#pragma unroll
    for (int u = 0; u < XL; ++u) {   // what lies behind k counts as zero
      const int k = 128 * c + 8 * (col ^ ((4 * (u * WN + wave) + g) & 15));
      load_lds16(k < a.k ? xc + xs[u] : reinterpret_cast<const char*>(kZeros), dst + u * WN * 1024);
    }
    // (a lane behind the last group reads that one, a chunk behind the last one that chunk;
    // scales are set to one there and x is zero)
    const int cw = min(c, (a.w.groups - 1) / 4);
    const uint32_t back = 16 * max(4 * cw + g - (a.w.groups - 1), 0);
    const uint8_t* cb = codes0 + (long)cw * 64;
#pragma unroll
    for (int f = 0; f < NF; ++f)
      codes[b][f] = *reinterpret_cast<const u32x4*>(cb + (f >= H ? up_codes : 0) + (wc[f] - back));
  };
  auto load_scales = [&](int b, int i) {    // of turn i
    const int s = walk(i);
    const uint8_t* sb = scales0 + (long)(PLANES ? s % walks : s) * 16;
#pragma unroll
    for (int f = 0; f < NF; ++f)
      scales[b][f] = *reinterpret_cast<const u32x4*>(sb + (f >= H ? up_scales : 0) + ws[f]);
  };
  auto compute = [&](int b, int sb, int i, int c4, bool infinite) {
    const int s = walk(i), c = 4 * (PLANES ? s % walks : s) + c4;
    const int left = a.w.groups - 4 * c;   // groups of the chunk
    const uint32_t keep = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1;
    u32x4 cd[NF];
    uint32_t sc[NF];
    if (TAIL && c == (a.w.groups - 1) / 4 && 4 * c + g == a.w.groups - 1) {
#pragma unroll
      for (int f = 0; f < NF; ++f) codes[b][f] = keep_codes(codes[b][f], a.tail);
    }
    if (PLANES && infinite) {
#pragma unroll
      for (int f = 0; f < NF; ++f) {
        const uint32_t e = (scales[sb][f][c4] >> (8 * g)) & 255u;
        if (mx_may_be_infinite(e)) codes[b][f] = finite_or_zero(codes[b][f], e);
      }
    }
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      cd[f] = transpose_groups(codes[b][f]);
      sc[f] = (scales[sb][f][c4] & keep) | (0x7f7f7f7fu & ~keep);
    }
    // In the large tiles the fragments of step j + 1 are read and unpacked between the
    // MFMAs of step j.
    constexpr int AHEAD = MT >= 8 ? 1 : 0;
    bf16x8 xv[AHEAD + 1][MT], w[AHEAD + 1][NF];
    auto fetch = [&](int j) {
#pragma unroll
      for (int t = 0; t < MT; ++t)
        xv[j & AHEAD][t] = *reinterpret_cast<const bf16x8*>(smem + slot[j] + b * STAGE + t * 4096);
#pragma unroll
      for (int f = 0; f < NF; ++f)
        w[j & AHEAD][f] = mx_bf16x8(cd[f][j], mx_scale((sc[f] >> (8 * j)) & 255u));
    };
    if (AHEAD) fetch(0);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (j + AHEAD < 4) fetch(j + AHEAD);
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int f = 0; f < NF; ++f)
          acc[t][f] = mfma16_bf16(xv[j & AHEAD][t], w[j & AHEAD][f], acc[t][f]);
    }
    if constexpr (AHEAD) {   // the order asked for: LDS reads, MFMAs and vector work in turn
      __builtin_amdgcn_sched_group_barrier(0x100, MT, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, 8 * NF, 0);
#pragma unroll
      for (int i = 0; i < 3 * MT; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, NF, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, (6 * NF + MT - 1) / MT, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, MT * NF, 0);
    }
  };
  // Every step issues the loads of a chunk, past the end those of the last walk again: the
  // waits count loads, and one that some path skips would have to be counted out. (Scales
  // are not counted: the waits are then longer by them where they are in flight.)
  load_scales(0, 0);
#pragma unroll
  for (int b = 0; b < NS - 1; ++b) {
    load(b, 0, b);
    __builtin_amdgcn_sched_barrier(0);
  }
  auto turn = [&](int i, auto parity) {
    constexpr int P = decltype(parity)::value;
    bool infinite = false;   // whether a weight of this walk meets zeros that it would make NaN
#pragma unroll
    for (int c4 = 0; c4 < 4; ++c4) {
      wait_vmcnt<(NS - 2) * LOADS>();      // the chunk is here, later ones may be in flight,
      __builtin_amdgcn_s_barrier();        // and every wave is done with the one before
      constexpr int D = NS - 1;
      load((c4 + D) % NS, i + (c4 + D) / 4, (c4 + D) % 4);
      if (PLANES && c4 == 0 && walk(i) >= walks) {   // the second and third plane
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
          for (int c = 0; c < 4; ++c) infinite |= mx_may_be_infinite((scales[P][f][c] >> (8 * g)) & 255u);
        infinite = __any(infinite);
      }
      if (c4 == 0) load_scales(1 - P, i + 1);
      __builtin_amdgcn_sched_barrier(0);
      compute(c4 % NS, P, i, c4, infinite);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  for (int i = 0; i < turns; i += 2) {
    turn(i, std::integral_constant<int, 0>{});
    if (i + 1 < turns) turn(i + 1, std::integral_constant<int, 1>{});
  }
  wait_vmcnt<0>();                         // (no load may reach LDS after the block has left it)

  const bool sliced = gridDim.z > 1;
  float* out = sliced ? a.slices + (long)blockIdx.z * a.m * a.w.n : reinterpret_cast<float*>(a.y);
  const long ldo = sliced ? a.w.n : a.ldy;
  if (a.swiglu && !sliced) {
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const int m = m0 + t * 16 + 4 * g;   // and the three rows behind
#pragma unroll
      for (int f = 0; f < H; ++f) {
        const int n = n0 + 16 * f + col;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (m + e < a.m && n < n_end)
            reinterpret_cast<T*>(a.y)[(m + e) * a.ldy + n] =
                from_f32<T>(silu_mul(acc[t][f][e], acc[t][f + H][e]));
      }
    }
    return;
  }
  float* o[NF];              // nullptr: a column behind the last
#pragma unroll
  for (int f = 0; f < NF; ++f) {
    const int n = n0 + 16 * (a.swiglu ? f % H : f) + col;
    o[f] = n < n_end ? out + (m0 + 4 * g) * ldo + n + (a.swiglu && f >= H ? n_end : 0) : nullptr;
  }
  if (a.add && !sliced && n0 < n_end) {   // all of the old values before the first store
    // In the large tiles no load is conditional, so that they go out together: 3369 x 4187
    // outputs of 382 inputs 65 us against 93. In the small ones the registers that this
    // takes would cost a block a CU: 300 rows of 3584 x 18944 71 us against 65.
    const float* p[NF];
#pragma unroll
    for (int f = 0; f < NF; ++f)   // (behind the last column: the wave's own first one, not used)
      p[f] = out + (n0 + 16 * f + col < n_end ? n0 + 16 * f + col : n0);
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int m = m0 + t * 16 + 4 * g + e;
          if constexpr (MT >= 8) {
            acc[t][f][e] += p[f][min(m, a.m - 1) * ldo];
          } else {
            if (o[f] && m < a.m) acc[t][f][e] += o[f][(t * 16 + e) * ldo];
          }
        }
  }
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (o[f] && m0 + t * 16 + 4 * g + e < a.m) o[f][(t * 16 + e) * ldo] = acc[t][f][e];
}

// The K slices of a product, added in order, and its epilogue: V columns of a row a
// thread (four where every row of the output starts at a multiple of 16 bytes).
template <typename T, int V>
__global__ __launch_bounds__(256) void mx_join_kernel(MxLinear a, int n_slices) {
  typedef float vec __attribute__((ext_vector_type(V)));
  const int n_out = a.swiglu ? a.w.n / 2 : a.w.n;
  const int n = (blockIdx.x * 256 + threadIdx.x) * V, m = blockIdx.y;
  if (n >= n_out) return;
  const long slice = (long)a.m * a.w.n;
  const float* p = a.slices + (long)m * a.w.n + n;
  vec v = *reinterpret_cast<const vec*>(p), u = {};
  if (a.swiglu) u = *reinterpret_cast<const vec*>(p + n_out);
#pragma unroll 4
  for (int s = 1; s < n_slices; ++s) {
    v += *reinterpret_cast<const vec*>(p + s * slice);
    if (a.swiglu) u += *reinterpret_cast<const vec*>(p + s * slice + n_out);
  }
  if (a.swiglu) {
    T* o = reinterpret_cast<T*>(a.y) + (long)m * a.ldy + n;
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = from_f32<T>(silu_mul(v[i], u[i]));
  } else {
    vec* o = reinterpret_cast<vec*>(reinterpret_cast<float*>(a.y) + (long)m * a.ldy + n);
    *o = a.add ? *o + v : v;
  }
}

// Launch of a planned product; x of NP planes.
template <int NP>
hipError_t launch_linear(MxLinear a, const MxTile& tl, bool join, const LaunchSpan& span, hipStream_t st) {
  const int n_out = a.swiglu ? a.w.n / 2 : a.w.n;
  const int cols = a.swiglu ? 8 : 16;    // output columns of a fragment
  a.planes = NP;
  dim3 grid;
  const int steps = ceil_div(a.w.groups, kWalk / kMxGroup) * (tl.kind == kMxFew ? 1 : NP);
  a.per_slice = ceil_div(steps, tl.slices);
  grid.z = ceil_div(steps, a.per_slice);
  if (tl.kind == kMxFew) {
    grid.x = ceil_div(n_out, cols * tl.nf), grid.y = ceil_div(a.m, 16);
#define MX_FEW(NF_, W_)                                                                            \
  if (tl.nf == NF_ && tl.waves == W_)                                                              \
  DLM_LAUNCH((mx_linear_kernel<NF_, W_, NP>), grid, dim3(W_ * 64), 0, st, a)
    MX_FEW(1, 8);
    MX_FEW(2, 8);
    MX_FEW(4, 8);
    if constexpr (NP == 1) MX_FEW(4, 4);
#undef MX_FEW
  } else {
#define MX_TILE(KIND_, WN_, MT_, NF_, NS_)                                                         \
  if (tl.kind == KIND_) {                                                                          \
    const int n_tiles = ceil_div(n_out, cols * NF_ * WN_), m_tiles = ceil_div(a.m, 16 * MT_);      \
    grid.x = ceil_div(n_tiles * m_tiles, kXcds) * kXcds, grid.y = 1;                                 \
    if (a.tail)                                                                                    \
      DLM_LAUNCH((mx_tile_kernel<WN_, MT_, NF_, NS_, (NP > 1), true>), grid, dim3(WN_ * 64), 0, st, \
                 a, n_tiles, m_tiles);                                                             \
    else                                                                                           \
      DLM_LAUNCH((mx_tile_kernel<WN_, MT_, NF_, NS_, (NP > 1), false>), grid, dim3(WN_ * 64), 0, st, \
                 a, n_tiles, m_tiles);                                                             \
  }
    MX_TILE(kMxTile32, 4, 2, 2, 4)
    MX_TILE(kMxTile64, 4, 4, 2, 2)
    MX_TILE(kMxTile128, 8, 8, 2, 2)
#undef MX_TILE
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || grid.z == 1 || !join) return e;
  span.last();
  typedef typename std::conditional<NP == 1, bf16, float>::type T;
  // (vector accesses of the slices and of fp32 outputs)
  const bool v4 = n_out % 4 == 0 && a.ldy % 4 == 0 && reinterpret_cast<uintptr_t>(a.y) % 16 == 0;
  if (v4)
    DLM_LAUNCH((mx_join_kernel<T, 4>), dim3(ceil_div(n_out, 1024), a.m), dim3(256), 0, st, a, (int)grid.z);
  else
    DLM_LAUNCH((mx_join_kernel<T, 1>), dim3(ceil_div(n_out, 256), a.m), dim3(256), 0, st, a, (int)grid.z);
  return hipGetLastError();
}

}  // namespace

// Way of a product. Times in us on MI355X (256 CUs), weights from HBM; what is modelled
// is what decides between the ways:
//  * blocks of 16 rows (mx_linear_kernel): 3.5 + the weights at 4.5 TB/s (less while blocks
//    leave CUs idle) + x, once for each column tile and K slice, at 9 TB/s out of the
//    L2s. So one row takes one column fragment a block and no slices (4096 x 4096 4.9,
//    two fragments 6.3), 32 rows two (9.1; tiles in four slices 11.5), and 10 rows of fp32
//    x over 4096 x 12288 four in four slices (20.3; two in two slices 24.6, tiles 30).
//    The model is off by up to a tenth: 16 rows of 4096 x 4096 get two slices (8.8; whole
//    7.9), one row of 24576 x 4096 four fragments (17.6; two 16.2).
//  * tiles (mx_tile_kernel): 4 + for each chunk of a slice 0.5, 0.84 or 1.7 (blocks of 32 x
//    128, 64 x 128 and 128 x 256), or 0.43, 0.55 or 1.7 for each block that a CU runs.
//    24576 x 4096: 32 rows 19.9 in the first, 128 rows 46, 38.5 and 54, 256 rows 84, 58
//    and 57; 37888 x 3584, 256 rows: 296 large blocks on 256 CUs 101, second 81.
//  * slices cost 2 + 0.8 a MB of them (mx_join_kernel and the stores), or, left to the
//    kernel that reads the output anyway, 0.5 + 0.3 a MB.
MxTile mx_tile(int elem, int rows, int n, int k, int groups, bool swiglu, bool join, int num_cu) {
  const int n_out = swiglu ? n / 2 : n, cols = swiglu ? 8 : 16, planes = elem == 2 ? 1 : 3;
  const double mb = (double)n * groups * 17e-6, x_mb = (double)rows * k * 2e-6 * planes;
  const int walks = ceil_div(groups, kWalk / kMxGroup);
  // (the tiles address their rows in 32 bits, the join its rows in one grid dimension)
  const bool wide = k > kMxTileK;
  MxTile best{};
  double best_t = 1e30;
  auto take = [&](MxTile t, int steps, double us) {
    t.slices = ceil_div(steps, ceil_div(steps, t.slices));   // none of them empty
    const double slices_mb = t.slices * rows * (double)n * 4e-6;
    if (t.slices > 1) us += join ? 2.0 + 0.8 * slices_mb : 0.5 + 0.3 * slices_mb;
    if (us < best_t) best_t = us, best = t;
  };
  struct Tile { int kind, bm, bn; double one, more; };
  static const Tile tiles[] = {{kMxTile32, 32, 128, 0.5, 0.43},
                               {kMxTile64, 64, 128, 0.84, 0.55},
                               {kMxTile128, 128, 256, 1.7, 1.7}};
  for (int s = 1; s <= (rows <= 4096 ? 8 : 1); s *= 2) {
    if ((rows <= 256 || wide) && s <= walks) {   // (small matrices: also for more than 16 rows)
      const int m_tiles = ceil_div(rows, 16);
      for (int nf = swiglu ? 2 : 1; nf <= 4; nf *= 2) {
        const int n_tiles = ceil_div(n_out, cols * nf);
        const double blocks = (double)n_tiles * m_tiles * s;
        const double idle = std::max(1.0, 0.875 * num_cu / blocks);
        const int waves = nf == 4 && planes == 1 && blocks > num_cu ? 4 : 8;
        take({kMxFew, nf, s, waves}, walks, 3.5 + mb * m_tiles * idle / 4.5 + x_mb * n_tiles / 9.0);
      }
    }
    if (wide || s > planes * walks) continue;
    const int chunks = 4 * ceil_div(planes * walks, s);
    for (const Tile& t : tiles) {
      const double fill =
          (double)ceil_div(rows, t.bm) * ceil_div(n_out, t.bn * cols / 16) * s / num_cu;
      const double share = fill < 4 || t.kind == kMxTile128 ? std::ceil(fill) : fill;
      take({t.kind, 0, s, 0}, planes * walks, 4 + chunks * std::max(t.one, t.more * share));
    }
  }
  return best;
}

// From this many rows on a bf16 matrix is unpacked once and goes through the GEMM kernels, where
// it holds kMxGemmValues or more and k is a multiple of 64, as the fast ones of those take it.
// Straight from the codes / unpacked (the unpacking included), us, at 2048, 3000 and 4096
// rows: 24576 x 4096 SwiGLU 361 / 354, 548 / 514, 752 / 645; 4096 x 12288 176 / 187, 343 /
// 297, 365 / 307; 4608 x 3584 87 / 79, 107 / 95, 160 / 121. Other k: 4096 x 4088 71 / 114,
// 133 / 174, 139 / 195; 24576 x 3608 SwiGLU 366 / 518, 540 / 771, 741 / 1029. Smaller
// matrices: 2048 x 2048 25 / 30, 34 / 48, 39 / 52; 1088 x 1024 15 / 19, 16 / 19, 21 / 26.
// (At 1024 rows 24576 x 4096 182 / 217, 12288 x 4096 110 / 105. fp32 stays with the codes:
// three bf16 products take half of an fp32 one, 24576 x 4096 at 1024 rows 503. Narrow
// matrices stay too: 41 x 2608 at 3636 rows 14 / 55.)
constexpr int kMxGemmRows = 2048, kMxGemmCols = 1024;
constexpr long kMxGemmValues = 1L << 23;

MxPlan mx_plan(int elem, int rows, int n, int k, long ldx, bool swiglu, bool x_aligned, bool y_aligned,
               bool join, int num_cu) {
  MxPlan p;
  // (the GEMM kernels address their operands by 32-bit element offsets)
  const bool near = std::max((double)rows * ldx, (double)n * k) < 4294967296.0;
  if (elem == 2 && near && x_aligned && y_aligned && rows >= kMxGemmRows && n >= kMxGemmCols && k % 64 == 0 &&
      (long)n * k >= kMxGemmValues && (!swiglu || n % 32 == 0)) {
    p.gemm = true;
    // (without the join, K slices as those of a dense projection)
    p.g = join ? gemm_plan(elem, rows, n, k, false, num_cu, !swiglu, true, !swiglu)
               : gemm_plan(elem, rows, n, k, true, num_cu);
    p.scratch = (size_t)n * k * elem;
    return p;
  }
  const int groups = ceil_div(k, kMxGroup), planes = elem == 2 ? 1 : 3;
  p.tile = mx_tile(elem, std::max(rows, 1), n, k, groups, swiglu, join, num_cu);
  p.join = join;
  p.staged = elem != 2 || !x_aligned || k % 8 != 0;
  if (p.staged) p.stage = ((size_t)rows * groups * kMxGroup * 2 * planes + 255) / 256 * 256;
  p.scratch = p.stage;
  if (join && p.tile.slices > 1) p.scratch += (size_t)p.tile.slices * rows * n * sizeof(float);
  return p;
}

template <typename T>
hipError_t mx_matmul(const MxPlan& plan, const T* x, long ldx, int rows, const MxView& w, int k,
                     int epilogue, void* y, long ldy, void* scratch, hipStream_t st) {
  if (rows <= 0 || w.n <= 0) return hipSuccess;
  const bool swiglu = epilogue == DLM_MX_SWIGLU, add = epilogue == DLM_MX_ADD;
  if (plan.gemm) {
    T* dense = reinterpret_cast<T*>(scratch);
    const LaunchSpan span(true);
    const hipError_t e = mx_unpack<T>(w, k, dense, k, st);
    if (e != hipSuccess) return e;
    span.last();
    if (swiglu)
      return gemm_swiglu<T>(plan.g, x, (int)ldx, dense, k, rows, w.n / 2, k, reinterpret_cast<T*>(y),
                            (int)ldy, st);
    float* c = reinterpret_cast<float*>(y);
    return add ? gemm_add_f32<T>(plan.g, x, (int)ldx, dense, k, rows, w.n, k, c, (int)ldy, st)
               : gemm_store_f32<T>(plan.g, x, (int)ldx, dense, k, rows, w.n, k, c, (int)ldy, st);
  }
  constexpr int NP = sizeof(T) == 2 ? 1 : 3;
  MxLinear a{};
  a.w = w, a.m = rows, a.k = k, a.tail = k % kMxGroup, a.swiglu = swiglu, a.add = add, a.y = y, a.ldy = ldy;
  a.slices = plan.join ? reinterpret_cast<float*>(reinterpret_cast<char*>(scratch) + plan.stage)
                       : reinterpret_cast<float*>(y);
  const bool joined = plan.join && plan.tile.slices > 1;
  const LaunchSpan span(plan.staged || joined);
  if (plan.staged) {
    const int kp = w.groups * kMxGroup;
    const long total = (long)rows * kp;
    bf16* xs = reinterpret_cast<bf16*>(scratch);
    DLM_LAUNCH((mx_stage_kernel<T, NP>), dim3(ceil_div(kp / 8, 256), std::min(rows, 65535)), dim3(256), 0,
               st, x, ldx, rows, k, kp, total, xs);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.x = xs, a.ldx = kp, a.plane = total, a.k = kp;
  } else if constexpr (NP == 1) {
    a.x = x, a.ldx = ldx;
  } else {
    return hipErrorInvalidValue;
  }
  if (!joined) span.last();
  return launch_linear<NP>(a, plan.tile, plan.join, span, st);
}

#define INST(T)                                                                                 \
  template hipError_t mx_matmul<T>(const MxPlan&, const T*, long, int, const MxView&, int, int, \
                                   void*, long, void*, hipStream_t);
INST(bf16)
INST(float)
#undef INST

}  // namespace dlm
