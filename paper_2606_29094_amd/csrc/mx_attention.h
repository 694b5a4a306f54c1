// Attention over a cache in 4 bits (mx_common.h). Part of attention.hip.
#pragma once

#include <algorithm>
#include <cmath>

#include "mx_common.h"
#include "mx_kernels.h"

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
typedef float f32x2 __attribute__((ext_vector_type(2)));

// V's part of LDS: kVRow bytes a key, 16-byte slot s (columns 8 s ..) of a key at v_slot.
// head_dim 128: the 32-byte blocks of a row and the halves of a block change places with
// the key, so that the eight rows that half a wave reads at one block, and the four keys
// that 16 lanes write, are in distinct banks. head_dim 64: rows 160 bytes apart, whose
// addresses are one base and constants. (With the weights in one term: rows 288 bytes
// apart at head_dim 128, 10240 rows of 32 heads over 1280 keys 239 us against 233; blocks
// exchanged at head_dim 64, 16 requests of 64 rows over 2000 keys 23.5 against 22.9.)
template <int DH>
constexpr int kVRow = DH == 128 ? 256 : DH * 2 + 32;
template <int DH>
__device__ __forceinline__ int v_slot(int key, int s) {
  if constexpr (DH == 128)
    s ^= ((key & 3) | (key >> 3 & 1) << 2) << 1 | (key >> 1 & 1);
  return key * kVRow<DH> + s * 16;
}

// eight keys (8 g .. 8 g + 7 of the 32 at `rows`) of V column d0 + lane % 16: two
// transposing reads, each of which hands a 16-lane group the columns of a [4 keys][16
// columns] block
template <int DH>
__device__ __forceinline__ bf16x8 v_columns(const char* rows, int d0, int lane) {
  typedef __attribute__((address_space(3))) s16x4* lds_t;
  const int key = 8 * (lane >> 4) + ((lane & 15) >> 2), s = d0 / 8 + (lane >> 1 & 1);
  const int at = v_slot<DH>(key, s) + (lane & 1) * 8;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(rows + at));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(rows + at + 4 * kVRow<DH>));
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  return __builtin_bit_cast(bf16x8, s16x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
}

// Online softmax of a lane's query over the 16 scores s[n][i] it owns of a 64-key tile (the
// other 48 are in the lanes 16, 32 and 48 further): the weights in NP bf16 terms as the B
// operands p[h] of the two 32-key steps, their sum added to l. m is a reference, not the
// maximum: it only moves (and l and the output are scaled) when a score exceeds it by
// more than 8 / c, so weights stay below 2^8 and most tiles skip the scaling. Returns
// what the output is to be multiplied by, where any query of the wave moves.
struct Rescale { bool any; float by; };
template <int NP>
__device__ __forceinline__ Rescale softmax_tile(const f32x4 (&s)[4], float c, float& m, float& l,
                                                bf16x8 (&p)[2][NP]) {
  float mx = s[0][0];
#pragma unroll
  for (int n = 0; n < 4; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[n][i]);
  mx = fmaxf(mx, __shfl_xor(mx, 16, kWave));
  mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
  Rescale r{false, 1.f};
  if (__any((mx - m) * c > 8.f)) {       // (m starts at -inf: the first tile with a score moves it)
    const float to = (mx - m) * c > 8.f ? mx : m;
    r.any = true;
    r.by = to == m ? 1.f : __builtin_amdgcn_exp2f((m - to) * c);
    l *= r.by;
    m = to;
  }
  const float mc = m == -INFINITY ? 0.f : m * c;   // (no key with a score yet)
#pragma unroll
  for (int n = 0; n < 4; ++n)
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
      const int e = 4 * (n & 1) + i;
      const f32x2 w = {__builtin_amdgcn_exp2f(s[n][i] * c - mc), __builtin_amdgcn_exp2f(s[n][i + 1] * c - mc)};
      l += w[0];
      l += w[1];
      if constexpr (NP == 2) {             // (one conversion instruction for a pair's terms)
        const bf16x2 hi = __builtin_convertvector(w, bf16x2);
        const bf16x2 lo = __builtin_convertvector(w - __builtin_convertvector(hi, f32x2), bf16x2);
        p[n >> 1][0][e] = hi[0], p[n >> 1][0][e + 1] = hi[1];
        p[n >> 1][1][e] = lo[0], p[n >> 1][1][e + 1] = lo[1];
      } else {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          bf16 hi, mid, lo;
          split3(w[u], hi, mid, lo);
          p[n >> 1][0][e + u] = hi;
          p[n >> 1][1][e + u] = mid;
          p[n >> 1][2][e + u] = lo;
        }
      }
    }
  return r;
}

// O^T += V^T P^T of a 64-key tile. The terms of a weight go into the same sums: two column
// blocks are taken together, so that an MFMA does not wait for the one right before it.
template <int DH, int QT, int PN>
__device__ __forceinline__ void add_values(const char* rows, int lane, const bf16x8 (&p)[QT][2][PN],
                                           f32x4 (&o)[DH / 16][QT]) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int d = 0; d < DH / 16; d += 2) {
      const bf16x8 v[2] = {v_columns<DH>(rows + 32 * h * kVRow<DH>, 16 * d, lane),
                           v_columns<DH>(rows + 32 * h * kVRow<DH>, 16 * d + 16, lane)};
#pragma unroll
      for (int w = PN - 1; w >= 0; --w)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int t = 0; t < QT; ++t) o[d + u][t] = mfma16_bf16(v[u], p[t][h][w], o[d + u][t]);
    }
}

// Few query rows: one block = 16 QT items of one key/value head, wave w
// takes the 64-key tiles w, w + W, ... of the block's key range, each with its own
// online softmax, merged in LDS at the end. Scores as S^T = K Q^T (16x16x32 MFMA, keys
// as the A operand straight from the codes in registers: lane l holds group l / 16 of key
// l % 16, whose dword j is the A fragment of step j), so a lane owns one query and 16
// keys; the keys of a tile are dealt to the rows of S^T so that a lane's weights are
// the B operand of O^T = V^T P^T as they stand. V is unpacked into the wave's part of
// LDS key by key (its scales belong to keys) and read back transposed. The next tile's
// codes are requested before the current one's are used. Bound by the chain of a wave's
// tiles and the join of the waves (32 rows of 32 heads: eight requests over 1280 keys 22.3
// us, five tiles a wave; one over 4256 keys in eight splits 19.3).
// bf16 queries: one term for an element, two for a weight (off by 2^-16 of itself at most,
// far below the output's rounding; one term, off by 2^-8, put an error of its own size beside
// that rounding). fp32 queries: three terms for each, which hold all 24 bits.
template <typename T, int DH, int QT, int W>
__global__ __launch_bounds__(W * 64, 2) void mx_attn_kernel(StepPlan p, const T* __restrict__ q,
                                                         MxAttn a, T* __restrict__ out) {
  constexpr int NP = sizeof(T) == 2 ? 1 : 3, PN = sizeof(T) == 2 ? 2 : 3;   // of a query, a weight
  constexpr int GROUPS = DH / kMxGroup;
  constexpr int KS = DH / 32;               // MFMA steps over dh
  constexpr int PER = DH / 4;               // elements of a key in a lane: 32 or 16
  constexpr int DT = DH / 16;
  constexpr int VBYTES = 64 * kVRow<DH>;
  static_assert(VBYTES >= QT * 16 * DH * 4, "the merge reuses the wave's part");
  __shared__ __attribute__((aligned(16))) char smem[W * VBYTES];
  __shared__ float2 stat[W][QT * 16];

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, g = lane >> 4;
  const int gh = a.hq / a.hkv;
  const int head = blockIdx.x % a.hkv;      // fastest: blocks of one head go to few XCDs
  const int tile = blockIdx.x / a.hkv;
  const int r = plan_req_of_tile(p, tile);
  const ReqPlan& rq = p.r[r];
  const int item0 = (tile - rq.tile0) * 16 * QT, items = rq.nrows * gh;
  const int split = blockIdx.z;
  const int len = rq.seq_len;
  const int tiles = ceil_div(len, 64), per = ceil_div(tiles, a.splits);
  const int t0 = min(split * per, tiles), t1 = min(t0 + per, tiles);

  const long base = ((long)rq.slot * a.hkv + head) * a.kv.s_max;
  const uint8_t* kc = a.kv.kc + base * (DH / 2);
  const uint8_t* vc = a.kv.vc + base * (DH / 2);
  const uint8_t* ks = a.kv.ks + base * GROUPS;
  const uint8_t* vs = a.kv.vs + base * GROUPS;
  char* vrows = smem + wave * VBYTES;

  // the codes of a tile: V in whole groups, key by key; of K this lane's part of the key
  // that is row l % 16 of each key tile n of S^T, 32 (n / 2) + 8 (x / 4) + 4 (n % 2) + x % 4.
  // (A slot holds a multiple of 64 positions: what lies behind the sequence is read.)
  constexpr int VN = GROUPS;
  typedef uint32_t kpart __attribute__((ext_vector_type(PER / 8)));
  struct Codes { u32x4 v[VN]; kpart k[4]; uint32_t ve[VN], ke[4]; };
  auto load = [&](Codes& x, int kt) {
    const long k0 = (long)kt * 64;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const long key = k0 + 32 * (n >> 1) + 8 * (col >> 2) + 4 * (n & 1) + (col & 3);
      x.k[n] = *reinterpret_cast<const kpart*>(kc + key * (DH / 2) + g * (PER / 2));
      x.ke[n] = ks[key * GROUPS + g * PER / kMxGroup];
    }
#pragma unroll
    for (int u = 0; u < VN; ++u) {
      x.v[u] = reinterpret_cast<const u32x4*>(vc)[k0 * GROUPS + u * 64 + lane];
      x.ve[u] = vs[k0 * GROUPS + u * 64 + lane];
    }
  };
  Codes cur, next;
  if (t0 + wave < t1) load(cur, t0 + wave);

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
    load(next, min(kt + W, t1 - 1));
    __builtin_amdgcn_sched_barrier(0);
    const bool last = k0 + 64 > len;        // the sequence ends inside: what is behind counts as nothing
#pragma unroll
    for (int u = 0; u < VN; ++u) {
      const int at = u * 64 + lane, key = at / GROUPS, gr = at % GROUPS;
      if (last && k0 + key >= len) cur.v[u] = u32x4{0u, 0u, 0u, 0u}, cur.ve[u] = 127u;
      const float s = mx_scale(cur.ve[u]);
#pragma unroll
      for (int w = 0; w < 4; ++w)
        *reinterpret_cast<bf16x8*>(vrows + v_slot<DH>(key, 4 * gr + w)) = mx_bf16x8(cur.v[u][w], s);
    }
    f32x4 s[QT][4];
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const float sc = mx_scale(cur.ke[n]);
#pragma unroll
      for (int t = 0; t < QT; ++t) s[t][n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < KS; ++j) {
        const bf16x8 kf = mx_bf16x8(cur.k[n][j], sc);
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int w = NP - 1; w >= 0; --w) s[t][n] = mfma16_bf16(kf, qf[t][j][w], s[t][n]);
      }
    }
    if (last) {
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (k0 + 32 * (n >> 1) + 8 * g + 4 * (n & 1) + i >= len)
#pragma unroll
            for (int t = 0; t < QT; ++t) s[t][n][i] = -INFINITY;
    }
    bf16x8 pf[QT][2][PN];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const Rescale f = softmax_tile<PN>(s[t], a.c, m[t], l[t], pf[t]);
      if (f.any)
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d][t] *= f.by;
    }
    // the wave's own stores to LDS, before it reads them
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    add_values<DH, QT, PN>(vrows, lane, pf, o);
    // and its reads, before the next tile's stores
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    cur = next;
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
      const float f = __builtin_amdgcn_exp2f((stat[w][x].x - ref) * a.c);
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

// Many query rows: one block = NW waves of 16 QT items each that share the 64-key tiles.
// The threads fetch a tile's codes two tiles ahead, and unpack them into one of two LDS
// stages while the other is multiplied, so each key and value is unpacked once for 16 QT
// NW queries. Scores and outputs as above; K rows are stored in the order in which
// S^T deals the keys (row 32 h + 16 b + 4 a + i holds key 32 h + 8 a + 4 b + i), their
// 16-byte slots at s ^ (row & mask), so that the rows a fragment reads come from
// distinct banks. Bound by the three pipes in turn (10240 rows of 32 heads over 1280 keys
// 290 us, 0.74 PFLOP/s; vector units 54 % busy, matrix cores 44, LDS 39; with the weights
// in one term 239).
template <int DH, int QT, int NW>
__global__ __launch_bounds__(NW * 64, 2) void mx_attn_shared_kernel(StepPlan p, const bf16* __restrict__ q,
                                                                 MxAttn a, bf16* __restrict__ out) {
  constexpr int GROUPS = DH / kMxGroup, KS = DH / 32, DT = DH / 16;
  constexpr int SLOTS = DH / 8;                    // 16-byte slots of a K row
  constexpr int KBYTES = 64 * DH * 2, VBYTES = 64 * kVRow<DH>;
  constexpr int NT = NW * 64, NG = 64 * GROUPS, PARTS = 2 * NG / NT;   // groups of K and of V
  static_assert(2 * NG % NT == 0 && (NG % NT == 0 || NT % NG == 0), "whole parts, of K or of V");
  __shared__ __attribute__((aligned(16))) char smem[2 * (KBYTES + VBYTES)];

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, g = lane >> 4;
  const int gh = a.hq / a.hkv;
  const int head = blockIdx.x % a.hkv;             // fastest: blocks of one head go to few XCDs
  const int tile = blockIdx.x / a.hkv;
  const int r = plan_req_of_tile(p, tile);
  const ReqPlan& rq = p.r[r];
  const int items = rq.nrows * gh;
  const int item0 = (tile - rq.tile0) * 16 * QT * NW + wave * 16 * QT;
  const int split = blockIdx.z;
  const int len = rq.seq_len;
  const int tiles = ceil_div(len, 64), per = ceil_div(tiles, a.splits);
  const int t0 = min(split * per, tiles), t1 = min(t0 + per, tiles);

  const long base = ((long)rq.slot * a.hkv + head) * a.kv.s_max;
  // this thread's groups of a tile: part u is group i = tid + u NT, the first NG of K
  struct Codes { u32x4 c[PARTS]; uint32_t e[PARTS]; };
  auto load = [&](Codes& x, int kt) {
#pragma unroll
    for (int u = 0; u < PARTS; ++u) {
      const int i = threadIdx.x + u * NT;
      const bool v = i >= NG;
      const long at = (base + (long)kt * 64) * GROUPS + i - (v ? NG : 0);
      x.c[u] = reinterpret_cast<const u32x4*>(v ? a.kv.vc : a.kv.kc)[at];
      x.e[u] = (v ? a.kv.vs : a.kv.ks)[at];
    }
  };
  auto unpack = [&](Codes& x, int kt, int stage) {
    char* st = smem + stage * (KBYTES + VBYTES);
#pragma unroll
    for (int u = 0; u < PARTS; ++u) {
      const int i = threadIdx.x + u * NT;
      const bool v = i >= NG;
      const int at = i - (v ? NG : 0), key = at / GROUPS, gr = at % GROUPS;
      if (v && kt * 64 + key >= len) x.c[u] = u32x4{0u, 0u, 0u, 0u}, x.e[u] = 127u;
      const float s = mx_scale(x.e[u]);
      const int row = (key & 32) | (key & 4) << 2 | (key & 24) >> 1 | (key & 3);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        char* to = v ? st + KBYTES + v_slot<DH>(key, 4 * gr + w)
                     : st + row * DH * 2 + ((4 * gr + w) ^ (row & (SLOTS - 1))) * 16;
        *reinterpret_cast<bf16x8*>(to) = mx_bf16x8(x.c[u][w], s);
      }
    }
  };
  Codes ahead;
  if (t0 < t1) load(ahead, t0);
  bf16x8 qf[QT][KS];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int it = max(min(item0 + 16 * t + col, items - 1), 0);
    const bf16* src = q + ((long)(rq.row0 + it / gh) * a.hq + head * gh + it % gh) * DH + 8 * g;
#pragma unroll
    for (int j = 0; j < KS; ++j) qf[t][j] = *reinterpret_cast<const bf16x8*>(src + 32 * j);
  }
  f32x4 o[DT][QT];
  float m[QT], l[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m[t] = -INFINITY;
    l[t] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  if (t0 < t1) {
    unpack(ahead, t0, 0);
    load(ahead, min(t0 + 1, t1 - 1));
  }
  for (int kt = t0; kt < t1; ++kt) {
    const int stage = (kt - t0) & 1, k0 = kt * 64;
    const char* st = smem + stage * (KBYTES + VBYTES);
    lds_barrier();                       // tile kt is in its stage, nobody reads the other one
    f32x4 s[QT][4];
#pragma unroll
    for (int n = 0; n < 4; ++n) {
#pragma unroll
      for (int t = 0; t < QT; ++t) s[t][n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < KS; ++j) {
        const bf16x8 kf = *reinterpret_cast<const bf16x8*>(
            st + (16 * n + col) * DH * 2 + ((4 * j + g) ^ (col & (SLOTS - 1))) * 16);
#pragma unroll
        for (int t = 0; t < QT; ++t) s[t][n] = mfma16_bf16(kf, qf[t][j], s[t][n]);
      }
    }
    if (kt + 1 < t1) {
      unpack(ahead, kt + 1, stage ^ 1);
      load(ahead, min(kt + 2, t1 - 1));
    }
    if (k0 + 64 > len) {
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (k0 + 32 * (n >> 1) + 8 * g + 4 * (n & 1) + i >= len)
#pragma unroll
            for (int t = 0; t < QT; ++t) s[t][n][i] = -INFINITY;
    }
    bf16x8 pf[QT][2][2];                 // weights in two terms, as above
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const Rescale f = softmax_tile<2>(s[t], a.c, m[t], l[t], pf[t]);
      if (f.any)
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d][t] *= f.by;
    }
    add_values<DH, QT, 2>(st + KBYTES, lane, pf, o);
  }
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    l[t] += __shfl_xor(l[t], 16, kWave);
    l[t] += __shfl_xor(l[t], 32, kWave);
    const int it = item0 + 16 * t + col;
    if (it >= items) continue;
    const long at = (long)(rq.row0 + it / gh) * a.hq + head * gh + it % gh;
    if (a.splits > 1) {
      const long rows = (long)p.n_rows * a.hq;
#pragma unroll
      for (int d = 0; d < DT; ++d)
        *reinterpret_cast<f32x4*>(a.po + (split * rows + at) * DH + 16 * d + 4 * g) = o[d][t];
      // a row over no keys: weight one on an output of zeros
      if (g == 0)
        a.ml[split * rows + at] = len == 0 && split == 0 ? make_float2(0.f, 1.f) : make_float2(m[t], l[t]);
      continue;
    }
    const float inv = len > 0 ? 1.f / l[t] : 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d)
      *reinterpret_cast<bf16x4*>(out + at * DH + 16 * d + 4 * g) =
          bf16x4{(bf16)(o[d][t][0] * inv), (bf16)(o[d][t][1] * inv), (bf16)(o[d][t][2] * inv),
                 (bf16)(o[d][t][3] * inv)};
  }
}

// The S key splits of each (row, head), added in order. A split without keys has
// weight zero. Bound by latency: everything is loaded before anything is used (12 heads,
// 16 splits: 8.2 us by a loop over them, 3.2 so).
template <typename T, int DH, int S>
__global__ __launch_bounds__(256) void mx_merge_kernel(MxAttn a, long items, T* __restrict__ out) {
  constexpr int QUADS = DH / 4;
  const long at = ((long)blockIdx.x * 256 + threadIdx.x) / QUADS;
  const int d = threadIdx.x % QUADS * 4;
  if (at >= items) return;
  float2 ml[S];
  f32x4 po[S];
#pragma unroll
  for (int s = 0; s < S; ++s) ml[s] = a.ml[s * items + at];
#pragma unroll
  for (int s = 0; s < S; ++s) po[s] = *reinterpret_cast<const f32x4*>(a.po + (s * items + at) * DH + d);
  float mx = ml[0].x;
#pragma unroll
  for (int s = 1; s < S; ++s) mx = fmaxf(mx, ml[s].x);
  const float ref = mx == -INFINITY ? 0.f : mx;
  float sum = 0.f;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const float f = __builtin_amdgcn_exp2f((ml[s].x - ref) * a.c);
    sum += ml[s].y * f;
    v += po[s] * f;
  }
  const float inv = 1.f / sum;
  typedef T T4 __attribute__((ext_vector_type(4)));
  *reinterpret_cast<T4*>(out + at * DH + d) = T4{from_f32<T>(v[0] * inv), from_f32<T>(v[1] * inv),
                                                 from_f32<T>(v[2] * inv), from_f32<T>(v[3] * inv)};
}

constexpr int kMxSplits = 16;   // at most, and a power of two

template <typename T, int DH>
hipError_t launch_attention(const StepPlan& p, const T* q, const MxAttn& a, MxAttnPlan plan, T* out,
                            hipStream_t st) {
  const int gh = a.hq / a.hkv;
  // items of a block
  const int per = plan.kind == kMxAttnShared128 ? 128 : plan.kind == kMxAttnShared64 ? 64 : sizeof(T) == 2 ? 32 : 16;
  const StepPlan t = plan_with_tiles(p, [&](int n) { return ceil_div(n * gh, per); });
  if (t.n_tiles == 0) return hipSuccess;
  const dim3 grid(t.n_tiles * a.hkv, 1, a.splits);
  const LaunchSpan span(a.splits > 1);
  if constexpr (sizeof(T) == 2) {
    if (plan.kind == kMxAttnShared128)
      DLM_LAUNCH((mx_attn_shared_kernel<DH, 2, 4>), grid, dim3(256), 0, st, t, q, a, out);
    else if (plan.kind == kMxAttnShared64)
      DLM_LAUNCH((mx_attn_shared_kernel<DH, 1, 4>), grid, dim3(256), 0, st, t, q, a, out);
    else
      DLM_LAUNCH((mx_attn_kernel<T, DH, 2, 4>), grid, dim3(256), 0, st, t, q, a, out);
  } else {
    DLM_LAUNCH((mx_attn_kernel<T, DH, 1, 4>), grid, dim3(256), 0, st, t, q, a, out);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  span.last();
  const long items = (long)p.n_rows * a.hq;
  const dim3 merge((unsigned)((items * (DH / 4) + 255) / 256));
#define MX_MERGE(S_) \
  if (a.splits == S_) DLM_LAUNCH((mx_merge_kernel<T, DH, S_>), merge, dim3(256), 0, st, a, items, out)
  MX_MERGE(2);
  MX_MERGE(4);
  MX_MERGE(8);
  MX_MERGE(16);
#undef MX_MERGE
  return hipGetLastError();
}

}  // namespace

size_t mx_attention_scratch(int rows, int hq, int dh, int splits) {
  if (splits <= 1) return 0;
  return (size_t)splits * rows * hq * (dh * sizeof(float) + sizeof(float2));
}

// Kernel and key splits. Times in us on MI355X (256 CUs), head_dim 128: 6.5, and for each
// 64-key tile that a block walks 0.555, 1.3 or 2.03 (32 items whose four waves split the
// keys, 64 and 128 items that share them) while every CU has one block, or 0.48, 1.04 or
// 1.62 for each block that a CU runs where it has more; a block's start and end (the join of
// its waves) count as 9, 1 and 1.5 tiles; head_dim 64 takes 0.67 and 0.6 of these, and 0.55 of
// the tiles for start and end. Splits add the joining kernel, 3.5, and their partials' way at
// 3 TB/s.
// So 32 rows over 1280 keys of 8 requests, 32 heads, take blocks of 32 (22.3; of 64: 33.7),
// 28/4 heads, 16 requests of 64 rows over 1024 keys blocks of 64 (40.4; 128: 41.5, 32: 47.6),
// 64 of them blocks of 128 (113; 64: 125, 32: 146), and one request of 32 rows over 4256 keys,
// 32 heads, eight splits (19.3; four 22.5).
// fp32 queries have the first kernel alone, with 16 items.
MxAttnPlan mx_attention_plan(const StepPlan& p, int hq, int hkv, int dh, size_t elem,
                             size_t scratch_bytes, int num_cu) {
  struct Kind { int kind, items, waves; double one, more, ends; };
  static const Kind kinds[] = {{kMxAttnFew, 32, 4, 0.555, 0.48, 9.0},
                               {kMxAttnShared64, 64, 1, 1.3, 1.04, 1.0},
                               {kMxAttnShared128, 128, 1, 2.03, 1.62, 1.5}};
  const int gh = hq / hkv;
  const double one = dh == 64 ? 0.67 : 1.0, more = dh == 64 ? 0.6 : 1.0, ends = dh == 64 ? 0.55 : 1.0;
  MxAttnPlan best;
  double best_t = 1e30;
  for (const Kind& k : kinds) {
    if (elem != 2 && k.kind != kMxAttnFew) break;
    const int items = elem == 2 ? k.items : 16;
    for (int s = 1; s <= kMxSplits; s *= 2) {
      long blocks = 0;
      double work = 0.0, longest = 0.0;
      for (int r = 0; r < p.n_req; ++r) {
        const long b = (long)hkv * ceil_div(p.r[r].nrows * gh, items) * s;
        int tiles = ceil_div(ceil_div(p.r[r].seq_len, 64), s);
        tiles = ceil_div(tiles, k.waves) * k.waves;
        blocks += b;
        const double walk = tiles + k.ends * ends;
        work += b * walk;
        if (b) longest = std::max(longest, walk);
      }
      if (s > 1 && (blocks > num_cu || mx_attention_scratch(p.n_rows, hq, dh, s) > scratch_bytes)) break;
      const double fill = (double)blocks / num_cu;   // blocks of a CU; few of them come whole
      const double share = fill > 1 && fill < 4 ? std::ceil(fill) / fill : 1.0;
      double t = 6.5 + std::max(longest * k.one * one, work * share * k.more * more / num_cu);
      if (s > 1) t += 3.5 + 2.0 * mx_attention_scratch(p.n_rows, hq, dh, s) / 3e6;
      if (t < best_t) best_t = t, best = MxAttnPlan{k.kind, s};
    }
  }
  return best;
}

template <typename T>
hipError_t mx_attention(const StepPlan& p, const T* q, const MxKv& kv, int hq, int hkv, int dh,
                        T* out, MxAttnPlan plan, float* scratch, hipStream_t st) {
  if (hkv < 1 || hq % hkv != 0 || plan.splits < 1 || plan.splits > kMxSplits ||
      (plan.splits & (plan.splits - 1)) != 0 ||
      (plan.splits > 1 && !scratch))
    return hipErrorInvalidValue;
  if (p.n_rows == 0) return hipSuccess;
  MxAttn a{kv, hq, hkv, plan.splits, 1.4426950408889634f / sqrtf((float)dh), scratch,
           reinterpret_cast<float2*>(scratch + (size_t)plan.splits * p.n_rows * hq * dh)};
  if (dh == 128) return launch_attention<T, 128>(p, q, a, plan, out, st);
  if (dh == 64) return launch_attention<T, 64>(p, q, a, plan, out, st);
  return hipErrorInvalidValue;
}

#define INST(T)                                                                                  \
  template hipError_t mx_attention<T>(const StepPlan&, const T*, const MxKv&, int, int, int, T*, \
                                      MxAttnPlan, float*, hipStream_t);
INST(bf16)
INST(float)
#undef INST

}  // namespace dlm
