// 4-bit matrices and caches (mx_common.h), row by row: packing, unpacking, appending
// rotated keys and values, reading them back. Part of rowwise.hip.
#pragma once

#include <algorithm>

#include "mx_common.h"
#include "mx_kernels.h"

namespace dlm {

namespace {

// ------------------------------------------------------------ pack, unpack --
// Bound by memory. A lane takes 16 bytes of the wide matrix, so a group is held by four
// lanes (bf16) or eight (fp32) that find its largest magnitude by exchanges within the
// row of lanes, and the wide matrix moves in whole lines. (One thread for each group, its
// lines in 64- and 128-byte strides: 4096 x 4096 bf16, both directions 25.5 us against
// 21.0, 37888 x 3584 fp32 340 against 237.) VEC: rows are whole 16-byte vectors; else
// their elements are loaded and stored one by one (2781 x 14407 bf16 both ways 108 us, 304 by
// a thread for each group).
constexpr int kPackVecs = 4;             // vectors of a thread, loaded together

// largest of the 16 / sizeof(T) lanes that hold a group
template <int LANES>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xb1, 0xf, 0xf, true));   // lane ^ 1
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4e, 0xf, 0xf, true));   // lane ^ 2
  if constexpr (LANES == 8)
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xf, 0xf, true));  // 7 - lane
  return v;
}

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void mx_pack_kernel(const T* __restrict__ w, long ldw, int k,
                                                      MxView o) {
  constexpr int V = 16 / sizeof(T), LANES = kMxGroup / V;
  typedef T vt __attribute__((ext_vector_type(V)));
  const int vecs = o.groups * LANES;
  const int at0 = blockIdx.x * 256 * kPackVecs + threadIdx.x;
  for (long row = blockIdx.y; row < o.n; row += gridDim.y) {
    vt x[kPackVecs];
#pragma unroll
    for (int u = 0; u < kPackVecs; ++u) {
      const int at = at0 + u * 256;
      const T* p = w + row * ldw + at * V;
      if constexpr (VEC) {
        x[u] = at * V < k ? *reinterpret_cast<const vt*>(p) : vt{};
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) x[u][i] = at * V + i < k ? p[i] : (T)0.f;
      }
    }
#pragma unroll
    for (int u = 0; u < kPackVecs; ++u) {
      const int at = at0 + u * 256;       // (all lanes of a group are in or out)
      uint32_t amax = 0;
#pragma unroll
      for (int i = 0; i < V; ++i) amax = max(amax, __float_as_uint(to_f32((T)x[u][i])) & 0x7fffffffu);
      const uint32_t e = mx_scale_byte(group_max<LANES>(amax));
      if (at >= vecs) continue;
      const float s = mx_scale(e);
      uint32_t c[V / 4];
#pragma unroll
      for (int i = 0; i < V / 4; ++i)
        c[i] = e == 255u ? 0u : mx_codes4(to_f32((T)x[u][4 * i]), to_f32((T)x[u][4 * i + 1]),
                                          to_f32((T)x[u][4 * i + 2]), to_f32((T)x[u][4 * i + 3]), s);
      uint8_t* codes = o.codes + row * o.groups * 16 + at * (V / 2);
      if constexpr (V == 8) *reinterpret_cast<uint32_t*>(codes) = c[0] | c[1] << 16;
      else *reinterpret_cast<uint16_t*>(codes) = (uint16_t)c[0];
      if (at % LANES == 0) o.scales[row * o.scale_ld + at / LANES] = (uint8_t)e;
    }
    const int g = o.groups + threadIdx.x;   // the row's padding scales
    if (blockIdx.x == 0 && g < o.scale_ld) o.scales[row * o.scale_ld + g] = 0;
  }
}

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void mx_unpack_kernel(MxView w, int k, T* __restrict__ out, long ldo) {
  constexpr int V = 16 / sizeof(T), LANES = kMxGroup / V;
  typedef T vt __attribute__((ext_vector_type(V)));
  const int at0 = blockIdx.x * 256 * kPackVecs + threadIdx.x;
  for (long row = blockIdx.y; row < w.n; row += gridDim.y) {
    uint32_t c[kPackVecs], e[kPackVecs];
#pragma unroll
    for (int u = 0; u < kPackVecs; ++u) {
      const int at = at0 + u * 256;
      if (at * V >= k) continue;
      const uint8_t* p = w.codes + row * w.groups * 16 + at * (V / 2);
      c[u] = V == 8 ? *reinterpret_cast<const uint32_t*>(p) : *reinterpret_cast<const uint16_t*>(p);
      e[u] = w.scales[row * w.scale_ld + at / LANES];
    }
#pragma unroll
    for (int u = 0; u < kPackVecs; ++u) {
      const int at = at0 + u * 256;
      if (at * V >= k) continue;
      const bf16x8 x = mx_bf16x8(c[u], mx_scale(e[u]));
      vt v;
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = (T)(float)x[i];
      T* p = out + row * ldo + at * V;
      if constexpr (VEC) {
        *reinterpret_cast<vt*>(p) = v;
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (at * V + i < k) p[i] = v[i];
      }
    }
  }
}

// ------------------------------------------------------------------ append --
// One block: 256 / QUADS heads of one row, QUADS = dh / 8 lanes a head; a lane takes
// four consecutive elements of the head's first half and the same four of the
// second, which are its rotary partners. Eight lanes hold a group of 32 of each
// half and find its largest magnitude with three lane exchanges. Bound by memory:
// it reads the product's fp32 slices once (10240 rows of 32 heads, one slice: 138 us,
// 4.6 TB/s; 32 rows, two slices: 3.6 us, the launch and two dependent loads).
//
// Every product of the rotation is rounded by itself (no fused multiply-add): the
// stored codes then follow from the inputs by plain fp32 operations, and a value on
// the border of two codes falls to the same side wherever it is computed.
template <typename T, int DH>
__global__ __launch_bounds__(256) void mx_append_kernel(StepPlan p, const float* __restrict__ qkv,
                                                        int splits, long split_stride,
                                                        const float2* __restrict__ cs, int hq,
                                                        int hkv, T* __restrict__ q_out, MxKv kv) {
#pragma clang fp contract(off)
  constexpr int HALF = DH / 2, QUADS = HALF / 4, GROUPS = DH / kMxGroup;
  const int row = blockIdx.x;
  const int r = plan_req_of_row(p, row);
  const int y = blockIdx.y * (256 / QUADS) + threadIdx.x / QUADS;   // head: q, then k, then v
  const int i = threadIdx.x % QUADS * 4;
  const int heads = hq + 2 * hkv;
  if (y >= heads) return;   // (whole groups of QUADS lanes: the exchanges stay among live lanes)
  const float* src = qkv + ((long)row * heads + y) * DH + i;
  f32x4 a = *reinterpret_cast<const f32x4*>(src);
  f32x4 b = *reinterpret_cast<const f32x4*>(src + HALF);
  for (int s = 1; s < splits; ++s) {
    a += *reinterpret_cast<const f32x4*>(src + s * split_stride);
    b += *reinterpret_cast<const f32x4*>(src + s * split_stride + HALF);
  }
  if (y < hq + hkv) {
    const f32x4 c0 = *reinterpret_cast<const f32x4*>(cs + (long)row * HALF + i);
    const f32x4 c1 = *reinterpret_cast<const f32x4*>(cs + (long)row * HALF + i + 2);
    const f32x4 c = {c0[0], c0[2], c1[0], c1[2]}, d = {c0[1], c0[3], c1[1], c1[3]};
    const f32x4 ac = a * c, bd = b * d, bc = b * c, ad = a * d;
    a = ac - bd;
    b = bc + ad;
  }
  if (y < hq) {
    T* o = q_out + ((long)row * hq + y) * DH + i;
    typedef T T4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<T4*>(o) = T4{from_f32<T>(a[0]), from_f32<T>(a[1]), from_f32<T>(a[2]), from_f32<T>(a[3])};
    *reinterpret_cast<T4*>(o + HALF) =
        T4{from_f32<T>(b[0]), from_f32<T>(b[1]), from_f32<T>(b[2]), from_f32<T>(b[3])};
    return;
  }
  const bool is_v = y >= hq + hkv;
  const ReqPlan& q = p.r[r];
  const long at = ((long)q.slot * hkv + (y - hq - (is_v ? hkv : 0))) * kv.s_max + q.pos0 + (row - q.row0);
  uint8_t* codes = (is_v ? kv.vc : kv.kc) + at * (DH / 2);
  uint8_t* scales = (is_v ? kv.vs : kv.ks) + at * GROUPS;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const f32x4 x = h ? b : a;
    uint32_t amax = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) amax = max(amax, __float_as_uint(x[j]) & 0x7fffffffu);
    amax = group_max<8>(amax);
    const uint32_t e = mx_scale_byte(amax);
    const uint32_t w = e == 255u ? 0u : mx_codes4(x[0], x[1], x[2], x[3], mx_scale(e));
    const int d = i + h * HALF;
    *reinterpret_cast<uint16_t*>(codes + d / 2) = (uint16_t)w;
    if (d % kMxGroup == 0) scales[d / kMxGroup] = (uint8_t)e;
  }
}

// The stored values: a lane writes 16 bytes of them, so that a wave's stores are whole lines.
// Bound by memory (10240 rows of 32 heads: 49 us, 4.3 TB/s).
template <typename T, int DH>
__global__ __launch_bounds__(256) void mx_read_kernel(StepPlan p, int hkv, MxKv kv,
                                                      T* __restrict__ k, T* __restrict__ v) {
  constexpr int GROUPS = DH / kMxGroup, V = 16 / sizeof(T), VECS = DH / V;   // vectors of a head
  typedef T vt __attribute__((ext_vector_type(V)));
  const int row = blockIdx.x;
  const int r = plan_req_of_row(p, row);
  const ReqPlan& q = p.r[r];
  const int i = blockIdx.y * 256 + threadIdx.x;
  if (i >= 2 * hkv * VECS) return;
  const bool is_v = i >= hkv * VECS;
  const int j = i - (is_v ? hkv * VECS : 0), head = j / VECS, x = j % VECS;
  const long at = ((long)q.slot * hkv + head) * kv.s_max + q.pos0 + (row - q.row0);
  const uint8_t* c = (is_v ? kv.vc : kv.kc) + at * (DH / 2) + x * (V / 2);
  const uint32_t w = V == 8 ? *reinterpret_cast<const uint32_t*>(c) : *reinterpret_cast<const uint16_t*>(c);
  const bf16x8 b = mx_bf16x8(w, mx_scale((is_v ? kv.vs : kv.ks)[at * GROUPS + x * V / kMxGroup]));
  vt o;
#pragma unroll
  for (int e = 0; e < V; ++e) o[e] = (T)(float)b[e];
  *reinterpret_cast<vt*>((is_v ? v : k) + (long)row * hkv * DH + j * V) = o;
}

}  // namespace

// whether rows of k elements, ld apart, are whole 16-byte vectors
template <typename T>
static bool whole_vectors(const T* p, long ld, int k) {
  constexpr int V = 16 / sizeof(T);
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % V == 0 && k % V == 0;
}

// blocks over the vectors of a row; the rows go round the second dimension
template <typename T>
static dim3 pack_grid(const MxView& w) {
  return dim3(ceil_div(w.groups * (kMxGroup / (16 / (int)sizeof(T))), 256 * kPackVecs), std::min(w.n, 65535));
}

template <typename T>
hipError_t mx_pack(const T* w, long ldw, int k, const MxView& o, hipStream_t st) {
  if (whole_vectors(w, ldw, k))
    DLM_LAUNCH((mx_pack_kernel<T, true>), pack_grid<T>(o), dim3(256), 0, st, w, ldw, k, o);
  else
    DLM_LAUNCH((mx_pack_kernel<T, false>), pack_grid<T>(o), dim3(256), 0, st, w, ldw, k, o);
  return hipGetLastError();
}

template <typename T>
hipError_t mx_unpack(const MxView& w, int k, T* out, long ldo, hipStream_t st) {
  if (whole_vectors(out, ldo, k))
    DLM_LAUNCH((mx_unpack_kernel<T, true>), pack_grid<T>(w), dim3(256), 0, st, w, k, out, ldo);
  else
    DLM_LAUNCH((mx_unpack_kernel<T, false>), pack_grid<T>(w), dim3(256), 0, st, w, k, out, ldo);
  return hipGetLastError();
}

template <typename T>
hipError_t mx_kv_append(const StepPlan& p, const float* qkv, int splits, long split_stride,
                        const float2* cs, int hq, int hkv, int dh, T* q_out, const MxKv& kv,
                        hipStream_t st) {
  if (p.n_rows == 0) return hipSuccess;
  const dim3 grid(p.n_rows, ceil_div((hq + 2 * hkv) * (dh / 8), 256));
  if (dh == 128)
    DLM_LAUNCH((mx_append_kernel<T, 128>), grid, dim3(256), 0, st, p, qkv, splits, split_stride, cs, hq,
               hkv, q_out, kv);
  else if (dh == 64)
    DLM_LAUNCH((mx_append_kernel<T, 64>), grid, dim3(256), 0, st, p, qkv, splits, split_stride, cs, hq,
               hkv, q_out, kv);
  else
    return hipErrorInvalidValue;
  return hipGetLastError();
}

template <typename T>
hipError_t mx_kv_read(const StepPlan& p, int hkv, int dh, const MxKv& kv, T* k, T* v,
                      hipStream_t st) {
  if (p.n_rows == 0) return hipSuccess;
  const dim3 grid(p.n_rows, ceil_div(2 * hkv * dh / (16 / (int)sizeof(T)), 256));
  if (dh == 128)
    DLM_LAUNCH((mx_read_kernel<T, 128>), grid, dim3(256), 0, st, p, hkv, kv, k, v);
  else if (dh == 64)
    DLM_LAUNCH((mx_read_kernel<T, 64>), grid, dim3(256), 0, st, p, hkv, kv, k, v);
  else
    return hipErrorInvalidValue;
  return hipGetLastError();
}

#define INST(T)                                                                                 \
  template hipError_t mx_pack<T>(const T*, long, int, const MxView&, hipStream_t);              \
  template hipError_t mx_unpack<T>(const MxView&, int, T*, long, hipStream_t);                  \
  template hipError_t mx_kv_append<T>(const StepPlan&, const float*, int, long, const float2*,  \
                                      int, int, int, T*, const MxKv&, hipStream_t);             \
  template hipError_t mx_kv_read<T>(const StepPlan&, int, int, const MxKv&, T*, T*, hipStream_t);
INST(bf16)
INST(float)
#undef INST

}  // namespace dlm
