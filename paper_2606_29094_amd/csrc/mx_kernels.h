// Launch functions of the kernels on 4-bit operands (mx_gemm.h, mx_rowwise.h, mx_attention.h;
// the format is in mx_common.h), internal to libdlm.so.
#pragma once

#include "common.h"
#include "kernels.h"

namespace dlm {

// For a call of several kernels: the first one carries the hook's start event, and the one
// launched after last() its stop event, so the time between them is the whole call's.
struct LaunchSpan {
  LaunchTiming all;
  explicit LaunchSpan(bool several) {
    if (several && g_launch_timing.start) {
      all = g_launch_timing;
      g_launch_timing.stop = nullptr;
    }
  }
  void last() const {
    if (all.stop) g_launch_timing = LaunchTiming{nullptr, all.stop};
  }
};

// A packed [n, k] matrix: groups = ceil(k / 32), codes [n, 16 groups] bytes, scales
// [n, scale_ld], scale_ld = groups rounded up to 16. Both 16-byte aligned.
struct MxView { uint8_t* codes; uint8_t* scales; int n, groups, scale_ld; };
template <typename T>
hipError_t mx_pack(const T* w, long ldw, int k, const MxView& o, hipStream_t st);
template <typename T>
hipError_t mx_unpack(const MxView& w, int k, T* out, long ldo, hipStream_t st);
// Products y = x w^T: fp32 [rows, n] stored or added, or silu(gate) * up in T
// ([rows, n / 2], rows [0, n / 2) of w the gate).
// A product's way: straight from the codes with K in `slices` (kMxFew: 16 rows x 16 nf
// columns a block of `waves` waves; tiles of 32 x 128, 64 x 128 and 128 x 256), or (gemm) over
// the matrix unpacked to the scratch and the GEMM kernels of its type. scratch: bytes,
// 256-byte aligned. staged: x is first copied into the scratch's first `stage` bytes (fp32 x,
// or rows that 16-byte loads cannot read).
enum { kMxFew, kMxTile32, kMxTile64, kMxTile128 };
constexpr int kMxTileK = 1 << 24;   // the tiles take rows (and row strides) of up to that many elements
struct MxTile { int kind, nf, slices, waves; };
struct MxPlan {
  bool gemm = false, staged = false, join = true;
  GemmPlan g{};
  MxTile tile{};
  size_t stage = 0, scratch = 0;
};
// x_aligned, y_aligned: the buffer and its rows start at multiples of 16 bytes (rows of x, ldx
// elements apart, at most kMxTileK). join: K slices are added by the product; otherwise (DLM_MX_STORE alone)
// y takes tile.slices (g.splits) of them, [slices, rows, n], for a consumer that adds them.
MxPlan mx_plan(int elem, int rows, int n, int k, long ldx, bool swiglu, bool x_aligned, bool y_aligned,
               bool join, int num_cu);
// epilogue: dlm_mx_epilogue
template <typename T>
hipError_t mx_matmul(const MxPlan& plan, const T* x, long ldx, int rows, const MxView& w, int k,
                     int epilogue, void* y, long ldy, void* scratch, hipStream_t st);
// kernel arguments of a product
struct MxLinear {
  const bf16* x;           // [m, ldx], NP planes `plane` elements apart
  long ldx, plane;
  MxView w;
  int m, k;                // k: elements of x a row holds (a multiple of 8)
  int tail;                // codes of the last group that belong to the matrix (0: all)
  void* y;
  long ldy;
  float* slices;           // [slice][m][n] partial sums, where K is sliced
  int per_slice;           // walks of 512 k in a slice
  int planes;
  bool swiglu, add;
};

// One layer of a 4-bit key/value cache: codes [slot][kv_head][pos][dh / 2] and scales
// [slot][kv_head][pos][dh / 32] of the keys and of the values, s_max positions a slot.
struct MxKv { uint8_t *kc, *vc, *ks, *vs; int s_max; };
// queries rotated to T, keys (rotated) and values packed at (slot, head, pos) of each row
template <typename T>
hipError_t mx_kv_append(const StepPlan& p, const float* qkv, int splits, long split_stride,
                        const float2* cs, int hq, int hkv, int dh, T* q_out, const MxKv& kv,
                        hipStream_t st);
// the stored keys and values of each row, [rows, hkv dh]
template <typename T>
hipError_t mx_kv_read(const StepPlan& p, int hkv, int dh, const MxKv& kv, T* k, T* v,
                      hipStream_t st);
// Attention of every row over [0, seq_len) of its request's slot (zeros where that is
// empty). splits > 1: the keys of a request are split over blocks, their partials go to
// scratch (mx_attention_scratch bytes) and a second kernel joins them.
// Blocks of 32 items (16 in fp32; an item is a query row of one head) whose four waves
// split the keys, or of 64 or 128 items whose waves share the keys.
enum MxAttnKind { kMxAttnFew, kMxAttnShared64, kMxAttnShared128 };
struct MxAttnPlan { int kind = kMxAttnFew; int splits = 1; };
MxAttnPlan mx_attention_plan(const StepPlan& p, int hq, int hkv, int dh, size_t elem,
                             size_t scratch_bytes, int num_cu);
size_t mx_attention_scratch(int rows, int hq, int dh, int splits);
template <typename T>
hipError_t mx_attention(const StepPlan& p, const T* q, const MxKv& kv, int hq, int hkv, int dh,
                        T* out, MxAttnPlan plan, float* scratch, hipStream_t st);

}  // namespace dlm
