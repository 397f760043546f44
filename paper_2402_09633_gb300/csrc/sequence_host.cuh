// Host-side pieces that the entry points of the sequence operators share: checks of views, and launches of the rotation.
#pragma once
#include <algorithm>
#include <cstring>
#include "host.cuh"
#include "rotary.cuh"

namespace gnn {

constexpr int32_t kRotaryMagic = 0x54524E47;       // "GNRT"

inline int elem_bytes(int dtype) { return dtype == GNN_DTYPE_FP32 ? 4 : 2; }

// A view whose elements are aligned, with strides that may be used; the furthest element stays within 2^62 bytes.
inline bool view_ok(const gnn_heads* h, int dtype) {
  if (!h || !h->data || h->n_heads < 1 || h->n_heads > (1 << 20) || h->reserved != 0) return false;
  if ((uintptr_t)h->data % elem_bytes(dtype) != 0) return false;
  return h->row_stride >= 0 && h->head_stride >= 0 && h->row_stride < (int64_t)1 << 39 &&
         h->head_stride < (int64_t)1 << 39;
}

inline HeadsView view(const gnn_heads& h, int dtype) {
  const int64_t e = elem_bytes(dtype);
  return {static_cast<char*>(h.data), h.row_stride * e, h.head_stride * e};
}

inline bool lies_on(const HeadsView& v, int64_t bytes) {
  return (uintptr_t)v.data % bytes == 0 && v.row_bytes % bytes == 0 && v.head_bytes % bytes == 0;
}

template <bool PAGED, typename T, int V>
cudaError_t launch_rotary(const RotaryParams& p, bool inter, bool norm, unsigned grid, cudaStream_t st) {
  if (norm)
    return inter ? launch_pdl(rotary_kernel<T, V, true, true, PAGED>, grid, kRotThreads, 0, st, p)
                 : launch_pdl(rotary_kernel<T, V, false, true, PAGED>, grid, kRotThreads, 0, st, p);
  return inter ? launch_pdl(rotary_kernel<T, V, true, false, PAGED>, grid, kRotThreads, 0, st, p)
               : launch_pdl(rotary_kernel<T, V, false, false, PAGED>, grid, kRotThreads, 0, st, p);
}

inline int device_sms() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
  return n;
}

// Fills the shared fields and launches; p.in, p.out, p.heads, p.gain, p.rows and p.eps are set.
template <bool PAGED>
int run_rotary(const gnn_rotary* rot, int dtype, int head_dim, RotaryParams& p, bool norm, const void* positions,
               int positions_float, int64_t n_rows, cudaStream_t st) {
  p.dim = head_dim;
  p.rot = rot->rot_dim;
  p.tokens = n_rows;
  p.pos = positions;
  p.pos_float = positions && positions_float;
  p.amplitude = rot->amplitude;
  std::memcpy(p.fixed, rot->turn_fixed, sizeof p.fixed);
  std::memcpy(p.hi, rot->turn_hi, sizeof p.hi);
  std::memcpy(p.lo, rot->turn_lo, sizeof p.lo);
  const bool inter = rot->layout == GNN_ROTARY_INTERLEAVED;
  const int e = elem_bytes(dtype);
  // the most pairs to a unit (8 in 16-bit types, 4, 2 or 1) that head_dim, rot_dim and how the views lie allow
  int V = dtype == GNN_DTYPE_FP32 ? 4 : 8;
  for (; V > 1; V /= 2) {
    bool ok = head_dim % (2 * V) == 0 && p.rot % (2 * V) == 0;
    for (int i = 0; i < 3; ++i)
      if (p.heads[i]) ok = ok && lies_on(p.in[i], V * e) && lies_on(p.out[i], V * e);
    if (ok) break;
  }
  p.units = head_dim / (2 * V);
  p.group = 1;
  while (p.group < p.units && p.group < 32) p.group *= 2;
  const int sms = device_sms();
  if (!sms) return cuda_fail(cudaGetLastError());
  // Blocks for one round of all tasks (two heads of a token), six to an SM at most, shared out by heads.
  const int heads = p.heads[0] + p.heads[1] + p.heads[2], per_block = kRotThreads / p.group;
  unsigned grid = 0;
  for (int i = 0; i < 3; ++i) {
    p.block0[i] = grid;
    if (!p.heads[i]) continue;
    const int64_t blocks = (n_rows * ((p.heads[i] + 1) / 2) + per_block - 1) / per_block;
    grid += (unsigned)std::min<int64_t>(blocks, std::max<int64_t>(1, (int64_t)sms * 6 * p.heads[i] / heads));
  }
  p.block0[3] = grid;
  cudaError_t err;
  if (dtype == GNN_DTYPE_FP32)
    err = V == 4   ? launch_rotary<PAGED, float, 4>(p, inter, norm, grid, st)
          : V == 2 ? launch_rotary<PAGED, float, 2>(p, inter, norm, grid, st)
                   : launch_rotary<PAGED, float, 1>(p, inter, norm, grid, st);
  else if (dtype == GNN_DTYPE_BF16)
    err = V == 8   ? launch_rotary<PAGED, __nv_bfloat16, 8>(p, inter, norm, grid, st)
          : V == 4 ? launch_rotary<PAGED, __nv_bfloat16, 4>(p, inter, norm, grid, st)
          : V == 2 ? launch_rotary<PAGED, __nv_bfloat16, 2>(p, inter, norm, grid, st)
                   : launch_rotary<PAGED, __nv_bfloat16, 1>(p, inter, norm, grid, st);
  else
    err = V == 8   ? launch_rotary<PAGED, __half, 8>(p, inter, norm, grid, st)
          : V == 4 ? launch_rotary<PAGED, __half, 4>(p, inter, norm, grid, st)
          : V == 2 ? launch_rotary<PAGED, __half, 2>(p, inter, norm, grid, st)
                   : launch_rotary<PAGED, __half, 1>(p, inter, norm, grid, st);
  return err == cudaSuccess ? GNN_OK : cuda_fail(err);
}

inline bool rotary_args_ok(const gnn_rotary* rot, int dtype, int head_dim, int64_t n_rows, const void* positions) {
  if (!rot || rot->magic != kRotaryMagic || dtype < GNN_DTYPE_FP32 || dtype > GNN_DTYPE_FP16) return false;
  if (head_dim < rot->rot_dim || head_dim > 2 * kRotMaxPairs || head_dim % 2 != 0) return false;
  return count_ok(n_rows) && (uintptr_t)positions % 4 == 0;
}

}  // namespace gnn
