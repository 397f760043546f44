// Entry points for hits read as a sequence: rotary positions, norms of queries and keys with the rotation, and
// attention with a sliding window (include/gnn.h).
#include <cudaTypedefs.h>
#include <cuda_runtime.h>
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "../../include/gnn.h"
#include "attend.cuh"
#include "attend_few.cuh"
#include "attend_tile.cuh"
#include "host.cuh"
#include "rotary.cuh"
#include "sequence_host.cuh"

using namespace gnn;

struct gnn_attention {
  int device = 0;
  int n_sm = 0;
  uint32_t* d_err = nullptr;
  PFN_cuTensorMapEncodeTiled_v12000 encode = nullptr;
  float* d_parts = nullptr;
  int* d_tickets = nullptr;
};

namespace {

void free_attention(gnn_attention* a) {
  if (a->d_err) cudaFree(a->d_err);
  if (a->d_parts) cudaFree(a->d_parts);
  if (a->d_tickets) cudaFree(a->d_tickets);
  delete a;
}

constexpr double kTwoPi = 6.283185307179586476925286766559;

// Boxes of box_rows rows x 64 elements of one head, in the 128-byte swizzle; what lies outside reads as zeros.
bool encode_map(const gnn_attention* a, CUtensorMap* map, const gnn_heads& h, int64_t rows, int dtype, int dim,
                int box_rows) {
  const cuuint64_t size[3] = {(cuuint64_t)dim, (cuuint64_t)h.n_heads, (cuuint64_t)std::max<int64_t>(rows, 1)};
  const cuuint64_t one = (cuuint64_t)(dim * 2 + 15) / 16 * 16;      // for a dimension of one, whose stride is not used
  const cuuint64_t stride[2] = {h.n_heads > 1 ? (cuuint64_t)h.head_stride * 2 : one,
                                rows > 1 ? (cuuint64_t)h.row_stride * 2 : one};
  const cuuint32_t box[3] = {64, 1, (cuuint32_t)box_rows}, step[3] = {1, 1, 1};
  return a->encode(map, dtype == GNN_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
                   h.data, size, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                   CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int DP>
cudaError_t launch_attend(unsigned grid, cudaStream_t st, const AttendParams& p, const AttendGrid& g,
                          const CUtensorMap* maps) {
  const cudaError_t err = cudaFuncSetAttribute(attend_tile_kernel<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               attend_smem_bytes<DP>());
  if (err != cudaSuccess) return err;
  return launch_pdl(attend_tile_kernel<T, DP>, grid, kAttendThreads, attend_smem_bytes<DP>(), st, p, g, maps[0], maps[1],
                    maps[2]);
}

int run_tiles(gnn_attention* a, const gnn_attention_call* c, const gnn_heads* views, const AttendParams& p,
              cudaStream_t st) {
  AttendGrid g = {};
  g.group = p.heads / p.kv_heads;
  // A block's tiles share the keys that are loaded, but fewer in a block are faster: as few as keep all SMs busy
  // (event of 2,000 hits, 32 tiles, one or two to a block: 11.7 and 13.8 us).
  const int64_t tiles = (c->n_q_rows / kTileQ + c->n_seqs) * p.heads;
  g.tiles = (int)std::min<int64_t>(kMostTiles, std::max<int64_t>(1, (tiles + a->n_sm - 1) / a->n_sm));
  const int64_t slots = (c->n_q_rows / kTileQ + c->n_seqs) * g.group / g.tiles + c->n_seqs;
  if ((c->n_q_rows / kTileQ + c->n_seqs) * g.group + c->n_seqs >= (int64_t)1 << 31) return GNN_ERR_INVALID_ARG;
  g.items = slots * p.kv_heads;
  CUtensorMap maps[3];
  if (!encode_map(a, &maps[0], views[0], c->n_q_rows, c->dtype, c->head_dim, kTileQ) ||
      !encode_map(a, &maps[1], views[1], c->n_kv_rows, c->dtype, c->head_dim, kKeys) ||
      !encode_map(a, &maps[2], views[2], c->n_kv_rows, c->dtype, c->head_dim, kKeys))
    return GNN_ERR_INVALID_ARG;
  const unsigned grid = (unsigned)std::min<int64_t>(g.items, a->n_sm);
  cudaError_t err;
  if (c->dtype == GNN_DTYPE_BF16)
    err = p.dim <= 64 ? launch_attend<__nv_bfloat16, 64>(grid, st, p, g, maps)
                      : launch_attend<__nv_bfloat16, 128>(grid, st, p, g, maps);
  else
    err = p.dim <= 64 ? launch_attend<__half, 64>(grid, st, p, g, maps) : launch_attend<__half, 128>(grid, st, p, g, maps);
  return err == cudaSuccess ? GNN_OK : cuda_fail(err);
}

template <typename T>
cudaError_t launch_few(unsigned grid, cudaStream_t st, const AttendParams& p, const FewGrid& f, bool sixteen) {
  auto go = [&](auto kernel) { return launch_pdl(kernel, grid, 32 * kFewWarps, 0, st, p, f); };
  switch ((p.dim + 31) / 32) {
    case 1: return sixteen ? go(attend_few_kernel<T, 1, 2>) : go(attend_few_kernel<T, 1, 1>);
    case 2: return sixteen ? go(attend_few_kernel<T, 2, 2>) : go(attend_few_kernel<T, 2, 1>);
    case 3: return sixteen ? go(attend_few_kernel<T, 3, 2>) : go(attend_few_kernel<T, 3, 1>);
    default: return sixteen ? go(attend_few_kernel<T, 4, 2>) : go(attend_few_kernel<T, 4, 1>);
  }
}

// The most keys that queries of one sequence see.
int64_t most_keys(const gnn_attention_call* c, const AttendParams& p, int64_t max_q) {
  int64_t keys = c->kv_len ? c->n_kv_rows : max_q;
  if (c->max_kv > 0) keys = std::min<int64_t>(keys, c->max_kv);
  if (p.left >= 0 && p.right >= 0) keys = std::min<int64_t>(keys, (int64_t)p.sinks + p.left + p.right + max_q);
  return keys;
}

// Whether the rows by mma.sync, which stream a sequence's keys once for every 16 of them and spread them over all SMs,
// take less time than tiles of 128 queries, each of which has one block go through its keys.  Measured: a stream takes
// 5.9 GB/ms behind 6 us (11 with 16 rows to a tile); a block of 128 keys takes a tile 0.83 us (heads up to 64) or 1.23
// behind 6.5 us, two tiles in one block half as much again.  32 queries of four heads over one cache of 65,536 keys, two key heads of 128: 92 and 631 us; 64 caches of 8,192,
// 16 queries: 373 and 194.
bool few_is_faster(const gnn_attention* a, const gnn_attention_call* c, const AttendParams& p, int64_t max_q) {
  const double group = p.heads / p.kv_heads, seqs = p.n_seqs, rows = max_q * group;
  if (seqs * p.kv_heads > 1 << 24 || rows > 1 << 20) return false;
  double keys = (double)most_keys(c, p, max_q);
  if (c->kv_len && c->max_kv == 0) keys = std::min(keys, (double)c->n_kv_rows / seqs + 1);   // evenly shared, for want of better
  const double streams = std::ceil(rows / (rows > 8 ? 16 : 8));
  const double few = (rows > 8 ? 11 : 6) + streams * seqs * keys * p.kv_heads * p.dim * 4 / 5.9e6;
  const double tiles = std::min((double)c->n_q_rows / kTileQ + seqs, seqs * std::ceil(max_q / (double)kTileQ)) * p.heads;
  const double per = p.dim <= 64 ? 0.83 : 1.23;
  // a causal tile of a long sequence sees half of it
  const double blocks = std::ceil((p.left < 0 && p.right >= 0 && !c->kv_len ? keys / 2 : keys) / kKeys);
  const double rounds = tiles <= a->n_sm ? 1 : 1.5 * std::ceil(tiles / 2 / a->n_sm);
  return few <= 6.5 + rounds * blocks * per;
}

// Few queries to a sequence: one round of blocks, which share the keys out among them.
int run_few(gnn_attention* a, const gnn_attention_call* c, const AttendParams& p, int64_t max_q, cudaStream_t st) {
  FewGrid f = {};
  f.group = p.heads / p.kv_heads;
  const bool sixteen = max_q * f.group > 8;
  f.row_tiles = (int)((max_q * f.group + (sixteen ? 15 : 7)) / (sixteen ? 16 : 8));
  f.parts = a->d_parts;
  f.tickets = a->d_tickets;
  // no more blocks than there are units of keys, where the keys are known to be few
  const int64_t keys = most_keys(c, p, max_q);
  const int64_t units = (int64_t)p.n_seqs * p.kv_heads * f.row_tiles * ((keys + kFewUnit) / kFewUnit);
  const unsigned grid = (unsigned)std::min<int64_t>(units, (int64_t)a->n_sm * (sixteen && p.dim > 64 ? 2 : 3));
  const cudaError_t err = c->dtype == GNN_DTYPE_BF16 ? launch_few<__nv_bfloat16>(grid, st, p, f, sixteen)
                                                     : launch_few<__half>(grid, st, p, f, sixteen);
  return err == cudaSuccess ? GNN_OK : cuda_fail(err);
}

}  // namespace

extern "C" {

int gnn_rotary_init(const gnn_rotary_config* cfg, gnn_rotary* out) {
  if (!cfg || !out || cfg->reserved != 0) return GNN_ERR_INVALID_ARG;
  const int R = cfg->rot_dim;
  if (R < 2 || R > 2 * kRotMaxPairs || R % 2 != 0) return GNN_ERR_INVALID_ARG;
  if (cfg->layout != GNN_ROTARY_HALF && cfg->layout != GNN_ROTARY_INTERLEAVED) return GNN_ERR_INVALID_ARG;
  if (cfg->scaling < GNN_ROTARY_PLAIN || cfg->scaling > GNN_ROTARY_BY_TURNS) return GNN_ERR_INVALID_ARG;
  auto positive = [](double x) { return std::isfinite(x) && x > 0; };
  if (!positive(cfg->base) || !std::isfinite(cfg->amplitude)) return GNN_ERR_INVALID_ARG;
  if (cfg->scaling != GNN_ROTARY_PLAIN && !positive(cfg->factor)) return GNN_ERR_INVALID_ARG;
  if (cfg->scaling == GNN_ROTARY_BY_TURNS &&
      (!positive(cfg->length) || !(cfg->slow >= 0) || !std::isfinite(cfg->fast) || !(cfg->fast > cfg->slow)))
    return GNN_ERR_INVALID_ARG;
  gnn_rotary r;
  std::memset(&r, 0, sizeof r);
  r.rot_dim = R;
  r.layout = cfg->layout;
  r.amplitude = (float)cfg->amplitude;
  for (int i = 0; i < R / 2; ++i) {
    double f = std::pow(cfg->base, -2.0 * i / R);
    if (cfg->scaling == GNN_ROTARY_LINEAR) f /= cfg->factor;
    if (cfg->scaling == GNN_ROTARY_BY_TURNS) {
      const double g = std::min(1.0, std::max(0.0, (cfg->length * f / kTwoPi - cfg->slow) / (cfg->fast - cfg->slow)));
      f *= g + (1.0 - g) / cfg->factor;
    }
    const double turns = f / kTwoPi;
    r.turn_hi[i] = (float)turns;
    r.turn_lo[i] = (float)(turns - (double)r.turn_hi[i]);
    if (!std::isfinite(r.turn_hi[i])) return GNN_ERR_INVALID_ARG;
    const double part = std::ldexp(turns - std::floor(turns), 64);     // [0, 2^64]: a whole turn is none
    r.turn_fixed[i] = part >= 18446744073709551616.0 ? 0 : (uint64_t)part;
  }
  r.magic = kRotaryMagic;
  *out = r;
  return GNN_OK;
}

int gnn_rope(const gnn_rotary* rot, int dtype, int head_dim, const gnn_heads* x, const gnn_heads* y,
             const void* positions, int positions_float, int64_t n_rows, gnn_stream_t stream) {
  if (!rotary_args_ok(rot, dtype, head_dim, n_rows, positions)) return GNN_ERR_INVALID_ARG;
  if (n_rows == 0) return GNN_OK;
  if (!view_ok(x, dtype) || !view_ok(y, dtype) || x->n_heads != y->n_heads) return GNN_ERR_INVALID_ARG;
  RotaryParams p = {};
  p.in[0] = view(*x, dtype);
  p.out[0] = view(*y, dtype);
  p.heads[0] = x->n_heads;
  return run_rotary<false>(rot, dtype, head_dim, p, false, positions, positions_float, n_rows, (cudaStream_t)stream);
}

int gnn_qk_norm_rope(const gnn_rotary* rot, int dtype, int head_dim, float eps, const float* q_gain,
                     const float* k_gain, const gnn_heads* q, const gnn_heads* k, const gnn_heads* v,
                     const gnn_heads* q_out, const gnn_heads* k_out, const gnn_heads* v_out, const void* positions,
                     int positions_float, const int64_t* rows, int64_t out_rows, int64_t n_rows,
                     gnn_stream_t stream) {
  if (!rotary_args_ok(rot, dtype, head_dim, n_rows, positions)) return GNN_ERR_INVALID_ARG;
  if (!std::isfinite(eps) || !(eps > 0.f) || (uintptr_t)q_gain % 4 || (uintptr_t)k_gain % 4 || (uintptr_t)rows % 8)
    return GNN_ERR_INVALID_ARG;
  if ((rows && !count_ok(out_rows)) || (v != nullptr) != (v_out != nullptr)) return GNN_ERR_INVALID_ARG;
  if (n_rows == 0) return GNN_OK;
  const gnn_heads* in[3] = {q, k, v};
  const gnn_heads* out[3] = {q_out, k_out, v_out};
  RotaryParams p = {};
  for (int i = 0; i < (v ? 3 : 2); ++i) {
    if (!view_ok(in[i], dtype) || !view_ok(out[i], dtype) || in[i]->n_heads != out[i]->n_heads)
      return GNN_ERR_INVALID_ARG;
    p.in[i] = view(*in[i], dtype);
    p.out[i] = view(*out[i], dtype);
    p.heads[i] = in[i]->n_heads;
  }
  if (v && v->n_heads != k->n_heads) return GNN_ERR_INVALID_ARG;
  p.gain[0] = q_gain;
  p.gain[1] = k_gain;
  p.rows = rows;
  p.out_rows = out_rows;
  p.eps = eps;
  return run_rotary<false>(rot, dtype, head_dim, p, true, positions, positions_float, n_rows, (cudaStream_t)stream);
}

int gnn_attention_create(gnn_attention** out) {
  if (!out) return GNN_ERR_INVALID_ARG;
  *out = nullptr;
  gnn_attention* a = new (std::nothrow) gnn_attention;
  if (!a) return GNN_ERR_OOM;
  cudaError_t err = cudaGetDevice(&a->device);
  if (err == cudaSuccess) err = cudaDeviceGetAttribute(&a->n_sm, cudaDevAttrMultiProcessorCount, a->device);
  cudaDriverEntryPointQueryResult found;
  if (err == cudaSuccess)
    err = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", (void**)&a->encode, 12000, cudaEnableDefault, &found);
  if (err == cudaSuccess && (found != cudaDriverEntryPointSuccess || !a->encode)) err = cudaErrorNotSupported;
  if (err == cudaSuccess) err = dev_alloc((void**)&a->d_err, 4);
  if (err == cudaSuccess) err = cudaMemset(a->d_err, 0, 4);
  const size_t blocks = 3 * (size_t)a->n_sm;         // of a call with few queries: two parts and a ticket each
  if (err == cudaSuccess) err = dev_alloc((void**)&a->d_parts, blocks * 2 * kFewRows * (128 + 2) * 4);
  if (err == cudaSuccess) err = dev_alloc((void**)&a->d_tickets, blocks * 4);
  if (err == cudaSuccess) err = cudaMemset(a->d_tickets, 0, blocks * 4);
  // the zeros are in place before any stream's first call: streams need not wait for the one they are written in
  if (err == cudaSuccess) err = cudaStreamSynchronize(cudaStreamLegacy);
  if (err != cudaSuccess) {
    free_attention(a);
    return cuda_fail(err);
  }
  *out = a;
  return GNN_OK;
}

int gnn_attention_run(gnn_attention* att, const gnn_attention_call* c, gnn_stream_t stream) {
  if (!att || !c || c->reserved != 0) return GNN_ERR_INVALID_ARG;
  if ((c->dtype != GNN_DTYPE_BF16 && c->dtype != GNN_DTYPE_FP16) || c->head_dim < 8 || c->head_dim > 128 ||
      c->head_dim % 8 != 0 || !std::isfinite(c->scale) || c->sinks < 0)
    return GNN_ERR_INVALID_ARG;
  if (!count_ok(c->n_q_rows) || !count_ok(c->n_kv_rows) || !count_ok(c->n_seqs) || c->max_q < 0 || c->max_kv < 0 ||
      (c->kv_start != nullptr) != (c->kv_len != nullptr))
    return GNN_ERR_INVALID_ARG;
  if (c->n_q_rows == 0 || c->n_seqs == 0) return GNN_OK;
  if (!c->q_start || (uintptr_t)c->q_start % 4 || (uintptr_t)c->kv_start % 4 || (uintptr_t)c->kv_len % 4)
    return GNN_ERR_INVALID_ARG;
  gnn_heads views[4] = {c->q, c->k, c->v, c->out};
  if (c->n_kv_rows == 0) views[1].data = views[2].data = c->out.data;   // nothing is read of them
  for (const gnn_heads& v : views)
    if (!view_ok(&v, c->dtype) || (uintptr_t)v.data % 16 || v.row_stride % 8 || v.head_stride % 8)
      return GNN_ERR_INVALID_ARG;
  if (c->n_seqs > 1 << 28 || c->q.n_heads > 4096) return GNN_ERR_INVALID_ARG;
  for (const gnn_heads& v : views)                 // one row or head for several is not a view that can be read here
    if ((v.n_heads > 1 && v.head_stride == 0) || v.row_stride == 0) return GNN_ERR_INVALID_ARG;
  if (c->k.n_heads != c->v.n_heads || c->q.n_heads != c->out.n_heads || c->q.n_heads % c->k.n_heads)
    return GNN_ERR_INVALID_ARG;
  AttendParams p = {};
  p.q = view(c->q, c->dtype);
  p.k = view(views[1], c->dtype);
  p.v = view(views[2], c->dtype);
  p.out = view(c->out, c->dtype);
  p.q_start = c->q_start;
  p.kv_start = c->kv_start;
  p.kv_len = c->kv_len;
  p.n_q_rows = (int)c->n_q_rows;
  p.n_kv_rows = (int)c->n_kv_rows;
  p.n_seqs = c->n_seqs;
  p.max_q = (int)(c->max_q > 0 ? std::min<int64_t>(c->max_q, c->n_q_rows) : c->n_q_rows);
  p.heads = c->q.n_heads;
  p.kv_heads = c->k.n_heads;
  p.dim = c->head_dim;
  p.left = c->left;
  p.right = c->right;
  p.sinks = c->sinks;
  // a scale of zero as one too small to be seen, so that -inf, a score that is not seen, stays -inf
  p.scale_log2 = c->scale == 0.f ? 1e-30f : (float)((double)c->scale * 1.4426950408889634);
  p.err = att->d_err;
  int device = 0;                                  // the handle's memory and SMs are its device's
  const cudaError_t err = cudaGetDevice(&device);
  if (err != cudaSuccess) return cuda_fail(err);
  if (device != att->device) return GNN_ERR_INVALID_ARG;
  if (few_is_faster(att, c, p, p.max_q)) return run_few(att, c, p, p.max_q, (cudaStream_t)stream);
  return run_tiles(att, c, views, p, (cudaStream_t)stream);
}

int gnn_attention_status(gnn_attention* att, gnn_stream_t stream) {
  if (!att) return GNN_ERR_INVALID_ARG;
  // In the caller's stream, so that the word is read behind its calls so far and cleared before the next.
  const cudaStream_t st = (cudaStream_t)stream;
  uint32_t word = 0;
  cudaError_t err = cudaMemcpyAsync(&word, att->d_err, 4, cudaMemcpyDeviceToHost, st);
  if (err == cudaSuccess) err = cudaMemsetAsync(att->d_err, 0, 4, st);
  const cudaError_t done = cudaStreamSynchronize(st);          // whatever failed: the copy writes to this frame
  if (err == cudaSuccess) err = done;
  if (err != cudaSuccess) return cuda_fail(err);
  if (word & DEV_ERR_TIMEOUT) return GNN_ERR_DEVICE_TIMEOUT;
  if (word & DEV_ERR_INDEX_RANGE) return GNN_ERR_INDEX_RANGE;
  return GNN_OK;
}

void gnn_attention_destroy(gnn_attention* att) {
  if (!att) return;
  cudaDeviceSynchronize();
  free_attention(att);
}

}  // extern "C"
