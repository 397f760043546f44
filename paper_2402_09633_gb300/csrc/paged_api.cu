// Entry points for several hypotheses of a sequence: caches in pages, the choice of continuations, and moving states
// (include/gnn.h).
#include <cudaTypedefs.h>
#include <cuda_runtime.h>
#include <algorithm>
#include <cmath>

#include "../../include/gnn.h"
#include "beam.cuh"
#include "host.cuh"
#include "paged.cuh"
#include "paged_tile.cuh"
#include "sequence_host.cuh"

using namespace gnn;

namespace {

constexpr int kPageLeast = 16, kPageMost = 1024;

bool pages_ok(const gnn_pages* c) {
  if (!c || c->reserved != 0 || c->dtype < GNN_DTYPE_FP32 || c->dtype > GNN_DTYPE_FP16) return false;
  if (c->page_size < kPageLeast || c->page_size > kPageMost || (c->page_size & (c->page_size - 1))) return false;
  if (c->n_pages < 1 || !count_ok(c->n_pages) || !count_ok(c->n_pages * c->page_size)) return false;
  if (c->n_seqs < 0 || c->n_seqs > 1 << 28 || c->table_width < 1 || !count_ok(c->table_width)) return false;
  if (c->table_stride < 0 || c->table_stride >= (int64_t)1 << 39) return false;
  if (c->n_seqs > 0 && (!c->table || !c->kv_len || (uintptr_t)c->table % 4 || (uintptr_t)c->kv_len % 4)) return false;
  if (c->head_dim < 1 || c->head_dim > 2 * kRotMaxPairs) return false;
  return c->status && (uintptr_t)c->status % 4 == 0 && view_ok(&c->k, c->dtype) && view_ok(&c->v, c->dtype) &&
         c->k.n_heads == c->v.n_heads;
}

int log2_of(int n) {
  int s = 0;
  while (1 << s < n) ++s;
  return s;
}

// A view that the attention reads in pieces of 16 bytes.
bool wide_ok(const gnn_heads& v, int dtype) {
  return view_ok(&v, dtype) && (uintptr_t)v.data % 16 == 0 && v.row_stride > 0 && v.row_stride % 8 == 0 && v.head_stride % 8 == 0 &&
         (v.n_heads == 1 || v.head_stride > 0);
}

bool attend_ok(const gnn_pages* c, const gnn_paged_call* a) {
  if (!pages_ok(c) || !a || a->reserved != 0 || c->dtype == GNN_DTYPE_FP32) return false;
  if (c->head_dim < 8 || c->head_dim > 128 || c->head_dim % 8 != 0 || !std::isfinite(a->scale)) return false;
  if (!count_ok(a->n_q_rows) || a->max_q < 0 || a->n_groups < 0 || a->n_groups > 1 << 28) return false;
  if ((a->n_groups > 0) != (a->group_start != nullptr) || (a->group_start != nullptr) != (a->shared_len != nullptr)) return false;
  if ((uintptr_t)a->group_start % 4 || (uintptr_t)a->shared_len % 4) return false;
  if (!wide_ok(c->k, c->dtype) || !wide_ok(c->v, c->dtype)) return false;
  if (a->n_q_rows == 0 || c->n_seqs == 0) return true;
  if (!a->q_start || (uintptr_t)a->q_start % 4 || !wide_ok(a->q, c->dtype) || !wide_ok(a->out, c->dtype)) return false;
  if (a->q.n_heads != a->out.n_heads || a->q.n_heads > 4096 || a->q.n_heads % c->k.n_heads) return false;
  return a->q.n_heads / c->k.n_heads <= 128;
}

int paged_chunks(int64_t n_seqs, int64_t n_groups) {
  return (int)((n_seqs + kAttendThreads - 1) / kAttendThreads + (n_groups + kAttendThreads - 1) / kAttendThreads);
}
// How a call is cut into tiles, and where its parts lie in the workspace; the bytes that takes.
struct PagedPlan { PagedGrid g; uint64_t bytes; unsigned blocks; };
PagedPlan paged_plan(const gnn_pages* c, const gnn_paged_call* a, int n_sm) {
  PagedPlan r = {};
  PagedGrid& g = r.g;
  const int64_t n = a->n_q_rows, max_q = a->max_q > 0 ? std::min<int64_t>(a->max_q, n) : n;
  r.blocks = (unsigned)n_sm;
  g.group = a->q.n_heads / c->k.n_heads;
  g.tile_q = kTileQ / g.group;
  g.box_a = (int)std::min<int64_t>(g.tile_q, n);
  g.pack = 1;
  // (and keys that are counted in 32 bits)
  while (g.pack < kPackMost && 2 * g.pack * max_q <= g.tile_q && 2 * g.pack * ((int64_t)c->table_width * c->page_size) <= 1 << 30) g.pack *= 2;
  g.box_b = (int)std::min<int64_t>(g.tile_q, g.pack * max_q);
  g.box = std::min(c->page_size, kKeys);
  g.rows_a = g.box_a * g.group;
  g.rows_b = g.box_b * g.group;
  const int64_t n_a = a->n_groups > 0 ? (n / (2 * g.tile_q) + a->n_groups) * c->k.n_heads : 0;
  const int64_t n_b = (g.pack > 1 ? (c->n_seqs + g.pack - 1) / g.pack : n / g.tile_q + c->n_seqs) * (int64_t)c->k.n_heads;
  const int64_t sums_a = n_a > 0 ? 2 * (n * a->q.n_heads + (int64_t)r.blocks * g.rows_a) : 0,
                sums_b = 2 * (n * a->q.n_heads + (int64_t)r.blocks * g.rows_b);
  char* at = static_cast<char*>(a->workspace);
  auto take = [&](int64_t bytes) {
    char* here = at;
    const int64_t whole = (bytes + 31) / 32 * 32;
    at = reinterpret_cast<char*>((uintptr_t)at + whole);
    r.bytes += whole;
    return here;
  };
  g.out_a = reinterpret_cast<float*>(take(sums_a * c->head_dim * 4));
  g.out_b = reinterpret_cast<float*>(take(sums_b * c->head_dim * 4));
  g.sum_a = reinterpret_cast<float2*>(take(sums_a * 8));
  g.sum_b = reinterpret_cast<float2*>(take(sums_b * 8));
  if (c->n_seqs > kPagedKept || a->n_groups > kAttendThreads) g.chunks = reinterpret_cast<int64_t*>(take((int64_t)paged_chunks(c->n_seqs, a->n_groups) * 8));
  g.first_a = reinterpret_cast<int2*>(take(n_a * 8));
  g.first_b = reinterpret_cast<int2*>(take(n_b * 8));
  return r;
}

PFN_cuTensorMapEncodeTiled_v12000 map_encoder() {
  static const PFN_cuTensorMapEncodeTiled_v12000 found = [] {
    PFN_cuTensorMapEncodeTiled_v12000 f = nullptr;
    cudaDriverEntryPointQueryResult r;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", (void**)&f, 12000, cudaEnableDefault, &r) != cudaSuccess ||
        r != cudaDriverEntryPointSuccess)
      f = nullptr;
    return f;
  }();
  return found;
}

// Boxes of box_rows rows x box_heads heads x 64 elements, in the 128-byte swizzle; what lies outside reads as zeros.
bool paged_map(CUtensorMap* map, const gnn_heads& h, int64_t rows, int dtype, int dim, int box_heads, int box_rows) {
  const cuuint64_t size[3] = {(cuuint64_t)dim, (cuuint64_t)h.n_heads, (cuuint64_t)rows};
  const cuuint64_t one = (cuuint64_t)(dim * 2 + 15) / 16 * 16;      // for a dimension of one, whose stride is not used
  const cuuint64_t stride[2] = {h.n_heads > 1 ? (cuuint64_t)h.head_stride * 2 : one, rows > 1 ? (cuuint64_t)h.row_stride * 2 : one};
  const cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_rows}, step[3] = {1, 1, 1};
  return map_encoder()(map, dtype == GNN_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, h.data,
                       size, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                       CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int DP>
cudaError_t launch_paged(const PagedParams& p, const PagedPlan& plan, const CUtensorMap* maps, cudaStream_t st) {
  cudaError_t err = allow_smem<paged_tile_kernel<T, DP>>(paged_smem_bytes<DP>());
  if (err == cudaSuccess && plan.g.chunks)
    err = launch_pdl(paged_weigh_kernel, (unsigned)paged_chunks(p.n_seqs, p.n_groups), kAttendThreads, 0, st, p, plan.g);
  if (err == cudaSuccess)
    err = launch_pdl(paged_tile_kernel<T, DP>, plan.blocks, kAttendThreads, paged_smem_bytes<DP>(), st, p, plan.g, maps[0], maps[1],
                     maps[2], maps[3], maps[4], maps[5]);
  if (err != cudaSuccess) return err;
  // One warp goes through a row's parts (up to one of every block) eight at a time; where rows are few, eight warps share a row's (8 rows
  // over 32,768 keys, one key head: 56.8 -> 27.8 us).  Where the former does not find room for all rows at once, more warps
  // with two parts each in flight do better (131,072 rows of up to three: 357 -> 298 us for the call; 1,024 rows of 38: 32.6 -> 38.1).
  const int64_t rows = (int64_t)p.n_q_rows * p.heads;
  const unsigned blocks = (unsigned)((rows + kPagedJoinWarps - 1) / kPagedJoinWarps);
  const int n = (int)plan.blocks;
  if (rows <= 2 * n) return launch_pdl(paged_join_kernel<T, kPagedJoinSplit, 8, 1>, (unsigned)rows, 32 * kPagedJoinSplit, 0, st, p, plan.g, n);
  if (rows <= 20 * n) return launch_pdl(paged_join_kernel<T, 1, 8, 1>, blocks, 32 * kPagedJoinWarps, 0, st, p, plan.g, n);
  return launch_pdl(paged_join_kernel<T, 1, 2, 10>, blocks, 32 * kPagedJoinWarps, 0, st, p, plan.g, n);
}

bool beam_ok(const gnn_beam_call* c) {
  if (!c || c->reserved != 0 || c->dtype < GNN_DTYPE_FP32 || c->dtype > GNN_DTYPE_FP16) return false;
  if (c->beams < 1 || c->beams > kBeamMost || c->best < 1 || c->best > kBeamMost || c->vocab < 1 || !count_ok(c->vocab))
    return false;
  return count_ok(c->n_groups) && count_ok(c->n_groups * c->beams) && c->row_stride >= 0 && c->row_stride < (int64_t)1 << 39;
}

// Strips of a row.  A strip takes its rounds of elements and about eight more for its first lists and its end; two blocks of an SM run
// beside each other for nothing, more share its issue slots.  In microseconds, by strips of a row (fp32, of 300,000 elements):
//   16 rows:  1: 53.4  2: 37.0  4: 27.2  9: 21.8  19: 22.4 (taken)  32: 28.4
//   64 rows:  1: 55.9  2: 39.3  4: 32.8 (taken)  9: 35.6  32: 58.4
//   256 rows: 1: 67.1 (taken)  2: 74.4  4: 75.8  7: 98.9
int beam_strips(const gnn_beam_call* c, int n_sm) {
  const int64_t rows = c->n_groups * c->beams, round = kStripThreads * kLaneElements;
  const int64_t rounds = (c->vocab + round - 1) / round;
  int64_t best = 1, least = 0;
  for (int64_t s = 1; s <= std::min<int64_t>(kStripsMost, rounds); ++s) {
    const int64_t time = std::max<int64_t>(2, (rows * s + n_sm - 1) / n_sm) * ((rounds + s - 1) / s + 8);
    if (s == 1 || time < least) best = s, least = time;
  }
  return (int)best;
}

constexpr int kMostSms = 152;        // that strips are counted for where no device need be asked

uint64_t beam_bytes(const gnn_beam_call* c) {
  const uint64_t strips = (uint64_t)c->n_groups * c->beams * beam_strips(c, kMostSms);
  return strips * (sizeof(BeamSum) + 8 * (uint64_t)c->best);
}

// Keys (even i) or values of the caches that move together.  Layers may have one cache, and a cache one pool of keys and values: such are
// moved once.
const gnn_heads& pool_of(const gnn_pages* caches, int i) { return i % 2 ? caches[i / 2].v : caches[i / 2].k; }
int pool_before(const gnn_pages* caches, int i) {
  for (int j = 0; j < i; ++j)
    if (pool_of(caches, j).data == pool_of(caches, i).data) return j;
  return -1;
}
bool same_pool(const gnn_pages* caches, int i, int j) {
  const gnn_pages &a = caches[i / 2], &b = caches[j / 2];
  const gnn_heads &x = pool_of(caches, i), &y = pool_of(caches, j);
  return a.dtype == b.dtype && a.head_dim == b.head_dim && x.n_heads == y.n_heads && x.row_stride == y.row_stride &&
         (x.n_heads == 1 || x.head_stride == y.head_stride);
}

int width_of(uintptr_t bits) { return bits % 16 == 0 ? 16 : bits % 4 == 0 ? 4 : 1; }

// Launches over `what` states or pools of columns of at most `columns` each.
int run_moves(MoveParams& p, int what, int64_t columns, cudaStream_t st) {
  const int sms = device_sms();
  if (!sms) return cuda_fail(cudaGetLastError());
  // segments for a few rounds of all SMs, at least a block's columns each
  const int64_t want = (16 * (int64_t)sms + p.groups * what - 1) / (p.groups * what);
  p.segments = (int)std::max<int64_t>(1, std::min<int64_t>(want, (columns + kMoveThreads - 1) / kMoveThreads));
  const size_t smem = (size_t)p.beams * kMoveThreads * 16;
  cudaError_t err = allow_smem<beam_move_kernel>(kBeamMost * kMoveThreads * 16);
  if (err == cudaSuccess)
    err = launch_pdl(beam_move_kernel, (unsigned)(p.groups * what * p.segments), kMoveThreads, smem, st, p);
  return err == cudaSuccess ? GNN_OK : cuda_fail(err);
}

}  // namespace

extern "C" {

int gnn_paged_status(uint32_t* status, gnn_stream_t stream) {
  if (!status || (uintptr_t)status % 4) return GNN_ERR_INVALID_ARG;
  const cudaStream_t st = (cudaStream_t)stream;
  uint32_t word = 0;
  cudaError_t err = cudaMemcpyAsync(&word, status, 4, cudaMemcpyDeviceToHost, st);
  if (err == cudaSuccess) err = cudaMemsetAsync(status, 0, 4, st);
  const cudaError_t done = cudaStreamSynchronize(st);          // whatever failed: the copy writes to this frame
  if (err == cudaSuccess) err = done;
  if (err != cudaSuccess) return cuda_fail(err);
  if (word & DEV_ERR_TIMEOUT) return GNN_ERR_DEVICE_TIMEOUT;
  if (word & DEV_ERR_INDEX_RANGE) return GNN_ERR_INDEX_RANGE;
  return GNN_OK;
}

int gnn_paged_append(const gnn_pages* c, const gnn_rotary* rot, const gnn_append_call* a, gnn_stream_t stream) {
  if (!a || !pages_ok(c) || !rotary_args_ok(rot, c->dtype, c->head_dim, a->n_rows, a->positions)) return GNN_ERR_INVALID_ARG;
  if (!std::isfinite(a->eps) || a->eps < 0.f || (uintptr_t)a->q_gain % 4 || (uintptr_t)a->k_gain % 4 || (uintptr_t)a->q_start % 4)
    return GNN_ERR_INVALID_ARG;
  if (a->eps == 0.f && (a->q_gain || a->k_gain)) return GNN_ERR_INVALID_ARG;
  if (a->n_rows == 0 || c->n_seqs == 0) return GNN_OK;
  if (!a->q_start || (a->q.data != nullptr) != (a->q_out.data != nullptr)) return GNN_ERR_INVALID_ARG;
  const gnn_heads* in[3] = {&a->q, &a->k, &a->v};
  const gnn_heads* out[3] = {&a->q_out, &c->k, &c->v};
  RotaryParams p = {};
  for (int i = a->q.data ? 0 : 1; i < 3; ++i) {
    if (!view_ok(in[i], c->dtype) || !view_ok(out[i], c->dtype) || in[i]->n_heads != out[i]->n_heads) return GNN_ERR_INVALID_ARG;
    p.in[i] = view(*in[i], c->dtype);
    p.out[i] = view(*out[i], c->dtype);
    p.heads[i] = in[i]->n_heads;
  }
  p.gain[0] = a->q_gain;
  p.gain[1] = a->k_gain;
  p.eps = a->eps;
  p.pages = {a->q_start, c->kv_len, c->table, c->table_stride, c->n_pages, c->n_seqs, c->table_width, log2_of(c->page_size), c->status};
  return run_rotary<true>(rot, c->dtype, c->head_dim, p, a->eps > 0.f, a->positions, a->positions_float, a->n_rows,
                          (cudaStream_t)stream);
}

int gnn_paged_workspace(const gnn_pages* c, const gnn_paged_call* a, uint64_t* bytes) {
  if (!bytes || !attend_ok(c, a)) return GNN_ERR_INVALID_ARG;
  *bytes = 0;
  if (a->n_q_rows == 0 || c->n_seqs == 0) return GNN_OK;
  const int sms = device_sms();
  if (!sms) return cuda_fail(cudaGetLastError());
  *bytes = paged_plan(c, a, sms).bytes;
  return GNN_OK;
}

int gnn_paged_attend(const gnn_pages* c, const gnn_paged_call* a, gnn_stream_t stream) {
  if (!attend_ok(c, a)) return GNN_ERR_INVALID_ARG;
  if (a->n_q_rows == 0 || c->n_seqs == 0) return GNN_OK;
  if (!a->workspace || (uintptr_t)a->workspace % 32 || a->n_q_rows * a->q.n_heads >= (int64_t)1 << 32) return GNN_ERR_INVALID_ARG;
  const int sms = device_sms();
  if (!sms) return cuda_fail(cudaGetLastError());
  if (!map_encoder()) return GNN_ERR_CUDA;
  const PagedPlan plan = paged_plan(c, a, sms);
  if (a->workspace_bytes < plan.bytes) return GNN_ERR_INVALID_ARG;
  PagedParams p = {};
  p.q = view(a->q, c->dtype);
  p.k = view(c->k, c->dtype);
  p.v = view(c->v, c->dtype);
  p.out = view(a->out, c->dtype);
  p.q_start = a->q_start;
  p.kv_len = c->kv_len;
  p.table = c->table;
  p.group_start = a->group_start;
  p.shared_len = a->shared_len;
  p.table_stride = c->table_stride;
  p.n_pages = c->n_pages;
  p.n_q_rows = (int)a->n_q_rows;
  p.n_seqs = c->n_seqs;
  p.n_groups = a->n_groups;
  p.width = c->table_width;
  p.shift = log2_of(c->page_size);
  p.max_q = (int)(a->max_q > 0 ? std::min<int64_t>(a->max_q, a->n_q_rows) : a->n_q_rows);
  p.heads = a->q.n_heads;
  p.kv_heads = c->k.n_heads;
  p.dim = c->head_dim;
  // a scale of zero as one too small to be seen, so that -inf, a score that is not seen, stays -inf
  p.scale_log2 = a->scale == 0.f ? 1e-30f : (float)((double)a->scale * 1.4426950408889634);
  p.err = c->status;
  // the packs' queries, keys and values; the groups', which are the same where the loads are
  CUtensorMap maps[6];
  const int64_t rows = c->n_pages * c->page_size;
  if (!paged_map(&maps[1], a->q, a->n_q_rows, c->dtype, p.dim, plan.g.group, plan.g.box_b) ||
      !paged_map(&maps[4], c->k, rows, c->dtype, p.dim, 1, kPiece) || !paged_map(&maps[5], c->v, rows, c->dtype, p.dim, 1, kPiece))
    return GNN_ERR_INVALID_ARG;
  maps[0] = maps[1];
  maps[2] = maps[4];
  maps[3] = maps[5];
  if (p.n_groups > 0) {
    if (plan.g.box_a != plan.g.box_b && !paged_map(&maps[0], a->q, a->n_q_rows, c->dtype, p.dim, plan.g.group, plan.g.box_a))
      return GNN_ERR_INVALID_ARG;
    if (plan.g.box != kPiece && (!paged_map(&maps[2], c->k, rows, c->dtype, p.dim, 1, plan.g.box) ||
                                 !paged_map(&maps[3], c->v, rows, c->dtype, p.dim, 1, plan.g.box)))
      return GNN_ERR_INVALID_ARG;
  }
  const cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t err = c->dtype == GNN_DTYPE_BF16
                              ? p.dim <= 64 ? launch_paged<__nv_bfloat16, 64>(p, plan, maps, st) : launch_paged<__nv_bfloat16, 128>(p, plan, maps, st)
                              : p.dim <= 64 ? launch_paged<__half, 64>(p, plan, maps, st) : launch_paged<__half, 128>(p, plan, maps, st);
  return err == cudaSuccess ? GNN_OK : cuda_fail(err);
}

int gnn_beam_workspace(const gnn_beam_call* c, uint64_t* bytes) {
  if (!bytes || !beam_ok(c)) return GNN_ERR_INVALID_ARG;
  *bytes = c->n_groups == 0 ? 0 : beam_bytes(c);
  return GNN_OK;
}

int gnn_beam_select(const gnn_beam_call* c, gnn_stream_t stream) {
  if (!beam_ok(c)) return GNN_ERR_INVALID_ARG;
  if (c->n_groups == 0) return GNN_OK;
  if (!c->logits || !c->scores || !c->out_scores || !c->out_parents || !c->out_tokens || !c->workspace) return GNN_ERR_INVALID_ARG;
  if ((uintptr_t)c->logits % elem_bytes(c->dtype) || (uintptr_t)c->scores % 4 || (uintptr_t)c->out_scores % 4 ||
      (uintptr_t)c->out_parents % 4 || (uintptr_t)c->out_tokens % 4 || (uintptr_t)c->workspace % 16 ||
      c->workspace_bytes < beam_bytes(c))
    return GNN_ERR_INVALID_ARG;
  BeamParams p = {};
  p.x = c->logits;
  p.stride = c->row_stride;
  p.score = c->scores;
  p.ended = c->ended;
  p.end = c->end_token;
  p.beams = c->beams;
  p.vocab = c->vocab;
  p.best = c->best;
  p.strips = beam_strips(c, kMostSms);
  p.rows = c->n_groups * c->beams;
  if (p.rows * p.strips >= (int64_t)1 << 31) p.strips = 1;
  p.sums = static_cast<BeamSum*>(c->workspace);
  p.lists = reinterpret_cast<uint64_t*>(p.sums + p.rows * p.strips);
  p.out_score = c->out_scores;
  p.out_parent = c->out_parents;
  p.out_token = c->out_tokens;
  const cudaStream_t st = (cudaStream_t)stream;
  const unsigned grid = (unsigned)(p.rows * p.strips);
  auto strips = [&](auto element) {
    using T = decltype(element);
    const cudaError_t set = allow_smem<beam_strip_kernel<T>>(strip_smem<T>());
    return set != cudaSuccess ? set : launch_pdl(beam_strip_kernel<T>, grid, kStripThreads, strip_smem<T>(), st, p);
  };
  cudaError_t err = c->dtype == GNN_DTYPE_FP32 ? strips(float()) : c->dtype == GNN_DTYPE_BF16 ? strips(__nv_bfloat16()) : strips(__half());
  const int smem = join_smem(p.beams, p.strips, p.best);
  if (err == cudaSuccess) err = allow_smem<beam_join_kernel>(join_smem(kBeamMost, kStripsMost, kBeamMost));
  if (err == cudaSuccess) err = launch_pdl(beam_join_kernel, (unsigned)c->n_groups, kJoinThreads, smem, st, p);
  return err == cudaSuccess ? GNN_OK : cuda_fail(err);
}

int gnn_beam_reorder(const int32_t* parents, int64_t n_groups, int32_t beams, const gnn_beam_state* states, int32_t n_states,
                     gnn_stream_t stream) {
  if (beams < 1 || beams > kBeamMost || n_groups < 0 || n_groups > 1 << 26 || n_states < 0 || (n_states > 0 && !states) ||
      (uintptr_t)parents % 4)
    return GNN_ERR_INVALID_ARG;
  for (int i = 0; i < n_states; ++i) {
    const gnn_beam_state& s = states[i];
    const int64_t most = (int64_t)1 << 39;
    if (s.row_bytes < 0 || s.stride < s.row_bytes || s.out_stride < s.row_bytes || s.stride >= most || s.out_stride >= most ||
        (s.out == s.data && s.out_stride != s.stride))
      return GNN_ERR_INVALID_ARG;
    if (n_groups > 0 && s.row_bytes > 0 && (!s.data || !s.out)) return GNN_ERR_INVALID_ARG;
    for (int j = 0; j < i && s.row_bytes > 0; ++j)
      if (states[j].row_bytes > 0 && states[j].out == s.out) return GNN_ERR_INVALID_ARG;     // moved twice at once
  }
  if (n_groups == 0) return GNN_OK;
  if (!parents) return GNN_ERR_INVALID_ARG;
  MoveParams p = {};
  p.parent = parents;
  p.groups = n_groups;
  p.beams = beams;
  int64_t columns = 0;
  for (int i = 0; i < n_states; ++i) {
    const gnn_beam_state& s = states[i];
    if (s.row_bytes > 0) {
      const int w = width_of((uintptr_t)s.data | (uintptr_t)s.out | (uintptr_t)s.stride | (uintptr_t)s.out_stride | (uintptr_t)s.row_bytes);
      p.state[p.states++] = {static_cast<char*>(s.data), static_cast<char*>(s.out), s.stride, s.out_stride, s.row_bytes, w};
      columns = std::max(columns, s.row_bytes / w);
    }
    if (p.states == 0 || (p.states < kMoveStates && i + 1 < n_states)) continue;
    const int rc = run_moves(p, p.states, columns, (cudaStream_t)stream);
    if (rc != GNN_OK) return rc;
    p.states = 0;
    columns = 0;
  }
  return GNN_OK;
}

int gnn_paged_reorder(const gnn_pages* caches, int32_t n_caches, const int32_t* parents, int64_t n_groups,
                      int32_t beams, gnn_stream_t stream) {
  if (n_caches < 1 || !caches || beams < 1 || beams > kBeamMost || n_groups < 0 || n_groups > 1 << 26 ||
      (uintptr_t)parents % 4)
    return GNN_ERR_INVALID_ARG;
  const gnn_pages& c = caches[0];
  for (int i = 0; i < n_caches; ++i) {
    const gnn_pages& x = caches[i];
    if (!pages_ok(&x) || x.n_seqs != n_groups * beams || x.table != c.table || x.kv_len != c.kv_len || x.page_size != c.page_size ||
        x.table_stride != c.table_stride || x.table_width != c.table_width || x.n_pages != c.n_pages)
      return GNN_ERR_INVALID_ARG;
  }
  for (int i = 1; i < 2 * n_caches; ++i) {
    const int j = pool_before(caches, i);
    if (j >= 0 && !same_pool(caches, i, j)) return GNN_ERR_INVALID_ARG;
  }
  if (n_groups == 0) return GNN_OK;
  if (!parents) return GNN_ERR_INVALID_ARG;
  MoveParams p = {};
  p.parent = parents;
  p.groups = n_groups;
  p.beams = beams;
  p.table = const_cast<int*>(c.table);
  p.kv_len = c.kv_len;
  p.table_stride = c.table_stride;
  p.n_pages = c.n_pages;
  p.table_width = c.table_width;
  p.shift = log2_of(c.page_size);
  p.err = c.status;
  for (int i = 0; i < 2 * n_caches;) {
    int64_t columns = 1;
    p.pools = 0;
    for (; i < 2 * n_caches && p.pools < kMoveStates; ++i) {
      if (pool_before(caches, i) >= 0) continue;
      const gnn_pages& x = caches[i / 2];
      const HeadsView v = view(pool_of(caches, i), x.dtype);
      const int bytes = x.head_dim * elem_bytes(x.dtype);
      const int w = width_of((uintptr_t)v.data | (uintptr_t)v.row_bytes | (uintptr_t)v.head_bytes | (uintptr_t)bytes);
      if (p.pools > 0 && bytes != p.dim_bytes) break;
      p.dim_bytes = bytes;
      p.pool[p.pools++] = {v.data, v.row_bytes, v.head_bytes, x.k.n_heads, w};
      columns = std::max<int64_t>(columns, (int64_t)x.page_size * x.k.n_heads * (bytes / w));
    }
    // the table last: the launches before only read it
    const int err = run_moves(p, p.pools + (i == 2 * n_caches ? 1 : 0), columns, (cudaStream_t)stream);
    if (err != GNN_OK) return err;
  }
  return GNN_OK;
}

}  // extern "C"
