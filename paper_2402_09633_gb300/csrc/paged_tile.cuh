// Attention over keys in pages, by tiles of 128 rows on tcgen05: what hypotheses share is read once for all of them.
//
// The query heads that read a key head lie side by side as rows (row r of a tile: query r / G of the tile, head r % G of
// the group).  A group's shared keys are an item of work for every two tiles of its hypotheses' rows: S = Q K^T and
// O = P V.  The sequences' own keys are items too, of a pack of consecutive sequences whose rows fit a tile: their keys follow
// each other in pieces of 16 rows, and a row sees the range that is its sequence's.  A tile costs the same with few
// rows as with 128, so that packing costs nothing, and short sequences fill blocks of keys together.  Items of one tile have
// their blocks in turn on the two tiles of tensor memory, so that one block's products run beside the other's softmax.
//
// All blocks of all items are one list, of which every thread block takes an equal share: it sums up the lengths, finds its
// place and goes on from there, so the host knows no lengths and no SM idles over ragged ones.  A share's part of an item leaves
// its outputs, maxima and sums in the workspace, and a second kernel joins the parts of every row, in order.
//
// Softmax as in the other tiled kernel: P = exp2(scale (S - m)) with a running maximum m that follows only when it is outgrown
// by 2^8 / scale.
//
// Measured (bf16, 16 query heads on 4 key heads of 128).  Bound by the tensor cores' operands and each tile's wait for its softmax:
// 512 sequences that share 65,536 keys, 234 us, 1,175 TFLOP/s, tensor pipe 60 % busy; a block for two tiles is 1.75 us.  Bound by HBM:
// 64 sequences of up to 8,192 keys of their own, 136 us, 5.9 TB/s.  Bound by its chain: 64 sequences that share 16,384 keys, 33 us,
// of which 6 are the start, 6 the blocks and 11 the join.  Packs of one sequence (where the most queries are not known) instead of 32:
// 262 us for the first, 36 for the last.
#pragma once
#include "attend_tile.cuh"
#include "paged.cuh"

namespace gnn {

constexpr int kPagedCost = 2;        // what an item's start and end take, in blocks (4: +1.3 %, 6: +3.2 % over 35 calls of all sizes)
constexpr int kPiece = 16;           // keys of a piece: pages have whole pieces
constexpr int kPieces = kKeys / kPiece;
constexpr int kPackMost = 32;        // sequences of a pack: a lane to each
constexpr int kPagedKept = 768, kGroupsKept = 64;              // sequences and groups that a thread block keeps what it has found out about

struct PagedGrid {
  int tile_q, box_a, box_b;          // queries of a tile; queries that a load of a group's, of a pack's brings
  int box;                           // rows of a load of shared keys: of a page, at most a block's
  int group;                         // query heads to a key head
  int pack;                          // sequences of a pack, a power of two; 1: a sequence may have several tiles
  int rows_a, rows_b;                // the most rows of a tile
  int64_t* chunks;                   // weights of kAttendThreads groups each, then of as many sequences; null where there are few of both
  int2 *first_a, *first_b;           // [ordinal]: the first thread block of an item, and how many have a part
  float *out_a, *out_b;              // outputs of parts, [rows][dim]: see paged_places
  float2 *sum_a, *sum_b;             // [rows]: scaled maximum and sum (with a minus: some output is not finite)
};

// What a group has to do over its shared keys, or a pack over its own: `twos` items of two tiles and `ones` of one for each key
// head, over `blocks` blocks of keys.
struct PagedWork { int q0, nq, table, len, blocks, twos, ones; };

__device__ __forceinline__ PagedWork paged_group_work(const PagedParams& p, const PagedGrid& g, int i, bool* bad) {
  PagedWork w = {};
  const int a = p.group_start[i], z = p.group_start[i + 1];
  const int s0 = min(max(a, 0), p.n_seqs), s1 = min(max(z, s0), p.n_seqs);
  *bad = *bad || a != s0 || z != s1;
  const int first = p.q_start[s0], last = p.q_start[s1];
  w.q0 = min(max(first, 0), p.n_q_rows);
  w.nq = min(max(last, w.q0), p.n_q_rows) - w.q0;
  w.table = s0;
  bool outside = false;
  w.len = paged_shared(p, i, &outside);
  *bad = *bad || (outside && s1 > s0);
  w.blocks = (w.len + kKeys - 1) / kKeys;
  const int tiles = (w.nq + g.tile_q - 1) / g.tile_q;
  w.twos = tiles / 2;
  w.ones = tiles % 2;
  return w;
}

// A sequence's own keys: positions shared .. len - 1, in `pieces` pieces from position base on.
struct PagedOwn { int q0, nq, base, shared, len, pieces; };
__device__ __forceinline__ PagedOwn paged_own(const PagedParams& p, int b, bool* bad) {
  const PagedSequence s = paged_sequence(p, b, bad);
  *bad = *bad || s.nq > p.max_q;
  const int base = s.shared / kPiece * kPiece;
  // queries below the shared length are left to the join, row by row
  const int pieces = s.nq == 0 || s.len - s.nq < s.shared ? 0 : (s.len - base + kPiece - 1) / kPiece;
  return {s.q0, s.nq, base, s.shared, s.len, pieces};
}

// A pack's work, on every one of its lanes (a lane to a sequence, `pack` lanes side by side); prefix: pieces of those before.
__device__ __forceinline__ PagedWork paged_pack_work(const PagedGrid& g, const PagedOwn& o, int* prefix) {
  const int lane = threadIdx.x & 31;
  int upto = o.pieces, all = o.pieces, q0 = o.q0, q1 = o.q0 + o.nq;
  for (int d = 1; d < g.pack; d *= 2) {
    const int y = __shfl_up_sync(0xffffffffu, upto, d);
    if ((lane & (g.pack - 1)) >= d) upto += y;
    all += __shfl_xor_sync(0xffffffffu, all, d);
    q0 = min(q0, __shfl_xor_sync(0xffffffffu, q0, d));
    q1 = max(q1, __shfl_xor_sync(0xffffffffu, q1, d));
  }
  *prefix = upto - o.pieces;
  PagedWork w = {};
  w.q0 = q0;
  w.nq = q1 - q0;
  w.blocks = (all + kPieces - 1) / kPieces;
  w.ones = g.pack > 1 ? (w.nq > 0 ? 1 : 0) : (w.nq + g.tile_q - 1) / g.tile_q;
  return w;
}

__device__ __forceinline__ int64_t paged_weight(const PagedParams& p, const PagedWork& w) {
  if (w.blocks == 0) return 0;
  return (int64_t)p.kv_heads * (w.twos + w.ones) * (w.blocks + kPagedCost);
}

// Of group i, or of the pack of sequence i on its first sequence's thread; all of a warp call it.
__device__ __forceinline__ int64_t paged_weight_of(const PagedParams& p, const PagedGrid& g, bool own, int i, bool* bad, PagedWork& w, PagedOwn& o) {
  if (!own) {
    if (i >= p.n_groups) return 0;
    w = paged_group_work(p, g, i, bad);
    return paged_weight(p, w);
  }
  o = {p.n_q_rows, 0, 0, 0, 0, 0};
  if (i < p.n_seqs) o = paged_own(p, i, bad);
  int prefix;
  w = paged_pack_work(g, o, &prefix);
  return (threadIdx.x & 31 & (g.pack - 1)) == 0 ? paged_weight(p, w) : 0;
}

// Ordinals leave room for every item, whatever lies before it: no sum over the groups or sequences is needed.
__device__ __forceinline__ int64_t paged_ordinal_a(const PagedGrid& g, int group, int q0) { return (int64_t)(q0 / (2 * g.tile_q)) + group; }
__device__ __forceinline__ int64_t paged_ordinal_b(const PagedGrid& g, int pack, int q0) {
  return g.pack > 1 ? (int64_t)pack : (int64_t)(q0 / g.tile_q) + pack;
}
// Where a part of an item leaves its outputs: tile t's (or of one tile, those of its blocks on tile t of tensor memory) row r in row
// first + thread block * 2 * (the most rows of a tile) + 2 r + t.  Items have room for twice their own rows, behind those of all items
// before them in the list: a thread block's parts follow its earlier ones, and an item's parts lie a whole part apart.  So all
// that is needed is two places for each row and head, and two to a thread block, whatever number of sequences or groups the rows are of.
// row0, have: the item's first query, and how many there are from it on in the group, pack or sequence.
__device__ __forceinline__ int64_t paged_places(const PagedParams& p, const PagedGrid& g, bool own, int row0, int have, int head) {
  return (int64_t)row0 * (2 * p.heads) + head * min(have, own ? g.box_b : 2 * g.tile_q) * (2 * g.group);
}
// Divisions of what is not negative, in 32 bits where that does: 64 bits take a warp with few registers thousands of cycles.
__device__ __forceinline__ int64_t paged_divide(int64_t a, int64_t b) {
  return (a | b) >> 32 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}

// A part of an item, as the softmax and the products need it.  Query i of the tile, of the last segment with q0 <= i, sees the
// keys from lo to below limit + (i - q0) * step.
struct PagedSegment { int q0, lo, limit; };
struct PagedItem {
  int n, first;                      // blocks of this part (-1: there is no more work), and the first one's number
  int whole;                         // blocks whose rows all are keys, as far as that is known
  int both, start;                   // two tiles over the same blocks; or one tile, the first block on tile `start`
  int rows[2];                       // of each tile
  int query[2];                      // each tile's first
  int segments, step;
  float* out;
  float2* sum;
  PagedSegment seg[kPackMost];
};

struct PagedBars {
  uint64_t q_full[4], q_empty[4], kv_full[8], kv_empty[8], drain[2];
  uint64_t s_full[2], s_free[2], p_half[2], p_full[2], pv_done[2];
  uint64_t item_full[kItemSlots], item_empty[kItemSlots];
  PagedItem item[kItemSlots];
  int64_t scan[2][kAttendThreads / 32];
  int64_t before;
  int at;
  PagedOwn own[kPagedKept];          // the first sequences
  PagedWork shared[kGroupsKept];     // the first groups
  uint16_t there[8][kPieces];        // of a stage of values: the rows of a piece that are keys, first | end << 8
  uint32_t tmem;
  int abort;
};
template <int DP>
constexpr int paged_smem_bytes() { return AttendShape<DP>::kSmem + (int)sizeof(PagedBars) + 1024; }

// Block b's share of the list: positions [start, end), the group or pack (own) that start falls on, and its position.
struct PagedShare { int64_t start, end, share, before; int at; bool own; };
__device__ __forceinline__ PagedShare paged_share(const PagedParams& p, const PagedGrid& g, PagedBars& s) {
  constexpr int W = kAttendThreads / 32;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  constexpr int KEEP = kPagedKept / kAttendThreads;
  bool bad = false;
  auto weight = [&](bool own, int i) {               // and what is kept
    PagedWork w;
    PagedOwn o;
    const int64_t n = paged_weight_of(p, g, own, i, &bad, w, o);
    if (own && i < kPagedKept) s.own[i] = o;
    if (!own && i < min(p.n_groups, kGroupsKept)) s.shared[i] = w;
    return n;
  };
  int64_t sum[2] = {0, 0}, kept[KEEP] = {};
  const int group_chunks = (p.n_groups + kAttendThreads - 1) / kAttendThreads, seq_chunks = (p.n_seqs + kAttendThreads - 1) / kAttendThreads;
  if (g.chunks) {
    for (int c = tid; c < group_chunks; c += kAttendThreads) sum[0] += g.chunks[c];
    for (int c = tid; c < seq_chunks; c += kAttendThreads) sum[1] += g.chunks[group_chunks + c];
  } else {
    // (groups from the last thread on: where there are few of both, other warps look at them)
    if (p.n_groups > 0) sum[0] = weight(false, kAttendThreads - 1 - tid);
#pragma unroll
    for (int k = 0; k < KEEP; ++k)
      if (k * kAttendThreads < p.n_seqs) sum[1] += kept[k] = weight(true, k * kAttendThreads + tid);
  }
  if (bad && blockIdx.x == 0 && !g.chunks) atomicOr(p.err, DEV_ERR_INDEX_RANGE);
  if (tid == 0) s.at = 0, s.before = LLONG_MAX;      // lengths that change under the kernel: no work
#pragma unroll
  for (int k = 0; k < 2; ++k) {
#pragma unroll
    for (int d = 16; d > 0; d /= 2) sum[k] += __shfl_xor_sync(0xffffffffu, sum[k], d);
    if (lane == 0) s.scan[k][warp] = sum[k];
  }
  __syncthreads();
  sum[0] = sum[1] = 0;
  for (int w = 0; w < W; ++w) {
    sum[0] += s.scan[0][w];
    sum[1] += s.scan[1][w];
  }
  __syncthreads();
  PagedShare r;
  const int64_t all = sum[0] + sum[1];
  r.share = max((int64_t)1, paged_divide(all + gridDim.x - 1, gridDim.x));
  r.start = min(all, (int64_t)blockIdx.x * r.share);
  r.end = min(all, r.start + r.share);
  r.own = r.start >= sum[0];
  r.before = r.own ? sum[0] : 0;
  r.at = 0;
  if (r.start >= r.end) {
    r.before = r.end;
    return r;
  }
  // Of a value of every thread: those up to this thread's, and all.
  auto scan = [&](int64_t w, int64_t& upto, int64_t& all) {
    upto = w;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int64_t y = __shfl_up_sync(0xffffffffu, upto, d);
      if (lane >= d) upto += y;
    }
    if (lane == 31) s.scan[0][warp] = upto;
    __syncthreads();
    all = 0;
    for (int x = 0; x < W; ++x) {
      if (x < warp) upto += s.scan[0][x];
      all += s.scan[0][x];
    }
  };
  int64_t upto, part;
  int c0 = 0;
  if (g.chunks) {                                    // the chunk that the start is in
    const int64_t* chunks = g.chunks + (r.own ? group_chunks : 0);
    for (int c = 0, n = r.own ? seq_chunks : group_chunks; c < n; c += kAttendThreads) {
      const int64_t w = c + tid < n ? chunks[c + tid] : 0, here = r.start - r.before;
      scan(w, upto, part);
      if (here >= upto - w && here < upto) {
        s.at = c + tid;
        s.before = r.before + upto - w;
      }
      __syncthreads();
      if (here < part) break;
      r.before += part;
    }
    c0 = s.at * kAttendThreads;
    r.before = s.before;
    __syncthreads();
  }
  for (int c = c0, n = r.own ? p.n_seqs : p.n_groups; c < n; c += kAttendThreads) {
    int64_t w = 0;
    if (r.own && !g.chunks) {
#pragma unroll
      for (int k = 0; k < KEEP; ++k)
        if (c == k * kAttendThreads) w = kept[k];
    } else {
      w = weight(r.own, c + tid);
    }
    scan(w, upto, part);
    const int64_t here = r.start - r.before;
    if (here >= upto - w && here < upto) {
      s.at = r.own ? (c + tid) / g.pack : c + tid;
      s.before = r.before + upto - w;
    }
    __syncthreads();
    if (here < part) break;
    r.before += part;
  }
  r.at = s.at;
  r.before = s.before;
  __syncthreads();
  return r;
}

// Where there are many groups or sequences: their weights, kAttendThreads to a block, so that not every block of the next kernel looks at
// all of them.  (20,000 sequences: 277 us without it, 192 with it.)
__global__ void __launch_bounds__(kAttendThreads) paged_weigh_kernel(const __grid_constant__ PagedParams p, const __grid_constant__ PagedGrid g) {
  __shared__ int64_t sum_s[kAttendThreads / 32];
  const int group_chunks = (p.n_groups + kAttendThreads - 1) / kAttendThreads, c = (int)blockIdx.x, tid = threadIdx.x;
  const bool own = c >= group_chunks;
  bool bad = false;
  PagedWork w;
  PagedOwn o;
  pdl_wait();
  pdl_trigger();
  int64_t sum = paged_weight_of(p, g, own, (own ? c - group_chunks : c) * kAttendThreads + tid, &bad, w, o);
  if (bad) atomicOr(p.err, DEV_ERR_INDEX_RANGE);
#pragma unroll
  for (int d = 16; d > 0; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if ((tid & 31) == 0) sum_s[tid / 32] = sum;
  __syncthreads();
  if (tid > 0) return;
  for (int x = 1; x < kAttendThreads / 32; ++x) sum += sum_s[x];
  g.chunks[c] = sum;
}

// Goes through a share, by one warp: part(work, own, group or pack, its item s, the item's blocks [b0, b1) that the share has,
// where its first block stands in the list, the sequence of the pack that is this lane's and the pieces before it), until ok is
// false.
template <typename F>
__device__ __forceinline__ void paged_walk(const PagedParams& p, const PagedGrid& g, const PagedShare& share, const PagedBars& s_bars, F& part, bool& ok) {
  const int lane = threadIdx.x & 31;
  int64_t at = share.before;                         // where the next group or pack stands in the list
  bool own = share.own;
  int index = share.at, chunk0 = -1;
  PagedWork chunk = {};                              // of group chunk0 + lane, or of the pack of sequence chunk0 + lane
  PagedOwn seq = {};
  int before = 0;
  while (ok && at < share.end) {
    const int first = own ? index * g.pack : index, n = own ? p.n_seqs : p.n_groups;
    if (first >= n) {
      if (own) break;
      own = true;
      index = 0;
      chunk0 = -1;
      continue;
    }
    if (chunk0 < 0 || first >= chunk0 + 32) {
      chunk0 = first;
      bool bad = false;
      if (own) {
        seq = {p.n_q_rows, 0, 0, 0, 0, 0};
        if (chunk0 + lane < n) seq = !g.chunks && chunk0 + lane < kPagedKept ? s_bars.own[chunk0 + lane] : paged_own(p, chunk0 + lane, &bad);
        chunk = paged_pack_work(g, seq, &before);
      } else {
        chunk = PagedWork{};
        if (chunk0 + lane < n) chunk = !g.chunks && chunk0 + lane < kGroupsKept ? s_bars.shared[chunk0 + lane] : paged_group_work(p, g, chunk0 + lane, &bad);
      }
    }
    const int from = first - chunk0;
    PagedWork w;
    w.q0 = __shfl_sync(0xffffffffu, chunk.q0, from);
    w.nq = __shfl_sync(0xffffffffu, chunk.nq, from);
    w.table = __shfl_sync(0xffffffffu, chunk.table, from);
    w.len = __shfl_sync(0xffffffffu, chunk.len, from);
    w.blocks = __shfl_sync(0xffffffffu, chunk.blocks, from);
    w.twos = __shfl_sync(0xffffffffu, chunk.twos, from);
    w.ones = __shfl_sync(0xffffffffu, chunk.ones, from);
    const int64_t weight = paged_weight(p, w);
    if (weight > 0 && at + weight > share.start) {
      PagedOwn mine = {};                            // lane l of the pack's: its sequence l
      int prefix = 0;
      if (own) {
        const int l = (from + lane) & 31;
        mine.q0 = __shfl_sync(0xffffffffu, seq.q0, l);
        mine.nq = __shfl_sync(0xffffffffu, seq.nq, l);
        mine.base = __shfl_sync(0xffffffffu, seq.base, l);
        mine.shared = __shfl_sync(0xffffffffu, seq.shared, l);
        mine.len = __shfl_sync(0xffffffffu, seq.len, l);
        mine.pieces = __shfl_sync(0xffffffffu, seq.pieces, l);
        prefix = __shfl_sync(0xffffffffu, before, l);
        w.table = first;
      }
      const int64_t one = w.blocks + kPagedCost, all = (int64_t)(w.twos + w.ones) * p.kv_heads;
      int64_t s = 0, pos = at;                       // the item, and where it stands
      if (share.start > at) {
        s = paged_divide(share.start - at, one);
        pos = at + s * one;
      }
      for (; ok && s < all && pos < share.end; ++s, pos += one) {
        const int64_t u0 = pos + kPagedCost;
        const int b0 = (int)min((int64_t)w.blocks, max((int64_t)0, share.start - u0)), b1 = (int)min((int64_t)w.blocks, max((int64_t)0, share.end - u0));
        if (b1 > b0) part(w, own, index, (uint32_t)s, b0, b1, u0, mine, prefix);
      }
    }
    at += weight;
    ++index;
  }
}

template <typename T, int DP>
__global__ void __launch_bounds__(kAttendThreads, 1)
    paged_tile_kernel(const __grid_constant__ PagedParams p, const __grid_constant__ PagedGrid g,
                      const __grid_constant__ CUtensorMap map_qa, const __grid_constant__ CUtensorMap map_qb,
                      const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                      const __grid_constant__ CUtensorMap map_k16, const __grid_constant__ CUtensorMap map_v16) {
  using S = AttendShape<DP>;
  constexpr int QT = 2 * S::kQBufs;                  // places of a tile's queries
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint8_t* q_buf = smem;
  uint8_t* kv_buf = smem + QT * S::kQBytes;
  PagedBars& b = *reinterpret_cast<PagedBars*>(smem + S::kSmem);
  const int warp = uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
  volatile int* abort = &b.abort;

  if (warp == kCopyWarp && lane == 0) {
    for (int i = 0; i < 4; ++i) {
      mbar_init(&b.q_full[i], 1);
      mbar_init(&b.q_empty[i], S::kMmaWarps);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&b.s_full[i], 1);
      mbar_init(&b.s_free[i], 4);
      mbar_init(&b.p_half[i], 4);
      mbar_init(&b.p_full[i], 4);
      mbar_init(&b.pv_done[i], 1);
    }
    for (int i = 0; i < 8; ++i) {
      mbar_init(&b.kv_full[i], 1);
      mbar_init(&b.kv_empty[i], S::kMmaWarps);
    }
    for (int i = 0; i < kItemSlots; ++i) {
      mbar_init(&b.item_full[i], 1);
      mbar_init(&b.item_empty[i], kSoftmaxWarps + S::kMmaWarps);
    }
    for (int i = 0; i < 2; ++i) mbar_init(&b.drain[i], 1);
    b.abort = 0;
    fence_mbar_init();
  }
  if (warp == kMmaWarp) {
    tmem_alloc(&b.tmem, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = (uint32_t)uniform((int)*reinterpret_cast<volatile uint32_t*>(&b.tmem));
  pdl_wait();
  pdl_trigger();
  const PagedShare share = paged_share(p, g, b);

  const int halves = p.dim > 64 ? 2 : 1;
  // The whole warp, for the completion of the bar's phase, within the library's limit.
  auto wait = [&](uint64_t* bar, uint32_t phase) {
    uint64_t t0 = 0;
#pragma unroll 1
    for (;;) {
      if (warp_all(mbar_wait_hint(bar, phase & 1, 200000))) return true;
      const uint64_t now = global_timer_ns();
      if (t0 == 0) t0 = now;
      const bool late = now - t0 > kWaitLimitNs;
      if (late) {
        atomicOr(p.err, DEV_ERR_TIMEOUT);
        *abort = 1;
      }
      if (__any_sync(0xffffffffu, late || *abort)) return false;
    }
  };
  if (warp >= kSoftmaxWarps) {
    regs_down<kControlRegs>();
    if (warp >= kCopyWarp) {
      // ---------------- the work, part by part: one warp hands it on and fetches queries and keys, the other values.  (A load of
      // pieces is 8 or 16 boxes, and a warp issues them one after another, at some 40 ns each.)
      const int kind = warp - kCopyWarp;
      uint32_t kv = kind, q = 0, items = 0, turn = 0;   // turn: the tile of tensor memory that the next block of one tile is on
      bool ok = true;
      // A block's keys or values: this lane's box of `rows` rows, from `row` on (mine: there are such), to row `to` of the stage.
      auto load = [&](bool mine, int row, int to, int rows, int half, int head, const CUtensorMap* mk, const CUtensorMap* mv,
                      uint32_t there) {
        const uint32_t bytes = __popc(__ballot_sync(0xffffffffu, mine)) * (uint32_t)rows * 128;
        const uint32_t st = kv % S::kStages;
        if (kv >= S::kStages) ok = wait(&b.kv_empty[st], kv / S::kStages - 1);
        if (!ok) return;
        if (kind && lane < kPieces) b.there[st][lane] = (uint16_t)there;
        __syncwarp();
        if (lane == 0) mbar_arrive_expect_tx(&b.kv_full[st], bytes);
        __syncwarp();
        if (mine)
          tma_load_3d(kv_buf + st * S::kKvBytes + half * kKeys * 128 + to * 128, kind ? mv : mk, 64 * half, head, row, &b.kv_full[st]);
        __syncwarp();
        kv += 2;
      };
      // The page of position pos of a sequence, and the row there; nowhere, where zeros are read, if there is no such page.
      auto page_of = [&](bool mine, int seq, int pos) { return mine ? p.table[(int64_t)seq * p.table_stride + (pos >> p.shift)] : 0; };
      auto row_of = [&](int page, int pos) {
        if (page >= 0 && page < p.n_pages) return (page << p.shift) + (pos & ((1 << p.shift) - 1));
        atomicOr(p.err, DEV_ERR_INDEX_RANGE);
        return (int)(p.n_pages << p.shift);
      };
      auto clip = [](int x) { return (uint32_t)min(max(x, 0), kPiece); };
      auto hand_over = [&](const PagedItem& it, const PagedSegment& segment) {
        const uint32_t slot = items % kItemSlots;
        if (items >= kItemSlots) ok = wait(&b.item_empty[slot], items / kItemSlots - 1);
        if (!ok) return;
        if (lane == 0) {
          PagedItem& to = b.item[slot];
          to.n = it.n; to.first = it.first; to.whole = it.whole; to.both = it.both; to.start = it.start; to.segments = it.segments; to.step = it.step;
#pragma unroll
          for (int t = 0; t < 2; ++t) to.rows[t] = it.rows[t], to.query[t] = it.query[t];
          to.out = it.out; to.sum = it.sum;
        }
        if (lane < it.segments) b.item[slot].seg[lane] = segment;
        __syncwarp();
        if (lane == 0) mbar_arrive(&b.item_full[slot]);
        ++items;
      };
      // Item s of what w has to do, its blocks [b0, b1); u0: where its first block stands in the list.
      auto part = [&](const PagedWork& w, bool own, int index, uint32_t s, int b0, int b1, int64_t u0, const PagedOwn& mine, int prefix) {
        const uint32_t e = s / (uint32_t)p.kv_heads;
        const int head = (int)(s - e * (uint32_t)p.kv_heads);
        PagedItem it;
        it.n = b1 - b0;
        it.first = b0;
        it.whole = own ? 0 : w.len / kKeys;
        it.both = e < (uint32_t)w.twos;
        it.start = (int)(turn & 1);
        if (!it.both) turn += (uint32_t)it.n;
        const int tile = own ? (int)e : 2 * (int)e, row0 = w.q0 + tile * g.tile_q, have = w.nq - tile * g.tile_q;
        const int most = own ? g.box_b : g.box_a;
        it.rows[0] = min(have, most) * g.group;
        it.rows[1] = it.both ? min(have - g.tile_q, most) * g.group : it.rows[0];
        it.query[0] = tile * g.tile_q;
        it.query[1] = it.both ? it.query[0] + g.tile_q : it.query[0];
        it.step = own ? 1 : 0;
        it.segments = own ? g.pack : 1;
        PagedSegment segment = {0, 0, w.len};
        if (own) {                                   // this lane's sequence; one without pieces sees nothing
          const int key0 = prefix * kPiece - mine.base;
          segment = {mine.q0 - w.q0, mine.pieces ? key0 + mine.shared : INT_MAX, mine.pieces ? key0 + mine.len - mine.nq + 1 : 0};
        }
        const int64_t ordinal = ((own ? paged_ordinal_b(g, index, w.q0) : paged_ordinal_a(g, index, w.q0)) + e) * p.kv_heads + head;
        const int64_t place = paged_places(p, g, own, row0, have, head) + (int64_t)blockIdx.x * (2 * (own ? g.rows_b : g.rows_a));
        it.out = (own ? g.out_b : g.out_a) + place * p.dim;
        it.sum = (own ? g.sum_b : g.sum_a) + place;
        if (b0 == 0 && lane == 0 && kind == 0) {
          const int64_t last = u0 + w.blocks - 1;
          (own ? g.first_b : g.first_a)[ordinal] =
              make_int2(blockIdx.x, last < share.end ? 1 : (int)paged_divide(last - share.start, share.share) + 1);
        }
        if (kind == 0) hand_over(it, segment);
        if (!ok) return;
        const int tiles = kind ? 0 : it.both ? 2 : 1;
#pragma unroll 1
        for (int t = 0; t < tiles; ++t, ++q) {
          const uint32_t qb = q % QT;
          if (q >= QT) ok = wait(&b.q_empty[qb], q / QT - 1);
          if (!ok) return;
          if (lane == 0) mbar_arrive_expect_tx(&b.q_full[qb], (uint32_t)(halves * most * g.group * 128));
          __syncwarp();
          if (lane < halves)
            tma_load_3d(q_buf + qb * S::kQBytes + lane * kTileQ * 128, own ? &map_qb : &map_qa, 64 * lane, head * g.group,
                        row0 + t * g.tile_q, &b.q_full[qb]);
          __syncwarp();
        }
        // A lane to a box, the halves of a head one after another; the next block's pages are looked up while this one's stage is
        // waited for.
        const int piece = lane & (kPieces - 1);
        if (own) {
          const int half = lane / kPieces;
          const int shift = mine.base - prefix * kPiece, end = mine.pieces ? mine.len : 0;
          auto place = [&](int i, int* pos, uint32_t* there, int* page) {
            const int at = i * kPieces + piece;
            int f = 0;                               // the last sequence with so many pieces before it
#pragma unroll 1
            for (int d = g.pack / 2; d > 0; d /= 2) {
              const int before = __shfl_sync(0xffffffffu, prefix, f + d);
              if (before <= at) f += d;
            }
            *pos = __shfl_sync(0xffffffffu, shift, f) + at * kPiece;
            const int lo = __shfl_sync(0xffffffffu, mine.shared, f), hi = __shfl_sync(0xffffffffu, end, f);
            const bool have = *pos < hi;
            *there = have ? clip(lo - *pos) | clip(hi - *pos) << 8 : 0;
            *page = page_of(have && half < halves, w.table + f, *pos);
            return have && half < halves;
          };
          int pos, page;
          uint32_t there;
          bool have_it = place(b0, &pos, &there, &page);
#pragma unroll 1
          for (int i = b0; i < b1 && ok; ++i) {
            const bool now = have_it;
            const int row = now ? row_of(page, pos) : 0;
            const uint32_t rows_there = there;
            if (i + 1 < b1) have_it = place(i + 1, &pos, &there, &page);
            load(now, row, piece * kPiece, kPiece, half, head, &map_k16, &map_v16, rows_there);
          }
        } else {
          const int boxes = kKeys / g.box, half = lane / boxes, box = lane - half * boxes;
          int pos = b0 * kKeys + box * g.box, page = page_of(half < halves && pos < w.len, w.table, pos);
#pragma unroll 1
          for (int i = b0; i < b1 && ok; ++i) {
            const bool now = half < halves && pos < w.len;
            const int row = now ? row_of(page, pos) : 0;
            pos += kKeys;
            if (i + 1 < b1) page = page_of(half < halves && pos < w.len, w.table, pos);
            load(now, row, box * g.box, g.box, half, head, &map_k, &map_v, clip(w.len - i * kKeys - piece * kPiece) << 8);
          }
        }
      };
      paged_walk(p, g, share, b, part, ok);
      if (ok && kind == 0) {
        PagedItem end = {};
        end.n = -1;
        hand_over(end, PagedSegment{});
      }
      // every copy lands before the block leaves
#pragma unroll 1
      for (uint32_t i = 2; i <= S::kStages; i += 2)
        if (kv >= i + kind) drain_wait(&b.kv_full[(kv - i) % S::kStages], (kv - i) / S::kStages & 1);
#pragma unroll 1
      for (uint32_t i = 0; i < QT; ++i)
        if (q > i) drain_wait(&b.q_full[(q - 1 - i) % QT], (q - 1 - i) / QT & 1);
    } else if (warp < kMmaWarp + S::kMmaWarps) {
      // ---------------- the products of tiles mine .. mine + NT - 1
      constexpr int NT = 2 / S::kMmaWarps;
      const int mine = NT == 1 ? warp - kMmaWarp : 0;
      const int steps = (p.dim + 15) / 16;
      constexpr uint32_t id_qk = idesc_attend<T>(kTileQ, kKeys, false);
      const uint32_t id_pv = idesc_attend<T>(kTileQ, (uint32_t)steps * 16, true);
      // in uniform registers: see the other tiled kernel
      const uint32_t q_base = (uint32_t)uniform((int)smem_u32(q_buf)), kv_base = (uint32_t)uniform((int)smem_u32(kv_buf));
      const uint64_t q_desc = sdesc_kmajor_sw128(q_base), k_desc = sdesc_kmajor_sw128(kv_base),
                     v_desc = sdesc_nmajor_sw128(kv_base, kKeys * 128);
      uint32_t kv = 0, q = 0, items = 0, qk_n[NT] = {}, pv_n[NT] = {};
      bool ok = true;
      while (ok) {
        const uint32_t slot = items % kItemSlots;
        ok = wait(&b.item_full[slot], items / kItemSlots);
        if (!ok) break;
        const int n = uniform(b.item[slot].n), both = uniform(b.item[slot].both), start = uniform(b.item[slot].start),
                  whole = uniform(b.item[slot].whole) - uniform(b.item[slot].first);
        __syncwarp();
        if (lane == 0) mbar_arrive(&b.item_empty[slot]);
        ++items;
        if (n < 0) break;
        bool fresh[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) fresh[t] = true;
        auto has = [&](int t, int i) { return both || ((i + start) & 1) == mine + t; };       // block i of the part
        auto qk = [&](int t, uint32_t st) {          // S = Q K^T, once the last scores have been read
          if (S::kApart && qk_n[t] > 0) ok = wait(&b.s_free[mine + t], qk_n[t] - 1);
          if (!ok) return;
          tc_fence_after();
          const uint64_t qa = q_desc + (((q + (both ? mine + t : 0)) % QT) * S::kQBytes >> 4), ka = k_desc + (st * S::kKvBytes >> 4);
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < DP / 16; ++k) {
              if (k >= steps) break;
              const uint64_t off = ((k >> 2) * 128 * 128 + (k & 3) * 32) >> 4;
              mma_bf16_ss(tmem + kKeys * (mine + t), qa + off, ka + off, id_qk, k > 0);
            }
            mma_commit(&b.s_full[mine + t]);
          }
          __syncwarp();
          ++qk_n[t];
        };
        // Scores in places of their own, or of the tile whose turn it is next, need not wait for the weights of this block.
        const bool ahead = S::kApart || !both;
        ok = wait(&b.q_full[q % QT], q / QT) && (!both || wait(&b.q_full[(q + 1) % QT], (q + 1) / QT));
        for (int i = -1; i < n && ok; ++i) {
          const bool more = i + 1 < n;
          const uint32_t kn = kv + 2 * (i + 1), vn = kv + 2 * i + 1;
          const uint32_t ks = kn % S::kStages, vs = vn % S::kStages;
          if (more) ok = wait(&b.kv_full[ks], kn / S::kStages);
          if (!ok) break;
          if (ahead && more) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
              if (ok && has(t, i + 1)) qk(t, ks);
            if (!ok) break;
            if (elect_one()) mma_commit(&b.kv_empty[ks]);
            __syncwarp();
          }
          if (i >= 0) {
            ok = wait(&b.kv_full[vs], vn / S::kStages);
            if (!ok) break;
            // Values of rows that are no keys: zeros, so that weights of zero leave no trace of them.  (Where several warps do this,
            // each does before its own products.)
            if (i >= whole) {
              const uint32_t there = b.there[vs][lane / 4], row4 = lane % 4 * 4;                // lane l: rows 4 l .. 4 l + 3
              uint32_t gone = 0;
#pragma unroll
              for (uint32_t r = 0; r < 4; ++r) gone |= row4 + r < (there & 255) || row4 + r >= there >> 8 ? 1u << r : 0u;
              uint32_t some = __ballot_sync(0xffffffffu, gone != 0);
              if (some) {
#pragma unroll 1
                for (; some; some &= some - 1) {
                  const int four = __ffs(some) - 1, r = lane / 8;
                  if (__shfl_sync(0xffffffffu, gone, four) >> r & 1u)
                    for (int h = 0; h < halves; ++h)
                      *reinterpret_cast<uint4*>(kv_buf + vs * S::kKvBytes + h * kKeys * 128 + (4 * four + r) * 128 + lane % 8 * 16) =
                          make_uint4(0, 0, 0, 0);
                }
                fence_async_shared();
                __syncwarp();
              }
            }
          }
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            if (i >= 0 && has(t, i)) {               // O += P V, the first 64 keys and the others
              const uint64_t va = v_desc + (vs * S::kKvBytes >> 4);
              const uint32_t acc = fresh[t] ? 0u : 1u;
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                ok = ok && wait(h ? &b.p_full[mine + t] : &b.p_half[mine + t], pv_n[t]);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                  for (int k = h ? 4 : 0; k < (h ? kKeys / 16 : 4); ++k)
                    mma_bf16_ts(tmem + S::kO + DP * (mine + t), tmem + S::kP + S::kPStep * (mine + t) + 8 * k,
                                va + (k * 2048 >> 4), id_pv, k > 0 ? 1u : acc);
                  if (h) mma_commit(&b.pv_done[mine + t]);
                }
                __syncwarp();
              }
              if (!ok) break;
              fresh[t] = false;
              ++pv_n[t];
            }
            if (!ahead && more) qk(t, ks);
            if (!ok) break;
          }
          if (!ok) break;
          if (elect_one()) {
            if (more && !ahead) mma_commit(&b.kv_empty[ks]);
            if (i >= 0) mma_commit(&b.kv_empty[vs]);
            if (i + 2 == n) {                        // the part's last Q K^T is out
              mma_commit(&b.q_empty[q % QT]);
              if (both) mma_commit(&b.q_empty[(q + 1) % QT]);
            }
          }
          __syncwarp();
        }
        kv += 2 * n;
        q += both ? 2 : 1;
      }
      if (elect_one()) mma_commit(&b.drain[mine]);
      __syncwarp();
      drain_wait(&b.drain[mine], 0);
    }
  } else {
    regs_up<kSoftmaxRegs>();
    // ---------------- softmax: a warpgroup to a tile, a row to a thread
    const int wg = warp >> 2, w0 = (warp & 3) * 32, row = w0 + lane, row_query = row / g.group;
    const uint32_t lanes = (uint32_t)w0 << 16;
    constexpr int PARTS = kKeys / 32;
    const uint32_t ts = tmem + lanes + kKeys * wg, tp = tmem + lanes + S::kP + S::kPStep * wg, to = tmem + lanes + S::kO + DP * wg;
    const float scale = fabsf(p.scale_log2);
    const float slack = 8.f / scale;                 // scores may outgrow the running maximum by 2^8
    // Weights in fp16 are taken up by 2^7, to 2^15 at most, which the sum has too, so that those down to 2^-31 of the largest are still
    // held (a weight of 2^-26 to within 2^-6 of itself) and many faint keys count in the product as they do in the sum.
    constexpr float kUp = std::is_same_v<T, __half> ? 7.f : 0.f;
    uint32_t n = 0, items = 0;                       // blocks this tile has gone through
    bool ok = true;
    while (ok) {
      const uint32_t slot = items % kItemSlots;
      ok = wait(&b.item_full[slot], items / kItemSlots);
      if (!ok) break;
      const PagedItem& item = b.item[slot];
      const int all = item.n, both = item.both, rows = item.rows[wg];
      const int skip = both || item.start == wg ? 0 : 1, first = item.first + skip;
      float* out = item.out + (2 * row + wg) * p.dim;
      float2* sum_at = item.sum + 2 * row + wg;
      int lo = INT_MAX, limit = 0;                   // the keys that the row sees; none where the tile has no such row
      if (all > 0 && row < rows) {
        const int query = item.query[wg] + row_query;
        int a = 0, z = item.segments;
#pragma unroll 1
        while (z - a > 1) {
          const int mid = (a + z) / 2;
          if (item.seg[mid].q0 <= query) a = mid; else z = mid;
        }
        lo = item.seg[a].lo;
        limit = item.seg[a].limit + (query - item.seg[a].q0) * item.step;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&b.item_empty[slot]);
      ++items;
      if (all < 0) break;
      const int blocks = both ? all : (all + 1 - skip) / 2;
      // what all rows of the warp see, and what some row does
      const int whole_lo = __reduce_max_sync(0xffffffffu, row < rows ? lo : 0), whole_hi = __reduce_min_sync(0xffffffffu, row < rows ? limit : INT_MAX);
      const int some_lo = __reduce_min_sync(0xffffffffu, lo), some_hi = __reduce_max_sync(0xffffffffu, limit);
      float m = row < rows ? -INFINITY : INFINITY, l = 0.f;        // rows that the tile does not have weigh nothing
      auto stored = [&](uint64_t* bar) {             // the weights so far are in place
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar);
      };
      auto weigh = [&](const float* s, float2 off2, float2* sum, uint32_t* w) {
        const float2 scale2 = make_float2(scale, scale);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float2 x = __ffma2_rn(make_float2(s[2 * e], s[2 * e + 1]), scale2, off2);
          x.x = exp2_approx(x.x);
          x.y = exp2_approx(x.y);
          sum[e & 1] = __fadd2_rn(sum[e & 1], x);
          w[e] = pack2<T>(x.x, x.y);
        }
      };
      for (int i = 0; i < blocks; ++i, ++n) {
        const int key0 = (first + (both ? i : 2 * i)) * kKeys;
        ok = wait(&b.s_full[wg], n);
        if (!ok) break;
        tc_fence_after();
        if (key0 >= some_hi || key0 + kKeys <= some_lo) {
          // No row of the warp sees any of it.  Not before the others are through with the last block: their arrivals are
          // counted together, and the weights before are used.
          if (i > 0) ok = wait(&b.pv_done[wg], n - 1);
          if (!ok) break;
          tc_fence_after();
          const uint32_t none[16] = {};
#pragma unroll
          for (int c = 0; c < PARTS; ++c) tmem_st_32x16(tp + 16 * c, none);
          if (S::kApart && lane == 0) mbar_arrive(&b.s_free[wg]);
          stored(&b.p_half[wg]);
          if (lane == 0) mbar_arrive(&b.p_full[wg]);
          __syncwarp();
          continue;
        }
        float s[kKeys];
#pragma unroll
        for (int c = 0; c < PARTS; ++c) tmem_ld_32x32(ts + 32 * c, s + 32 * c);
#pragma unroll
        for (int c = 0; c < PARTS; ++c) tmem_wait_ld_32(s + 32 * c);
        if (S::kApart) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&b.s_free[wg]);
        }
        if (p.scale_log2 < 0.f) {
#pragma unroll
          for (int e = 0; e < kKeys; ++e) s[e] = -s[e];
        }
        if (key0 < whole_lo || key0 + kKeys > whole_hi) {            // not every row sees all of it
          auto below = [](int x) { return x >= 32 ? 0xffffffffu : x <= 0 ? 0u : (1u << x) - 1u; };
#pragma unroll
          for (int c = 0; c < PARTS; ++c) {
            const uint32_t see = below(limit - key0 - 32 * c) & ~below(lo - key0 - 32 * c);
#pragma unroll
            for (int e = 0; e < 32; ++e) s[32 * c + e] = see >> e & 1u ? s[32 * c + e] : -INFINITY;
          }
        }
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int c = 0; c < kKeys; c += 8)
#pragma unroll
          for (int x = 0; x < 4; ++x) mx[x] = max3(mx[x], s[c + x], s[c + 4 + x]);
        const float high = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]);
        const bool grow = high > m + slack || (m == -INFINITY && high > m);
        // the last product with these weights' columns, and into these outputs, is over
        if (i > 0) {
          ok = wait(&b.pv_done[wg], n - 1);
          if (!ok) break;
          tc_fence_after();
        }
        if (__any_sync(0xffffffffu, grow)) {
          const float mn = grow ? high : m;
          const float shrink = !grow ? 1.f : m == -INFINITY ? 0.f : exp2_approx((m - mn) * scale);
          m = mn;
          l *= shrink;
          if (i > 0) {
#pragma unroll 1
            for (int c = 0; c < DP; c += 8) tmem_scale_32x8(to + c, shrink);
          }
        }
        const float off = m == -INFINITY ? kUp : fmaf(-m, scale, kUp);
        float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
        for (int c = 0; c < PARTS; ++c) {
          uint32_t w[16];
          weigh(s + 32 * c, make_float2(off, off), sum, w);
          if (c == 2) stored(&b.p_half[wg]);
          tmem_st_32x16(tp + 16 * c, w);
        }
        l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
        stored(&b.p_full[wg]);
      }
      if (!ok) break;
      const bool some = blocks > 0 && row < rows && m > -INFINITY;   // NaN too: a sum of it is, with the maximum of what is not
      const bool odd = blocks > 0 && row < rows && l != 0.f;
      // Whether the row sees keys of the part at all: then its outputs are there, though they may weigh nothing, and a sum below zero
      // says that not all of them are finite, which the join has to know whatever they weigh.
      const bool sees = blocks > 0 && lo < limit && limit > first * kKeys && lo < (first + (both ? blocks : 2 * blocks - 1)) * kKeys;
      float2 spoilt = make_float2(0.f, 0.f);         // stays zero, or becomes NaN
      if (blocks > 0) {
        ok = wait(&b.pv_done[wg], n - 1);
        if (!ok) break;
        tc_fence_after();
        if (__any_sync(0xffffffffu, sees)) {
#pragma unroll 1
          for (int c = 0; c < DP; c += 32) {
            float o[32];
            tmem_ld_32x32(to + c, o);
            tmem_wait_ld_32(o);
            if (sees) {
#pragma unroll
              for (int e = 0; e < 32; e += 8)
                if (c + e < p.dim) {
                  st_global_32b(out + c + e, reinterpret_cast<const uint32_t*>(o + e));
#pragma unroll
                  for (int x = 0; x < 8; x += 2) spoilt = __ffma2_rn(make_float2(o[e + x], o[e + x + 1]), make_float2(0.f, 0.f), spoilt);
                }
            }
          }
        }
        tc_fence_before();
      }
      if (row < rows)
        *sum_at = make_float2(some ? m * scale : odd ? 0.f : -INFINITY, spoilt.x + spoilt.y == 0.f ? l : -l);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kMmaWarp) tmem_dealloc(tmem, 512);
}

// ------------------------------------------------------------------ join
constexpr int kPagedJoinWarps = 4, kPagedJoinSplit = 8;

// A row of a head to a warp: the parts of its shared and of its own keys into one, four elements to a lane: with the largest maximum
// m of the parts, o = sum 2^(m_x - m) o_x / sum 2^(m_x - m) l_x.  Bound by its chain of dependent loads, so each step's go out
// together: what is known of the sequence and group that the row would be of if all were as large (others are searched for), first
// blocks, sums, outputs (PARTS in flight).  SPLIT warps share a row where there are few.  1,024 rows of 38 parts (20 MB): 11 us behind
// the first kernel, which leaves no room for it to be there before; 8 rows of 152 parts: 10 us, 38 with a warp to a row.
template <typename T, int SPLIT, int PARTS, int BLOCKS>
__global__ void __launch_bounds__(32 * (SPLIT > 1 ? SPLIT : kPagedJoinWarps), BLOCKS) paged_join_kernel(const __grid_constant__ PagedParams p,
                                                                              const __grid_constant__ PagedGrid g, int blocks) {
  constexpr int WARPS = SPLIT > 1 ? SPLIT : kPagedJoinWarps;       // warps of a block that meet at a barrier have one row
  __shared__ __align__(16) float q_s[WARPS][128];
  __shared__ int odd_s[WARPS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = warp % SPLIT;
  const int64_t at = (int64_t)blockIdx.x * (WARPS / SPLIT) + warp / SPLIT;
  const int row = (int)paged_divide(at, p.heads), head = (int)(at - (int64_t)row * p.heads), kv = head / g.group;
  int seq = min((int)((float)row / (float)p.n_q_rows * (float)p.n_seqs), p.n_seqs - 1);
  int group = p.n_groups > 0 ? min((int)((float)seq / (float)p.n_seqs * (float)p.n_groups), p.n_groups - 1) : -1;
  // What the caller gave is there before the first kernel ends, as all of that one's blocks have waited for it before this may start.
  // (Whoever leaves early waits too, so that this kernel does not end before that one.)
  if (at >= (int64_t)p.n_q_rows * p.heads) {
    pdl_wait();
    return;
  }
  // of the sequence's pack: its first row, and the one behind its last (a pack that is not full goes on to the array's end)
  auto pack_end = [&] {
    const int64_t end = ((int64_t)(seq / g.pack) + 1) * g.pack;
    return end <= p.n_seqs ? p.q_start[end] : p.n_q_rows;
  };
  int s0 = p.q_start[seq], s1 = p.q_start[seq + 1], len = p.kv_len[seq], pack0 = p.q_start[seq / g.pack * g.pack], pack1 = pack_end();
  int g0 = 0, g1 = 0, shared = 0;
  if (group >= 0) {
    g0 = p.group_start[group];
    g1 = p.group_start[group + 1];
    shared = p.shared_len[group];
  }
  if (row < s0 || row >= s1) {
    seq = sequence_of(p.q_start, p.n_seqs, p.n_q_rows, row);
    if (seq < 0) {
      pdl_wait();
      return;
    }
    s0 = p.q_start[seq];
    s1 = p.q_start[seq + 1];
    len = p.kv_len[seq];
    pack0 = p.q_start[seq / g.pack * g.pack];
    pack1 = pack_end();
  }
  if (group >= 0 && (seq < g0 || seq >= g1)) {
    group = sequence_of(p.group_start, p.n_groups, p.n_seqs, seq);
    if (group >= 0) {
      g0 = p.group_start[group];
      g1 = p.group_start[group + 1];
      shared = p.shared_len[group];
    }
  }
  int2 rows = make_int2(0, 0);                       // the group's: its first, and how many
  if (group >= 0) {
    const int a = min(max(g0, 0), p.n_seqs), z = min(max(g1, a), p.n_seqs), first = p.q_start[a], last = p.q_start[z];
    rows.x = min(max(first, 0), p.n_q_rows);
    rows.y = min(max(last, rows.x), p.n_q_rows) - rows.x;
  }
  // as the first kernel cuts them to the arrays
  PagedSequence sq;
  sq.q0 = min(max(s0, 0), p.n_q_rows);
  sq.nq = min(max(s1, sq.q0), p.n_q_rows) - sq.q0;
  sq.len = min(max(len, 0), paged_room(p));
  sq.group = group;
  sq.first = group >= 0 ? max(g0, 0) : seq;
  sq.shared = group >= 0 ? min(max(shared, 0), paged_room(p)) : 0;
  pack0 = min(max(pack0, 0), p.n_q_rows);
  pack1 = min(max(pack1, pack0), p.n_q_rows);
  const int i = row - sq.q0;
  pdl_wait();
  if (i >= p.max_q) return;
  auto slowly = [&] {
    const T* src = reinterpret_cast<const T*>(p.q.data + (int64_t)row * p.q.row_bytes + (int64_t)head * p.q.head_bytes);
    for (int d = lane; d < p.dim; d += 32) q_s[warp][d] = to_f(src[d]);
    __syncwarp();
    paged_attend_row<T>(p, sq, seq, i, head, q_s[warp]);
  };
  if (sq.len - sq.nq < sq.shared) {                  // a sequence with queries among the shared positions, or without keys
    if (sub == 0) slowly();
    return;
  }
  // where the row's parts lie: of the shared keys, [0, na), and of its own, [na, na + nb)
  int64_t ordinal_a = 0, ordinal_b;
  int64_t row_a = 0, row_b;
  int every = 1;                                     // shared parts of both places (1), or of one (2)
  if (sq.shared > 0) {
    if (row < rows.x || row >= rows.x + rows.y) return;            // offsets that contradict each other
    const int tile = (row - rows.x) / g.tile_q, tiles = (rows.y + g.tile_q - 1) / g.tile_q, before = tile / 2 * 2 * g.tile_q;
    every = (tile | 1) < tiles ? 2 : 1;
    row_a = paged_places(p, g, false, rows.x + before, rows.y - before, kv) + 2 * ((row - rows.x - tile * g.tile_q) * g.group + head % g.group) + (every == 2 ? tile & 1 : 0);
    ordinal_a = (paged_ordinal_a(g, group, rows.x) + tile / 2) * p.kv_heads + kv;
  }
  {
    const int pack = seq / g.pack, q0 = g.pack > 1 ? pack0 : sq.q0, tile = g.pack > 1 ? 0 : i / g.tile_q, query = row - q0 - tile * g.tile_q;
    const int have = (g.pack > 1 ? pack1 - pack0 : sq.nq) - tile * g.tile_q;
    if (query < 0 || query >= have) return;          // offsets that contradict each other
    if (query >= g.box_b) {                          // behind a sequence of the pack that has more queries than announced
      if (sub == 0) slowly();
      return;
    }
    row_b = paged_places(p, g, true, q0 + tile * g.tile_q, have, kv) + 2 * (query * g.group + head % g.group);
    ordinal_b = (paged_ordinal_b(g, pack, q0) + tile) * p.kv_heads + kv;
  }
  const int2 fa = sq.shared > 0 ? g.first_a[ordinal_a] : make_int2(0, 0), fb = g.first_b[ordinal_b];
  const int first_a = min(max(fa.x, 0), blocks - 1), first_b = min(max(fb.x, 0), blocks - 1);
  const int na = min(max(fa.y, 0), blocks - first_a) * (2 / every), nb = min(max(fb.y, 0), blocks - first_b) * 2;
  const int step_a = 2 * g.rows_a, step_b = 2 * g.rows_b;          // from one thread block's part to the next's
  row_a += first_a * step_a;
  row_b += first_b * step_b;
  const float2 *sa = g.sum_a + row_a, *sb = g.sum_b + row_b;
  const float *oa = g.out_a + row_a * p.dim, *ob = g.out_b + row_b * p.dim;
  auto at_a = [&](int k) { return every == 2 ? k * step_a : (k >> 1) * step_a + (k & 1); };
  auto at_b = [&](int k) { return (k >> 1) * step_b + (k & 1); };
  auto sums = [&](int k) { return k < na ? sa[at_a(k)] : sb[at_b(k - na)]; };
  const float2 mine = lane < na + nb ? sums(lane) : make_float2(-INFINITY, 0.f);           // the first parts, kept
  float top = mine.x;
  for (int k = lane + 32; k < na + nb; k += 32) top = fmaxf(top, sums(k).x);
#pragma unroll
  for (int d = 16; d > 0; d /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  const float ref = top == -INFINITY ? 0.f : top;
  float l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  const bool have = 4 * lane < p.dim;
  bool odd = false;                                  // something of its own keys' part is not finite
  for (int k0 = 0; k0 < na + nb; k0 += 32) {
    float z = 0.f;
    bool spoilt = false;
    if (k0 + lane < na + nb) {
      const float2 s = k0 == 0 ? mine : sums(k0 + lane);
      z = s.x == -INFINITY ? 0.f : exp2f(s.x - ref);
      l = fmaf(fabsf(s.y), z, l);
      spoilt = __float_as_int(s.y) < 0;              // a minus: its outputs are not all finite
      odd = odd || (k0 + lane >= na && (spoilt || !(fabsf(s.y) < INFINITY)));
    }
    // those that count, some at a time with their loads together; outputs that are not finite count even where they weigh nothing
    uint32_t left = __ballot_sync(0xffffffffu, z != 0.f || spoilt);
    if (SPLIT > 1) left &= (0xffffffffu / ((1u << SPLIT) - 1)) << sub;             // every SPLIT-th
    while (left) {
      float4 x[PARTS];
      float f[PARTS];
      bool own[PARTS];
#pragma unroll
      for (int e = 0; e < PARTS; ++e) {
        const int k = left ? __ffs(left) - 1 : 0;
        f[e] = __shfl_sync(0xffffffffu, z, k);
        if (left == 0) f[e] = 0.f;
        own[e] = k0 + k >= na;
        x[e] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (have && left != 0)
          x[e] = __ldcs(reinterpret_cast<const float4*>(own[e] ? ob + at_b(k0 + k - na) * p.dim : oa + at_a(k0 + k) * p.dim) + lane);
        left &= left - 1;
      }
#pragma unroll
      for (int e = 0; e < PARTS; ++e) {
        o.x = fmaf(x[e].x, f[e], o.x); o.y = fmaf(x[e].y, f[e], o.y);
        o.z = fmaf(x[e].z, f[e], o.z); o.w = fmaf(x[e].w, f[e], o.w);
        odd = odd || (own[e] && !(fabsf(x[e].x) + fabsf(x[e].y) + fabsf(x[e].z) + fabsf(x[e].w) < INFINITY));
      }
    }
  }
#pragma unroll
  for (int d = 16; d > 0; d /= 2) l += __shfl_xor_sync(0xffffffffu, l, d);
  odd = __any_sync(0xffffffffu, odd);
  if (SPLIT > 1) {                                   // a row's warps have all left before here, or none
    if (have) *reinterpret_cast<float4*>(&q_s[warp][4 * lane]) = o;
    if (lane == 0) odd_s[warp] = odd;
    __syncthreads();
    if (sub != 0) return;
#pragma unroll
    for (int w = 1; w < SPLIT; ++w) {
      const float4 x = *reinterpret_cast<const float4*>(&q_s[warp + w][have ? 4 * lane : 0]);
      o = make_float4(o.x + x.x, o.y + x.y, o.z + x.z, o.w + x.w);
      odd = odd || odd_s[warp + w];
    }
    __syncwarp();
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  o = l == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  // A weight of zero times a value that is not finite is NaN.  A pack's keys, and new rows, are seen by some of its queries only, so
  // a row whose part of its own keys is not finite is done again, key by visible key; shared keys are seen by all.
  if (odd) {
    slowly();
    return;
  }
  if (have)
    *reinterpret_cast<uint2*>(p.out.data + (int64_t)row * p.out.row_bytes + (int64_t)head * p.out.head_bytes + 8 * lane) =
        make_uint2(pack2<T>(o.x, o.y), pack2<T>(o.z, o.w));
}

}  // namespace gnn
