// Attention over keys in pages, by tiles of 128 rows on tcgen05: what hypotheses share is read once for all of them.
//
// The query heads that read a key head lie side by side as rows (row r of a tile: query r / G of the tile, head r % G of
// the group), so that the hypotheses of a group fill tiles together: S = Q K^T and O = P V over the group's shared keys, two
// tiles of rows at a time (an item).  A sequence's own keys are items of their own, with the rows of that sequence.  Items
// of one tile have their blocks of 128 keys in turn on the two tiles of tensor memory, so that one block's products run
// beside the other's softmax.
//
// All blocks of all items are one list, of which every thread block takes an equal share: it sums up the lengths, finds its
// place and goes on from there, so the host knows no lengths and no SM idles over ragged ones.  A share's part of an item leaves
// its outputs, maxima and sums in the workspace, and a second kernel joins the parts of every row, in order.
//
// Softmax as in the other tiled kernel: P = exp2(scale (S - m)) with a running maximum m that follows only when it is outgrown
// by 2^8 / scale.
#pragma once
#include "attend_tile.cuh"
#include "paged.cuh"

namespace gnn {

constexpr int kPagedCost = 1;        // what an item's start and end take, in blocks of one tile

struct PagedGrid {
  int tile_q, box_a, box_b;          // queries of a tile; queries that a load of a group's, of a sequence's brings
  int box;                           // rows of a load of keys: of a page, at most a block's
  int group;                         // query heads to a key head
  int rows_a, rows_b;                // rows of a place
  int64_t n_a;                       // ordinals of shared items
  int2 *first_a, *first_b;           // [ordinal]: the first thread block of an item, and how many have a part
  float *out_a, *out_b;              // [ordinal + thread block][2 places][rows][dim]
  float2 *sum_a, *sum_b;             // the same, [rows]: scaled maximum and sum
};

// What a group (of its shared keys) or a sequence (of its own) has to do: `twos` items of two tiles and `ones` of one for each key
// head, over `blocks` blocks of keys from position `base` on.
struct PagedWork { int q0, nq, table, base, lo, len, blocks, twos, ones; };

__device__ __forceinline__ PagedWork paged_group_work(const PagedParams& p, const PagedGrid& g, int i, bool* bad) {
  PagedWork w = {};
  const int a = p.group_start[i], z = p.group_start[i + 1];
  const int s0 = min(max(a, 0), p.n_seqs), s1 = min(max(z, s0), p.n_seqs);
  *bad = *bad || a != s0 || z != s1;
  const int first = p.q_start[s0], last = p.q_start[s1];
  w.q0 = min(max(first, 0), p.n_q_rows);
  w.nq = min(max(last, w.q0), p.n_q_rows) - w.q0;
  w.table = s0;
  w.len = paged_shared(p, i, bad);
  w.blocks = (w.len + kKeys - 1) / kKeys;
  const int tiles = (w.nq + g.tile_q - 1) / g.tile_q;
  w.twos = tiles / 2;
  w.ones = tiles % 2;
  return w;
}

__device__ __forceinline__ PagedWork paged_own_work(const PagedParams& p, const PagedGrid& g, int b, bool* bad) {
  PagedWork w = {};
  const PagedSequence s = paged_sequence(p, b, bad);
  *bad = *bad || s.nq > p.max_q;
  w.q0 = s.q0;
  w.nq = min(s.nq, p.max_q);
  w.table = b;
  w.len = s.len;
  w.base = s.shared / g.box * g.box;                 // a load begins where a page does
  w.lo = s.shared - w.base;
  // queries below the shared length are left to the join, row by row
  w.blocks = s.len - s.nq < s.shared ? 0 : (w.len - w.base + kKeys - 1) / kKeys;
  w.ones = (w.nq + g.tile_q - 1) / g.tile_q;
  return w;
}

__device__ __forceinline__ int64_t paged_weight(const PagedParams& p, const PagedWork& w) {
  if (w.blocks == 0) return 0;
  return (int64_t)p.kv_heads * ((int64_t)w.twos * (2 * (int64_t)w.blocks + kPagedCost) + (int64_t)w.ones * (w.blocks + kPagedCost));
}

// Ordinals leave room for every item, whatever lies before it: no sum over the groups or sequences is needed.
__device__ __forceinline__ int64_t paged_ordinal_a(const PagedGrid& g, int group, int q0) { return (int64_t)q0 / (2 * g.tile_q) + group; }
__device__ __forceinline__ int64_t paged_ordinal_b(const PagedGrid& g, int seq, int q0) { return (int64_t)q0 / g.tile_q + seq; }

// A part of an item, as the softmax and the products need it.
struct PagedItem {
  int n, first;                      // blocks of this part (-1: there is no more work), and the first one's number
  int both;                          // two tiles over the same blocks, or one tile over every second
  int rows[2];                       // of each tile
  int lo, len;                       // keys that there are, from the item's first block on
  int limit[2], step;                // row r of a tile sees keys below limit + (r / G) * step
  float* out[2];
  float2* sum[2];
};

struct PagedBars {
  uint64_t q_full[2], q_empty[2], kv_full[8], kv_empty[8], drain[2];
  uint64_t s_full[2], s_free[2], p_half[2], p_full[2], pv_done[2];
  uint64_t item_full[kItemSlots], item_empty[kItemSlots];
  PagedItem item[kItemSlots];
  int64_t scan[2][kAttendThreads / 32];
  int64_t before;
  int at, own;
  uint32_t tmem;
  int abort;
};
template <int DP>
constexpr int paged_smem_bytes() { return AttendShape<DP>::kSmem + (int)sizeof(PagedBars) + 1024; }

// Block b's share of the list: positions [start, end), the group or sequence (own) that start falls on, and its position.
struct PagedShare { int64_t start, end, share, before; int at; bool own; };
__device__ __forceinline__ PagedShare paged_share(const PagedParams& p, const PagedGrid& g, PagedBars& s) {
  constexpr int W = kAttendThreads / 32;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  int64_t sum[2] = {0, 0};
  bool bad = false;
  for (int i = tid; i < p.n_groups; i += kAttendThreads) sum[0] += paged_weight(p, paged_group_work(p, g, i, &bad));
  for (int i = tid; i < p.n_seqs; i += kAttendThreads) sum[1] += paged_weight(p, paged_own_work(p, g, i, &bad));
  if (bad && blockIdx.x == 0) atomicOr(p.err, DEV_ERR_INDEX_RANGE);
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
  r.share = max((int64_t)2, (all + gridDim.x - 1) / gridDim.x);      // two: every share that an item spans has a block of it
  r.start = min(all, (int64_t)blockIdx.x * r.share);
  r.end = min(all, r.start + r.share);
  r.own = r.start >= sum[0];
  r.before = r.own ? sum[0] : 0;
  r.at = 0;
  if (r.start >= r.end) return r;
  const int n = r.own ? p.n_seqs : p.n_groups;
  for (int c = 0; c < n; c += kAttendThreads) {
    const int i = c + tid;
    int64_t w = 0;
    if (i < n) w = paged_weight(p, r.own ? paged_own_work(p, g, i, &bad) : paged_group_work(p, g, i, &bad));
    int64_t upto = w;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int64_t y = __shfl_up_sync(0xffffffffu, upto, d);
      if (lane >= d) upto += y;
    }
    if (lane == 31) s.scan[0][warp] = upto;
    __syncthreads();
    int64_t chunk = 0;
    for (int x = 0; x < W; ++x) {
      if (x < warp) upto += s.scan[0][x];
      chunk += s.scan[0][x];
    }
    const int64_t here = r.start - r.before;
    if (here >= upto - w && here < upto) {
      s.at = i;
      s.before = r.before + upto - w;
    }
    __syncthreads();
    if (here < chunk) break;
    r.before += chunk;
  }
  r.at = s.at;
  r.before = s.before;
  __syncthreads();
  return r;
}

// Goes through a share, by one warp: part(work, own, group or sequence, its item s, the item's blocks [b0, b1) that the share has,
// where its first block stands in the list), until ok is false.
template <typename F>
__device__ __forceinline__ void paged_walk(const PagedParams& p, const PagedGrid& g, const PagedShare& share, F& part, bool& ok) {
  const int lane = threadIdx.x & 31;
  int64_t at = share.before;                         // where the next group or sequence stands in the list
  bool own = share.own;
  int index = share.at, chunk0 = -1;
  PagedWork chunk = {};                              // of chunk0 + lane
  while (ok && at < share.end) {
    const int n = own ? p.n_seqs : p.n_groups;
    if (index >= n) {
      if (own) break;
      own = true;
      index = 0;
      chunk0 = -1;
      continue;
    }
    if (chunk0 < 0 || index >= chunk0 + 32) {
      chunk0 = index;
      bool bad = false;
      chunk = PagedWork{};
      if (chunk0 + lane < n) chunk = own ? paged_own_work(p, g, chunk0 + lane, &bad) : paged_group_work(p, g, chunk0 + lane, &bad);
    }
    PagedWork w;
    const int from = index - chunk0;
    w.q0 = __shfl_sync(0xffffffffu, chunk.q0, from);
    w.nq = __shfl_sync(0xffffffffu, chunk.nq, from);
    w.table = __shfl_sync(0xffffffffu, chunk.table, from);
    w.base = __shfl_sync(0xffffffffu, chunk.base, from);
    w.lo = __shfl_sync(0xffffffffu, chunk.lo, from);
    w.len = __shfl_sync(0xffffffffu, chunk.len, from);
    w.blocks = __shfl_sync(0xffffffffu, chunk.blocks, from);
    w.twos = __shfl_sync(0xffffffffu, chunk.twos, from);
    w.ones = __shfl_sync(0xffffffffu, chunk.ones, from);
    const int64_t weight = paged_weight(p, w);
    if (weight > 0 && at + weight > share.start) {
      const int64_t two = 2 * (int64_t)w.blocks + kPagedCost, one = w.blocks + kPagedCost;
      const int64_t twos = (int64_t)w.twos * p.kv_heads, all = twos + (int64_t)w.ones * p.kv_heads;
      int64_t s = 0, pos = at;                       // the item, and where it stands
      if (share.start > at) {
        s = min((share.start - at) / two, twos);
        pos = at + s * two;
        if (s == twos) {
          const int64_t more = (share.start - pos) / one;
          s += more;
          pos += more * one;
        }
      }
      for (; ok && s < all && pos < share.end; ++s) {
        const int step = s < twos ? 2 : 1;
        const int64_t u0 = pos + kPagedCost;
        const int64_t skip = max((int64_t)0, share.start - u0), upto = max((int64_t)0, share.end - u0);
        const int b0 = (int)min((int64_t)w.blocks, (skip + step - 1) / step), b1 = (int)min((int64_t)w.blocks, (upto + step - 1) / step);
        if (b1 > b0) part(w, own, index, (uint32_t)s, b0, b1, u0);
        pos += step == 2 ? two : one;
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
                      const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  using S = AttendShape<DP>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint8_t* q_buf = smem;
  uint8_t* kv_buf = smem + S::kQBufs * 2 * S::kQBytes;
  PagedBars& b = *reinterpret_cast<PagedBars*>(smem + S::kSmem);
  const int warp = uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
  volatile int* abort = &b.abort;

  if (warp == kCopyWarp && lane == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&b.q_full[i], 1);
      mbar_init(&b.q_empty[i], S::kMmaWarps);
      mbar_init(&b.s_full[i], 1);
      mbar_init(&b.s_free[i], 4);
      mbar_init(&b.p_half[i], 4);
      mbar_init(&b.p_full[i], 4);
      mbar_init(&b.pv_done[i], 1);
      mbar_init(&b.drain[i], 1);
    }
    for (int i = 0; i < 8; ++i) {
      mbar_init(&b.kv_full[i], 1);
      mbar_init(&b.kv_empty[i], S::kMmaWarps);
    }
    for (int i = 0; i < kItemSlots; ++i) {
      mbar_init(&b.item_full[i], 1);
      mbar_init(&b.item_empty[i], kSoftmaxWarps + S::kMmaWarps);
    }
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
    if (warp == kCopyWarp) {
      // ---------------- the work, part by part; its queries, and its keys and values through the ring
      const int boxes = kKeys / g.box;               // of a block, a lane to each and each half of a head
      const int box = lane / halves, half = lane % halves;
      uint32_t kv = 0, q = 0, items = 0;
      bool ok = true;
      auto hand_over = [&](const PagedItem& it) {
        const uint32_t slot = items % kItemSlots;
        if (items >= kItemSlots) ok = wait(&b.item_empty[slot], items / kItemSlots - 1);
        if (!ok) return;
        if (lane == 0) {
          b.item[slot] = it;
          mbar_arrive(&b.item_full[slot]);
        }
        ++items;
      };
      // Item s of what w has to do, its blocks [b0, b1); u0: where its first block stands in the list.
      auto part = [&](const PagedWork& w, bool own, int index, uint32_t s, int b0, int b1, int64_t u0) {
        const uint32_t e = s / (uint32_t)p.kv_heads;
        const int head = (int)(s - e * (uint32_t)p.kv_heads);
        PagedItem it = {};
        it.n = b1 - b0;
        it.first = b0;
        it.both = e < (uint32_t)w.twos;
        const int tile = own ? (int)e : 2 * (int)e, row0 = w.q0 + tile * g.tile_q;
        const int have = w.nq - tile * g.tile_q;
        it.rows[0] = min(have, g.tile_q) * g.group;
        it.rows[1] = it.both ? min(have - g.tile_q, g.tile_q) * g.group : it.rows[0];
        it.lo = w.lo;
        it.len = w.len - w.base;
        it.step = own ? 1 : 0;
        it.limit[0] = own ? w.len - w.nq + tile * g.tile_q + 1 - w.base : it.len;
        it.limit[1] = it.limit[0];
        const int64_t ordinal = ((own ? paged_ordinal_b(g, index, w.q0) : paged_ordinal_a(g, index, w.q0)) + e) * p.kv_heads + head;
        const int64_t place = 2 * (ordinal + blockIdx.x);
        const int place_rows = own ? g.rows_b : g.rows_a;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          it.out[t] = (own ? g.out_b : g.out_a) + (place + t) * place_rows * p.dim;
          it.sum[t] = (own ? g.sum_b : g.sum_a) + (place + t) * place_rows;
        }
        if (b0 == 0 && lane == 0) {
          const int64_t last = u0 + (int64_t)(w.blocks - 1) * (it.both ? 2 : 1);
          (own ? g.first_b : g.first_a)[ordinal] = make_int2(blockIdx.x, (int)((last - share.start) / share.share) + 1);
        }
        hand_over(it);
        if (!ok) return;
        const uint32_t qb = q % S::kQBufs;
        if (q >= S::kQBufs) ok = wait(&b.q_empty[qb], q / S::kQBufs - 1);
        if (!ok) return;
        const int tiles = it.both ? 2 : 1, q_box = own ? g.box_b : g.box_a;
        if (lane == 0) mbar_arrive_expect_tx(&b.q_full[qb], (uint32_t)(tiles * halves * q_box * g.group * 128));
        __syncwarp();
        if (lane < tiles * halves)
          tma_load_3d(q_buf + (qb * 2 + lane / halves) * S::kQBytes + (lane % halves) * kTileQ * 128, own ? &map_qb : &map_qa,
                      64 * (lane % halves), head * g.group, row0 + lane / halves * g.tile_q, &b.q_full[qb]);
        ++q;
        const int* table = p.table + (int64_t)w.table * p.table_stride;
#pragma unroll 1
        for (int i = b0; i < b1 && ok; ++i) {
          const int pos = w.base + i * kKeys + box * g.box;
          const bool mine = box < boxes && pos < w.len;
          int row = 0;
          if (mine) {
            const int page = table[pos >> p.shift];
            if (page >= 0 && page < p.n_pages) {
              row = (page << p.shift) + (pos & ((1 << p.shift) - 1));
            } else {                                 // nowhere: zeros
              row = (int)(p.n_pages << p.shift);
              atomicOr(p.err, DEV_ERR_INDEX_RANGE);
            }
          }
          const uint32_t bytes = __popc(__ballot_sync(0xffffffffu, mine)) * (uint32_t)g.box * 128;
#pragma unroll 1
          for (int kind = 0; kind < 2; ++kind, ++kv) {
            const uint32_t st = kv % S::kStages;
            if (kv >= S::kStages) ok = wait(&b.kv_empty[st], kv / S::kStages - 1);
            if (!ok) break;
            if (lane == 0) mbar_arrive_expect_tx(&b.kv_full[st], bytes);
            __syncwarp();
            if (mine)
              tma_load_3d(kv_buf + st * S::kKvBytes + half * kKeys * 128 + box * g.box * 128, kind ? &map_v : &map_k, 64 * half, head,
                          row, &b.kv_full[st]);
            __syncwarp();
          }
        }
      };
      paged_walk(p, g, share, part, ok);
      if (ok) {
        PagedItem end = {};
        end.n = -1;
        hand_over(end);
      }
      // every copy lands before the block leaves
#pragma unroll 1
      for (uint32_t i = 0; i < S::kStages; ++i)
        if (kv > i) drain_wait(&b.kv_full[(kv - 1 - i) % S::kStages], (kv - 1 - i) / S::kStages & 1);
#pragma unroll 1
      for (uint32_t i = 0; i < S::kQBufs; ++i)
        if (q > i) drain_wait(&b.q_full[(q - 1 - i) % S::kQBufs], (q - 1 - i) / S::kQBufs & 1);
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
        const int n = uniform(b.item[slot].n), first = uniform(b.item[slot].first), both = uniform(b.item[slot].both),
                  lo = uniform(b.item[slot].lo), len = uniform(b.item[slot].len);
        __syncwarp();
        if (lane == 0) mbar_arrive(&b.item_empty[slot]);
        ++items;
        if (n < 0) break;
        const uint32_t qb = q % S::kQBufs;
        bool fresh[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) fresh[t] = true;
        auto has = [&](int t, int i) { return both || (i & 1) == mine + t; };      // block i of the part
        auto qk = [&](int t, uint32_t st) {          // S = Q K^T, once the last scores have been read
          if (S::kApart && qk_n[t] > 0) ok = wait(&b.s_free[mine + t], qk_n[t] - 1);
          if (!ok) return;
          tc_fence_after();
          const uint64_t qa = q_desc + ((qb * 2 + (both ? mine + t : 0)) * S::kQBytes >> 4), ka = k_desc + (st * S::kKvBytes >> 4);
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
        ok = wait(&b.q_full[qb], q / S::kQBufs);
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
            // Values of rows that are no keys of the item: zeros, so that weights of zero leave no trace of them.  (Where
            // several warps do this, each does before its own products.)
            const int key0 = (first + i) * kKeys;
            if (key0 < lo || key0 + kKeys > len) {
#pragma unroll 1
              for (int r = lane; r < kKeys * 8; r += 32)
                if (key0 + r / 8 < lo || key0 + r / 8 >= len)
                  for (int h = 0; h < halves; ++h)
                    *reinterpret_cast<uint4*>(kv_buf + vs * S::kKvBytes + h * kKeys * 128 + r * 16) = make_uint4(0, 0, 0, 0);
              fence_async_shared();
              __syncwarp();
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
            if (i + 2 == n) mma_commit(&b.q_empty[qb]);      // the part's last Q K^T is out
          }
          __syncwarp();
        }
        kv += 2 * n;
        ++q;
      }
      if (elect_one()) mma_commit(&b.drain[mine]);
      __syncwarp();
      drain_wait(&b.drain[mine], 0);
    }
  } else {
    regs_up<kSoftmaxRegs>();
    // ---------------- softmax: a warpgroup to a tile, a row to a thread
    const int wg = warp >> 2, w0 = (warp & 3) * 32, row = w0 + lane, query = row / g.group;
    const uint32_t lanes = (uint32_t)w0 << 16;
    constexpr int PARTS = kKeys / 32;
    const uint32_t ts = tmem + lanes + kKeys * wg, tp = tmem + lanes + S::kP + S::kPStep * wg, to = tmem + lanes + S::kO + DP * wg;
    const float scale = fabsf(p.scale_log2);
    const float slack = 8.f / scale;                 // scores may outgrow the running maximum by 2^8
    uint32_t n = 0, items = 0;                       // blocks this tile has gone through
    bool ok = true;
    while (ok) {
      const uint32_t slot = items % kItemSlots;
      ok = wait(&b.item_full[slot], items / kItemSlots);
      if (!ok) break;
      const PagedItem& item = b.item[slot];
      const int all = item.n, both = item.both, rows = item.rows[wg], len = item.len, lo = item.lo;
      const int low = item.limit[wg], limit = min(len, low + query * item.step);      // the tile's first row's, and the row's
      const int first = item.first + (both ? 0 : wg);
      float* out = item.out[wg] + (int64_t)row * p.dim;
      float2* sum_at = item.sum[wg] + row;
      __syncwarp();
      if (lane == 0) mbar_arrive(&b.item_empty[slot]);
      ++items;
      if (all < 0) break;
      const int blocks = both ? all : (all + 1 - wg) / 2;
      const bool idle = w0 >= rows;                  // the warp has no rows: what lies in its weights touches no other row
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
        if (idle) {
          // not before the others are through with the last block: their arrivals are counted together
          if (i > 0) ok = wait(&b.pv_done[wg], n - 1);
          if (!ok) break;
          tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            if (S::kApart) mbar_arrive(&b.s_free[wg]);
            mbar_arrive(&b.p_half[wg]);
            mbar_arrive(&b.p_full[wg]);
          }
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
        if (key0 < lo || key0 + kKeys > low) {       // not every row sees all of it
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
        const float off = m == -INFINITY ? 0.f : -m * scale;
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
      if (blocks > 0) {
        ok = wait(&b.pv_done[wg], n - 1);
        if (!ok) break;
        tc_fence_after();
        if (!idle) {
#pragma unroll 1
          for (int c = 0; c < DP; c += 32) {
            float o[32];
            tmem_ld_32x32(to + c, o);
            tmem_wait_ld_32(o);
            if (row < rows) {
#pragma unroll
              for (int e = 0; e < 32; e += 8)
                if (c + e < p.dim) st_global_32b(out + c + e, reinterpret_cast<const uint32_t*>(o + e));
            }
          }
        }
        tc_fence_before();
      }
      if (row < rows) *sum_at = blocks > 0 ? make_float2(m * scale, l) : make_float2(-INFINITY, 0.f);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kMmaWarp) tmem_dealloc(tmem, 512);
}

// ------------------------------------------------------------------ join
constexpr int kPagedJoinWarps = 4;

// A row of a head to a warp: the parts of its shared and of its own keys into one, four elements to a lane.
template <typename T>
__global__ void __launch_bounds__(32 * kPagedJoinWarps) paged_join_kernel(const __grid_constant__ PagedParams p,
                                                                           const __grid_constant__ PagedGrid g, int blocks) {
  __shared__ float q_s[kPagedJoinWarps][128];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t at = (int64_t)blockIdx.x * kPagedJoinWarps + warp;
  pdl_wait();
  if (at >= (int64_t)p.n_q_rows * p.heads) return;
  const int row = (int)(at / p.heads), head = (int)(at - (int64_t)row * p.heads), kv = head / g.group;
  const int seq = sequence_of(p.q_start, p.n_seqs, p.n_q_rows, row);
  if (seq < 0) return;
  bool bad = false;
  const PagedSequence sq = paged_sequence(p, seq, &bad);
  const int i = row - sq.q0;
  if (i >= p.max_q) return;
  auto slowly = [&] {
    const T* src = reinterpret_cast<const T*>(p.q.data + (int64_t)row * p.q.row_bytes + (int64_t)head * p.q.head_bytes);
    for (int d = lane; d < p.dim; d += 32) q_s[warp][d] = to_f(src[d]);
    __syncwarp();
    paged_attend_row<T>(p, sq, seq, i, head, q_s[warp]);
  };
  if (sq.len - sq.nq < sq.shared) {                  // a sequence with queries among the shared positions, or without keys
    slowly();
    return;
  }
  // where the row's parts lie: of the shared keys, [0, na), and of its own, [na, na + nb)
  const float *oa = nullptr, *ob = nullptr;
  const float2 *sa = nullptr, *sb = nullptr;
  int na = 0, nb = 0, every = 1;                     // every: shared parts of both places, or of one
  if (sq.shared > 0) {
    const int group = sequence_of(p.group_start, p.n_groups, p.n_seqs, seq);
    const PagedWork w = paged_group_work(p, g, max(group, 0), &bad);
    if (group < 0 || row < w.q0 || row >= w.q0 + w.nq) return;         // offsets that contradict each other
    const int tile = (row - w.q0) / g.tile_q, e = tile / 2, r = (row - w.q0 - tile * g.tile_q) * g.group + head % g.group;
    every = e < w.twos ? 2 : 1;
    const int64_t ordinal = (paged_ordinal_a(g, group, w.q0) + e) * p.kv_heads + kv;
    const int2 f = g.first_a[ordinal];
    const int first = min(max(f.x, 0), blocks - 1);
    const int64_t place = 2 * (ordinal + first) + (every == 2 ? tile & 1 : 0);
    na = min(max(f.y, 0), blocks - first) * (2 / every);
    oa = g.out_a + (place * g.rows_a + r) * p.dim;
    sa = g.sum_a + place * g.rows_a + r;
  }
  {
    const int tile = i / g.tile_q, r = (i - tile * g.tile_q) * g.group + head % g.group;
    const int64_t ordinal = (paged_ordinal_b(g, seq, sq.q0) + tile) * p.kv_heads + kv;
    const int2 f = g.first_b[ordinal];
    const int first = min(max(f.x, 0), blocks - 1);
    const int64_t place = 2 * (ordinal + first);
    nb = min(max(f.y, 0), blocks - first) * 2;
    ob = g.out_b + (place * g.rows_b + r) * p.dim;
    sb = g.sum_b + place * g.rows_b + r;
  }
  const int64_t step_a = (int64_t)every * g.rows_a, step_b = g.rows_b;
  auto sums = [&](int k) { return k < na ? sa[k * step_a] : sb[(k - na) * step_b]; };
  float top = -INFINITY;
  for (int k = lane; k < na + nb; k += 32) top = fmaxf(top, sums(k).x);
#pragma unroll
  for (int d = 16; d > 0; d /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  const float ref = top == -INFINITY ? 0.f : top;
  float l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  const bool mine = 4 * lane < p.dim;
  for (int k0 = 0; k0 < na + nb; k0 += 32) {
    float z = 0.f;
    if (k0 + lane < na + nb) {
      const float2 s = sums(k0 + lane);
      z = s.x == -INFINITY ? 0.f : exp2f(s.x - ref);
      l = fmaf(s.y, z, l);
    }
    const int n = min(32, na + nb - k0);
    for (int k = 0; k < n; k += 4) {
      float4 x[4];
      float f[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int part = k0 + k + e;
        f[e] = __shfl_sync(0xffffffffu, z, (k + e) & 31);
        x[e] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (k + e < n && mine && f[e] != 0.f)
          x[e] = __ldcs(reinterpret_cast<const float4*>(part < na ? oa + part * step_a * p.dim : ob + (part - na) * step_b * p.dim) + lane);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (k + e < n) {
          o.x = fmaf(x[e].x, f[e], o.x); o.y = fmaf(x[e].y, f[e], o.y);
          o.z = fmaf(x[e].z, f[e], o.z); o.w = fmaf(x[e].w, f[e], o.w);
        }
    }
  }
#pragma unroll
  for (int d = 16; d > 0; d /= 2) l += __shfl_xor_sync(0xffffffffu, l, d);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  o = l == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  // A weight of zero times a value that is not finite is NaN.  New rows are seen by some of a sequence's queries only, so a
  // row that is not finite is done again, key by visible key.
  const bool odd = mine && !(fabsf(o.x) + fabsf(o.y) + fabsf(o.z) + fabsf(o.w) < INFINITY);
  if (sq.nq > 1 && __any_sync(0xffffffffu, odd)) {
    slowly();
    return;
  }
  if (mine)
    *reinterpret_cast<uint2*>(p.out.data + (int64_t)row * p.out.row_bytes + (int64_t)head * p.out.head_bytes + 8 * lane) =
        make_uint2(pack2<T>(o.x, o.y), pack2<T>(o.z, o.w));
}

}  // namespace gnn
