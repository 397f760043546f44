// The tiled attention kernel: 128 queries to a tile, two tiles to a block, tcgen05 for both products.
//
// S = Q K^T and O = P V block of keys by block of keys, P = exp2(scale (S - m)) with a running maximum m for each row:
// where m grows by more than 2^8 / scale, O and the sum so far are multiplied by what that takes; else the weights
// stay on the old m, above 1 if need be.  Only blocks that some row of the tile sees are loaded; of those, parts that
// no row of a warp sees cost no exponentials.
//
// What bounds it (event of 300,000 hits, two bf16 heads of 64, 512 neighbours to each side: 0.200 ms, 800 TFLOP/s of
// visible products, tensor cores 36 % busy; causal 16,384, heads of 128, window 4,096: 0.186 ms, 1,330 TFLOP/s, 62 %):
// a block's softmax is one chain of 1,200 cycles in a warp with 512 of them exponentials, two warps share a scheduler,
// and tensor memory holds no third tile beside two.  Other splits lost: 16 rows to a warp in sixteen warps 0.36 ms,
// two threads to a row 0.25, three tiles of 96 keys 0.26, one warp that issues whatever is ready 0.36 (its polls take
// issue slots).
#pragma once
#include <cuda.h>
#include <climits>
#include "attend.cuh"
#include "attend_ptx.cuh"

namespace gnn {

constexpr int kTileQ = 128;                        // queries of a tile
constexpr int kMostTiles = 2;                      // tiles of a block
constexpr int kKeys = 128;                         // keys of a block of keys
constexpr int kStageBytes = 32 * 64;               // 32 rows of 32 columns of output, of a softmax warp
constexpr int kItemSlots = 4;                      // items that the copy warp is ahead by, at most

// A softmax warpgroup to a tile, and one for control: warps that issue the products and one that finds the work and
// issues the copies.  All are launched with 168 registers a thread, of which the last hands over what it does not
// need: 2 * 216 + 72 = 3 * 168.
constexpr int kAttendThreads = 384, kSoftmaxRegs = 216, kControlRegs = 72;
constexpr int kSoftmaxWarps = 8, kMmaWarp = 8, kCopyWarp = 10;

// DP: head_dim rounded up to 64 or 128.  Tensor memory has 512 columns for two tiles: the scores S in fp32 take 128
// each, the outputs O DP.  With DP = 64 the weights P have 64 columns of their own, so that the next scores are
// computed while the softmax runs; with DP = 128 they lie over the scores that they come from, and a tile's P V and
// next Q K^T are one chain.
template <int DP>
struct AttendShape {
  static constexpr bool kApart = DP == 64;
  // Apart, a tile's products wait for nothing of the other tile's: a warp to each.  Two chains in turn keep the tensor
  // cores busy, while two side by side end together, and both tiles wait.
  static constexpr int kMmaWarps = kApart ? 2 : 1;
  static constexpr int kQBufs = DP == 64 ? 2 : 1;
  static constexpr int kStages = DP == 64 ? 8 : 4; // of a block of keys or of values each
  static constexpr int kQBytes = kTileQ * DP * 2, kKvBytes = kKeys * DP * 2;
  static constexpr int kP = kApart ? 256 : 0, kPStep = kApart ? 64 : 128, kO = kApart ? 384 : 256;
  static constexpr int kSmem = kQBufs * kMostTiles * kQBytes + kStages * kKvBytes;
};

// ------------------------------------------------------------------ work
// The rows of the sequence that a tile has, and the blocks of keys it goes through: [0, sinks) and [lo, hi).  A
// block is seen whole by every row when it is below whole_hi and either from whole_lo on or below whole_sinks.
// Row r of the tile sees the keys j <= top + r and (j >= low + r or j < sinks of the call).
struct AttendTile { int row, n, head, sinks, lo, hi, whole_sinks, whole_lo, whole_hi, top, low; };
struct AttendItem {
  Sequence sq;
  AttendTile t[kMostTiles];
  int kv_head, sinks, lo, n;         // the item's blocks: [0, sinks), then n - sinks from lo on
  __device__ __forceinline__ int block(int i) const { return i < sinks ? i : lo + (i - sinks); }
};
// An item is up to `tiles` tiles of a sequence that read the same key head: its query heads side by side, 128 rows
// after 128 rows.
struct AttendGrid {
  int tiles, group;                  // group: query heads to a key head
  int64_t items;
};

__device__ __forceinline__ bool tile_sees(const AttendTile& t, int kb) {
  return kb < t.sinks || (kb >= t.lo && kb < t.hi);
}

__device__ __forceinline__ AttendTile attend_tile(const AttendParams& p, const Sequence& sq, int row, int head) {
  AttendTile t = {row, min(max(sq.nq - row, 0), kTileQ), head, 0, 0, 0, 0, 0, 0, 0, 0};
  if (t.n == 0) return t;
  const int pos = sq.len - sq.nq + row;
  const Seen a = seen_keys(pos, sq.len, p.left, p.right, p.sinks);
  const Seen z = seen_keys(pos + t.n - 1, sq.len, p.left, p.right, p.sinks);
  if (z.hi <= 0) return t;
  t.hi = (z.hi + kKeys - 1) / kKeys;
  t.lo = min(a.lo, z.hi) / kKeys;
  t.sinks = min((z.first + kKeys - 1) / kKeys, t.lo);
  t.whole_hi = a.hi / kKeys;
  t.whole_lo = (z.lo + kKeys - 1) / kKeys;
  t.whole_sinks = p.sinks / kKeys;
  // some row sees a key, so a negative pos + right is above -kTileQ
  t.top = p.right < 0 ? INT_MAX - kTileQ : (int)min((int64_t)INT_MAX - kTileQ, (int64_t)pos + p.right);
  t.low = p.left < 0 ? -kTileQ : (int)max((int64_t)-kTileQ, (int64_t)pos - p.left);
  return t;
}

// Item `at`: false when it has no rows.  Sequence b's items start at slot group (q0 / 128 + b) / tiles + b, which leaves
// room for all of them and needs no sum over the sequences before it.  (Slots and tiles are below 2^31; the divisions
// are in 32 bits, as 64 bits take thousands of cycles here.)
static __device__ __noinline__ bool attend_item(const AttendParams& p, const AttendGrid& g, int64_t at, AttendItem& it) {
  const uint32_t heads = (uint32_t)p.kv_heads, group = (uint32_t)g.group, tiles = (uint32_t)g.tiles;
  const uint32_t slot = at >> 32 ? (uint32_t)(at / heads) : (uint32_t)at / heads;
  it.kv_head = (int)(at - (int64_t)slot * heads);
  auto start = [&](int b, int q0) { return group * (uint32_t)(q0 / kTileQ + b) / tiles + (uint32_t)b; };
  int a = 0, z = p.n_seqs;
#pragma unroll 1
  while (z - a > 1) {
    const int mid = (int)(((int64_t)a + z) / 2);
    if (start(mid, min(max(p.q_start[mid], 0), p.n_q_rows)) <= slot) a = mid; else z = mid;
  }
  bool bad;
  it.sq = sequence(p, a, &bad);
  const uint32_t from = start(a, it.sq.q0), all = group * (uint32_t)((it.sq.nq + kTileQ - 1) / kTileQ);
  if (slot < from || (slot - from) * tiles >= all) return false;
  const uint32_t first = (slot - from) * tiles;
  int lo = INT_MAX, hi = 0;
  it.sinks = 0;
#pragma unroll 1
  for (uint32_t t = 0; t < kMostTiles; ++t) {
    const uint32_t e = first + t, row = e / group;
    const bool have = t < tiles && e < all;
    it.t[t] = attend_tile(p, it.sq, have ? (int)row * kTileQ : it.sq.nq, it.kv_head * g.group + (int)(e - row * group));
    if (it.t[t].hi > 0) {
      lo = min(lo, it.t[t].lo);
      hi = max(hi, it.t[t].hi);
      it.sinks = max(it.sinks, it.t[t].sinks);
    }
  }
  if (hi == 0) lo = 0;
  it.sinks = min(it.sinks, lo);
  it.lo = lo;
  it.n = it.sinks + (hi - lo);
  return true;
}

// ------------------------------------------------------------------ kernel
struct AttendBars {
  uint64_t q_full[2], q_empty[2], kv_full[8], kv_empty[8], drain[kMostTiles];
  uint64_t s_full[kMostTiles], s_free[kMostTiles], p_half[kMostTiles], p_full[kMostTiles], pv_done[kMostTiles];
  uint64_t item_full[kItemSlots], item_empty[kItemSlots];
  AttendItem item[kItemSlots];
  uint32_t tmem;
  int abort;
};
template <int DP>
constexpr int attend_smem_bytes() {
  return AttendShape<DP>::kSmem + kSoftmaxWarps * kStageBytes + (int)sizeof(AttendBars) + 1024;
}

template <typename T, int DP>
__global__ void __launch_bounds__(kAttendThreads, 1)
    attend_tile_kernel(const __grid_constant__ AttendParams p, const __grid_constant__ AttendGrid g,
                       const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                       const __grid_constant__ CUtensorMap map_v) {
  using S = AttendShape<DP>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint8_t* q_buf = smem;
  uint8_t* kv_buf = smem + S::kQBufs * kMostTiles * S::kQBytes;
  uint8_t* stage = smem + S::kSmem;                // 32 rows of 32 columns of output to a softmax warp
  AttendBars& b = *reinterpret_cast<AttendBars*>(stage + kSoftmaxWarps * kStageBytes);
  const int warp = uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
  volatile int* abort = &b.abort;

  if (warp == kCopyWarp && lane == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&b.q_full[i], 1);
      mbar_init(&b.q_empty[i], S::kMmaWarps);
    }
    for (int i = 0; i < kMostTiles; ++i) {
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
    for (int i = 0; i < kMostTiles; ++i) mbar_init(&b.drain[i], 1);
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
      // ---------------- the work, item by item; its queries, and its keys and values through the ring
      const uint32_t q_bytes = (uint32_t)halves * kTileQ * 128, kv_bytes = (uint32_t)halves * kKeys * 128;
      uint32_t kv = 0, q = 0, items = 0;
      bool ok = true;
      for (int64_t at = blockIdx.x; ok; at += gridDim.x) {
        AttendItem it;
        const bool end = at >= g.items;
        if (end) it.n = -1;
        else if (!attend_item(p, g, at, it)) continue;
        const uint32_t slot = items % kItemSlots;
        if (items >= kItemSlots) ok = wait(&b.item_empty[slot], items / kItemSlots - 1);
        if (!ok) break;
        if (lane == 0) {
          b.item[slot] = it;
          mbar_arrive(&b.item_full[slot]);
        }
        ++items;
        if (end) break;
        if (it.n == 0) continue;
        const uint32_t qb = q % S::kQBufs;
        if (q >= S::kQBufs) ok = wait(&b.q_empty[qb], q / S::kQBufs - 1);
        if (!ok) break;
        if (lane == 0) {
          uint32_t some = 0;
#pragma unroll
          for (int t = 0; t < kMostTiles; ++t) some += it.t[t].hi > 0 ? 1 : 0;
          mbar_arrive_expect_tx(&b.q_full[qb], q_bytes * some);
#pragma unroll
          for (int t = 0; t < kMostTiles; ++t)
            if (it.t[t].hi > 0)
#pragma unroll 1
              for (int h = 0; h < halves; ++h)
                tma_load_3d(q_buf + (qb * kMostTiles + t) * S::kQBytes + h * kTileQ * 128, &map_q, 64 * h, it.t[t].head,
                            it.sq.q0 + it.t[t].row, &b.q_full[qb]);
        }
        ++q;
#pragma unroll 1
        for (int i = 0; i < it.n && ok; ++i) {
          const int row = it.sq.k0 + it.block(i) * kKeys;
#pragma unroll 1
          for (int kind = 0; kind < 2; ++kind, ++kv) {
            const uint32_t st = kv % S::kStages;
            if (kv >= S::kStages) ok = wait(&b.kv_empty[st], kv / S::kStages - 1);
            if (!ok) break;
            if (lane == 0) {
              mbar_arrive_expect_tx(&b.kv_full[st], kv_bytes);
              for (int h = 0; h < halves; ++h)
                tma_load_3d(kv_buf + st * S::kKvBytes + h * kKeys * 128, kind ? &map_v : &map_k, 64 * h, it.kv_head,
                            row, &b.kv_full[st]);
            }
          }
        }
        __syncwarp();
      }
      // every copy lands before the block leaves
#pragma unroll 1
      for (uint32_t i = 0; i < S::kStages; ++i)
        if (kv > i) drain_wait(&b.kv_full[i], (kv - 1 - i) / S::kStages & 1);
#pragma unroll 1
      for (uint32_t i = 0; i < S::kQBufs; ++i)
        if (q > i) drain_wait(&b.q_full[i], (q - 1 - i) / S::kQBufs & 1);
      // offsets that point outside the views, and more queries than were announced
#pragma unroll 1
      for (int64_t s = (int64_t)blockIdx.x * 32 + lane; s < p.n_seqs; s += (int64_t)gridDim.x * 32) {
        bool bad;
        const Sequence sq = sequence(p, (int)s, &bad);
        if (bad || sq.nq > p.max_q) atomicOr(p.err, DEV_ERR_INDEX_RANGE);
      }
    } else if (warp < kMmaWarp + S::kMmaWarps) {
      // ---------------- the products of tiles mine .. mine + NT - 1
      constexpr int NT = kMostTiles / S::kMmaWarps;
      const int mine = NT == 1 ? warp - kMmaWarp : 0;
      const int steps = (p.dim + 15) / 16;
      constexpr uint32_t id_qk = idesc_attend<T>(kTileQ, kKeys, false);
      const uint32_t id_pv = idesc_attend<T>(kTileQ, (uint32_t)steps * 16, true);
      // Descriptors and addresses are computed by the whole warp, outside the elected thread's branch, so that they
      // stay in uniform registers: inside it an MMA takes several times as long to issue.
      const uint32_t q_base = (uint32_t)uniform((int)smem_u32(q_buf)), kv_base = (uint32_t)uniform((int)smem_u32(kv_buf));
      const uint64_t q_desc = sdesc_kmajor_sw128(q_base), k_desc = sdesc_kmajor_sw128(kv_base),
                     v_desc = sdesc_nmajor_sw128(kv_base, kKeys * 128);
      uint32_t kv = 0, q = 0, items = 0, qk_n[NT] = {}, pv_n[NT] = {};
      bool ok = true;
      while (ok) {
        const uint32_t slot = items % kItemSlots;
        ok = wait(&b.item_full[slot], items / kItemSlots);
        if (!ok) break;
        AttendTile tile[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const AttendTile& from = b.item[slot].t[mine + t];
          tile[t].sinks = uniform(from.sinks);
          tile[t].lo = uniform(from.lo);
          tile[t].hi = uniform(from.hi);
        }
        const int n = uniform(b.item[slot].n), sinks = uniform(b.item[slot].sinks), lo = uniform(b.item[slot].lo),
                  len = uniform(b.item[slot].sq.len);
        __syncwarp();
        if (lane == 0) mbar_arrive(&b.item_empty[slot]);
        ++items;
        if (n < 0) break;
        if (n == 0) continue;
        const uint32_t qb = q % S::kQBufs;
        bool fresh[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) fresh[t] = true;
        auto qk = [&](int t, uint32_t st) {          // S = Q K^T, once the last scores have been read
          if (S::kApart && qk_n[t] > 0) ok = wait(&b.s_free[mine + t], qk_n[t] - 1);
          if (!ok) return;
          tc_fence_after();
          const uint64_t qa = q_desc + ((qb * kMostTiles + mine + t) * S::kQBytes >> 4),
                         ka = k_desc + (st * S::kKvBytes >> 4);
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
        ok = wait(&b.q_full[qb], q / S::kQBufs);
        for (int i = -1; i < n && ok; ++i) {
          const bool more = i + 1 < n;
          const int kb = i < sinks ? i : lo + (i - sinks), next = i + 1 < sinks ? i + 1 : lo + (i + 1 - sinks);
          const uint32_t kn = kv + 2 * (i + 1), vn = kv + 2 * i + 1;
          const uint32_t ks = kn % S::kStages, vs = vn % S::kStages;
          if (more) ok = wait(&b.kv_full[ks], kn / S::kStages);
          if (!ok) break;
          if (S::kApart && more && tile_sees(tile[0], next)) qk(0, ks);
          if (!ok) break;
          if (i >= 0) {
            ok = wait(&b.kv_full[vs], vn / S::kStages);
            if (!ok) break;
            // Values of rows behind the sequence's last key: zeros, so that weights of zero leave no trace of them.
            // (Where several warps do this, each does before its own products.)
            const int have = len - kb * kKeys;
            if (have < kKeys) {
#pragma unroll 1
              for (int r = have * 8 + lane; r < kKeys * 8; r += 32)
                for (int h = 0; h < halves; ++h)
                  *reinterpret_cast<uint4*>(kv_buf + vs * S::kKvBytes + h * kKeys * 128 + r * 16) = make_uint4(0, 0, 0, 0);
              fence_async_shared();
              __syncwarp();
            }
          }
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            if (i >= 0 && tile_sees(tile[t], kb)) {  // O += P V, the first 64 keys and the others
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
            if (!S::kApart && more && tile_sees(tile[t], next)) qk(t, ks);
          }
          if (!ok) break;
          if (elect_one()) {
            if (more) mma_commit(&b.kv_empty[ks]);
            if (i >= 0) mma_commit(&b.kv_empty[vs]);
            if (i + 2 == n) mma_commit(&b.q_empty[qb]);      // the item's last Q K^T is out
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
    // ---------------- softmax and output: a warpgroup to a tile, a row to a thread
    const int wg = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    constexpr int PARTS = kKeys / 32;
    const uint32_t ts = tmem + lanes + kKeys * wg, tp = tmem + lanes + S::kP + S::kPStep * wg,
                   to = tmem + lanes + S::kO + DP * wg;
    const float scale = fabsf(p.scale_log2);
    const float slack = 8.f / scale;                 // scores may outgrow the running maximum by 2^8
    uint32_t n = 0, items = 0;                       // blocks this tile has gone through
    bool ok = true, dirty = false;
    while (ok) {
      const uint32_t slot = items % kItemSlots;
      ok = wait(&b.item_full[slot], items / kItemSlots);
      if (!ok) break;
      const AttendItem& item = b.item[slot];
      const int rows = item.t[wg].n, len = item.sq.len, item_n = item.n;
      const int sinks = item.t[wg].sinks, lo = item.t[wg].lo, blocks = sinks + (item.t[wg].hi - lo);
      const int whole_sinks = item.t[wg].whole_sinks, whole_lo = item.t[wg].whole_lo, whole_hi = item.t[wg].whole_hi;
      // the row's keys, and the warp's: of its first row, and of its last that the tile has
      const int tile_top = item.t[wg].top, tile_low = item.t[wg].low, w0 = (warp & 3) * 32, w1 = min(rows, w0 + 32) - 1;
      const int top = min(len - 1, tile_top + row), low = max(0, tile_low + row);
      char* out = p.out.data + (int64_t)(item.sq.q0 + item.t[wg].row + w0) * p.out.row_bytes +   // the warp's first row's
                  (int64_t)item.t[wg].head * p.out.head_bytes;
      __syncwarp();
      if (lane == 0) mbar_arrive(&b.item_empty[slot]);
      ++items;
      if (item_n < 0) break;
      if (rows == 0) continue;
      float m = row < rows ? -INFINITY : INFINITY, l = 0.f;        // rows that the tile does not have weigh nothing
      const float2 scale2 = make_float2(scale, scale);
      bool plain = false;                            // every row has a maximum that the next block may be weighed by
      auto read = [&](float* s) {                    // the block's scores
        tc_fence_after();
#pragma unroll
        for (int c = 0; c < PARTS; ++c) tmem_ld_32x32(ts + 32 * c, s + 32 * c);
#pragma unroll
        for (int c = 0; c < PARTS; ++c) tmem_wait_ld_32(s + 32 * c);
      };
      auto scores_read = [&] {
        if (!S::kApart) return;
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&b.s_free[wg]);
      };
      auto stored = [&](uint64_t* bar) {             // the weights so far are in place
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar);
      };
      // 32 scores to weights, and their sum
      auto weigh = [&](const float* s, float2 off2, float2* sum, uint32_t* w) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float2 x = __ffma2_rn(make_float2(s[2 * e], s[2 * e + 1]), scale2, off2);
          x.x = exp2_approx(x.x);
          x.y = exp2_approx(x.y);
          sum[e & 1] = __fadd2_rn(sum[e & 1], x);
          w[e] = pack2<T>(x.x, x.y);
        }
      };
      // Part c (32 keys) of block kb: true when no row of the warp sees any of it; else what a row does not see becomes -inf.
      const int sink = min(p.sinks, len);
      auto hide = [&](int kb, int c, float* s) {
        const int j = kb * kKeys + 32 * c;
        const int first_top = min(len - 1, tile_top + w0), last_top = min(len - 1, tile_top + w1);
        if (w1 < w0 || j > last_top || (j + 31 < tile_low + w0 && j >= sink)) return true;
        if (j + 31 > first_top || (j < tile_low + w1 && j + 32 > sink)) {
          auto below = [](int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; };
          const uint32_t see = below(top + 1 - j) & (~below(low - j) | below(sink - j));
#pragma unroll
          for (int e = 0; e < 32; ++e) s[e] = see >> e & 1u ? s[e] : -INFINITY;
        }
        return false;
      };
      // Blocks on the guess that their scores do not outgrow the running maximum (which they rarely do after the first).
      // In bf16 nothing depends on the guess: weights above 1 lose no precision, and their sum tells whether the next
      // block has to look for the maximum, and how far that was left behind.  Scores that outgrow it by 2^128 in one block
      // overflow the weights, their sum or the outputs: such a row is left not finite and done again.  In fp16, whose
      // weights end at 2^16, the maximum is computed beside the weights of a block that every row sees whole: false,
      // with nothing changed, when the guess was wrong.
      constexpr bool LOOSE = std::is_same<T, __nv_bfloat16>::value;
      auto loose = [&](int kb, auto edge) {
        constexpr bool EDGE = decltype(edge)::value;   // a block that not every row sees whole
        const float off = -m * scale;
        const float2 off2 = make_float2(off, off);
        float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
        if constexpr (!EDGE && S::kApart) {
          // All scores first, so that the next product over them runs beside the weights (213 -> 205 us).
          float s[kKeys];
          read(s);
          scores_read();
          uint32_t w[2][16];
#pragma unroll
          for (int c = 0; c < PARTS; ++c) {
            weigh(s + 32 * c, off2, sum, w[c & 1]);
            if (c == 0) {
              ok = wait(&b.pv_done[wg], n - 1);
              if (!ok) return true;
              tc_fence_after();
            }
            if (c == 2) stored(&b.p_half[wg]);
            tmem_st_32x16(tp + 16 * c, w[c & 1]);
          }
          stored(&b.p_full[wg]);
        } else {
          tc_fence_after();
          // 64 keys at a time, or 32 where the first weights' product waits for them, in a loop: with the code of all 128
          // in one piece for these blocks too, the kernel misses the instruction caches.
          constexpr int STEP = S::kApart ? 2 : 1;
#pragma unroll 1
          for (int c0 = 0; c0 < PARTS; c0 += STEP) {
            float s[32 * STEP];
#pragma unroll
            for (int c = 0; c < STEP; ++c) tmem_ld_32x32(ts + 32 * (c0 + c), s + 32 * c);
#pragma unroll
            for (int c = 0; c < STEP; ++c) tmem_wait_ld_32(s + 32 * c);
            if (c0 + STEP == PARTS) scores_read();
#pragma unroll
            for (int c = 0; c < STEP; ++c) {
              uint32_t w[16];
              if (EDGE && hide(kb, c0 + c, s + 32 * c)) {
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e] = 0u;
              } else {
                weigh(s + 32 * c, off2, sum, w);
              }
              if (c == 0 && c0 == 0) {
                // the last product with these weights' columns, and into these outputs, is over
                ok = wait(&b.pv_done[wg], n - 1);
                if (!ok) return true;
                tc_fence_after();
              }
              if (!S::kApart && c0 == 2) stored(&b.p_half[wg]);
              tmem_st_32x16(tp + 16 * (c0 + c), w);
            }
            if (S::kApart) stored(c0 ? &b.p_full[wg] : &b.p_half[wg]);
          }
          if (!S::kApart) stored(&b.p_full[wg]);
        }
        const float all = (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
        l += all;
        plain = warp_all(all <= 256.f || row >= rows);
        return true;
      };
      auto guess = [&]() {
        float s[kKeys];
        read(s);
        const float off = -m * scale;
        const float2 off2 = make_float2(off, off);
        float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
        uint32_t w[2][16];
        weigh(s, off2, sum, w[0]);
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int c = 0; c < kKeys; c += 8)
#pragma unroll
          for (int x = 0; x < 4; ++x) mx[x] = max3(mx[x], s[c + x], s[c + 4 + x]);
        const float high = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]);
        weigh(s + 32, off2, sum, w[1]);
        if (!warp_all(high <= m + slack)) return false;
        scores_read();
        ok = wait(&b.pv_done[wg], n - 1);
        if (!ok) return true;
        tc_fence_after();
        tmem_st_32x16(tp, w[0]);
        tmem_st_32x16(tp + 16, w[1]);
#pragma unroll
        for (int c = 2; c < PARTS; ++c) {
          weigh(s + 32 * c, off2, sum, w[c & 1]);
          if (c == 2) stored(&b.p_half[wg]);
          tmem_st_32x16(tp + 16 * c, w[c & 1]);
        }
        l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
        stored(&b.p_full[wg]);
        return true;
      };
      // Any block.
      auto block = [&](int kb, bool start) {
        if (p.scale_log2 < 0.f) {                    // rare, and so in little code
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < kKeys; c += 8) tmem_scale_32x8(ts + c, -1.f);
          tmem_st_wait();
        }
        float s[kKeys];
        read(s);
        scores_read();
        uint32_t hidden = 0;                         // parts of the block that no row of the warp sees
#pragma unroll
        for (int c = 0; c < PARTS; ++c)
          if (hide(kb, c, s + 32 * c)) hidden |= 1u << c;
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int c = 0; c < PARTS; ++c)
          if (!(hidden >> c & 1u)) {
#pragma unroll
            for (int e = 0; e < 32; e += 8)
#pragma unroll
              for (int x = 0; x < 4; ++x) mx[x] = max3(mx[x], s[32 * c + e + x], s[32 * c + e + 4 + x]);
          }
        const float high = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]);
        const bool grow = high > m + slack || (m == -INFINITY && high > m);
        // the last product with these weights' columns, and into these outputs, is over
        if (!start && !wait(&b.pv_done[wg], n - 1)) return false;
        tc_fence_after();
        if (__any_sync(0xffffffffu, grow)) {
          const float mn = grow ? high : m;
          const float shrink = !grow ? 1.f : m == -INFINITY ? 0.f : exp2_approx((m - mn) * scale);
          m = mn;
          l *= shrink;
          if (!start) {
#pragma unroll 1
            for (int c = 0; c < DP; c += 8) tmem_scale_32x8(to + c, shrink);
          }
        }
        const float off = m == -INFINITY ? 0.f : -m * scale;
        float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
        for (int c = 0; c < PARTS; ++c) {
          uint32_t w[16];
          if (hidden >> c & 1u) {
#pragma unroll
            for (int e = 0; e < 16; ++e) w[e] = 0u;
          } else {
            weigh(s + 32 * c, make_float2(off, off), sum, w);
          }
          if (c == 2) stored(&b.p_half[wg]);
          tmem_st_32x16(tp + 16 * c, w);
        }
        l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
        stored(&b.p_full[wg]);
        plain = warp_all(m > -INFINITY);
        return true;
      };
      // After weights on a maximum left far behind: it catches up by the powers of two in their sum, which comes down by as
      // many, and the outputs with it.  Otherwise the step from the old maximum to a new one could be past 2^-126,
      // which is zero, and drop sums that count.
      auto catch_up = [&] {
        if (!wait(&b.pv_done[wg], n - 1)) return false;
        tc_fence_after();
        const bool late = l > 65536.f;
        const float mn = late ? m + (float)min((__float_as_int(l) >> 23) - 127, 120) / scale : m;
        const float shrink = late ? exp2_approx((m - mn) * scale) : 1.f;
        m = mn;
        l *= shrink;
#pragma unroll 1
        for (int c = 0; c < DP; c += 8) tmem_scale_32x8(to + c, shrink);
        tmem_st_wait();
        return true;
      };
      for (int i = 0; i < blocks; ++i, ++n) {
        const int kb = i < sinks ? i : lo + (i - sinks);
        ok = wait(&b.s_full[wg], n);
        if (!ok) break;
        if (plain && p.scale_log2 >= 0.f) {
          const bool whole = kb < whole_hi && (kb >= whole_lo || kb < whole_sinks);
          if (LOOSE ? (whole ? loose(kb, std::false_type()) : loose(kb, std::true_type())) : whole && guess()) {
            if (!ok) break;
            continue;
          }
        }
        if (LOOSE && __any_sync(0xffffffffu, l > 65536.f)) {
          ok = catch_up();
          if (!ok) break;
        }
        ok = block(kb, i == 0);
        if (!ok) break;
      }
      if (!ok) break;
      // output
      if (blocks > 0) {
        ok = wait(&b.pv_done[wg], n - 1);
        if (!ok) break;
        tc_fence_after();
      }
      const bool none = blocks == 0 || l == 0.f;
      const float r = none ? 0.f : LOOSE && !(l < INFINITY) ? NAN : 1.f / l;   // a sum that overflowed: done again
      float2 odd = make_float2(0.f, 0.f);            // not finite once a value is not
      uint8_t* mine = stage + warp * kStageBytes;
#pragma unroll S::kApart ? 2 : 1                      // 204 -> 201 us; four in one piece cost as much as they save
      for (int c = 0; c < DP; c += 32) {
        // A thread has a row, and rows lie apart: written from here, every store would touch 32 lines.  Through shared
        // memory, 16 bytes at a place that the row turns by its number, four threads write 64 bytes of a row.
        float o[32];
        if (blocks > 0) {
          tmem_ld_32x32(to + c, o);
          tmem_wait_ld_32(o);
        }
        __syncwarp();
#pragma unroll
        for (int e = 0; e < 32; e += 8) {
          uint32_t u[4];
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const float2 y = none ? make_float2(0.f, 0.f) : make_float2(o[e + 2 * x] * r, o[e + 2 * x + 1] * r);
            odd = __fadd2_rn(odd, y);
            u[x] = pack2<T>(y.x, y.y);
          }
          *reinterpret_cast<uint4*>(mine + lane * 64 + (e / 8 ^ lane / 2 % 4) * 16) = make_uint4(u[0], u[1], u[2], u[3]);
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int at = 8 * i + lane / 4;
          if (w0 + at < rows && c + lane % 4 * 8 < p.dim)
            *reinterpret_cast<uint4*>(out + at * p.out.row_bytes + (c + lane % 4 * 8) * 2) =
                *reinterpret_cast<const uint4*>(mine + at * 64 + (lane % 4 ^ at / 2 % 4) * 16);
        }
      }
      tc_fence_before();
      dirty = dirty || (row < rows && !(fabsf(odd.x + odd.y) < INFINITY));
    }
    // A weight of zero times a value that is not finite is NaN: rows that hold one are done again, key by visible
    // key, also where the result cannot be finite.  After everything else, so that nothing waits for it.  (Event of 300,000
    // hits: one NaN that 1,025 rows see takes it from 0.2 to 6.7 ms, one in a first token, which all rows see, to 100 ms.)
    if (ok && __any_sync(0xffffffffu, dirty)) {
      float* qs = reinterpret_cast<float*>(stage + warp * kStageBytes);
      __syncwarp();
      for (int64_t at = blockIdx.x; at < g.items; at += gridDim.x) {
        AttendItem it;
        if (!attend_item(p, g, at, it)) continue;
        const AttendTile t = it.t[wg];
        bool again = false;
        if (row < t.n) {
          const T* out = reinterpret_cast<const T*>(p.out.data + (int64_t)(it.sq.q0 + t.row + row) * p.out.row_bytes +
                                                    (int64_t)t.head * p.out.head_bytes);
#pragma unroll 1
          for (int d = 0; d < p.dim; ++d) again = again || !(fabsf(to_f(out[d])) < INFINITY);
        }
        for (uint32_t rows = __ballot_sync(0xffffffffu, again); rows; rows &= rows - 1) {
          const int i = t.row + (warp & 3) * 32 + __ffs(rows) - 1;
          const T* q = reinterpret_cast<const T*>(p.q.data + (int64_t)(it.sq.q0 + i) * p.q.row_bytes +
                                                  (int64_t)t.head * p.q.head_bytes);
          __syncwarp();
#pragma unroll 1
          for (int d = lane; d < p.dim; d += 32) qs[d] = to_f(q[d]);
          __syncwarp();
          attend_row<T>(p, it.sq, i, t.head, qs);
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kMmaWarp) tmem_dealloc(tmem, 512);
}

}  // namespace gnn
