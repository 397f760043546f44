// The tiled attention kernel: 128 queries to a tile, two tiles to a block, tcgen05 for both products.
#pragma once
#include <cuda.h>
#include <climits>
#include <type_traits>
#include "attend.cuh"

namespace gnn {

constexpr int kTileQ = 128, kTileK = 128;          // queries of a tile, keys of a block of keys
// Two softmax warpgroups, and one whose first warp issues the products and whose second the copies.  All are
// launched with 168 registers a thread; the last one hands over what it does not need: 2 * 200 + 104 = 3 * 168.
constexpr int kAttendThreads = 384, kSoftmaxRegs = 200, kControlRegs = 104;

template <int DP>
struct AttendShape {
  static constexpr bool kApart = DP == 64;         // P has columns of its own; otherwise it lies over S
  static constexpr int kQBufs = DP == 64 ? 2 : 1;
  static constexpr int kStages = DP == 64 ? 8 : 4; // of a block of keys or of values each
  static constexpr int kTileBytes = kTileQ * DP * 2;
  static constexpr int kS = 0, kP = kApart ? 256 : 0, kPStep = kApart ? 64 : 128, kO = kApart ? 384 : 256;
  static constexpr int kSmem = kQBufs * 2 * kTileBytes + kStages * kTileBytes;
};
struct AttendBars {
  uint64_t q_full[2], q_empty[2], kv_full[8], kv_empty[8], s_full[2], s_free[2], p_full[2], pv_done[2], drain;
  uint32_t tmem;
  int abort;
};
template <int DP>
constexpr int attend_smem_bytes() { return AttendShape<DP>::kSmem + 8 * 128 * 4 + (int)sizeof(AttendBars) + 1024; }

// ------------------------------------------------------------------ PTX
__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar)) : "memory");
}
template <int N> __device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// 32 lanes x 32 columns: thread t gets lane t's columns.  Defined only after tmem_wait32 on the same array.
__device__ __forceinline__ void tmem_ld_32x32(uint32_t a, float* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,"
      "%30,%31}, [%32];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
        "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]),
        "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]),
        "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(a));
}
__device__ __forceinline__ void tmem_wait_ld_32(float* v) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]),
                 "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]),
                 "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]),
                 "+f"(v[23]), "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]),
                 "+f"(v[30]), "+f"(v[31])
               :
               : "memory");
}
// 32 lanes x 8 columns, scaled by each lane's factor, in place.
__device__ __forceinline__ void tmem_scale_32x8(uint32_t a, float f) {
  float v[8];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
      : "r"(a)
      : "memory");
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] *= f;
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(a), "f"(v[0]), "f"(v[1]),
               "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
               : "memory");
}
__device__ __forceinline__ void tmem_st_32x32(uint32_t a, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,"
      "%30,%31,%32};" ::"r"(a),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
      "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]),
      "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]),
      "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
      : "memory");
}
__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) { return pack_bf16x2(a, b); }
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Instruction descriptor, kind::f16: A and B of type T, D fp32, A K-major, B K-major or (b_mn) N-major.
template <typename T>
__device__ __forceinline__ uint32_t idesc_attend(uint32_t M, uint32_t N, bool b_mn) {
  const uint32_t f = sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
  return (1u << 4) | (f << 7) | (f << 10) | ((b_mn ? 1u : 0u) << 16) | ((N >> 3) << 17) | ((M >> 4) << 24);
}
// Shared-memory descriptor, N-major rows of 128 bytes (64 elements) with the 128-byte swizzle: 8-row groups along
// K 1024 bytes apart (stride byte offset), the next 64 elements of N `half` bytes further (leading byte offset).
__device__ __forceinline__ uint64_t sdesc_nmajor_sw128(uint32_t saddr, uint32_t half) {
  return (uint64_t)((saddr >> 4) & 0x3FFFu) | (uint64_t)(half >> 4) << 16 | (uint64_t)(1024u >> 4) << 32 |
         (uint64_t)1u << 46 | (uint64_t)2u << 61;
}

// ------------------------------------------------------------------ work
// The rows of the sequence that a tile has, and the blocks of keys it goes through: [0, sinks) and [lo, hi).
struct AttendTile { int row, n, pos, head, sinks, lo, hi; };
struct AttendItem {
  Sequence sq;
  AttendTile t[2];
  int kv_head, sinks, lo, n;         // the item's blocks: [0, sinks), then n - sinks from lo on
  __device__ __forceinline__ int block(int i) const { return i < sinks ? i : lo + (i - sinks); }
};
struct AttendGrid {
  int pair_heads;                    // the two tiles: the same rows of two heads, or 256 rows of one
  int rows;                          // queries of an item: 128 or 256
  int heads;                         // items side by side: heads or pairs of heads
  int64_t items;
};

__device__ __forceinline__ bool tile_sees(const AttendTile& t, int kb) {
  return kb < t.sinks || (kb >= t.lo && kb < t.hi);
}

__device__ __forceinline__ AttendTile attend_tile(const AttendParams& p, const Sequence& sq, int row, int head) {
  AttendTile t = {row, min(max(sq.nq - row, 0), kTileQ), sq.len - sq.nq + row, head, 0, 0, 0};
  if (t.n == 0) return t;
  const Seen a = seen_keys(t.pos, sq.len, p.left, p.right, p.sinks);
  const Seen z = seen_keys(t.pos + t.n - 1, sq.len, p.left, p.right, p.sinks);
  if (z.hi <= 0) return t;
  t.hi = (z.hi + kTileK - 1) / kTileK;
  t.lo = min(a.lo, z.hi) / kTileK;
  t.sinks = min((z.first + kTileK - 1) / kTileK, t.lo);
  return t;
}

// Item `at`: false when it has no rows.  A sequence's items start at slot q0 / rows + b, which leaves room for
// ceil(nq / rows) of them and needs no sum over the sequences before it.
__device__ __forceinline__ bool attend_item(const AttendParams& p, const AttendGrid& g, int64_t at, AttendItem& it) {
  const int slot = (int)(at / g.heads), h = (int)(at - (int64_t)slot * g.heads);
  int a = 0, z = p.n_seqs;
  while (z - a > 1) {
    const int mid = (int)(((int64_t)a + z) / 2);
    if (min(max(p.q_start[mid], 0), p.n_q_rows) / g.rows + mid <= slot) a = mid; else z = mid;
  }
  bool bad;
  it.sq = sequence(p, a, &bad);
  const int64_t row = (int64_t)(slot - (it.sq.q0 / g.rows + a)) * g.rows;
  if (row < 0 || row >= it.sq.nq) return false;
  const int head = g.pair_heads ? 2 * h : h;
  it.kv_head = head / (p.heads / p.kv_heads);
  it.t[0] = attend_tile(p, it.sq, (int)row, head);
  it.t[1] = g.pair_heads ? attend_tile(p, it.sq, (int)row, head + 1) : attend_tile(p, it.sq, (int)row + kTileQ, head);
  int lo = INT_MAX, hi = 0;
  it.sinks = 0;
#pragma unroll
  for (int t = 0; t < 2; ++t)
    if (it.t[t].hi > 0) {
      lo = min(lo, it.t[t].lo);
      hi = max(hi, it.t[t].hi);
      it.sinks = max(it.sinks, it.t[t].sinks);
    }
  if (hi == 0) lo = 0;
  it.sinks = min(it.sinks, lo);
  it.lo = lo;
  it.n = it.sinks + (hi - lo);
  return true;
}

// ------------------------------------------------------------------ kernel
template <typename T, int DP>
__global__ void __launch_bounds__(kAttendThreads, 1)
    attend_tile_kernel(const __grid_constant__ AttendParams p, const __grid_constant__ AttendGrid g,
                       const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                       const __grid_constant__ CUtensorMap map_v) {
  using S = AttendShape<DP>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint8_t* q_buf = smem;
  uint8_t* kv_buf = smem + S::kQBufs * 2 * S::kTileBytes;
  float* q_rows = reinterpret_cast<float*>(smem + S::kSmem);             // a row per softmax warp, for the repair
  AttendBars& b = *reinterpret_cast<AttendBars*>(q_rows + 8 * 128);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abort = &b.abort;

  if (warp == 9 && lane == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&b.q_full[i], 1);
      mbar_init(&b.q_empty[i], 1);
      mbar_init(&b.s_full[i], 1);
      mbar_init(&b.s_free[i], 4);
      mbar_init(&b.p_full[i], 4);
      mbar_init(&b.pv_done[i], 1);
    }
    for (int i = 0; i < 8; ++i) {
      mbar_init(&b.kv_full[i], 1);
      mbar_init(&b.kv_empty[i], 1);
    }
    mbar_init(&b.drain, 1);
    b.abort = 0;
    fence_mbar_init();
  }
  if (warp == 8) {
    tmem_alloc(&b.tmem, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&b.tmem);
  pdl_wait();

  const int halves = p.dim > 64 ? 2 : 1;
  auto wait = [&](uint64_t* bar, int64_t phase) {  // the whole warp, for the completion of the bar's phase
    return warp_all(bounded_wait(bar, (uint32_t)(phase & 1), abort, p.err));
  };
  if (warp >= 8) {
    regs_down<kControlRegs>();
    if (warp == 9) {
      // ---------------- copies: queries, then keys and values block by block, through the ring
      const uint32_t bytes = (uint32_t)halves * kTileQ * 128;
      int64_t kv = 0, q = 0;
      bool ok = true;
      for (int64_t at = blockIdx.x; ok && at < g.items; at += gridDim.x) {
        AttendItem it;
        if (!attend_item(p, g, at, it) || it.n == 0) continue;
        const int qb = (int)(q % S::kQBufs);
        if (q >= S::kQBufs) ok = wait(&b.q_empty[qb], q / S::kQBufs - 1);
        if (!ok) break;
        if (lane == 0) {
          const bool two = it.t[1].hi > 0, one = it.t[0].hi > 0;
          mbar_arrive_expect_tx(&b.q_full[qb], bytes * ((one ? 1 : 0) + (two ? 1 : 0)));
  #pragma unroll
          for (int t = 0; t < 2; ++t)
            if (t ? two : one)
              for (int h = 0; h < halves; ++h)
                tma_load_3d(q_buf + (qb * 2 + t) * S::kTileBytes + h * kTileQ * 128, &map_q, 64 * h, it.t[t].head,
                            it.sq.q0 + it.t[t].row, &b.q_full[qb]);
        }
        ++q;
        for (int i = 0; i < it.n && ok; ++i) {
          const int row = it.sq.k0 + it.block(i) * kTileK;
          for (int kind = 0; kind < 2 && ok; ++kind, ++kv) {
            const int st = (int)(kv % S::kStages);
            if (kv >= S::kStages) ok = wait(&b.kv_empty[st], kv / S::kStages - 1);
            if (!ok) break;
            if (lane == 0) {
              mbar_arrive_expect_tx(&b.kv_full[st], bytes);
              for (int h = 0; h < halves; ++h)
                tma_load_3d(kv_buf + st * S::kTileBytes + h * kTileK * 128, kind ? &map_v : &map_k, 64 * h, it.kv_head, row,
                            &b.kv_full[st]);
            }
          }
        }
        __syncwarp();
      }
      // every copy lands before the block leaves
      for (int i = 0; i < S::kStages; ++i) {
        const int64_t uses = (kv - i + S::kStages - 1) / S::kStages;
        if (kv > i) drain_wait(&b.kv_full[i], (uint32_t)((uses - 1) & 1));
      }
      for (int i = 0; i < S::kQBufs; ++i) {
        const int64_t uses = (q - i + S::kQBufs - 1) / S::kQBufs;
        if (q > i) drain_wait(&b.q_full[i], (uint32_t)((uses - 1) & 1));
      }
      // offsets that point outside the views
      for (int64_t s = (int64_t)blockIdx.x * 32 + lane; s < p.n_seqs; s += (int64_t)gridDim.x * 32) {
        bool bad;
        sequence(p, (int)s, &bad);
        if (bad) atomicOr(p.err, DEV_ERR_INDEX_RANGE);
      }
    } else if (warp == 8) {
      // ---------------- products
      const int steps = (p.dim + 15) / 16;
      const uint32_t id_qk = idesc_attend<T>(kTileQ, kTileK, false);
      const uint32_t id_pv = idesc_attend<T>(kTileQ, (uint32_t)steps * 16, true);
      int64_t kv = 0, q = 0;
      int64_t qk_n[2] = {0, 0}, pv_n[2] = {0, 0};
      bool ok = true;
      for (int64_t at = blockIdx.x; ok && at < g.items; at += gridDim.x) {
        AttendItem it;
        if (!attend_item(p, g, at, it) || it.n == 0) continue;
        const int qb = (int)(q % S::kQBufs);
        bool fresh[2] = {true, true};
        auto qk = [&](int t, int st) {                 // S_t = Q_t K^T, once S_t's last scores have been read
          if (S::kApart && qk_n[t] > 0) ok = ok && wait(&b.s_free[t], qk_n[t] - 1);
          if (!ok) return;
          tc_fence_after();
          if (elect_one()) {
            const uint32_t qa = smem_u32(q_buf + (qb * 2 + t) * S::kTileBytes), ka = smem_u32(kv_buf + st * S::kTileBytes);
            for (int k = 0; k < steps; ++k) {
              const uint32_t off = (k >> 2) * kTileQ * 128 + (k & 3) * 32;
              mma_bf16_ss(tmem + S::kS + 128 * t, sdesc_kmajor_sw128(qa + off), sdesc_kmajor_sw128(ka + off), id_qk, k > 0);
            }
            mma_commit(&b.s_full[t]);
          }
          __syncwarp();
          ++qk_n[t];
        };
        ok = wait(&b.q_full[qb], q / S::kQBufs);
        if (!ok) break;
        for (int i = -1; i < it.n && ok; ++i) {
          // keys of block i + 1
          const bool more = i + 1 < it.n;
          const int kb = i >= 0 ? it.block(i) : 0, next = more ? it.block(i + 1) : 0;
          const int64_t kn = kv + 2 * (i + 1), vn = kv + 2 * i + 1;
          const int ks = (int)(kn % S::kStages), vs = (int)(vn % S::kStages);
          if (more) ok = wait(&b.kv_full[ks], kn / S::kStages);
          if (!ok) break;
          if (S::kApart && more)
  #pragma unroll
            for (int t = 0; t < 2; ++t)
              if (tile_sees(it.t[t], next)) qk(t, ks);
          if (!ok) break;
          if (i >= 0) {
            ok = wait(&b.kv_full[vs], vn / S::kStages);
            if (!ok) break;
            // values of rows behind the sequence's last key: zeros, so that weights of zero leave no trace of them
            const int have = it.sq.len - kb * kTileK;
            if (have < kTileK) {
              for (int r = max(have, 0) * 8 + lane; r < kTileK * 8; r += 32)
                for (int h = 0; h < halves; ++h)
                  *reinterpret_cast<uint4*>(kv_buf + vs * S::kTileBytes + h * kTileK * 128 + r * 16) = make_uint4(0, 0, 0, 0);
              fence_async_shared();
              __syncwarp();
            }
          }
  #pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (!ok) break;
            if (i >= 0 && tile_sees(it.t[t], kb)) {
              ok = wait(&b.p_full[t], pv_n[t]);
              if (!ok) break;
              tc_fence_after();
              if (elect_one()) {
                const uint32_t va = smem_u32(kv_buf + vs * S::kTileBytes);
                for (int k = 0; k < kTileK / 16; ++k)
                  mma_bf16_ts(tmem + S::kO + DP * t, tmem + S::kP + S::kPStep * t + 8 * k,
                              sdesc_nmajor_sw128(va + k * 2048, kTileK * 128), id_pv, !fresh[t] || k > 0);
                mma_commit(&b.pv_done[t]);
              }
              __syncwarp();
              fresh[t] = false;
              ++pv_n[t];
            }
            if (!S::kApart && more && tile_sees(it.t[t], next)) qk(t, ks);
          }
          if (!ok) break;
          if (elect_one()) {
            if (more) mma_commit(&b.kv_empty[ks]);
            if (i >= 0) mma_commit(&b.kv_empty[vs]);
            if (i + 2 == it.n) mma_commit(&b.q_empty[qb]);   // the item's last Q K^T is out
          }
          __syncwarp();
        }
        kv += 2 * (int64_t)it.n;
        ++q;
      }
      if (elect_one()) mma_commit(&b.drain);
      __syncwarp();
      drain_wait(&b.drain, 0);
    }
  } else {
    regs_up<kSoftmaxRegs>();
    // ---------------- softmax and output: a warpgroup to a tile, a row to a thread
    const int wg = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + lanes + S::kS + 128 * wg, tp = tmem + lanes + S::kP + S::kPStep * wg,
                   to = tmem + lanes + S::kO + DP * wg;
    const bool negative = p.scale_log2 < 0.f;
    const float sign = negative ? -1.f : 1.f;
    const float scale = fabsf(p.scale_log2);
    const float slack = 8.f / scale;                 // scores may outgrow the running maximum by 2^8
    int64_t n = 0;                                   // blocks this tile has gone through
    bool ok = true, dirty = false;
    for (int64_t at = blockIdx.x; ok && at < g.items; at += gridDim.x) {
      AttendItem it;
      if (!attend_item(p, g, at, it)) continue;
      const AttendTile t = wg ? it.t[1] : it.t[0];
      if (t.n == 0) continue;
      const int pos = t.pos + row;
      float m = -INFINITY, l = 0.f;
      bool first = true;
      for (int i = 0; i < it.n && ok; ++i) {
        const int kb = it.block(i);
        if (!tile_sees(t, kb)) continue;
        ok = wait(&b.s_full[wg], n);
        if (!ok) break;
        tc_fence_after();
        float s[128];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld_32x32(ts + 32 * c, s + 32 * c);
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_wait_ld_32(s + 32 * c);
        if (S::kApart) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&b.s_free[wg]);
        }
        const int j0 = kb * kTileK, last = t.pos + t.n - 1;
        const bool whole = j0 + kTileK <= it.sq.len && (p.right < 0 || j0 + kTileK - 1 <= (int64_t)t.pos + p.right) &&
                           (p.left < 0 || j0 >= (int64_t)last - p.left || j0 + kTileK <= p.sinks);
        if (!whole || negative) {
          // columns c <= top and (c >= low or c < sink) are seen; as bits, 32 columns to a word
          auto column = [&](int64_t j) { return (int)max((int64_t)-1, min((int64_t)kTileK, j - j0)); };
          const int top = min(column(it.sq.len - 1), p.right < 0 ? kTileK : column((int64_t)pos + p.right));
          const int low = p.left < 0 ? 0 : column((int64_t)pos - p.left), sink = column(p.sinks);
          auto below = [](int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; };
#pragma unroll
          for (int c = 0; c < 128; c += 32) {
            const uint32_t see = below(top + 1 - c) & (~below(low - c) | below(sink - c));
#pragma unroll
            for (int e = 0; e < 32; ++e) s[c + e] = see >> e & 1u ? s[c + e] * sign : -INFINITY;
          }
        }
        float mx[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) mx[c] = s[c];
#pragma unroll
        for (int c = 4; c < 128; c += 8)
#pragma unroll
          for (int e = 0; e < 4; ++e) mx[e] = fmaxf(fmaxf(mx[e], s[c + e]), s[min(c + 4 + e, 127)]);
        const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
        const bool grow = top > m + slack || (m == -INFINITY && top > m);
        const float mn = grow ? top : m;
        const float shrink = !grow ? 1.f : m == -INFINITY ? 0.f : exp2_approx((m - mn) * scale);
        m = mn;
        const float off = m == -INFINITY ? 0.f : -m * scale;
        l *= shrink;
        // the last product with these weights' columns, and into these outputs, is over
        if (!first) ok = wait(&b.pv_done[wg], n - 1);
        if (!ok) break;
        tc_fence_after();
        if (!first && __any_sync(0xffffffffu, grow)) {
#pragma unroll 1
          for (int c = 0; c < DP; c += 8) tmem_scale_32x8(to + c, shrink);
        }
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t w[32];
#pragma unroll
          for (int c = 0; c < 32; ++c) {
            const float a = exp2_approx(fmaf(s[64 * h + 2 * c], scale, off));
            const float d = exp2_approx(fmaf(s[64 * h + 2 * c + 1], scale, off));
            sum[(2 * c) & 3] += a;
            sum[(2 * c + 1) & 3] += d;
            w[c] = pack2<T>(a, d);
          }
          tmem_st_32x32(tp + 32 * h, w);
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&b.p_full[wg]);
        first = false;
        ++n;
      }
      if (!ok) break;
      // output
      if (!first) {
        ok = wait(&b.pv_done[wg], n - 1);
        if (!ok) break;
        tc_fence_after();
      }
      const bool none = first || l == 0.f;
      const float r = none ? 0.f : 1.f / l;
      T* out = reinterpret_cast<T*>(p.out.data + (int64_t)(it.sq.q0 + t.row + min(row, t.n - 1)) * p.out.row_bytes +
                                    (int64_t)t.head * p.out.head_bytes);
      float odd = 0.f;                               // NaN once a value is not finite
#pragma unroll
      for (int c = 0; c < DP; c += 32) {
        float o[32];
        if (!first) {
          tmem_ld_32x32(to + c, o);
          tmem_wait_ld_32(o);
        }
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          o[e] = none ? 0.f : o[e] * r;
          odd = fmaf(o[e], 0.f, odd);
        }
        if (row < t.n)
#pragma unroll
          for (int e = 0; e < 32; e += 8)
            if (c + e < p.dim) {
              uint4 u;
              u.x = pack2<T>(o[e], o[e + 1]);
              u.y = pack2<T>(o[e + 2], o[e + 3]);
              u.z = pack2<T>(o[e + 4], o[e + 5]);
              u.w = pack2<T>(o[e + 6], o[e + 7]);
              *reinterpret_cast<uint4*>(out + c + e) = u;
            }
      }
      tc_fence_before();
      dirty = dirty || (row < t.n && odd != odd);
    }
    // A weight of zero times a value that is not finite is NaN: rows that hold one are done again, key by visible
    // key.  After everything else, so that nothing waits for it.
    if (ok && __any_sync(0xffffffffu, dirty)) {
      float* qs = q_rows + warp * 128;
      for (int64_t at = blockIdx.x; at < g.items; at += gridDim.x) {
        AttendItem it;
        if (!attend_item(p, g, at, it)) continue;
        const AttendTile t = wg ? it.t[1] : it.t[0];
        bool again = false;
        if (row < t.n) {
          const T* out = reinterpret_cast<const T*>(p.out.data + (int64_t)(it.sq.q0 + t.row + row) * p.out.row_bytes +
                                                    (int64_t)t.head * p.out.head_bytes);
          for (int d = 0; d < p.dim; ++d) again = again || !(fabsf(to_f(out[d])) < INFINITY);
        }
        for (uint32_t rows = __ballot_sync(0xffffffffu, again); rows; rows &= rows - 1) {
          const int i = t.row + (warp & 3) * 32 + __ffs(rows) - 1;
          const T* q = reinterpret_cast<const T*>(p.q.data + (int64_t)(it.sq.q0 + i) * p.q.row_bytes +
                                                  (int64_t)t.head * p.q.head_bytes);
          __syncwarp();
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
  if (warp == 8) tmem_dealloc(tmem, 512);
}

}  // namespace gnn
